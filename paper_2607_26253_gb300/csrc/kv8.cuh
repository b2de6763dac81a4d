// The 8-bit paged KV cache: quantising tokens as they are written, reading them back.
//   value = code * 2^e, e per 32 positions, KV head and K or V: the smallest integer with amax <= top * 2^e
// A power of two costs e4m3 nothing (its steps are relative) and int8 half a bit on average, and it makes raising a scale
// exact but for the bits that fall off the lower end: the errors of any number of raises add up to at most
// 1/2 + 1/4 + ... of one smallest step, where a free scale would round every code again each time.
// Both directions are bound by memory: 64 x 1,024 tokens of 8 heads of 128 are written in 61 us (403 MB, 6.6 TB/s), 48 x 4,096 read back
// in 178 (1,208 MB, 6.8 TB/s); one token each of 26 rows 3.5 us, a chain of three dependent loads.
#pragma once
#include "device_common.cuh"
#include "host_util.h"

namespace sara {

constexpr int kKv8Page = SARA_KV8_PAGE;
constexpr int kKv8Block = SARA_KV8_SCALE;
constexpr int kKv8PageBlocks = kKv8Page / kKv8Block;
constexpr int kKv8LowestExp = -100;
constexpr int kKv8MaxSeqs = 1 << 30;  // of a call: the search for a unit's sequence counts in 32 bits

struct Kv8Cache {
    uint8_t *codes;
    float *scales;
    const int32_t *table;
    int64_t table_stride;
    int n_blocks, max_blocks, KVH;
};

__device__ __forceinline__ int64_t kv8_tile(const Kv8Cache &c, int block, int kv, int h) {
    return ((int64_t)block * 2 + kv) * c.KVH + h;
}
__device__ __forceinline__ void kv8_report(int32_t *status) {
    if (status) *status = SARA_EINVAL;
}

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }
// The largest integer e with 2^e <= s of a scale s > 0 (below the normal range: -127)
__device__ __forceinline__ int scale_exp(float s) { return ((__float_as_int(s) >> 23) & 0xff) - 127; }

// The smallest e >= kKv8LowestExp with amax <= top * 2^e: amax = f * 2^x with 1 <= f < 2, 448 = 1.75 * 2^8,
// 127 = 1.984375 * 2^6.
template <int FMT>
__device__ __forceinline__ int exponent_for(float amax) {
    const int bits = __float_as_int(amax), x = (bits >> 23) - 127, frac = bits & 0x7fffff;
    const int e = FMT == SARA_KV8_E4M3 ? x - 8 + (frac > 0x600000) : x - 6 + (frac > 0x7e0000);
    return max(e, kKv8LowestExp);
}

// Codes of four fp32 values times f (|x f| at most the format's top; the product is exact), to the nearest, ties to even: first
// value in the low byte.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(float2 a, float2 b, float f) {
    if constexpr (FMT == SARA_KV8_E4M3) {
        uint16_t lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(a.y * f), "f"(a.x * f));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(b.y * f), "f"(b.x * f));
        return (uint32_t)lo | (uint32_t)hi << 16;
    } else {
        constexpr float kUnits = 12582912.f;  // 1.5 * 2^23: the sum's last bits are the rounded whole number
        const uint32_t x = __float_as_uint(fmaf(a.x, f, kUnits)), y = __float_as_uint(fmaf(a.y, f, kUnits));
        const uint32_t z = __float_as_uint(fmaf(b.x, f, kUnits)), w = __float_as_uint(fmaf(b.y, f, kUnits));
        return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
    }
}
// Two codes (low 16 bits of w) as an fp16 pair: exact in both formats (e4m3 is a subset of fp16).
template <int FMT>
__device__ __forceinline__ uint32_t decode2_half(uint32_t w) {
    if constexpr (FMT == SARA_KV8_E4M3) {
        uint32_t r;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
        return r;
    } else {
        // byte + 128 as the low bits of fp16 1024 .. 1279, minus 1152
        const uint32_t u = __byte_perm(w ^ 0x8080u, 0x64646464u, 0x4140);
        const __half2 r = __hsub2(*reinterpret_cast<const __half2 *>(&u), __floats2half2_rn(1152.f, 1152.f));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
}
template <int FMT>
__device__ __forceinline__ float2 decode2(uint32_t w) {
    const uint32_t h = decode2_half<FMT>(w);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

// 16-bit element pairs
template <int TYPE>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    if constexpr (TYPE == SARA_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (TYPE == SARA_BF16) return (uint32_t)f32_to_bf16(a) | ((uint32_t)f32_to_bf16(b) << 16);
    else return (uint32_t)__half_as_ushort(__float2half_rn(a)) | ((uint32_t)__half_as_ushort(__float2half_rn(b)) << 16);
}

// The larger magnitudes of two pairs; a NaN stays
template <int TYPE>
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
    uint32_t r;
    if constexpr (TYPE == SARA_BF16)
        asm("{\n\t.reg .b32 x, y;\n\tabs.bf16x2 x, %1;\n\tabs.bf16x2 y, %2;\n\tmax.NaN.bf16x2 %0, x, y;\n\t}" : "=r"(r) : "r"(a), "r"(b));
    else
        asm("{\n\t.reg .b32 x, y;\n\tabs.f16x2 x, %1;\n\tabs.f16x2 y, %2;\n\tmax.NaN.f16x2 %0, x, y;\n\t}" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// The packed tokens of n sequences in units of one scale block: sequence i's units begin at start[i] / 32 + 2 i, which
// leaves room for the most blocks that its tokens can touch ((n_i - 1) / 32 + 2), so a unit finds its sequence
// by search and no prefix sums are needed.  A warp narrows the search 32-fold a step.
__host__ __device__ __forceinline__ int64_t kv8_first_unit(int start, int i) { return (int64_t)(start / kKv8Block) + 2 * (int64_t)i; }
inline int64_t kv8_units(int total, int n) { return kv8_first_unit(total, n); }

struct Kv8Range {
    const int32_t *pos0, *start;
    int n, total;
};
struct Kv8Unit {
    int seq, lo, hi;  // positions lo .. hi of the sequence, within one scale block
    int row;          // packed row of position lo
    bool held;        // the block holds earlier tokens
    bool bad;         // the sequence's positions are wrong
};
// Warp w < n looks at sequence w's range, whichever unit is its own: starts that fall may leave a sequence without one.
__device__ __forceinline__ void kv8_check(const Kv8Range &r, int max_blocks, int64_t w, int32_t *status) {
    if (w >= r.n || (threadIdx.x & 31) != 0 || !status) return;
    const int a = __ldg(r.start + w), b = __ldg(r.start + w + 1), p0 = __ldg(r.pos0 + w);
    if (a < 0 || b < a || b > r.total || (b > a && (p0 < 0 || (int64_t)p0 + (b - a) > (int64_t)max_blocks * kKv8Page))) kv8_report(status);
}
// Whole warps call this with the same u.  False: nothing to do.
__device__ __forceinline__ bool kv8_find(const Kv8Range &r, int max_blocks, int64_t u, Kv8Unit &x) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = r.n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32;
        const int64_t i = lo + (int64_t)(lane + 1) * step;
        const bool before = i < hi && kv8_first_unit(__ldg(r.start + i), (int)i) <= u;
        const int k = __popc(__ballot_sync(0xffffffffu, before));
        lo += k * step;
        hi = min(hi, lo + step);
    }
    const int a = __ldg(r.start + lo), b = __ldg(r.start + lo + 1), p0 = __ldg(r.pos0 + lo);
    if (a < 0 || b < a || b > r.total) return false;
    const int64_t local = u - kv8_first_unit(a, lo);
    if (local < 0 || b == a) return false;
    const int64_t end = (int64_t)p0 + (b - a);
    x.seq = lo;
    x.bad = p0 < 0 || end > (int64_t)max_blocks * kKv8Page;
    const int base = x.bad ? 0 : p0;  // (a wrong range: its rows, counted from 0)
    const int64_t blk = base / kKv8Block + local, last = base + (int64_t)(b - a);
    if (blk * kKv8Block >= last) return false;
    x.lo = (int)max((int64_t)base, blk * kKv8Block);
    x.hi = (int)min(last, (blk + 1) * kKv8Block);
    x.row = a + (x.lo - base);
    x.held = x.lo % kKv8Block != 0;
    return true;
}

// One warp per scale block, KV head and K or V: the block's new tokens wait in registers for their largest
// magnitude, so k and v are read once.  (64 registers a lane at 128 dims: 20 warps an SM hold 160 KB, more than the
// bandwidth times the latency.)
template <int HD, int FMT, int TYPE>
__global__ void __launch_bounds__(128) kv8_write_kernel(Kv8Cache c, Kv8Range r, const uint16_t *k, int64_t k_stride,
                                                        const uint16_t *v, int64_t v_stride, int64_t warps, int32_t *status) {
    constexpr int LT = HD / 8, TW = 32 / LT, IT = kKv8Block / TW;  // lanes a token, tokens at a time, times
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (w >= warps) return;
    const int lane = threadIdx.x & 31, h = (int)(w % c.KVH), kv = (int)(w / c.KVH % 2);
    kv8_check(r, c.max_blocks, w, status);
    Kv8Unit x;
    if (!kv8_find(r, c.max_blocks, w / (2 * c.KVH), x)) return;
    if (x.bad) return;  // (reported above)
    const int block = __ldg(c.table + x.seq * c.table_stride + x.lo / kKv8Page);
    if (block < 0 || block >= c.n_blocks) {
        kv8_report(status);
        return;
    }
    const int64_t tile = kv8_tile(c, block, kv, h);
    const int base = x.lo / kKv8Block * kKv8Block, dim = lane % LT * 8;
    uint8_t *codes = c.codes + (tile * kKv8Page + base % kKv8Page) * HD + dim;  // of the block's first position
    float *scale = c.scales + tile * kKv8PageBlocks + base % kKv8Page / kKv8Block;
    const uint16_t *src = (kv ? v : k) + h * HD + dim;
    const int64_t stride = kv ? v_stride : k_stride;
    uint4 e[IT];
    uint32_t top = 0;
    const bool full = x.hi - x.lo == kKv8Block;
    src += (x.row + (base - x.lo) + lane / LT) * stride;  // (of the block's first position: the loads stay behind x.lo)
    if (full) {
#pragma unroll
        for (int i = 0; i < IT; ++i) e[i] = __ldg(reinterpret_cast<const uint4 *>(src + i * (TW * stride)));
    } else {
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int p = base + i * TW + lane / LT;
            e[i] = p >= x.lo && p < x.hi ? __ldg(reinterpret_cast<const uint4 *>(src + i * (TW * stride))) : make_uint4(0, 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) top = max_abs2<TYPE>(top, max_abs2<TYPE>(max_abs2<TYPE>(e[i].x, e[i].y), max_abs2<TYPE>(e[i].z, e[i].w)));
    // magnitudes order as their bits do, NaN above infinity
    top = __reduce_max_sync(0xffffffffu, max(top & 0xffff, top >> 16));
    const float amax = unpack2<TYPE>(top).x;
    const float was = x.held ? *scale : 0.f;
    if (!(amax <= 3.4028235e38f) || was != was || was > 3.4028235e38f) {  // (codes no longer mean anything)
        __syncwarp();
        if (lane == 0) *scale = __int_as_float(0x7fc00000);
        return;
    }
    int ex = exponent_for<FMT>(amax);
    if (x.held) {
        const int old = scale_exp(was);
        if (old >= ex) {
            ex = old;
        } else {
            const float f = old - ex < -126 ? 0.f : pow2f(old - ex);
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const int p = base + i * TW + lane / LT;
                if (p < x.lo) {
                    uint2 *at = reinterpret_cast<uint2 *>(codes + (p - base) * HD);
                    uint2 o = *at;
                    uint32_t n[2] = {o.x, o.y};
#pragma unroll
                    for (int j = 0; j < 2; ++j) n[j] = encode4<FMT>(decode2<FMT>(n[j] & 0xffff), decode2<FMT>(n[j] >> 16), f);
                    *at = make_uint2(n[0], n[1]);
                }
            }
        }
    }
    const float f = pow2f(-ex);
    codes += lane / LT * HD;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int p = base + i * TW + lane / LT;
        if (full || (p >= x.lo && p < x.hi))
            *reinterpret_cast<uint2 *>(codes + i * TW * HD) =
                make_uint2(encode4<FMT>(unpack2<TYPE>(e[i].x), unpack2<TYPE>(e[i].y), f),
                           encode4<FMT>(unpack2<TYPE>(e[i].z), unpack2<TYPE>(e[i].w), f));
    }
    __syncwarp();
    if (lane == 0) *scale = pow2f(ex);
}

// Eight codes times s to 8 `type` elements at p (16-byte aligned)
template <int FMT, int TYPE>
__device__ __forceinline__ void store8(uint8_t *p, uint2 o, float s) {
    float2 y[4] = {decode2<FMT>(o.x & 0xffff), decode2<FMT>(o.x >> 16), decode2<FMT>(o.y & 0xffff), decode2<FMT>(o.y >> 16)};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        y[j].x *= s;
        y[j].y *= s;
    }
    if constexpr (TYPE == SARA_FP32) {
#pragma unroll
        for (int j = 0; j < 2; ++j) reinterpret_cast<float4 *>(p)[j] = make_float4(y[2 * j].x, y[2 * j].y, y[2 * j + 1].x, y[2 * j + 1].y);
    } else {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<TYPE>(y[0].x, y[0].y), pack2<TYPE>(y[1].x, y[1].y), pack2<TYPE>(y[2].x, y[2].y),
                                                   pack2<TYPE>(y[3].x, y[3].y));
    }
}

// One warp per scale block, KV head and K or V, 16 codes a lane, the block's in flight together.  Two neighbouring lanes
// exchange halves, so that each of their stores fills a 32-byte sector.
template <int HD, int FMT, int TYPE>
__global__ void __launch_bounds__(128) kv8_read_kernel(Kv8Cache c, Kv8Range r, uint8_t *k, int64_t k_stride, uint8_t *v,
                                                       int64_t v_stride, int64_t warps, int32_t *status) {
    constexpr int LT = HD / 16, TW = 32 / LT, IT = kKv8Block / TW, SIZE = TYPE == SARA_FP32 ? 4 : 2;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (w >= warps) return;
    const int lane = threadIdx.x & 31, h = (int)(w % c.KVH), kv = (int)(w / c.KVH % 2);
    kv8_check(r, c.max_blocks, w, status);
    Kv8Unit x;
    if (!kv8_find(r, c.max_blocks, w / (2 * c.KVH), x)) return;
    bool bad = x.bad;
    int block = 0;
    if (!bad) {
        block = __ldg(c.table + x.seq * c.table_stride + x.lo / kKv8Page);
        bad = block < 0 || block >= c.n_blocks;
    }
    if (bad) kv8_report(status);
    const int64_t tile = kv8_tile(c, bad ? 0 : block, kv, h);
    const int base = x.lo / kKv8Block * kKv8Block, dim = lane % LT / 2 * 32 + 8 * (lane & 1);
    const uint8_t *codes = c.codes + (tile * kKv8Page + base % kKv8Page + lane / LT) * HD + lane % LT * 16;
    const float s = bad ? __int_as_float(0x7fc00000) : __ldg(c.scales + tile * kKv8PageBlocks + base % kKv8Page / kKv8Block);
    const int64_t stride = (kv ? v_stride : k_stride) * SIZE;
    uint8_t *dst = (kv ? v : k) + (x.row + (base - x.lo) + lane / LT) * stride + (h * HD + dim) * SIZE;
    const bool full = x.hi - x.lo == kKv8Block;
    uint4 o[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int p = base + i * TW + lane / LT;
        o[i] = make_uint4(0, 0, 0, 0);
        if (!bad && (full || (p >= x.lo && p < x.hi))) o[i] = __ldg(reinterpret_cast<const uint4 *>(codes + i * TW * HD));
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int p = base + i * TW + lane / LT;
        const bool odd = lane & 1;
        const uint2 give = odd ? make_uint2(o[i].x, o[i].y) : make_uint2(o[i].z, o[i].w);
        const uint2 got = make_uint2(__shfl_xor_sync(0xffffffffu, give.x, 1), __shfl_xor_sync(0xffffffffu, give.y, 1));
        if (!full && (p < x.lo || p >= x.hi)) continue;
        uint8_t *at = dst + i * TW * stride;
        store8<FMT, TYPE>(at, odd ? got : make_uint2(o[i].x, o[i].y), s);
        store8<FMT, TYPE>(at + 16 * SIZE, odd ? make_uint2(o[i].z, o[i].w) : got, s);
    }
}

}  // namespace sara
