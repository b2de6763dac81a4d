// Log-probabilities of given tokens under softmax(logits), with entropy and top alternatives, and the gradient of both.
//   m = max z, S = sum e^(z - m), T = sum e^(z - m) (z - m)
//   logprob = z[token] - m - log S,   entropy = log S - T / S
//   dz_v = g (1[v = token] - p_v) - g' p_v (log p_v + entropy)
// The gradient is bound by reading and writing the logits once (2,048 x 151,936, a tenth of the rows padding: fp32 334 us, 7.1 TB/s,
// bf16 174, 6.8).  The scores read them once, 16 bytes a lane, a step's loads in flight during the one before; 16-bit
// logits come so fast that the instructions per logit count, so they are taken two at a time and in base 2:
//   e^(z - m) = 2^(z log2(e) - r) 2^-c,  r = m log2(e) as rounded, c what the rounding took: one fused operation a logit,
// and c, the same for all, is put right once, in log S.  Sums in fp32 against the thread's own running maximum.  c is half a step of r
// at most: 1/16 up to |m| = 10^6, but 440 at 10^10 (a mask's usual values), where 2^c has no room.  Larger maxima take z - m first, logit by logit.
// Scores of 2,048 x 151,936 in bf16: 88 us, 6.4 TB/s (rows end in waves); with 8 alternatives 115; 26 rows with
// 8 alternatives 9.6, 5.4 without: the bound on them, their ranks and the cluster's join are latencies.
#pragma once
#include "device_common.cuh"
#include "host_util.h"

namespace sara {

constexpr int kScoreMaxTop = 32, kScoreMaxCtas = 8, kScoreWarpVectors = 512, kScoreTopWarpVectors = 1024;
constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;

__device__ __forceinline__ float exp2_approx(float y) {  // 2^-22 relative, 0 below 2^-126
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(y));
    return e;
}
__device__ __forceinline__ float exp2_full(float y) {  // the same down to the subnormal range
    float e;
    asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(y));
    return e;
}

// A row's elements as the aligned 16-byte vectors that hold them: vector k has elements k E - off .. + E - 1, of
// which those in [0, V) are the row's.
template <int TYPE>
struct RowVectors {
    static constexpr int kSize = TYPE == SARA_FP32 ? 4 : 2, E = 16 / kSize;
    static constexpr uint32_t kNone = TYPE == SARA_FP32 ? 0xff800000u : TYPE == SARA_BF16 ? 0xff80ff80u : 0xfc00fc00u;  // -inf
    const uint8_t *base;  // of vector 0
    uint32_t off, V;
    __device__ __forceinline__ RowVectors(const void *z, int64_t row, int64_t stride, int V_) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(z) + (uintptr_t)(row * stride * kSize);
        off = (uint32_t)(a & 15) / kSize;
        base = reinterpret_cast<const uint8_t *>(a & ~(uintptr_t)15);
        V = (uint32_t)V_;
    }
    __device__ __forceinline__ int vectors() const { return (int)((off + V + (E - 1)) / E); }
    __device__ __forceinline__ uint32_t first(int k) const { return (uint32_t)k * E - off; }  // (wraps below 0 for k = 0)
    __device__ __forceinline__ bool whole(int k) const { return first(k) < V && V - first(k) >= (uint32_t)E; }
    // The vectors whose elements are all the row's are [whole_from, whole_to).
    __device__ __forceinline__ int whole_from() const { return off ? 1 : 0; }
    __device__ __forceinline__ int whole_to() const { return (int)((off + V) / E); }
    // The row's elements of vector k, -inf in the place of others.  (Plain loads: the gradient may take the logits' place.)
    __device__ __forceinline__ uint4 load(int k) const {
        const uint8_t *p = base + (int64_t)k * 16;
        if (whole(k)) return *reinterpret_cast<const uint4 *>(p);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = kNone;
            if constexpr (TYPE == SARA_FP32) {
                if (first(k) + i < V) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
            } else {
                if (first(k) + 2 * i < V) w[i] = (w[i] & 0xffff0000u) | reinterpret_cast<const uint16_t *>(p)[2 * i];
                if (first(k) + 2 * i + 1 < V) w[i] = (w[i] & 0xffffu) | (uint32_t)reinterpret_cast<const uint16_t *>(p)[2 * i + 1] << 16;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <int TYPE>
__device__ __forceinline__ void unpack_vector(const uint4 &x, float (&z)[16 / (TYPE == SARA_FP32 ? 4 : 2)]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (TYPE == SARA_FP32) {
            z[i] = __uint_as_float(w[i]);
        } else if constexpr (TYPE == SARA_BF16) {
            z[2 * i] = __uint_as_float(w[i] << 16);
            z[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            z[2 * i] = f.x;
            z[2 * i + 1] = f.y;
        }
    }
}
// The larger of two words' logits (of 16-bit types: pairs); a NaN gives way
template <int TYPE>
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
    if constexpr (TYPE == SARA_FP32) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    } else {
        uint32_t r;
        if constexpr (TYPE == SARA_BF16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
}
// Logits (of 16-bit types: pairs) raised to at least `least` (a word of the same type); a NaN stays
template <int TYPE>
__device__ __forceinline__ uint32_t raise_word(uint32_t a, uint32_t least) {
    uint32_t r;
    if constexpr (TYPE == SARA_FP32) asm("max.NaN.f32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(least));
    else if constexpr (TYPE == SARA_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(least));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(least));
    return r;
}
template <int TYPE>
__device__ __forceinline__ uint4 raise_vector(const uint4 &x, uint32_t least) {
    return make_uint4(raise_word<TYPE>(x.x, least), raise_word<TYPE>(x.y, least), raise_word<TYPE>(x.z, least), raise_word<TYPE>(x.w, least));
}
__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 unpack_f32x2(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
template <int TYPE>
__device__ __forceinline__ float load_logit(const void *z, int64_t i) {
    if constexpr (TYPE == SARA_FP32) return static_cast<const float *>(z)[i];
    else if constexpr (TYPE == SARA_BF16) return bf16_to_f32(static_cast<const uint16_t *>(z)[i]);
    else return f16_to_f32(static_cast<const uint16_t *>(z)[i]);
}

struct ScoreParams {
    const void *z;
    int64_t stride;
    int R, V, top;
    const int32_t *tokens;
    float *logprob, *entropy, *stats;
    int32_t *top_token;
    float *top_logprob;
    int ctas;  // a row
    int turn;  // 1: the grid of the last rows may start when this one's CTAs all have; 2: the grid of the last rows; 0: alone
};

// ------------------------------------------------------------------------------- alternatives
// A logit's place in their order: by value, then the lower token; 0 for one that is not listed.
__device__ __forceinline__ uint64_t score_key(float z, uint32_t v) {
    if (!(z > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(z + 0.f);  // (-0 as 0)
    return ((uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32) | (0x7fffffffu - v);
}
__device__ __forceinline__ float score_key_value(uint64_t k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return k == 0 ? -INFINITY : __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int score_key_token(uint64_t k) { return k == 0 ? -1 : 0x7fffffff - (int)(uint32_t)k; }

__device__ __forceinline__ uint64_t exchange_key(uint64_t key, int d, bool larger) {
    const uint64_t o = __shfl_xor_sync(0xffffffffu, key, d);
    return larger == (key > o) ? key : o;
}
// A warp's 32 best keys so far, lane i the i-th.  Candidates are collected in shared memory and joined 32 at a
// time: sorted the other way round, the element-wise larger keys are the best 32 of both and a bitonic sequence, which five
// exchanges sort.
struct ScoreList {
    uint64_t key = 0;
    __device__ __forceinline__ void join(uint64_t other) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
            for (int d = size / 2; d > 0; d >>= 1) other = exchange_key(other, d, ((lane & d) == 0) == ((lane & size) != 0 && size < 32));
        key = key > other ? key : other;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) key = exchange_key(key, d, (lane & d) == 0);
    }
};
// The `top` best of n keys to their places in `out` (zeroed before), a key's place being the number of larger ones: four threads a
// key.  Whole CTAs.
__device__ __forceinline__ void rank_keys(const uint64_t *keys, int n, int top, uint64_t *out) {
    const int part = threadIdx.x & 3;
    for (int i0 = 0; i0 < n; i0 += blockDim.x / 4) {
        const int i = i0 + (int)threadIdx.x / 4;
        const uint64_t k = i < n ? keys[i] : 0;
        int rank = 0;
#pragma unroll 4
        for (int j = part; j < n; j += 4) rank += keys[j] > k;
        rank += __shfl_xor_sync(0xffffffffu, rank, 1);
        rank += __shfl_xor_sync(0xffffffffu, rank, 2);
        if (part == 0 && rank < top && k) out[rank] = k;
    }
}
// The `top`-th largest of the lanes' values
__device__ __forceinline__ float warp_nth_largest(float v, int top) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int d = size / 2; d > 0; d >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, v, d);
            const bool larger_here = ((lane & d) == 0) == ((lane & size) == 0 || size == 32);
            v = larger_here ? fmaxf(v, o) : fminf(v, o);
        }
    return __shfl_sync(0xffffffffu, v, top - 1);
}

// ------------------------------------------------------------------------------- sums
// Maximum m, s = sum 2^(z log2(e) - r), t = sum 2^y y with y that exponent.  Where m is so large that c would count (or logits below m
// have no room in their type), r is exact (c = 0) and logits are taken one by one.
template <int TYPE>
struct ScoreSums {
    static constexpr uint32_t kLeast = TYPE == SARA_FP32 ? 0xfe967699u : TYPE == SARA_BF16 ? 0xfe96fe96u : 0xfbfffbffu;  // -1e38; fp16: its lowest
    float m = -3.4028235e38f, s = 0.f, t = 0.f;
    static __device__ __forceinline__ bool plain(float m) { return fabsf(m) < 1e6f && (TYPE != SARA_FP16 || m > -6e4f); }
    static __device__ __forceinline__ float carry(float m) { return plain(m) ? fmaf(m, kLog2e, -(m * kLog2e)) : 0.f; }  // c
    // to a maximum n >= m.  (The bound keeps 0 times infinity out where the maxima are that far apart.)
    __device__ __forceinline__ void rebase(float n) {
        const float d = fmaxf(fmaf(m - n, kLog2e, carry(n) - carry(m)), -1e4f), f = exp2_approx(d);
        t = (t + s * d) * f;
        s *= f;
        m = n;
    }
    // of LANES neighbouring lanes, the first lane's among them
    template <int LANES>
    __device__ __forceinline__ void join_lanes() {
        float n = m;
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) n = fmaxf(n, __shfl_xor_sync(0xffffffffu, n, d));
        rebase(n);
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, d);
            t += __shfl_xor_sync(0xffffffffu, t, d);
        }
    }
    // of the first n <= COLUMNS columns of a table, in every lane of a warp
    template <int COLUMNS>
    __device__ __forceinline__ void join_table(const float (*x)[COLUMNS], int n) {
        const int lane = threadIdx.x & (COLUMNS - 1);
        m = lane < n ? x[0][lane] : -3.4028235e38f;
        s = lane < n ? x[1][lane] : 0.f;
        t = lane < n ? x[2][lane] : 0.f;
        join_lanes<COLUMNS>();
    }
    // a vector's logits, none above m: one of -inf, raised to a finite one, still adds nothing to either sum; a NaN stays
    __device__ __forceinline__ void add(const uint4 &x, uint64_t &s2, uint64_t &t2) const {
        constexpr int E = RowVectors<TYPE>::E;
        const float r = -(m * kLog2e);
        const uint64_t r2 = pack_f32x2(r, r), l2 = pack_f32x2(kLog2e, kLog2e);
        float z[E];
        unpack_vector<TYPE>(raise_vector<TYPE>(x, kLeast), z);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const uint64_t y2 = fma_f32x2(pack_f32x2(z[e], z[e + 1]), l2, r2);
            const float2 y = unpack_f32x2(y2);
            const uint64_t w2 = pack_f32x2(exp2_approx(y.x), exp2_approx(y.y));
            s2 = add_f32x2(s2, w2);
            t2 = fma_f32x2(w2, y2, t2);
        }
    }
    __device__ __forceinline__ void add_far(const uint4 &x) {  // where !plain(m)
        constexpr int E = RowVectors<TYPE>::E;
        float z[E];
        unpack_vector<TYPE>(x, z);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float y = (z[e] - m) * kLog2e, w = exp2_approx(y);
            s += w;
            t = fmaf(w, fmaxf(y, -1000.f), t);
        }
    }
};

// Whether a value, of 64 in x, is the `top`-th largest (top <= 32): fewer than `top` are above it and, with its equals, at least
// `top` not below.  Four threads a value (256 in all).
__device__ __forceinline__ bool is_nth_of_64(const float *x, int top, float &v) {
    const int part = threadIdx.x & 3;
    v = x[threadIdx.x / 4];
    int above = 0, least = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 y = *reinterpret_cast<const float4 *>(x + 16 * j + 4 * part);
        above += (y.x > v) + (y.y > v) + (y.z > v) + (y.w > v);
        least += (y.x >= v) + (y.y >= v) + (y.z >= v) + (y.w >= v);
    }
    int n = above << 16 | least;
    n += __shfl_xor_sync(0xffffffffu, n, 1);
    n += __shfl_xor_sync(0xffffffffu, n, 2);
    return (n >> 16) < top && (n & 0xffff) >= top;
}
// Floats as integers of the same order
__device__ __forceinline__ int ordered(float f) {
    const int b = __float_as_int(f);
    return b < 0 ? b ^ 0x7fffffff : b;
}
__device__ __forceinline__ float from_ordered(int i) { return __int_as_float(i < 0 ? i ^ 0x7fffffff : i); }

// One row per group of WARPS warps (1: eight rows to a CTA; else a CTA), or, where p.ctas > 1, per cluster of that many
// CTAs, each a contiguous share of its vectors.
// CTAs an SM that the registers have to leave room for.  (The alternatives of 16-bit logits would spill at four: 2,048 x 151,936, top 8:
// 132 us, 148 with four.  A warp a row in fp32 spills 12 bytes at six.)
constexpr int score_sm_ctas(int type, bool top, int warps) {
    return warps == 4 ? 8 : warps == 1 && !top ? 6 : warps == 8 && top && type != SARA_FP32 ? 3 : 4;
}
template <int TYPE, bool TOP, int WARPS>
__global__ void __launch_bounds__(WARPS > 1 ? 32 * WARPS : 256, score_sm_ctas(TYPE, TOP, WARPS)) score_kernel(ScoreParams p) {
    constexpr int CW = WARPS > 1 ? WARPS : 8;  // the CTA's warps
    using Row = RowVectors<TYPE>;
    constexpr int E = Row::E, U = WARPS > 1 ? 4 : 2, STEP = 32 * WARPS;
    __shared__ float s_sums[3][CW];
    __shared__ uint64_t s_cand[TOP ? CW : 1][64];             // candidates that a warp has not joined yet
    __shared__ uint64_t s_key[TOP ? CW * 32 : 1], s_best[32];  // the warps' candidates; the CTA's alternatives
    __shared__ __align__(16) float s_group[64];
    __shared__ int s_floor;  // no alternative is below this (ordered)
    __shared__ int s_held[CW];
    __shared__ __align__(8) uint32_t c_sums[3][kScoreMaxCtas], c_key[TOP ? kScoreMaxCtas * 32 : 1][2];  // (rank 0) the cluster's
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = threadIdx.x % STEP;
    const bool cluster = WARPS > 1 && p.ctas > 1;
    if (p.turn == 1) pdl_allow_dependents();
    if (cluster) cluster_arrive();  // (waited for before the stores into rank 0's shared memory)
    const int64_t r64 = WARPS > 1 ? (int64_t)(blockIdx.x / (unsigned)p.ctas) : (int64_t)blockIdx.x * 8 + warp;
    const int rank = WARPS > 1 ? (int)(blockIdx.x % (unsigned)p.ctas) : 0;
    if (r64 >= p.R) return;
    const int r = (int)r64, tok = p.tokens ? p.tokens[r] : 0;
    const bool pad = tok < 0;
    const Row row(p.z, r, p.stride, p.V);
    const float nan = __int_as_float(0x7fc00000);
    const float ztok = part == 0 && rank == 0 && !pad && tok < p.V ? load_logit<TYPE>(p.z, r * p.stride + tok) : nan;

    ScoreSums<TYPE> a;
    ScoreList list;
    int nb = 0, held = 0;                       // steps; candidates in s_cand
    uint64_t kth = 0;                           // the list's entry `top`
    float kth_v = -INFINITY, floor = -INFINITY;  // its value; no alternative is below this
    const int nv = pad ? 0 : row.vectors(), per = (nv + p.ctas - 1) / p.ctas, v1 = min(nv, (rank + 1) * per);
    uint4 next[U];
    const int w0 = row.whole_from(), w1 = min(v1, row.whole_to());
    auto load = [&](int b, uint4 (&x)[U]) {  // the step of vectors from b on
        if (b >= w0 && b + U * STEP <= w1) {
            const uint4 *q = reinterpret_cast<const uint4 *>(row.base) + b + part;
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = q[u * STEP];
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = b + part + u * STEP;
                x[u] = k < v1 ? row.load(k) : make_uint4(Row::kNone, Row::kNone, Row::kNone, Row::kNone);
            }
        }
    };
    auto join = [&](int least) {  // candidates into the list, 32 at a time
        while (held >= least) {
            __syncwarp();
            const int at = max(held - 32, 0);
            list.join(at + lane < held ? s_cand[warp][at + lane] : 0);
            held = at;
        }
        kth = __shfl_sync(0xffffffffu, list.key, p.top - 1);
        kth_v = score_key_value(kth);
        floor = fmaxf(floor, kth_v);
        if (WARPS > 1 && lane == 0) atomicMax(&s_floor, ordered(floor));
        __syncwarp();
    };
    if (TOP && WARPS > 1 && threadIdx.x == 0) s_floor = ordered(-INFINITY);
    const int v0 = min(rank * per, v1);
    load(v0, next);
#pragma unroll 1
    for (int b = v0; b < v1; b += U * STEP) {  // (every lane of a warp the same steps)
        const int k = b + part;
        uint4 cur[U];
        uint32_t most = Row::kNone;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            cur[u] = next[u];
            most = max_word<TYPE>(most, max_word<TYPE>(max_word<TYPE>(cur[u].x, cur[u].y), max_word<TYPE>(cur[u].z, cur[u].w)));
        }
        if (v1 - b > U * STEP) load(b + U * STEP, next);
        const float best = TYPE == SARA_FP32 ? __uint_as_float(most) : TYPE == SARA_BF16 ? fmaxf(__uint_as_float(most << 16), __uint_as_float(most & 0xffff0000u))
                                                                                          : fmaxf(f16_to_f32((uint16_t)most), f16_to_f32((uint16_t)(most >> 16)));
        if (best > a.m) a.rebase(best);
        if (a.plain(a.m)) {
            uint64_t s2 = pack_f32x2(a.s, 0.f), t2 = pack_f32x2(a.t, 0.f);
#pragma unroll
            for (int u = 0; u < U; ++u) a.add(cur[u], s2, t2);
            a.s = unpack_f32x2(s2).x + unpack_f32x2(s2).y;
            a.t = unpack_f32x2(t2).x + unpack_f32x2(t2).y;
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) a.add_far(cur[u]);
        }
        if constexpr (TOP) {
            // nothing below the top-th of some parts' maxima so far can matter (of the lanes, or of a 64th of the CTA each): taken
            // again whenever the steps have doubled, so that a long row's later steps hold few candidates
            if (++nb, (nb & (nb - 1)) == 0) {
                if constexpr (WARPS > 1) {
                    float four = fmaxf(a.m, __shfl_xor_sync(0xffffffffu, a.m, 1)), v;
                    four = fmaxf(four, __shfl_xor_sync(0xffffffffu, four, 2));
                    if (lane % 4 == 0) s_group[threadIdx.x / 4] = four;
                    __syncthreads();
                    if (is_nth_of_64(s_group, p.top, v)) atomicMax(&s_floor, ordered(v));
                    __syncthreads();
                } else {
                    floor = fmaxf(floor, warp_nth_largest(a.m, p.top));
                }
            }
            if (WARPS > 1) floor = fmaxf(floor, from_ordered(*(volatile int *)&s_floor));  // (a late one is a lower bound all the same)
            // earlier steps had the lower tokens, so equal to the own top-th is too late, equal to another warp's is not
            if (__any_sync(0xffffffffu, best > kth_v && best >= floor)) {
                uint32_t mask = 0;  // this lane's logits that may count
                const float least = fmaxf(floor, -3.4028235e38f);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float z[E];
                    unpack_vector<TYPE>(cur[u], z);
#pragma unroll
                    for (int e = 0; e < E; ++e) mask |= (uint32_t)(z[e] >= least) << (u * E + e);
                }
#pragma unroll 1
                while (__any_sync(0xffffffffu, mask != 0)) {  // (few: read again, from the cache)
                    const int i = mask ? __ffs(mask) - 1 : 0;
                    const uint32_t v = row.first(k + i / E * STEP) + i % E;
                    const uint64_t key = mask ? score_key(load_logit<TYPE>(p.z, r * p.stride + v), v) : 0;
                    mask &= mask - 1;
                    const uint32_t cand = __ballot_sync(0xffffffffu, key > kth);
                    if (key > kth) s_cand[warp][held + __popc(cand & ((1u << lane) - 1))] = key;
                    held += __popc(cand);
                    if (held >= 32) join(32);
                }
            }
        }
    }
    const bool sorted = WARPS == 1 || kth != 0;  // (only then the list holds something)
    if (TOP && sorted && held > 0) join(1);
    a.template join_lanes<32>();
    if constexpr (WARPS > 1) {
        if (lane == 0) {
            s_sums[0][warp] = a.m;
            s_sums[1][warp] = a.s;
            s_sums[2][warp] = a.t;
            if (TOP) s_held[warp] = sorted ? p.top : held;
        }
        if (TOP && warp == 0) s_best[lane] = 0;
        if (cluster) cluster_wait();  // every CTA of the cluster has started
        __syncthreads();
        if (warp == 0) a.join_table(s_sums, WARPS);
        if (TOP) {
            int from = 0, n = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                if (w < warp) from += s_held[w];
                n += s_held[w];
            }
            if (lane < s_held[warp]) s_key[from + lane] = sorted ? list.key : s_cand[warp][lane];
            __syncthreads();
            rank_keys(s_key, n, p.top, s_best);
            __syncthreads();
            list.key = s_best[lane];
        }
        if (cluster) {
            if (warp == 0) {
                if (lane < 3) st_cluster_u32(cluster_addr(&c_sums[lane][rank], 0), __float_as_uint(lane == 0 ? a.m : lane == 1 ? a.s : a.t));
                if (TOP && lane < p.top) {
                    st_cluster_u32(cluster_addr(&c_key[rank * p.top + lane][0], 0), (uint32_t)list.key);
                    st_cluster_u32(cluster_addr(&c_key[rank * p.top + lane][1], 0), (uint32_t)(list.key >> 32));
                }
            }
            cluster_sync();
            if (rank != 0) return;
            if (warp == 0) a.join_table(reinterpret_cast<const float (*)[kScoreMaxCtas]>(c_sums), p.ctas);
            if (TOP) {
                if (warp == 0) s_best[lane] = 0;
                __syncthreads();
                rank_keys(reinterpret_cast<const uint64_t *>(c_key), p.ctas * p.top, p.top, s_best);
                __syncthreads();
                list.key = s_best[lane];
            }
        }
        if (warp != 0) return;
    }
    if (p.turn == 2) pdl_wait_prior_grids();  // (so that who waits for these rows waits for the others too)
    const bool none = a.s == 0.f;  // every logit is -inf
    const float m = pad ? 0.f : none ? -INFINITY : a.m, ls = none ? 0.f : fmaf(-kLn2, ScoreSums<TYPE>::carry(a.m), logf(a.s));
    if (lane == 0) {
        if (p.logprob) p.logprob[r] = pad ? 0.f : none && tok < p.V ? -INFINITY : ztok - m - ls;
        if (p.entropy) p.entropy[r] = none ? 0.f : fmaf(-kLn2, a.t / a.s, logf(a.s));  // (c cancels)
        if (p.stats) {
            p.stats[2 * (int64_t)r] = m;
            p.stats[2 * (int64_t)r + 1] = ls;
        }
    }
    if (TOP && lane < p.top) {
        p.top_token[(int64_t)r * p.top + lane] = score_key_token(list.key);
        p.top_logprob[(int64_t)r * p.top + lane] = list.key ? score_key_value(list.key) - m - ls : -INFINITY;
    }
}

// Few rows are split over a cluster while a CTA would still hold more than 512 vectors and the CTAs fit the SMs at once (rows that
// fill the SMs lose by it: 2,048 x 151,936 96 us in one CTA each, 102 in two, 163 in eight).  With twice the CTAs that fit, in bf16: 152 x 151,936
// 15.7 us for 12.1, 304 21.3 for 18.8, 608 33.8 for 29.4, with 8 alternatives 29.5, 37.7 and 52.7 for 17.5, 24.1 and 43.1, 300 x 9,001 9.5 for
// 5.4; better there only just behind the line (160 x 151,936 12.5 for 13.5, 305 18.4 for 19.9, 305 x 60,001 9.8 for 13.5).  Many rows take a
// warp each up to 512 vectors, 4 warps up to 8,192 (8,192 x 8,192: 31 us, 43 with 8 warps; 4,096 x 50,304: 66, 72), 8 warps
// beyond (3,000 x 151,936: 131 us, 140 with 4).  The alternatives' bound wants the 256 threads.
// Where the last of the waves in which long rows end would leave more than half of the SMs' room empty, its rows are split over 2 or 4
// CTAs and start as the others end (2,048 x 151,936: 93 -> 89 us, 700 42 -> 36, 900 52 -> 44; 1,300, whose rows of padding leave
// no third wave, 57 -> 60; with 8 CTAs 95; with alternatives, whose bound costs each CTA its own, 114 -> 116, so not there).
template <int TYPE, bool TOP>
inline void launch_score(cudaStream_t s, int sms, ScoreParams p) {
    const int vectors = p.V / (TYPE == SARA_FP32 ? 4 : 8), wave = score_sm_ctas(TYPE, TOP, 8) * sms;
    p.ctas = 1;
    while (p.ctas < kScoreMaxCtas && vectors > 512 * p.ctas && (int64_t)p.R * 2 * p.ctas <= wave) p.ctas *= 2;
    if (p.ctas == 1 && vectors <= (TOP ? kScoreTopWarpVectors : kScoreWarpVectors)) {
        score_kernel<TYPE, TOP, 1><<<((unsigned)p.R + 7) / 8, 256, 0, s>>>(p);
        CK(cudaGetLastError());
        return;
    }
    if constexpr (!TOP) {
        if (p.ctas == 1 && vectors <= 8192) {
            score_kernel<TYPE, false, 4><<<(unsigned)p.R, 128, 0, s>>>(p);
            CK(cudaGetLastError());
            return;
        }
        const int last = p.R % wave;
        if (p.ctas == 1 && vectors > 8192 && p.R > wave && last > 0 && 2 * last <= wave) {
            p.turn = 1;
            p.R -= last;
            launch_cluster(s, false, dim3((unsigned)p.R), dim3(256), 0, 1, score_kernel<TYPE, false, 8>, p);
            const int64_t r = p.R;
            p.z = static_cast<const uint8_t *>(p.z) + r * p.stride * RowVectors<TYPE>::kSize;
            p.tokens += p.tokens ? r : 0;
            p.logprob += p.logprob ? r : 0;
            p.entropy += p.entropy ? r : 0;
            p.stats += p.stats ? 2 * r : 0;
            p.turn = 2;
            p.R = last;
            p.ctas = last * 4 <= wave ? 4 : 2;
            launch_cluster(s, true, dim3((unsigned)p.R * p.ctas), dim3(256), 0, (unsigned)p.ctas, score_kernel<TYPE, false, 8>, p);
            return;
        }
    }
    launch_cluster(s, false, dim3((unsigned)p.R * p.ctas), dim3(256), 0, (unsigned)p.ctas, score_kernel<TYPE, TOP, 8>, p);
}

// ------------------------------------------------------------------------------- gradient
struct ScoreGradParams {
    const void *z;
    int64_t stride;
    int R, V;
    const int32_t *tokens;
    const float *stats, *entropy, *glp, *gent;
    void *out;
    int64_t out_stride;
    int segs;       // of a row
    int64_t warps;  // R * segs
};
constexpr int kGradVectors = 4;  // a lane

template <int TYPE>
__device__ __forceinline__ uint32_t pack_grad(float a, float b) {  // both to the nearest, one conversion
    uint32_t r;
    if constexpr (TYPE == SARA_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

// What a row's gradients share: with R = (max + log S) log2(e) as rounded and c what the roundings added,
//   y = z log2(e) - R,  p = 2^y 2^c,  dz = -2^y (a y + b) with a = 2^c g' ln 2 and b = 2^c (g + g' (entropy + c ln 2))
// A subnormal p may meet a factor that makes a normal product.  fp32 takes the full exponential for it; bf16, whose 8 bits can spare
// the last of y's, has y 32 higher and the factor 2^-32 lower; fp16 has no room for such products.
template <int TYPE>
struct GradRow {
    static constexpr float kLift = TYPE == SARA_BF16 ? 32.f : 0.f;
    float r, a, b;
    uint32_t least;  // a logit below every one that counts: those of -inf are raised to it
    bool plain;      // else the logits are taken one by one
    __device__ __forceinline__ GradRow(float m, float ls, float g, float gh, float H) {
        plain = fabsf(m) < 1e6f && (TYPE != SARA_FP16 || m > -6e4f);
        const float p1 = m * kLog2e, p2 = ls * kLog2e, sum = p1 + p2;
        const float v = sum - p1;  // (the sum's own rounding, and the products')
        float c = -(((p1 - (sum - v)) + (p2 - v)) + (fmaf(m, kLog2e, -p1) + fmaf(ls, kLog2e, -p2)));
        r = sum - kLift;
        const float w = r - sum;  // (and the lift's)
        c -= (sum - (r - w)) + (-kLift - w);
        const float k = exp2_approx(c);
        a = k * gh * kLn2;
        b = k * fmaf(gh, fmaf(c, kLn2, H), g);
        if constexpr (kLift > 0.f) {
            b = fmaf(-kLift, a, b) * 2.3283064e-10f;  // 2^-32
            a *= 2.3283064e-10f;
        }
        const float low = m - 1000.f - fabsf(m) * 0.015625f;
        least = TYPE == SARA_FP32 ? __float_as_uint(low) : TYPE == SARA_BF16 ? f32_to_bf16(low) * 0x10001u : f32_to_f16_sat(low) * 0x10001u;
    }
};

// One warp per segment of 32 x 4 vectors of a row.  A thread reads what it writes before it writes it, so the gradient
// may take the logits' place.
template <int TYPE>
__global__ void __launch_bounds__(256) score_grad_kernel(ScoreGradParams p) {
    using Row = RowVectors<TYPE>;
    constexpr int E = Row::E;
    const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (w >= p.warps) return;
    const int r = (int)(w / p.segs), seg = (int)(w - (int64_t)r * p.segs), lane = threadIdx.x & 31;
    const Row row(p.z, r, p.stride, p.V);
    const int nv = row.vectors(), from = seg * (32 * kGradVectors), k0 = from + lane;
    const int tok = p.tokens ? p.tokens[r] : 0;
    uint8_t *out = static_cast<uint8_t *>(p.out) + ((int64_t)r * p.out_stride - row.off) * Row::kSize;  // of vector 0
    const bool vec = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
    const bool inside = from >= row.whole_from() && from + 32 * kGradVectors <= row.whole_to();  // whole vectors alone
    uint4 x[kGradVectors];
    if (tok >= 0) {
        if (inside) {
            const uint4 *q = reinterpret_cast<const uint4 *>(row.base) + k0;
#pragma unroll
            for (int u = 0; u < kGradVectors; ++u) x[u] = q[32 * u];
        } else {
#pragma unroll
            for (int u = 0; u < kGradVectors; ++u)
                if (k0 + 32 * u < nv) x[u] = row.load(k0 + 32 * u);
        }
    }
    const float m = p.stats[2 * (int64_t)r], ls = p.stats[2 * (int64_t)r + 1];
    const float g = p.glp ? p.glp[r] : 0.f, gh = p.gent ? p.gent[r] : 0.f, H = p.gent ? p.entropy[r] : 0.f;
    const bool zero = tok < 0 || (m == -INFINITY && ls == 0.f && tok < p.V), wrong = tok >= p.V;
    const GradRow<TYPE> c(m, ls, g, gh, H);
    const uint64_t l2 = pack_f32x2(kLog2e, kLog2e), r2 = pack_f32x2(-c.r, -c.r), a2 = pack_f32x2(-c.a, -c.a), b2 = pack_f32x2(-c.b, -c.b);
#pragma unroll
    for (int u = 0; u < kGradVectors; ++u) {
        const int k = k0 + 32 * u;
        if (!inside && k >= nv) continue;
        float y[E];
        if (zero || wrong) {
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = zero ? 0.f : __int_as_float(0x7fc00000);
        } else {
            if (c.plain) {
                unpack_vector<TYPE>(raise_vector<TYPE>(x[u], c.least), y);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const uint64_t y2 = fma_f32x2(pack_f32x2(y[e], y[e + 1]), l2, r2);
                    const float2 t = unpack_f32x2(y2), f = unpack_f32x2(fma_f32x2(y2, a2, b2));
                    y[e] = (TYPE == SARA_FP32 ? exp2_full(t.x) : exp2_approx(t.x)) * f.x;
                    y[e + 1] = (TYPE == SARA_FP32 ? exp2_full(t.y) : exp2_approx(t.y)) * f.y;
                }
            } else {
                unpack_vector<TYPE>(x[u], y);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float lp = (y[e] - m) - ls, q = exp2_full(lp * kLog2e);
                    y[e] = -q * fmaf(gh, fmaxf(lp, -1000.f) + H, g);  // (a logit of -inf has q = 0)
                }
            }
            const uint32_t at = (uint32_t)tok - row.first(k);
            if (at < (uint32_t)E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at == (uint32_t)e) y[e] += g;
            }
        }
        uint8_t *o = out + (int64_t)k * 16;
        if (vec && (inside || row.whole(k))) {
            if constexpr (TYPE == SARA_FP32)
                *reinterpret_cast<float4 *>(o) = make_float4(y[0], y[1], y[2], y[3]);
            else
                *reinterpret_cast<uint4 *>(o) = make_uint4(pack_grad<TYPE>(y[0], y[1]), pack_grad<TYPE>(y[2], y[3]),
                                                          pack_grad<TYPE>(y[4], y[5]), pack_grad<TYPE>(y[6], y[7]));
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (row.first(k) + e >= row.V) continue;
                if constexpr (TYPE == SARA_FP32) reinterpret_cast<float *>(o)[e] = y[e];
                else reinterpret_cast<uint16_t *>(o)[e] = (uint16_t)pack_grad<TYPE>(y[e], 0.f);
            }
        }
    }
}

template <int TYPE>
inline void launch_score_grad(cudaStream_t s, ScoreGradParams p) {
    constexpr int E = RowVectors<TYPE>::E, kSeg = 32 * kGradVectors;
    const int64_t vectors = ((int64_t)p.V + 2 * E - 2) / E;  // the most that a row's place can make of it
    p.segs = (int)((vectors + kSeg - 1) / kSeg);
    p.warps = (int64_t)p.R * p.segs;
    const int64_t ctas = (p.warps + 7) / 8;
    if (ctas > INT32_MAX) throw SaraError(SARA_EINVAL, "too many logits");
    score_grad_kernel<TYPE><<<(unsigned)ctas, 256, 0, s>>>(p);
    CK(cudaGetLastError());
}

}  // namespace sara
