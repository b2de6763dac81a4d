// Decode attention over the 8-bit paged KV cache: one query row per sequence,
//     out[i, h] = softmax(q[i, h] . K[first_i .. ctx_i)^T / sqrt(hd)) V[first_i .. ctx_i)
// Bound by reading the codes once (2 hd bytes a position and KV head), so every byte goes from memory to registers in
// the order in which the warp-level MMAs want it, 16 bytes a lane, and becomes fp16 there, which both
// formats fit exactly; a warp takes 16 positions of each page of 128.
//   - Scores: A = K (rows: positions), B = q^T (columns: the group's query heads, at most 8).  Lane (g, t) loads
//     16 consecutive dims of positions g and g + 8; which dims meet in a k-step does not matter as long as q is laid out
//     alike.  bf16 queries enter as fp16 after a power of two has brought the row's largest to 2^14.
//   - Output: A = V^T (rows: dims, lane (g, t) holds hd / 8 dims of 4 positions, byte permutes pair the positions),
//     B = P^T, the scores' own registers transposed by movmatrix.  P enters as an fp16 pair, hi + lo: 22 bits, and
//     multiples of 2^-31 of the maximum (probabilities are scaled by 2^7).
//   - A scale covers both of a warp's rows of 8 positions: K's is a factor of the scores, V's of P, relative to the largest so far
//     (vref), so that neither costs a multiplication per code.
// Online softmax in fp32 per warp; the maximum is re-based only when a probability would pass 2^8, so most pages
// skip the column maximum and the rescale.  Work: the (row, KV head, page) triples in one list, cut into equal
// shares, one per CTA; a (row, KV head) that several CTAs share is joined by the last of them to finish, in the list's order.
#pragma once
#include "kv8.cuh"

namespace sara {

constexpr int kAttnKv8Warps = 8;
constexpr int kAttnKv8Threads = 32 * kAttnKv8Warps;
constexpr int kAttnKv8MaxCtas = 512;

struct AttnKv8Params {
    Kv8Cache c;
    const uint16_t *q;
    int64_t q_stride;
    const int32_t *ctx, *first;
    uint16_t *out;
    float *lse;
    int32_t *status;
    int *count;   // [n][KVH] finished shares of a (row, KV head) that several CTAs work on; left zero
    float *part;  // [CTA][2][8 (hd + 2)] their states: max and sum of 8 heads, then their outputs
    int n, H, type;
    float scale_log2;  // log2(e) / sqrt(hd)
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Four codes as two fp16 pairs
template <int FMT>
__device__ __forceinline__ void decode4_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (FMT == SARA_KV8_E4M3) {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
            : "=r"(lo), "=r"(hi)
            : "r"(w));
    } else {
        const uint32_t u = w ^ 0x80808080u;  // (see decode2_half)
        const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 k = __floats2half2_rn(1152.f, 1152.f);
        const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&a), k), y = __hsub2(*reinterpret_cast<const __half2 *>(&b), k);
        lo = *reinterpret_cast<const uint32_t *>(&x);
        hi = *reinterpret_cast<const uint32_t *>(&y);
    }
}
template <int WORDS>
__device__ __forceinline__ void load_codes(const uint8_t *p, uint32_t *r) {
    if constexpr (WORDS == 4)
        asm("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
    else if constexpr (WORDS == 2)
        asm("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
    else
        asm("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(r[0]) : "l"(p));
}

// A row's positions, and the pages that hold them
struct AttnKv8Row {
    int first, ctx, page0, pages;
    bool bad;
};
__device__ __forceinline__ AttnKv8Row attn_kv8_row(const AttnKv8Params &p, int i) {
    AttnKv8Row r;
    r.ctx = __ldg(p.ctx + i);
    r.first = p.first ? min(__ldg(p.first + i), r.ctx) : 0;  // (past the end: no position)
    r.bad = r.ctx < 0 || r.first < 0 || r.ctx > (int64_t)p.c.max_blocks * kKv8Page;
    r.page0 = r.first / kKv8Page;
    r.pages = r.bad || r.ctx <= r.first ? 0 : (r.ctx - 1) / kKv8Page - r.page0 + 1;
    return r;
}

// Inclusive prefix of v over the CTA's threads, and the total
__device__ __forceinline__ int64_t attn_kv8_scan(int64_t v, int64_t &total, int64_t *room) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += y;
    }
    __syncthreads();
    if (lane == 31) room[warp] = v;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kAttnKv8Warps; ++w) {
        if (w < warp) before += room[w];
        total += room[w];
    }
    return before + v;
}

template <int HD, int FMT>
__global__ void __launch_bounds__(kAttnKv8Threads, 2) attn_kv8_kernel(AttnKv8Params p) {
    constexpr int KW = HD / 16, VW = HD / 32, NT = HD / 16;  // words a lane of a key row, of a value row; output tiles
    constexpr int KL = KW < 4 ? KW : 4;                      // words a load
    constexpr int PITCH = HD + 4;                            // (conflict-free 8-byte stores)
    constexpr float kShift = 7.f;
    __shared__ __align__(16) float s_o[kAttnKv8Warps][8][PITCH];
    __shared__ float s_m[kAttnKv8Warps][8], s_l[kAttnKv8Warps][8], s_M[8], s_L[8];
    __shared__ int64_t s_room[kAttnKv8Warps], s_base;
    __shared__ int s_row, s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int KVH = p.c.KVH, G = p.H / KVH;
    const float nan = __int_as_float(0x7fc00000);

    // rows without a position, and wrong ones
    for (int i = blockIdx.x; i < p.n; i += gridDim.x) {
        const AttnKv8Row r = attn_kv8_row(p, i);
        if (r.pages) continue;
        const float y = r.bad ? nan : 0.f;
        const uint32_t y2 = p.type == SARA_BF16 ? pack2<SARA_BF16>(y, y) : pack2<SARA_FP16>(y, y);
        uint32_t *o = reinterpret_cast<uint32_t *>(p.out + (int64_t)i * p.H * HD);
        for (int e = tid; e < p.H * HD / 2; e += kAttnKv8Threads) o[e] = y2;
        if (p.lse)
            for (int e = tid; e < p.H; e += kAttnKv8Threads) p.lse[(int64_t)i * p.H + e] = r.bad ? nan : -INFINITY;
        if (r.bad && tid == 0) kv8_report(p.status);
    }

    // this CTA's share of the list, and the row in which it begins
    int64_t total = 0;
    for (int b = 0; b < p.n; b += kAttnKv8Threads) {
        int64_t sum;
        attn_kv8_scan(b + tid < p.n ? attn_kv8_row(p, b + tid).pages : 0, sum, s_room);
        total += sum;
    }
    total *= KVH;
    const int64_t ctas = min((int64_t)gridDim.x, total);
    if (blockIdx.x >= ctas) return;
    const int64_t lo = blockIdx.x * total / ctas, hi = (blockIdx.x + 1) * total / ctas;
    for (int64_t b = 0, before = 0; b < p.n; b += kAttnKv8Threads) {
        int64_t sum;
        const int pages = b + tid < p.n ? attn_kv8_row(p, (int)b + tid).pages : 0;
        const int64_t end = (before + attn_kv8_scan(pages, sum, s_room)) * KVH;
        if (lo < end && lo >= end - (int64_t)pages * KVH) {
            s_row = (int)b + tid;
            s_base = end - (int64_t)pages * KVH;
        }
        before += sum;
        if (before * KVH > lo) break;
    }
    __syncthreads();
    int row = s_row;
    int64_t base = s_base;
    AttnKv8Row r = attn_kv8_row(p, row);

    for (int64_t at = lo; at < hi;) {
        const int h = (int)((at - base) / r.pages), a = (int)((at - base) % r.pages);
        const int64_t unit = base + (int64_t)h * r.pages;
        const int b = (int)min((int64_t)r.pages, hi - unit);  // pages a .. b of the row's, for KV head h

        // queries: head g of the group, the dims of this lane's key words
        uint32_t qb[KW][2];
        float mul0, mul1;  // from MMA sums to base-2 exponents, heads 2 t and 2 t + 1
        {
            const uint16_t *qp = p.q + row * p.q_stride + (int64_t)(h * G + min(g, G - 1)) * HD;
#pragma unroll
            for (int s = 0; s < KW; ++s) {
                const int d = KW == 8 ? 64 * (s / 4) + 16 * t + 4 * (s % 4) : HD / 4 * t + 4 * s;
                const uint2 x = __ldg(reinterpret_cast<const uint2 *>(qp + d));
                qb[s][0] = g < G ? x.x : 0;
                qb[s][1] = g < G ? x.y : 0;
            }
            float mul = p.scale_log2;
            if (p.type == SARA_BF16) {
                uint32_t top = 0;
#pragma unroll
                for (int s = 0; s < KW; ++s)
                    top = __vmaxu2(top, __vmaxu2(qb[s][0] & 0x7fff7fffu, qb[s][1] & 0x7fff7fffu));
                top = max(top & 0xffff, top >> 16);
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // 2^e: the largest magnitude's power of two becomes 2^14
                const int e = min(14 - ((int)(top >> 7) - 127), 126);
                const float f = pow2f(max(e, -113));
#pragma unroll
                for (int s = 0; s < KW; ++s)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 x = unpack2<SARA_BF16>(qb[s][i]);
                        qb[s][i] = pack_half2(x.x * f, x.y * f);
                    }
                mul *= pow2f(-max(e, -113));
            }
            mul0 = __shfl_sync(0xffffffffu, mul, 8 * t);
            mul1 = __shfl_sync(0xffffffffu, mul, 8 * t + 4);
        }

        float m0 = -3.4028235e38f, m1 = m0, l0 = 0.f, l1 = 0.f, vref = 0.f, vinv = 0.f, o[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][e] = 0.f;

        // this warp's positions of page x: 128 x + 16 warp .. + 15; the row's first and last page may have none
        int pa = r.page0 + a, pb = r.page0 + b;
        if (pa * kKv8Page + 16 * warp + 16 <= r.first) ++pa;
        if ((pb - 1) * kKv8Page + 16 * warp >= r.ctx) --pb;
        const int32_t *tab = p.c.table + row * p.c.table_stride;
        int ids = 0;     // this lane's entry of the 32 table entries from idbase on
        int idbase = 0;
        bool wrong = false;
        auto block_of = [&](int x, int begin) -> int64_t {
            if (((x - begin) & 31) == 0) {
                idbase = x;
                ids = x + lane < pb ? __ldg(tab + x + lane) : 0;
                const bool out = ids < 0 || ids >= p.c.n_blocks;
                wrong = wrong || out;
                ids = out ? -1 : ids;
            }
            return __shfl_sync(0xffffffffu, ids, x - idbase);
        };
        auto slot_of = [&](int x, int e) {  // (masked positions stand for the nearest that is not: their probability is 0)
            const int pos = x * kKv8Page + 16 * warp + e;
            return min(max(pos, r.first), r.ctx - 1) & (kKv8Page - 1);
        };
        uint32_t kr[2][KW];
        float ks = 0.f;
        int64_t blk = 0;
        auto load_k = [&](int x, int64_t id) {
            const int64_t tile = kv8_tile(p.c, (int)max(id, (int64_t)0), 0, h);
            ks = id < 0 ? nan : __ldg(p.c.scales + tile * kKv8PageBlocks + (warp >> 1));
            const uint8_t *k = p.c.codes + tile * (kKv8Page * HD) + (KW == 8 ? 16 : HD / 4) * t;
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < KW / KL; ++i) load_codes<KL>(k + slot_of(x, g + 8 * e) * HD + 64 * i, &kr[e][4 * i]);
        };
        if (pa < pb) {
            blk = block_of(pa, pa);
            load_k(pa, blk);
        }
#pragma unroll 1
        for (int x = pa; x < pb; ++x) {
            // values of this page, keys of the next
            uint32_t vr[4][VW];
            const int64_t vtile = kv8_tile(p.c, (int)max(blk, (int64_t)0), 1, h);
            const float vs = __ldg(p.c.scales + vtile * kKv8PageBlocks + (warp >> 1));
            const uint8_t *v = p.c.codes + vtile * (kKv8Page * HD) + HD / 8 * g;
#pragma unroll
            for (int e = 0; e < 4; ++e) load_codes<VW>(v + slot_of(x, 2 * t + (e & 1) + 8 * (e >> 1)) * HD, vr[e]);
            uint32_t kc[2][KW];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int s = 0; s < KW; ++s) kc[e][s] = kr[e][s];
            const float kscale = ks;
            if (x + 1 < pb) {
                blk = block_of(x + 1, pa);
                load_k(x + 1, blk);
            }
            float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                uint32_t f[4];
                decode4_half<FMT>(kc[0][i], f[0], f[2]);
                decode4_half<FMT>(kc[1][i], f[1], f[3]);
                mma_f16_16816(i & 1 ? s2 : s, f, qb[i][0], qb[i][1]);
            }
            // s[0], s[1]: position g, heads 2 t and 2 t + 1; s[2], s[3]: position g + 8
            const float f0 = kscale * mul0, f1 = kscale * mul1;
            s[0] = (s[0] + s2[0]) * f0;
            s[1] = (s[1] + s2[1]) * f1;
            s[2] = (s[2] + s2[2]) * f0;
            s[3] = (s[3] + s2[3]) * f1;
            const int p0 = x * kKv8Page + 16 * warp;
            if (p0 < r.first || p0 + 16 > r.ctx) {
                if (p0 + g < r.first || p0 + g >= r.ctx) s[0] = s[1] = -INFINITY;
                if (p0 + g + 8 < r.first || p0 + g + 8 >= r.ctx) s[2] = s[3] = -INFINITY;
            }
            if (__any_sync(0xffffffffu, fmaxf(s[0], s[2]) > m0 + 8.f || fmaxf(s[1], s[3]) > m1 + 8.f)) {
                float n0 = fmaxf(m0, fmaxf(s[0], s[2])), n1 = fmaxf(m1, fmaxf(s[1], s[3]));
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, d));
                    n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, d));
                }
                const float a0 = ex2(m0 - n0), a1 = ex2(m1 - n1);
                m0 = n0;
                m1 = n1;
                l0 *= a0;
                l1 *= a1;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    o[j][0] *= a0;
                    o[j][1] *= a1;
                    o[j][2] *= a0;
                    o[j][3] *= a1;
                }
            }
            const float c0 = m0 - kShift, c1 = m1 - kShift;
            float w0 = ex2(s[0] - c0), w1 = ex2(s[1] - c1), w2 = ex2(s[2] - c0), w3 = ex2(s[3] - c1);
            l0 += w0 + w2;
            l1 += w1 + w3;
            if (!(vs <= vref)) {  // the largest scale so far (or NaN)
                const float inv = 1.f / vs, f = vref * inv;
                vref = vs;
                vinv = inv;
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[j][e] *= f;
            }
            const float vf = vs * vinv;
            w0 *= vf;
            w1 *= vf;
            w2 *= vf;
            w3 *= vf;
            uint32_t ph[2] = {pack_half2(w0, w1), pack_half2(w2, w3)}, pl[2];
            const float2 h0 = __half22float2(*reinterpret_cast<const __half2 *>(&ph[0]));
            const float2 h1 = __half22float2(*reinterpret_cast<const __half2 *>(&ph[1]));
            pl[0] = movmatrix_trans(pack_half2(w0 - h0.x, w1 - h0.y));
            pl[1] = movmatrix_trans(pack_half2(w2 - h1.x, w3 - h1.y));
            ph[0] = movmatrix_trans(ph[0]);
            ph[1] = movmatrix_trans(ph[1]);
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                uint32_t f0[4], f1[4];  // dims 4 i, 4 i + 1 and 4 i + 2, 4 i + 3 of the lane's
                decode4_half<FMT>(__byte_perm(vr[0][i], vr[1][i], 0x5140), f0[0], f0[1]);
                decode4_half<FMT>(__byte_perm(vr[2][i], vr[3][i], 0x5140), f0[2], f0[3]);
                decode4_half<FMT>(__byte_perm(vr[0][i], vr[1][i], 0x7362), f1[0], f1[1]);
                decode4_half<FMT>(__byte_perm(vr[2][i], vr[3][i], 0x7362), f1[2], f1[3]);
                mma_f16_16816(o[2 * i], f0, ph[0], ph[1]);
                mma_f16_16816(o[2 * i + 1], f1, ph[0], ph[1]);
                mma_f16_16816(o[2 * i], f0, pl[0], pl[1]);
                mma_f16_16816(o[2 * i + 1], f1, pl[0], pl[1]);
            }
        }
        if (wrong) kv8_report(p.status);

        // the warps' states: o[j][e], o[j][2 + e]: head 2 t + e, dims hd / 8 g + 2 j and + 1, at place 16 j + 2 g
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        if (g == 0) {
            s_m[warp][2 * t] = m0;
            s_m[warp][2 * t + 1] = m1;
            s_l[warp][2 * t] = l0;
            s_l[warp][2 * t + 1] = l1;
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            *reinterpret_cast<float2 *>(&s_o[warp][2 * t][16 * j + 2 * g]) = make_float2(o[j][0] * vref, o[j][2] * vref);
            *reinterpret_cast<float2 *>(&s_o[warp][2 * t + 1][16 * j + 2 * g]) = make_float2(o[j][1] * vref, o[j][3] * vref);
        }
        __syncthreads();
        if (tid < 8) {
            float M = s_m[0][tid], L = 0.f;
#pragma unroll
            for (int w = 1; w < kAttnKv8Warps; ++w) M = fmaxf(M, s_m[w][tid]);
#pragma unroll
            for (int w = 0; w < kAttnKv8Warps; ++w) {
                const float f = ex2(s_m[w][tid] - M);
                L += f * s_l[w][tid];
                s_m[w][tid] = f;
            }
            s_M[tid] = M;
            s_L[tid] = L;
        }
        __syncthreads();
        const bool whole = a == 0 && b == r.pages;
        float *mine = p.part + ((int64_t)blockIdx.x * 2 + (a == 0)) * (8 * (HD + 2));
        for (int e = tid; e < G * HD / 2; e += kAttnKv8Threads) {
            const int hh = e / (HD / 2), i = e % (HD / 2) * 2;
            float y0 = 0.f, y1 = 0.f;
#pragma unroll
            for (int w = 0; w < kAttnKv8Warps; ++w) {
                const float2 x = *reinterpret_cast<const float2 *>(&s_o[w][hh][i]);
                const float f = s_m[w][hh];
                y0 += f * x.x;
                y1 += f * x.y;
            }
            if (whole) {
                const int dim = HD / 8 * (i % 16 / 2) + i / 16 * 2;
                y0 /= s_L[hh];
                y1 /= s_L[hh];
                *reinterpret_cast<uint32_t *>(p.out + ((int64_t)row * p.H + h * G + hh) * HD + dim) =
                    p.type == SARA_BF16 ? pack2<SARA_BF16>(y0, y1) : pack2<SARA_FP16>(y0, y1);
            } else {
                *reinterpret_cast<float2 *>(mine + 16 + hh * HD + i) = make_float2(y0, y1);
            }
        }
        if (tid < G) {
            if (!whole) {
                mine[tid] = s_M[tid];
                mine[8 + tid] = s_L[tid];
            } else if (p.lse) {
                p.lse[(int64_t)row * p.H + h * G + tid] = (s_M[tid] - kShift + log2f(s_L[tid])) * 0.69314718f;
            }
        }
        if (!whole) {
            // CTA of entry x: the largest c with c total / ctas <= x
            const int64_t c0 = ((unit + 1) * ctas - 1) / total, c1 = ((unit + r.pages) * ctas - 1) / total;
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                int *n = p.count + (int64_t)row * KVH + h;
                s_last = atomicAdd(n, 1) == (int)(c1 - c0);
                if (s_last) *n = 0;
            }
            __syncthreads();
            if (s_last) {
                __threadfence();
                auto state = [&](int64_t c) { return p.part + (c * 2 + (c == c0)) * (8 * (HD + 2)); };
                for (int e = tid; e < G * HD / 2; e += kAttnKv8Threads) {
                    const int hh = e / (HD / 2), i = e % (HD / 2) * 2;
                    float M = -3.4028235e38f, L = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll 4
                    for (int64_t c = c0; c <= c1; ++c) {
                        const float *x = state(c);
                        const float mc = __ldcg(x + hh), lc = __ldcg(x + 8 + hh);
                        const float2 yc = __ldcg(reinterpret_cast<const float2 *>(x + 16 + hh * HD + i));
                        const float N = fmaxf(M, mc), fa = ex2(M - N), fb = ex2(mc - N);
                        M = N;
                        L = L * fa + lc * fb;
                        y0 = y0 * fa + yc.x * fb;
                        y1 = y1 * fa + yc.y * fb;
                    }
                    const int dim = HD / 8 * (i % 16 / 2) + i / 16 * 2;
                    y0 /= L;
                    y1 /= L;
                    *reinterpret_cast<uint32_t *>(p.out + ((int64_t)row * p.H + h * G + hh) * HD + dim) =
                        p.type == SARA_BF16 ? pack2<SARA_BF16>(y0, y1) : pack2<SARA_FP16>(y0, y1);
                    if (p.lse && i == 0) p.lse[(int64_t)row * p.H + h * G + hh] = (M - kShift + log2f(L)) * 0.69314718f;
                }
            }
        }
        __syncthreads();  // (shared memory is the next share's)
        at = unit + b;
        if (at < hi && h == KVH - 1) {
            base += (int64_t)KVH * r.pages;
            do r = attn_kv8_row(p, ++row);
            while (r.pages == 0);
        }
    }
}

inline size_t attn_kv8_count_bytes(int n, int KVH) { return ((size_t)n * KVH * sizeof(int) + 255) / 256 * 256; }
inline size_t attn_kv8_workspace(int n, int KVH, int hd) {
    return attn_kv8_count_bytes(n, KVH) + (size_t)kAttnKv8MaxCtas * 2 * 8 * (hd + 2) * sizeof(float);
}

}  // namespace sara
