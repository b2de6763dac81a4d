// Log-probabilities of given tokens under softmax(scale H W^T), H [R][d] hidden states, W [V][d] the vocabulary's weights, with the
// entropy, and the gradient of both with respect to H and W.  No logits are kept:
//   forward:  the logits of a tile of rows and tokens are the accumulator of tensor-core products; its epilogue leaves a row's maximum
//             a, sum 2^y and sum 2^y y with y = (acc - a) scale log2(e), which a second kernel joins over the tiles
//   gradient: the vocabulary goes by in pieces.  A piece's logits are made again, its dZ = g (1[v = token] - p) - g' p (log p + H),
//             [R][piece], is stored in the operands' type, and feeds both products, dH += dZ W and dW = dZ^T H.
// Bound by the tensor cores from some 300 rows on, by reading W below.
//
// One persistent kernel does all the products (D = A B^T, fp32 in tensor memory): 256 columns, 128 rows a CTA, K in chunks of 64.
// With more than 128 rows two CTAs (a cluster) share a tile of 256 x 256, each bringing half of A's rows and half of B's: 64 bytes
// a cycle and SM from L2 for 96 alone.  Operands come by TMA with 128-byte swizzling, K-major or M/N-major as they lie in memory, so
// nothing is ever transposed: dZ is K-major for dH and M-major for dW, W is K-major for the logits and N-major for dH.
// Rows of padding (token < 0) are left out: the live rows are gathered first, so that they cost nothing and their contents,
// whatever they are, reach nothing.
//
// The tensor core cuts its sums off: about half a step of fp32 each 16 products, all towards zero.  A logit's products are therefore
// summed in parts, which the epilogue adds.
// dZ enters the products in 16 bits.  Its largest element by far is mostly the token's own: what that one's rounding left off is
// kept (delta) and added to both gradients in fp32.
//
// Warp roles (320 threads): warp 0 producer, warp 1 MMA issuer and tensor-memory owner, warps 2..9 epilogue (warp w: the rows of
// tensor-memory lanes 32 (w % 4) ..): of the scores every tile, 128 columns a thread, which are in registers before the accumulator is given
// back; of the others warps 2..5 and 6..9 alternate tiles, one of the two accumulators each.
#pragma once
#include <type_traits>

#include "device_common.cuh"
#include "host_util.h"
#include "kv8.cuh"
#include "logprob.cuh"

namespace sara {

constexpr int kLinThreads = 320;
constexpr int kLinRows = 128, kLinCols = 256, kLinK = 64;  // of a CTA's tile; of a chunk
constexpr int kLinMaxSplits = 32;
constexpr int kLinWorkers = 152;  // SMs that a plan counts on (on a GPU with others it is as right, if less even)

// What the kernels of a call share, at the start of the workspace
struct LinHeader {
    int err;   // bits of device_common.cuh; left zero
    int live;  // rows that are not padding
    int exp;   // the least power of two of a row's dZ (0 in bf16)
    int pad[61];
};

__host__ __device__ constexpr int lin_stage_bytes(int ctas) { return (kLinRows + kLinCols / ctas) * kLinK * 2; }
__host__ __device__ constexpr int lin_stages(int ctas) { return ctas == 2 ? 6 : 4; }
__host__ __device__ constexpr size_t lin_smem(int ctas) { return 1024 + (size_t)lin_stages(ctas) * lin_stage_bytes(ctas); }

enum LinMode : int {
    LIN_SCORE = 0,  // tiles of logits -> partial sums
    LIN_DZ = 1,     // tiles of logits -> dZ of a piece
    LIN_GRAD = 2,   // dZ of a piece -> dH's sums, dW
};

struct LinParams {
    LinHeader *head;
    int R, d, V;
    const int32_t *tokens;
    const int *src;    // compact row -> row, or null: the same
    const int *kexp;   // [row] power of two that dZ's row is raised by
    float scale;
    // LIN_SCORE
    float *part;       // [3][token tile][rows_cap]: a, s, t
    float *ztok;       // [rows_cap]
    int rows_cap, token_tiles;
    // LIN_DZ
    const float *stats, *entropy, *glp, *gent;
    uint16_t *dz;      // [rows_cap][piece]
    int piece, v0, cols;  // columns of dZ; the piece's first token and tokens
    float *delta;      // [rows_cap]: what rounding took from dZ at the row's token
    // LIN_GRAD
    const int *tokc;   // [rows_cap]: the compact rows' tokens
    const uint16_t *low;  // [rows_cap][d]: the rows that dW's product has
    float *acc;        // [split][rows_cap][d]
    int splits, first; // first: the first piece
    uint16_t *dw;      // or null
    int64_t dw_stride;
    bool dh;
};

// Chunks of a part of a logit's sum: with two CTAs a tile's epilogue has no time for more parts
__host__ __device__ constexpr int lin_part(int ctas) { return ctas == 2 ? 8 : 1; }
constexpr int kLinHits = 256;  // rows of a quarter whose tokens are in a tile of dW and whose delta is added there (the first ones)

struct LinSmem {
    uint64_t full[6], empty[6], acc_full[2], acc_empty[2], drain;
    uint32_t tmem_base;
    int abort, stop[2];                  // stop: the epilogue's, for two tiles in turn
};
struct LinScoreSmem {
    float sums[2][3][kLinRows];          // of the second half's columns, for two tiles in turn
};
struct LinGradSmem {
    int found[2][4];                     // of each epilogue warp's quarter of the rows
    int2 hit[2][4][kLinHits];            // place in the tile, row
};

// ------------------------------------------------------------------------------- PTX for a pair of CTAs
template <int CTAS>
__device__ __forceinline__ void lin_tmem_alloc(uint32_t *dst, uint32_t cols) {
    if constexpr (CTAS == 1) {
        tmem_alloc(dst, cols);
        tmem_relinquish();
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CTAS>
__device__ __forceinline__ void lin_tmem_free(uint32_t taddr, uint32_t cols) {
    if constexpr (CTAS == 1) tmem_dealloc(taddr, cols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
// A box to this CTA's shared memory; its bytes count at `bar` (a shared::cluster address: of the pair's first CTA)
template <int CTAS>
__device__ __forceinline__ void lin_load(void *dst, const CUtensorMap *tm, uint32_t bar, int x, int y, uint64_t policy) {
    if constexpr (CTAS == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(
                smem_u32(dst)),
            "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(bar), "l"(policy)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(
                smem_u32(dst)),
            "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(bar), "l"(policy)
            : "memory");
}
template <int CTAS>
__device__ __forceinline__ void lin_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CTAS == 1)
        tc_mma_bf16(d, a, b, idesc, accumulate);
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}
// Arrive on `bar` (of both CTAs) when every MMA issued so far has completed
template <int CTAS>
__device__ __forceinline__ void lin_commit(uint64_t *bar) {
    if constexpr (CTAS == 1)
        tc_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                     "h"((uint16_t)3)
                     : "memory");
}
// The same on this CTA's alone
template <int CTAS>
__device__ __forceinline__ void lin_commit_here(uint64_t *bar) {
    if constexpr (CTAS == 1) tc_commit(bar);
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major: 8 rows of 64 elements after sbo bytes.  M/N-major: lines of 64 rows or
// columns at one k, 8 k after sbo bytes, the next 64 rows after lbo bytes.
__device__ __forceinline__ uint64_t sdesc_sw128(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// ------------------------------------------------------------------------------- work
// A tile: rows m0 .. of A, rows n0 .. of B (n of them), chunks k0 .. k1
struct LinJob {
    int m0, n0, n, k0, k1;
    int kind;   // LIN_GRAD: 0 dH, 1 dW
    int split;  // dH
};

// The jobs of a CTA (or pair) `w` of `W`, by number.  Logits: rows fastest, so that the CTAs at work share tokens.
// LIN_GRAD: dH's jobs are long, so the workers that have one more of them get fewer of dW's.
template <int MODE, int CTAS>
struct LinWork {
    static constexpr int TM = kLinRows * CTAS;
    int w, W, mt, nt, count;
    int64_t tiles;
    // LIN_GRAD
    int kc, kr, splits, jh, extra, light;  // chunks of a piece, of the rows; dH's jobs; of dW's: those before the others join, this worker's
    int own_h, wide;                       // this worker's dH jobs; the workers with one less of them
    __device__ __forceinline__ LinWork(const LinParams &p, int live, int w_, int W_) : w(w_), W(W_) {
        mt = max((live + TM - 1) / TM, 1);
        if constexpr (MODE != LIN_GRAD) {
            nt = (p.cols + kLinCols - 1) / kLinCols;
            tiles = (int64_t)mt * nt;
            count = (int)(tiles > w ? (tiles - 1 - w) / W + 1 : 0);
        } else {
            nt = (p.d + kLinCols - 1) / kLinCols;
            kc = (p.cols + kLinK - 1) / kLinK;
            kr = max((live + kLinK - 1) / kLinK, 1);
            splits = min(p.splits, kc);
            jh = p.dh ? mt * nt * splits : 0;
            const int jw = p.dw ? (p.cols + TM - 1) / TM * nt : 0;
            const int rem = jh % W;
            wide = W - rem;
            own_h = jh / W + (w < rem);
            const int ratio = rem ? (kc / splits + kr - 1) / kr : 0;  // dW's jobs in the time of one of dH's
            int b = (int)(((int64_t)jw + (int64_t)rem * ratio + W - 1) / W), a = b - ratio;
            if (a < 0) {
                a = 0;
                b = (jw + wide - 1) / wide;
            }
            extra = b - a;  // of the workers with one dH job less
            light = a;
            tiles = jw;
            count = own_h + (w >= rem ? extra : 0) + light;
        }
    }
    // false: nothing (a number behind the last job)
    __device__ __forceinline__ bool job(const LinParams &p, int i, LinJob &j) const {
        if constexpr (MODE != LIN_GRAD) {
            const int64_t t = (int64_t)i * W + w;
            if (t >= tiles) return false;
            const int n = (int)(t / mt), m = (int)(t - (int64_t)n * mt);
            j = {m * TM, n * kLinCols, kLinCols, 0, (p.d + kLinK - 1) / kLinK, 0, 0};
            return true;
        } else {
            int n, m;
            if (i < own_h) {
                const int t = i * W + w;
                n = t % nt;
                m = t / nt % mt;
                const int s = t / nt / mt;
                j.kind = 0;
                j.split = s;
                j.k0 = (int)((int64_t)kc * s / splits);
                j.k1 = (int)((int64_t)kc * (s + 1) / splits);
            } else {
                const int rem = W - wide, before = w >= rem ? extra : 0, x = i - own_h;
                const int64_t t = x < before ? (int64_t)x * wide + (w - rem) : (int64_t)extra * wide + (int64_t)(x - before) * W + w;
                if (t >= tiles) return false;
                n = (int)(t % nt);
                m = (int)(t / nt);
                j.kind = 1;
                j.split = 0;
                j.k0 = 0;
                j.k1 = kr;
            }
            j.m0 = m * TM;
            j.n0 = n * kLinCols;
            j.n = min(kLinCols, (p.d - j.n0 + 64 * CTAS - 1) / (64 * CTAS) * (64 * CTAS));
            return true;
        }
    }
};

// ------------------------------------------------------------------------------- epilogues
// A row's maximum a and sums over some of its logits, s and t without one maximum's own terms (1 and 0), so that the logarithm of
// 1 + s keeps what is small beside the 1 of a row with one likely token
struct LinSums {
    float a = -3.4028235e38f, s = -1.f, t = 0.f;  // of none
    // (the bound keeps 0 times infinity out where the maxima are far apart)
    __device__ __forceinline__ void join(float b, float sb, float tb, float c) {
        const bool up = b > a;
        const float hi = up ? b : a, lo = up ? a : b, s0 = up ? sb : s, s1 = 1.f + (up ? s : sb), t0 = up ? tb : t, t1 = up ? t : tb;
        const float y = fmaxf((lo - hi) * c, -1e4f), f = exp2_approx(y);
        a = hi;
        s = fmaf(s1, f, s0);
        t = fmaf(fmaf(s1, y, t1), f, t0);
    }
};

// 32 columns of a lane, or their sum with v; the wait is part of the instruction, so that nothing uses the values before it
template <bool ADD>
__device__ __forceinline__ void lin_tmem_load(uint32_t taddr, float *v) {
    uint32_t r[32];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = ADD ? v[i] + __uint_as_float(r[i]) : __uint_as_float(r[i]);
}

template <int TYPE>
__device__ __forceinline__ float lin_float(uint16_t x) {
    return TYPE == SARA_BF16 ? bf16_to_f32(x) : f16_to_f32(x);
}
template <int TYPE>
__device__ __forceinline__ uint16_t lin_round(float x) {
    return TYPE == SARA_BF16 ? f32_to_bf16(x) : __half_as_ushort(__float2half_rn(x));
}

template <int MODE, int CTAS, int TYPE>
__global__ void __launch_bounds__(kLinThreads, 1)
lin_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmA2,
           const __grid_constant__ CUtensorMap tmB2, LinParams p) {
    constexpr int STAGES = lin_stages(CTAS), STAGE = lin_stage_bytes(CTAS), A_BYTES = kLinRows * kLinK * 2;
    constexpr int BN = kLinCols / CTAS, PART = lin_part(CTAS);  // a CTA's share of B's rows
    extern __shared__ uint8_t smem_raw[];
    __shared__ LinSmem S;
    __shared__ std::conditional_t<MODE == LIN_GRAD, LinGradSmem, LinScoreSmem> E;
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CTAS == 2 ? (int)cluster_rank() : 0;
    int *err = &p.head->err;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&S.full[s], 1);
            mbar_init(&S.empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&S.acc_full[a], 1);
            mbar_init(&S.acc_empty[a], (MODE == LIN_SCORE ? 8 : 4) * CTAS);
        }
        mbar_init(&S.drain, 1);
        S.abort = S.stop[0] = S.stop[1] = 0;
        fence_mbar_init();
    }
    if (warp == 1) lin_tmem_alloc<CTAS>(&S.tmem_base, 512);
    tc_fence_before();
    if constexpr (CTAS == 2) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = S.tmem_base;
    volatile int *ab = &S.abort;
    const int live = p.src ? p.head->live : p.R;
    const LinWork<MODE, CTAS> work(p, live, (int)blockIdx.x / CTAS, (int)gridDim.x / CTAS);

    if (warp == 0) {
        // ------------------------------------------------------------ producer
        const uint64_t keep = l2_policy_evict_last();
        uint64_t pass;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pass));
        int s = 0;
        uint32_t ph = 1, loads = 0;
        bool ok = true;
#pragma unroll 1
        for (int i = 0; i < work.count && ok; ++i) {
            LinJob j;
            if (!work.job(p, i, j)) break;
            const bool mn_a = MODE == LIN_GRAD && j.kind == 1, mn_b = MODE == LIN_GRAD;
            const int m = j.m0 + rank * kLinRows, bn = j.n / CTAS, n = j.n0 + rank * bn;
            const uint32_t bytes = (uint32_t)(A_BYTES + (mn_b ? bn : BN) * kLinK * 2) * CTAS;
#pragma unroll 1
            for (int k = j.k0; k < j.k1; ++k) {
                if (loads >= (uint32_t)STAGES) ok = __all_sync(0xffffffffu, mbar_wait(&S.empty[s], ph, err) && !*ab);
                if (!ok) break;
                if (elect_one()) {
                    uint8_t *a = ring + s * STAGE, *b = a + A_BYTES;
                    const uint32_t bar = CTAS == 2 ? cluster_addr(&S.full[s], 0) : smem_u32(&S.full[s]);
                    if (rank == 0) mbar_arrive_expect_tx(&S.full[s], bytes);
                    if (!mn_a) {
                        lin_load<CTAS>(a, &tmA, bar, k * kLinK, m, MODE == LIN_GRAD ? pass : keep);
                    } else {
                        lin_load<CTAS>(a, &tmA2, bar, m, k * kLinK, pass);
                        lin_load<CTAS>(a + A_BYTES / 2, &tmA2, bar, m + 64, k * kLinK, pass);
                    }
                    if (!mn_b) {
                        lin_load<CTAS>(b, &tmB, bar, k * kLinK, p.v0 + n, pass);
                    } else {
                        const CUtensorMap *tm = j.kind ? &tmB2 : &tmB;
                        const int y = k * kLinK + (j.kind ? 0 : p.v0);
                        for (int x = 0; x < bn; x += 64) lin_load<CTAS>(b + x * kLinK * 2, tm, bar, n + x, y, j.kind ? keep : pass);
                    }
                }
                __syncwarp();
                ++loads;
                if (++s == STAGES) {
                    s = 0;
                    ph ^= 1;
                }
            }
        }
        if (!ok) {  // every load already issued lands before the CTA (or pair) exits
            *ab = 1;
            if (rank == 0)
                for (uint32_t q = 0; q < (uint32_t)STAGES && q < loads; ++q) {
                    const uint32_t last = (loads - 1 - q) / STAGES * STAGES + q;
                    mbar_wait(&S.full[q], (last / STAGES) & 1, err);
                }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (of the pair's first CTA)
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        const uint32_t formats = 1u << 4 | (TYPE == SARA_BF16 ? 1u << 7 | 1u << 10 : 0u) | (uint32_t)(kLinRows * CTAS >> 4) << 24;
        int it = 0;  // parts
#pragma unroll 1
        for (int i = 0; rank == 0 && i < work.count && ok; ++i) {
            LinJob j;
            if (!work.job(p, i, j)) break;
            const bool mn_a = MODE == LIN_GRAD && j.kind == 1, mn_b = MODE == LIN_GRAD;
            const uint32_t idesc = formats | (uint32_t)mn_a << 15 | (uint32_t)mn_b << 16 | (uint32_t)(j.n >> 3) << 17;
            const uint32_t step_a = mn_a ? 2048 : 32, step_b = mn_b ? 2048 : 32;
            uint32_t dacc = 0;
            int a = 0;
#pragma unroll 1
            for (int k = j.k0; k < j.k1; ++k) {
                const bool begins = MODE == LIN_SCORE ? k % PART == 0 : k == j.k0, ends = k + 1 == j.k1 || (MODE == LIN_SCORE && (k + 1) % PART == 0);
                if (begins) {
                    a = it & 1;
                    dacc = tmem + (uint32_t)(a * kLinCols);
                    if (it >= 2) ok = __all_sync(0xffffffffu, mbar_wait(&S.acc_empty[a], (uint32_t)(((it >> 1) - 1) & 1), err) && !*ab);
                    if (!ok) break;
                    ++it;
                }
                ok = __all_sync(0xffffffffu, mbar_wait(&S.full[s], ph, err) && !*ab);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t at = smem_u32(ring) + (uint32_t)(s * STAGE);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        lin_mma<CTAS>(dacc, sdesc_sw128(at + kk * step_a, kLinK * 128, 1024), sdesc_sw128(at + A_BYTES + kk * step_b, kLinK * 128, 1024),
                                      idesc, !begins || kk > 0);
                    lin_commit<CTAS>(&S.empty[s]);
                    if (ends) lin_commit<CTAS>(&S.acc_full[a]);
                }
                __syncwarp();
                if (++s == STAGES) {
                    s = 0;
                    ph ^= 1;
                }
            }
        }
        if (!ok) *ab = 1;
        if (rank == 0) {
            if (elect_one()) lin_commit_here<CTAS>(&S.drain);
            mbar_wait(&S.drain, 0, err);  // every MMA has retired before tensor memory is released
        }
    } else {
        // ------------------------------------------------------------ epilogues
        const int quarter = warp & 3, mine = (warp - 2) >> 2, lrow = quarter * 32 + lane;
        const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16);
        bool ok = true;
        auto give = [&](int a) {  // the accumulator back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CTAS == 2) mbar_arrive_cluster(cluster_addr(&S.acc_empty[a], 0));
                else mbar_arrive(&S.acc_empty[a]);
            }
        };
        auto wait = [&](int a, int use) {
            ok = __all_sync(0xffffffffu, mbar_wait(&S.acc_full[a], (uint32_t)(use & 1), err) && !*ab);
            tc_fence_after();
        };
        if constexpr (MODE == LIN_SCORE) {
            const float c = p.scale * kLog2e;
            const int c0 = mine * 128;
            int it = 0;
#pragma unroll 1
            for (int i = 0; i < work.count; ++i) {
                LinJob j;
                if (!work.job(p, i, j)) break;
                const int m = j.m0 + rank * kLinRows + lrow;  // row of A
                const int tok = m < live && p.tokens ? p.tokens[p.src ? p.src[m] : m] : -1;
                float v[128];
                const int parts = (j.k1 + PART - 1) / PART;
#pragma unroll 1
                for (int q = 0; q < parts && ok; ++q, ++it) {
                    wait(it & 1, it >> 1);
                    if (!ok) break;
                    const uint32_t at = from + (uint32_t)((it & 1) * kLinCols + c0);
                    if (q == 0) {
#pragma unroll
                        for (int cc = 0; cc < 4; ++cc) lin_tmem_load<false>(at + 32 * cc, v + 32 * cc);
                    } else {
#pragma unroll
                        for (int cc = 0; cc < 4; ++cc) lin_tmem_load<true>(at + 32 * cc, v + 32 * cc);
                    }
                    give(it & 1);
                }
                LinSums x;
                const int left = p.V - j.n0 - c0, at = tok - j.n0 - c0;  // columns that are tokens; the row's token
                if ((unsigned)at < 128u) {
                    float z = 0.f;
#pragma unroll
                    for (int e = 0; e < 128; ++e) z = e == at ? v[e] : z;
                    p.ztok[m] = z;
                }
                if (left < 128) {
#pragma unroll
                    for (int e = 0; e < 128; ++e) v[e] = e < left ? v[e] : -INFINITY;
                }
                float n = v[0];
#pragma unroll
                for (int e = 1; e < 128; ++e) n = fmaxf(n, v[e]);
                x.a = fmaxf(x.a, n);
                float s0 = 0.f, s1 = 0.f, t1 = 0.f, tops = -1.f;
#pragma unroll
                for (int e = 0; e < 128; e += 2) {
                    const float y0 = (v[e] - x.a) * c, y1 = (v[e + 1] - x.a) * c;
                    float w0 = exp2_approx(y0), w1 = exp2_approx(y1);
                    x.t = fmaf(w0, fmaxf(y0, -1000.f), x.t);  // (a logit of -inf adds nothing)
                    t1 = fmaf(w1, fmaxf(y1, -1000.f), t1);
                    if constexpr (CTAS == 1) {  // (with more rows the epilogue has no time for it, and no row's small terms weigh as much)
                        const float o0 = y0 == 0.f ? 1.f : 0.f, o1 = y1 == 0.f ? 1.f : 0.f;
                        w0 -= o0;
                        w1 -= o1;
                        tops += o0 + o1;
                    }
                    s0 += w0;
                    s1 += w1;
                }
                x.s = s0 + s1 + tops;
                x.t += t1;
                if (mine) {
                    E.sums[i & 1][0][lrow] = x.a;
                    E.sums[i & 1][1][lrow] = x.s;
                    E.sums[i & 1][2][lrow] = x.t;
                }
                // one decision for all eight warps, so that none is left in a barrier (a warp that is a tile ahead has the other place and flag)
                if (!ok) S.stop[i & 1] = 1;
                named_bar_sync(1, 256);
                if (*(volatile int *)&S.stop[i & 1]) break;
                if (!mine && m < live) {
                    x.join(E.sums[i & 1][0][lrow], E.sums[i & 1][1][lrow], E.sums[i & 1][2][lrow], c);
                    float *o = p.part + (int64_t)(j.n0 / kLinCols) * p.rows_cap + m;
                    const int64_t plane = (int64_t)p.token_tiles * p.rows_cap;
                    o[0] = x.a;
                    o[plane] = x.s;
                    o[2 * plane] = x.t;
                }
            }
        } else if constexpr (MODE == LIN_DZ) {
#pragma unroll 1
            for (int i = mine; i < work.count && ok; i += 2) {
                LinJob j;
                if (!work.job(p, i, j)) break;
                const int m = j.m0 + rank * kLinRows + lrow;
                // what the row wants, read while the MMAs run
                int tok = -1;
                float mx = 0.f, ls = 0.f, g = 0.f, gh = 0.f, H = 0.f, raise = 1.f;
                bool zero = true, wrong = false;
                if (m < live) {
                    const int r = p.src[m];
                    tok = p.tokens ? p.tokens[r] : -1;
                    mx = p.stats[2 * (int64_t)r];
                    ls = p.stats[2 * (int64_t)r + 1];
                    if (p.glp) g = p.glp[r];
                    if (p.gent) {
                        gh = p.gent[r];
                        H = p.entropy[r];
                    }
                    raise = pow2f(p.kexp[r]);
                    wrong = tok >= p.V;
                    zero = mx == -INFINITY && ls == 0.f && !wrong;
                }
                wait(mine, i >> 1);
                if (!ok) break;
                const int left = p.cols - j.n0;
                uint16_t *o = p.dz + (int64_t)m * p.piece + j.n0;
#pragma unroll 1
                for (int cc = 0; cc < kLinCols; cc += 32) {
                    float v[32];
                    lin_tmem_load<false>(from + (uint32_t)(mine * kLinCols + cc), v);
                    const int at = tok - p.v0 - j.n0 - cc;
                    uint16_t h[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const float lp = fmaf(v[e], p.scale, -mx) - ls, x = exp2_approx(lp * kLog2e);
                        float y = -x * fmaf(gh, fmaxf(lp, -1000.f) + H, g);
                        if (e == at) y += g;
                        y = wrong ? __int_as_float(0x7fc00000) : y * raise;
                        v[e] = zero || cc + e >= left ? 0.f : y;
                        h[e] = lin_round<TYPE>(v[e]);
                    }
                    if ((unsigned)at < 32u && m < live) {
                        float off = 0.f;
#pragma unroll
                        for (int e = 0; e < 32; ++e) off = e == at ? v[e] - lin_float<TYPE>(h[e]) : off;
                        p.delta[m] = off;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint16_t(&g8)[8] = *reinterpret_cast<const uint16_t(*)[8]>(h + 8 * q);
                        *reinterpret_cast<uint4 *>(o + cc + 8 * q) = m < live ? pack8(g8) : make_uint4(0, 0, 0, 0);
                    }
                }
                give(mine);
            }
        } else {
            const float k = p.scale * pow2f(-p.head->exp);
#pragma unroll 1
            for (int i = mine; i < work.count; i += 2) {
                LinJob j;
                if (!work.job(p, i, j)) break;
                const int m = j.m0 + rank * kLinRows + lrow, left = min(p.d - j.n0, j.n);
                // one decision for the four warps, so that none is left in a barrier (the flag is read by all before the next one)
                if (!ok) S.stop[mine] = 1;
                named_bar_sync(1 + mine, 128);
                if (*(volatile int *)&S.stop[mine]) break;
                if (j.kind) {
                    // rows whose token is one of the tile's: each warp looks through a quarter, so that their order is the rows'
                    const int base = p.v0 + j.m0 + rank * kLinRows, each = ((live + 3) / 4 + 31) / 32 * 32;
                    int n = 0;
#pragma unroll 4
                    for (int x = 0; x < each; x += 32) {
                        const int r = quarter * each + x + lane;
                        const int at = r < live ? p.tokc[r] - base : -1;
                        const bool hit = (unsigned)at < (unsigned)kLinRows;
                        const uint32_t mask = __ballot_sync(0xffffffffu, hit);
                        const int to = n + __popc(mask & ((1u << lane) - 1));
                        if (hit && to < kLinHits) E.hit[mine][quarter][to] = make_int2(at, r);
                        n += __popc(mask);
                    }
                    if (lane == 0) E.found[mine][quarter] = min(n, kLinHits);
                }
                named_bar_sync(1 + mine, 128);
                wait(mine, i >> 1);
                if (!ok) continue;  // (to the barrier)
                const bool write = j.kind ? m < p.cols : m < live;
                int hits = 0;  // of the row
                if (j.kind) {
#pragma unroll 1
                    for (int w = 0; w < 4; ++w)
                        for (int x = 0; x < E.found[mine][w]; ++x) hits += E.hit[mine][w][x].x == lrow;
                }
                float *acc = p.acc + ((int64_t)j.split * p.rows_cap + m) * p.d + j.n0;
                uint16_t *o = j.kind ? p.dw + (int64_t)(p.v0 + m) * p.dw_stride + j.n0 : nullptr;
#pragma unroll 1
                for (int cc = 0; cc < left; cc += 32) {
                    float v[32];
                    lin_tmem_load<false>(from + (uint32_t)(mine * kLinCols + cc), v);
                    if (!write) continue;
                    if (hits) {
#pragma unroll 1
                        for (int w = 0; w < 4; ++w)
#pragma unroll 1
                            for (int x = 0; x < E.found[mine][w]; ++x) {
                                const int2 hit = E.hit[mine][w][x];
                                if (hit.x != lrow) continue;
                                const float f = p.delta[hit.y];
                                const uint16_t *h = p.low + (int64_t)hit.y * p.d + j.n0 + cc;
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    if (cc + 8 * q >= left) continue;
                                    const uint4 y = *reinterpret_cast<const uint4 *>(h + 8 * q);
                                    const uint32_t u[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const float2 z = unpack2<TYPE>(u[e]);
                                        v[8 * q + 2 * e] = fmaf(f, z.x, v[8 * q + 2 * e]);
                                        v[8 * q + 2 * e + 1] = fmaf(f, z.y, v[8 * q + 2 * e + 1]);
                                    }
                                }
                            }
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (cc + 8 * q >= left) continue;
                        if (j.kind) {
                            uint16_t h[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) h[e] = lin_round<TYPE>(v[8 * q + e] * k);
                            *reinterpret_cast<uint4 *>(o + cc + 8 * q) = pack8(h);
                        } else {
                            float4 *to = reinterpret_cast<float4 *>(acc + cc + 8 * q);
                            float4 x0 = make_float4(v[8 * q], v[8 * q + 1], v[8 * q + 2], v[8 * q + 3]);
                            float4 x1 = make_float4(v[8 * q + 4], v[8 * q + 5], v[8 * q + 6], v[8 * q + 7]);
                            if (!p.first) {
                                const float4 y0 = to[0], y1 = to[1];
                                x0 = make_float4(x0.x + y0.x, x0.y + y0.y, x0.z + y0.z, x0.w + y0.w);
                                x1 = make_float4(x1.x + y1.x, x1.y + y1.y, x1.z + y1.z, x1.w + y1.w);
                            }
                            to[0] = x0;
                            to[1] = x1;
                        }
                    }
                }
                give(mine);
            }
        }
        if (!ok) *ab = 1;
    }
    __syncwarp();
    tc_fence_before();
    if constexpr (CTAS == 2) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    if (warp == 1) lin_tmem_free<CTAS>(tmem, 512);
    if constexpr (CTAS == 2) cluster_sync();
}

// ------------------------------------------------------------------------------- rows
// One CTA: the live rows' places, and in fp16 the power of two that each row's dZ is raised by, so that the largest is of some 2^13
// and p down to 2^-27 of it is not a subnormal number.  (|dZ| <= |g| + |g'| p |log p + H|, the last factors below 16.)  bf16 has fp32's range.
struct LinRowParams {
    LinHeader *head;
    int R;
    const int32_t *tokens;
    const float *glp, *gent;  // null in the forward pass
    int *src, *pos, *kexp;    // [R]; kexp null in the forward pass
    bool raise;
};
__global__ void __launch_bounds__(1024) lin_rows_kernel(LinRowParams p) {
    __shared__ int s_warp[32], s_exp;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int base = 0, least = 1 << 20;
    if (threadIdx.x == 0) s_exp = 1 << 20;
#pragma unroll 1
    for (int r0 = 0; r0 < p.R; r0 += 1024) {
        const int r = r0 + threadIdx.x;
        const bool on = r < p.R && (!p.tokens || p.tokens[r] >= 0);
        const uint32_t mask = __ballot_sync(0xffffffffu, on);
        __syncthreads();
        if (lane == 0) s_warp[warp] = __popc(mask);
        __syncthreads();
        const int n = s_warp[lane];
        const int before = __reduce_add_sync(0xffffffffu, lane < warp ? n : 0), all = __reduce_add_sync(0xffffffffu, n);
        const int at = base + before + __popc(mask & ((1u << lane) - 1));
        base += all;
        if (r < p.R) p.pos[r] = on ? at : -1;
        if (on) p.src[at] = r;
        if (p.kexp && r < p.R) {
            int k = 0;
            if (on && p.raise) {
                const float b = (p.glp ? fabsf(p.glp[r]) : 0.f) + 16.f * (p.gent ? fabsf(p.gent[r]) : 0.f);
                // 2^e > b >= 2^(e - 1) (a NaN, an infinity or 0: 0)
                if (b > 0.f && b < INFINITY) {
                    k = max(min(13 - (ilogbf(b) + 1), 120), -120);
                    least = min(least, k);
                }
            }
            p.kexp[r] = k;
        }
    }
    least = __reduce_min_sync(0xffffffffu, least);
    if (lane == 0) atomicMin(&s_exp, least);
    __syncthreads();
    if (threadIdx.x == 0) {
        p.head->live = base;
        p.head->exp = s_exp == 1 << 20 ? 0 : s_exp;
    }
}

// The live rows side by side, zeros behind them up to a whole tile; in fp16, for dW, once more, each lowered by what its dZ is raised more
// than the least: rows whose gradients are far below the largest's lose bits that would not reach dW's either.
struct LinGatherParams {
    const LinHeader *head;
    const uint16_t *h;
    int64_t stride;
    int d, tile;
    const int *src, *kexp;
    const int32_t *tokens;  // may be null
    int *tokc;              // [rows_cap]: the compact rows' tokens, or null
    uint16_t *out, *low;    // [rows_cap][d]; low null: not wanted
};
__global__ void __launch_bounds__(256) lin_gather_kernel(LinGatherParams p) {
    const int live = p.head->live, row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= max((live + p.tile - 1) / p.tile, 1) * p.tile) return;
    uint16_t *o = p.out + (int64_t)row * p.d, *o2 = p.low ? p.low + (int64_t)row * p.d : nullptr;
    const int r = row < live ? p.src[row] : 0, down = o2 && row < live ? min(p.head->exp - p.kexp[r], 0) : 0;
    if (p.tokc && lane == 0) p.tokc[row] = row < live && p.tokens ? p.tokens[r] : -1;
    const uint16_t *h = p.h + r * p.stride;
    const float f = pow2f(max(down, -126));
    for (int x = 8 * lane; x < p.d; x += 256) {
        const uint4 v = row < live ? *reinterpret_cast<const uint4 *>(h + x) : make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(o + x) = v;
        if (!o2) continue;
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&w[e]));
            w[e] = pack_half2(y.x * f, y.y * f);
        }
        *reinterpret_cast<uint4 *>(o2 + x) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ------------------------------------------------------------------------------- joins
// ROWS rows a CTA, whose other threads share the tiles: 8 rows fill the sectors that are read, one is sooner done
struct LinJoinParams {
    LinHeader *head;
    int R, V, tiles, rows_cap;
    const int32_t *tokens;
    const int *pos;     // null: the same
    const float *part, *ztok;
    float scale;
    float *logprob, *entropy, *stats;
};
template <int ROWS>
__global__ void __launch_bounds__(256) lin_join_kernel(LinJoinParams p) {
    constexpr int G = 256 / ROWS;
    __shared__ float s_sums[3][G][ROWS];
    const int group = threadIdx.x / ROWS, lane = threadIdx.x % ROWS, r = blockIdx.x * ROWS + lane;
    const bool in = r < p.R;
    const int tok = in && p.tokens ? p.tokens[r] : 0, at = in && tok >= 0 ? (p.pos ? p.pos[r] : r) : -1;
    const float c = p.scale * kLog2e;
    const int64_t plane = (int64_t)p.tiles * p.rows_cap;
    LinSums x;
    if (at >= 0) {
#pragma unroll 4
        for (int n = group; n < p.tiles; n += G) {
            const float *q = p.part + (int64_t)n * p.rows_cap + at;
            x.join(q[0], q[plane], q[2 * plane], c);
        }
    }
#pragma unroll 1
    for (int g = G; g > 1; g /= 2) {  // by halves, always the same ones
        if (group >= g / 2 && group < g) {
            s_sums[0][group][lane] = x.a;
            s_sums[1][group][lane] = x.s;
            s_sums[2][group][lane] = x.t;
        }
        __syncthreads();
        if (group < g / 2) x.join(s_sums[0][group + g / 2][lane], s_sums[1][group + g / 2][lane], s_sums[2][group + g / 2][lane], c);
    }
    if (group || !in) return;
    const float a = x.a, s = x.s, t = x.t;
    const float nan = __int_as_float(0x7fc00000);
    const bool pad = tok < 0, none = s == -1.f, failed = p.head->err != 0;
    const float ls = none ? 0.f : log1pf(s);
    float lp = 0.f;
    if (at >= 0 && tok < p.V) lp = none ? -INFINITY : fmaf(p.ztok[at] - a, p.scale, -ls);
    else if (!pad) lp = nan;
    if (p.logprob) p.logprob[r] = failed ? nan : pad ? 0.f : lp;
    if (p.entropy) p.entropy[r] = failed ? nan : pad || none ? 0.f : fmaf(-kLn2, t / (1.f + s), ls);
    if (p.stats) {
        p.stats[2 * (int64_t)r] = failed ? nan : pad ? 0.f : none ? -INFINITY : a * p.scale;
        p.stats[2 * (int64_t)r + 1] = failed ? nan : pad ? 0.f : ls;
    }
}

// dH: the splits' sums in their order and what rounding took at the row's token, times scale and what dZ was raised by, to the rows' places; 0
// for rows of padding
struct LinOutParams {
    const LinHeader *head;
    int R, d, splits, rows_cap;
    const int *pos, *kexp;
    const float *acc, *delta;
    const int32_t *tokens;
    int V;
    const uint16_t *w;
    int64_t w_stride;
    float scale;
    uint16_t *out;
    int64_t stride;
};
template <int TYPE>
__global__ void __launch_bounds__(256) lin_out_kernel(LinOutParams p) {
    const int r = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (r >= p.R) return;
    const int at = p.pos[r];
    const float k = p.head->err ? __int_as_float(0x7fc00000) : p.scale * pow2f(-p.kexp[r]);
    uint16_t *o = p.out + r * p.stride;
    const int tok = p.tokens && at >= 0 ? p.tokens[r] : -1;
    const bool fix = tok >= 0 && tok < p.V;
    const float f = fix ? p.delta[at] : 0.f;
    for (int x = 8 * lane; x < p.d; x += 256) {
        float v[8] = {};
        if (fix) {
            const uint4 y = *reinterpret_cast<const uint4 *>(p.w + tok * p.w_stride + x);
            const uint32_t u[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 z = unpack2<TYPE>(u[e]);
                v[2 * e] = f * z.x;
                v[2 * e + 1] = f * z.y;
            }
        }
        if (at >= 0) {
            for (int s = 0; s < p.splits; ++s) {
                const float4 *q = reinterpret_cast<const float4 *>(p.acc + ((int64_t)s * p.rows_cap + at) * p.d + x);
                const float4 a = q[0], b = q[1];
                v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
                v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
            }
        }
        uint16_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = at >= 0 ? lin_round<TYPE>(v[e] * k) : (uint16_t)0;
        *reinterpret_cast<uint4 *>(o + x) = pack8(h);
    }
}

// ------------------------------------------------------------------------------- host: sizes
inline int64_t lin_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// How a call's work is cut, and where its parts stand in the workspace
struct LinPlan {
    int ctas, rows_cap, tiles;        // CTAs of a tile; rows up to whole tiles; tiles of tokens
    bool gather;                      // the live rows are gathered
    int piece, splits;                // gradient: tokens of a piece, parts of its dH
    size_t src, pos, kexp, tokc, delta, rows, low, part, ztok, dz, acc, bytes;
};
inline LinPlan lin_plan(int R, int d, int V, bool backward) {
    LinPlan q{};
    q.ctas = R > kLinRows ? 2 : 1;
    const int tm = kLinRows * q.ctas;
    q.rows_cap = (int)lin_up(R, tm);
    q.tiles = (int)lin_up(V, kLinCols) / kLinCols;
    q.gather = backward || R > kLinRows;
    size_t at = sizeof(LinHeader);
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += (bytes + 255) / 256 * 256;
        return was;
    };
    if (q.gather) {
        q.src = take((size_t)R * 4);
        q.pos = take((size_t)R * 4);
        q.rows = take((size_t)q.rows_cap * d * 2);
    }
    if (!backward) {
        q.part = take((size_t)3 * q.tiles * q.rows_cap * 4);
        q.ztok = take((size_t)q.rows_cap * 4);
    } else {
        q.kexp = take((size_t)R * 4);
        q.tokc = take((size_t)q.rows_cap * 4);
        q.delta = take((size_t)q.rows_cap * 4);
        q.low = take((size_t)q.rows_cap * d * 2);
        const int workers = kLinWorkers / q.ctas, mt = q.rows_cap / tm, nt = (int)lin_up(d, kLinCols) / kLinCols;
        int64_t piece = ((int64_t)192 << 20) / 2 / q.rows_cap;
        piece = piece / kLinCols * kLinCols;
        if (piece < 4 * kLinCols) piece = 4 * kLinCols;
        if (piece > 16384) piece = 16384;
        if (piece > lin_up(V, kLinCols)) piece = lin_up(V, kLinCols);
        q.piece = (int)piece;
        const int64_t kc = lin_up(piece < V ? piece : V, kLinK) / kLinK, kr = lin_up(R, kLinK) / kLinK, jw = lin_up(piece, tm) / tm * nt;
        const int64_t load = (jw * kr + (int64_t)mt * nt * kc) / workers + 1;
        int64_t s = workers / ((int64_t)mt * nt);
        if (s < (kc + load - 1) / load) s = (kc + load - 1) / load;
        if (s < 1) s = 1;
        if (s > kc) s = kc;
        if (s > kLinMaxSplits) s = kLinMaxSplits;
        q.splits = (int)s;
        q.dz = take((size_t)q.rows_cap * q.piece * 2);
        q.acc = take((size_t)q.splits * q.rows_cap * d * 4);
    }
    q.bytes = at;
    return q;
}

}  // namespace sara
