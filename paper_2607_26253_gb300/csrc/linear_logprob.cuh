// Log-probabilities of given tokens under softmax(scale H W^T), H [R][d] hidden states, W [V][d] the vocabulary's weights, with the
// entropy, and the gradient of both with respect to H and W.  No logits are kept:
//   forward:  the logits of a tile of rows and tokens are the accumulator of tensor-core products; its epilogue leaves a row's maximum
//             a, sum 2^y and sum 2^y y with y = (acc - a) scale log2(e), which a second kernel joins over the tiles
//   gradient: the vocabulary goes by in pieces.  A piece's logits are made again, its dZ = g (1[v = token] - p) - g' p (log p + H),
//             [R][piece], is stored in the operands' type, and feeds both products, dH += dZ W and dW = dZ^T H.
// Bound by the tensor cores from some 300 rows on, by reading W below.  us of a call in a CUDA graph (and of its floor): scores of 1 x 2,048 x 151,936 115 (92),
// of 26 x 1,536 x 151,936 93 (69), of 4,096 x 1,536 x 151,936 1,016 (910; 1,120 back to back); gradient of 301 x 2,048 x 32,001 in fp16 205 (56: 106 with rows
// in whole tiles), of 4,096 x 1,536 x 151,936 3,510 (2,730; 3,013 at the rate that the power cap leaves; 3,570 back to back).
//
// One persistent kernel does all the products (D = A B^T, fp32 in tensor memory): 256 columns, 128 rows a CTA, K in chunks of 64.
// With more than 128 rows two CTAs (a cluster) share a tile of 256 x 256, each bringing half of A's rows and half of B's: 64 bytes
// a cycle and SM from L2 for 96 alone.  Operands come by TMA with 128-byte swizzling, K-major or M/N-major as they lie in memory, so
// nothing is ever transposed: dZ is K-major for dH and M-major for dW, W is K-major for the logits and N-major for dH.
// Rows of padding (token < 0) are left out: the live rows are gathered first, so that they cost nothing and their contents,
// whatever they are, reach nothing.
//
// The tensor core cuts its sums off, all towards zero: sums of one sign lost 1.4 to 4 times 2^-24 of themselves each 16 products.  Long sums are therefore
// made in parts, which the epilogue adds.
// dZ enters the products in 16 bits.  Its largest element by far is mostly the token's own: what that one's rounding left off is
// kept (delta) and added to both gradients in fp32.
//
// Warp roles (320 threads): warp 0 producer, warp 1 MMA issuer and tensor-memory owner, warps 2..9 epilogue (warp w: the rows of
// tensor-memory lanes 32 (w % 4) .., columns 128 ((w - 2) / 4) ..).  A tile's 128 columns are in a thread's registers before its accumulator,
// one of two, is given back: the epilogue has a tile's time, not what is left of it (dZ of 4,096 rows: 161 us a piece with
// warps 2..5 and 6..9 on alternate tiles, reading their accumulator as they go).
#pragma once
#include <type_traits>

#include "device_common.cuh"
#include "host_util.h"
#include "kv8.cuh"
#include "logprob.cuh"

namespace sara {

constexpr int kLinThreads = 320;
constexpr int kLinRows = 128, kLinCols = 256, kLinK = 64;  // of a CTA's tile; elements of a chunk
constexpr int kLinMaxSplits = 32;
constexpr int kLinSort = 65536, kLinGatherCols = 1024;  // rows that are sorted together; columns of a warp that gathers
constexpr int kLinWorkers = 152;  // SMs that a plan counts on (on a GPU with others it is as right, if less even)

// What the kernels of a call share, at the start of the workspace
struct LinHeader {
    int err;   // bits of device_common.cuh; left zero
    int live;  // rows that are not padding
    int exp;   // dW's sums are raised by this power of two (0 in bf16)
    int up;    // kLinUp less the least that a row allows, of those seen so far; left zero
    int pad[60];
};

constexpr int kLinBlock = kLinRows * kLinK * 2;  // 16 KB: 128 rows of a chunk
enum LinMode : int {
    LIN_SCORE = 0,  // tiles of logits -> partial sums
    LIN_DZ = 1,     // tiles of logits -> dZ of a piece
    LIN_GRAD = 2,   // dZ of a piece -> dH's sums, dW
};
// How results leave: from registers, each thread its row's, which costs the memory pipe an access a lane; or STAGED, by way of shared memory, two blocks of
// 64 columns for each half of the epilogue, in whole lines, which costs stages of operands.  dW of 301 rows, 5 chunks a tile: 147 us / 118 staged; of
// 4,096, 58 chunks: 287 / 297; dZ of 4,096 rows: 136 / 140.
constexpr int kLinStagedRows = 1024;  // up to which dW is staged
__host__ __device__ constexpr int lin_stage_bytes(int ctas) { return kLinBlock * (1 + 2 / ctas); }
__host__ __device__ constexpr int lin_stages(int ctas, bool staged) { return ctas == 2 ? (staged ? 4 : 6) : staged ? 3 : 4; }
__host__ __device__ constexpr size_t lin_smem(int ctas, bool staged) {
    return 1024 + (size_t)lin_stages(ctas, staged) * lin_stage_bytes(ctas) + (staged ? 4 : 0) * kLinBlock;
}
constexpr int kLinDwCost = 9;
constexpr int kLinNoToken = 1 << 30;  // (behind every token)
constexpr int kLinHits = 8;  // rows of a tile of tokens that wait in shared memory for dW's epilogue

struct LinParams {
    LinHeader *head;
    int R, d, V;
    int a_rows;        // of a box of A (up to 128 rows in all: no more than there are; what the others hold does not matter)
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
    int v0, cols;      // the piece's first token, and tokens
    float *delta;      // [rows_cap]: what rounding took from dZ at the row's token
    // LIN_GRAD
    const int *start;  // see lin_gather_kernel
    const int2 *sorted;
    int buckets;
    const uint16_t *low;  // [rows_cap][d]: the rows as dW's product has them
    float *acc;        // [split][rows_cap][d]
    int splits, first; // first: the first piece
    bool dh, dw;
    uint16_t *out;     // DZ: dZ's blocks, [piece / 64][rows_cap][64]; GRAD: dW
    int64_t out_stride;
    bool wide;         // its rows' blocks are 32-byte aligned
};

// Chunks of a part of a logit's sum.  Scores and fp16: with two CTAs a tile's epilogue has no time for more parts; the errors of a few rows, which nothing averages
// away, get some more (1 x 2,048 x 151,936: 109 us with 2, 113 with 1; entropies of 1 x 944 x 32,990 off by 4.3e-6 and below 1e-6)
__device__ __forceinline__ int lin_part(int ctas, int rows) { return ctas == 2 ? 8 : rows <= 8 ? 1 : 2; }
// The gradient's in bf16, whose products have fewer bits to cut off and whose results have 8: one sum up to 2,048 dims, LONG sums of parts of as many beyond
// (65,536 products of one sign in one sum: a logit of 36 was off by 0.012, and p by as much of itself; a loop over one part costs 128 x 1,536 x 151,936 3 %).
constexpr int kLinLongPart = 32;
// Gradients of more than kLinLong chunks of rows or tokens are LONG too, in parts (fp16: dW of 262,144 rows, of one sign in one sum, was off by 1.7e-3, dH of a
// vocabulary of 780,000 by 1.1e-2).  Sums of one sign lost 2 to 4 times 2^-24 of themselves each 16 products: 3 to 6e-4 at kLinLong chunks.
constexpr int kLinLong = 640, kLinGradPart = 64;
struct LinSmem {
    uint64_t full[6], empty[6], acc_full[2], acc_empty[2], drain;
    uint32_t tmem_base;
    int abort, stop[2];                  // stop: the epilogue's, for two tiles in turn
};
struct LinScoreSmem {
    float sums[2][3][kLinRows];          // of the second half's columns, for two tiles in turn
};
struct LinGradSmem {
    uint16_t row[2][2][kLinHits][kLinCols / 2];  // for each half of the columns, two tiles in turn
};
struct LinNoSmem {};

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

__device__ __forceinline__ void lin_store(const CUtensorMap *tm, uint32_t src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<uint64_t>(tm)), "r"(x),
                 "r"(y), "r"(src)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// This thread's stores have been read from shared memory
__device__ __forceinline__ void lin_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void lin_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

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

// A job of dW's in chunks: its products, or its epilogue where those are few
__host__ __device__ __forceinline__ int lin_dw_cost(int kr) { return kr + 1 > kLinDwCost ? kr + 1 : kLinDwCost; }

// The jobs of a CTA (or pair) `w` of `W`, by number.  Logits: rows fastest, so that the CTAs at work share tokens.
// LIN_GRAD: dH's jobs are long, so the workers that have one more of them get fewer of dW's.
template <int MODE, int CTAS>
struct LinWork {
    static constexpr int TM = kLinRows * CTAS, COLS = kLinCols;
    int w, W, mt, nt, count;
    int64_t tiles;
    // LIN_GRAD
    int kc, kr, splits, jh, extra, light;  // chunks of a piece, of the rows; dH's jobs; of dW's: those before the others join, this worker's
    int own_h, wide;                       // this worker's dH jobs; the workers with one less of them
    __device__ __forceinline__ LinWork(const LinParams &p, int live, int w_, int W_) : w(w_), W(W_) {
        mt = max((live + TM - 1) / TM, 1);
        if constexpr (MODE != LIN_GRAD) {
            nt = (p.cols + COLS - 1) / COLS;
            tiles = (int64_t)mt * nt;
            count = (int)(tiles > w ? (tiles - 1 - w) / W + 1 : 0);
        } else {
            nt = (p.d + COLS - 1) / COLS;
            kc = (p.cols + kLinK - 1) / kLinK;
            kr = max((live + kLinK - 1) / kLinK, 1);
            splits = min(p.splits, kc);
            jh = p.dh ? mt * nt * splits : 0;
            const int jw = p.dw ? (p.cols + TM - 1) / TM * nt : 0;
            const int rem = jh % W;
            wide = W - rem;
            own_h = jh / W + (w < rem);
            const int cost = lin_dw_cost(kr), ratio = rem ? (kc / splits + cost - 1) / cost : 0;  // dW's jobs in the time of one of dH's
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
            j = {m * TM, n * COLS, COLS, 0, (p.d + kLinK - 1) / kLinK, 0, 0};
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
            j.n0 = n * COLS;
            j.n = min(COLS, (p.d - j.n0 + 64 * CTAS - 1) / (64 * CTAS) * (64 * CTAS));
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

// 32 columns of a lane are added to v; the wait is part of the instruction, so that nothing uses the values before it
__device__ __forceinline__ void lin_tmem_add(uint32_t taddr, float *v) {
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
    for (int i = 0; i < 32; ++i) v[i] += __uint_as_float(r[i]);
}

__device__ __forceinline__ float max_nan(float a, float b) {  // the larger; a NaN stays
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// 128 columns of a lane
__device__ __forceinline__ void lin_tmem_load128(uint32_t taddr, float (&v)[128]) {
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x128.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%3"
        "7,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63,%64,%65,%66,%67,%68,%69,%70,%71,%7"
        "2,%73,%74,%75,%76,%77,%78,%79,%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95,%96,%97,%98,%99,%100,%101,%102,%103,%104,%105,"
        "%106,%107,%108,%109,%110,%111,%112,%113,%114,%115,%116,%117,%118,%119,%120,%121,%122,%123,%124,%125,%126,%127}, [%128];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), 
          "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), 
          "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]), "=f"(v[32]), "=f"(v[33]), 
          "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]), "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), 
          "=f"(v[45]), "=f"(v[46]), "=f"(v[47]), "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]), 
          "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63]), "=f"(v[64]), "=f"(v[65]), "=f"(v[66]), 
          "=f"(v[67]), "=f"(v[68]), "=f"(v[69]), "=f"(v[70]), "=f"(v[71]), "=f"(v[72]), "=f"(v[73]), "=f"(v[74]), "=f"(v[75]), "=f"(v[76]), "=f"(v[77]), 
          "=f"(v[78]), "=f"(v[79]), "=f"(v[80]), "=f"(v[81]), "=f"(v[82]), "=f"(v[83]), "=f"(v[84]), "=f"(v[85]), "=f"(v[86]), "=f"(v[87]), "=f"(v[88]), 
          "=f"(v[89]), "=f"(v[90]), "=f"(v[91]), "=f"(v[92]), "=f"(v[93]), "=f"(v[94]), "=f"(v[95]), "=f"(v[96]), "=f"(v[97]), "=f"(v[98]), "=f"(v[99]), 
          "=f"(v[100]), "=f"(v[101]), "=f"(v[102]), "=f"(v[103]), "=f"(v[104]), "=f"(v[105]), "=f"(v[106]), "=f"(v[107]), "=f"(v[108]), "=f"(v[109]), 
          "=f"(v[110]), "=f"(v[111]), "=f"(v[112]), "=f"(v[113]), "=f"(v[114]), "=f"(v[115]), "=f"(v[116]), "=f"(v[117]), "=f"(v[118]), "=f"(v[119]), 
          "=f"(v[120]), "=f"(v[121]), "=f"(v[122]), "=f"(v[123]), "=f"(v[124]), "=f"(v[125]), "=f"(v[126]), "=f"(v[127])
        : "r"(taddr)
        : "memory");
}

template <int MODE, int CTAS, int TYPE, bool STAGED, bool LONG = false>
__global__ void __launch_bounds__(kLinThreads, 1)
lin_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmA2,
           const __grid_constant__ CUtensorMap tmB2, const __grid_constant__ CUtensorMap tmOut, LinParams p) {
    constexpr int STAGES = lin_stages(CTAS, STAGED), STAGE = lin_stage_bytes(CTAS), COLS = kLinCols;
    constexpr bool PARTED = LONG || MODE == LIN_SCORE || (MODE == LIN_DZ && TYPE == SARA_FP16);
    const int PART = !LONG ? lin_part(CTAS, p.R) : MODE == LIN_GRAD ? kLinGradPart : kLinLongPart;
    extern __shared__ uint8_t smem_raw[];
    __shared__ LinSmem S;
    __shared__ __align__(16) std::conditional_t<MODE == LIN_SCORE, LinScoreSmem, std::conditional_t<MODE == LIN_GRAD, LinGradSmem, LinNoSmem>> E;
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CTAS == 2 ? (int)cluster_rank() : 0;
    int *err = &p.head->err;
    // (a tile of dW's adds its rows' corrections one after the other: some 1 us each, 4 s where 2^22 rows have one token)
    const uint64_t limit = kWaitLimitNs + (MODE == LIN_GRAD ? (uint64_t)p.R * 4096 : 0);
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&S.full[s], 1);
            mbar_init(&S.empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&S.acc_full[a], 1);
            mbar_init(&S.acc_empty[a], 8 * CTAS);
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
    pdl_allow_dependents();
    pdl_wait_prior_grids();
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
            const uint32_t bytes = (uint32_t)((mn_a ? kLinBlock : p.a_rows * kLinK * 2) + bn * kLinK * 2) * CTAS;
#pragma unroll 1
            for (int k = j.k0; k < j.k1; ++k) {
                if (loads >= (uint32_t)STAGES) ok = __all_sync(0xffffffffu, mbar_wait(&S.empty[s], ph, err, limit) && !*ab);
                if (!ok) break;
                if (elect_one()) {
                    uint8_t *a = ring + s * STAGE, *b = a + kLinBlock;
                    const uint32_t bar = CTAS == 2 ? cluster_addr(&S.full[s], 0) : smem_u32(&S.full[s]);
                    if (rank == 0) mbar_arrive_expect_tx(&S.full[s], bytes);
                    if (mn_a) {  // (dZ: blocks of 64 columns one after the other)
                        lin_load<CTAS>(a, &tmA2, bar, 0, m / 64 * p.rows_cap + k * kLinK, pass);
                        lin_load<CTAS>(a + kLinBlock / 2, &tmA2, bar, 0, (m / 64 + 1) * p.rows_cap + k * kLinK, pass);
                    } else if (MODE == LIN_GRAD) {
                        lin_load<CTAS>(a, &tmA, bar, 0, k * p.rows_cap + m, pass);
                    } else {
                        lin_load<CTAS>(a, &tmA, bar, k * kLinK, m, keep);
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
                    mbar_wait(&S.full[q], (last / STAGES) & 1, err, limit);
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
                const bool begins = PARTED ? (k - j.k0) % PART == 0 : k == j.k0, ends = k + 1 == j.k1 || (PARTED && (k + 1 - j.k0) % PART == 0);
                if (begins) {
                    a = it & 1;
                    dacc = tmem + (uint32_t)(a * COLS);
                    if (it >= 2) ok = __all_sync(0xffffffffu, mbar_wait(&S.acc_empty[a], (uint32_t)((it / 2 - 1) & 1), err, limit) && !*ab);
                    if (!ok) break;
                    ++it;
                }
                ok = __all_sync(0xffffffffu, mbar_wait(&S.full[s], ph, err, limit) && !*ab);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t at = smem_u32(ring) + (uint32_t)(s * STAGE);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        lin_mma<CTAS>(dacc, sdesc_sw128(at + kk * step_a, kLinK * 128, 1024), sdesc_sw128(at + kLinBlock + kk * step_b, kLinK * 128, 1024),
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
            mbar_wait(&S.drain, 0, err, limit);  // every MMA has retired before tensor memory is released
        }
    } else {
        // ------------------------------------------------------------ epilogues
        const int quarter = warp & 3, mine = (warp - 2) >> 2, lrow = quarter * 32 + lane, c0 = mine * 128;  // mine: which half of the columns
        const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c0;
        bool ok = true;
        auto give = [&](int a) {  // the accumulator back
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CTAS == 2) mbar_arrive_cluster(cluster_addr(&S.acc_empty[a], 0));
                else mbar_arrive(&S.acc_empty[a]);
            }
        };
        auto wait = [&](int it) {  // for the it-th accumulator
            ok = __all_sync(0xffffffffu, mbar_wait(&S.acc_full[it & 1], (uint32_t)(it / 2 & 1), err, limit) && !*ab);
            tc_fence_after();
        };
        if constexpr (MODE == LIN_SCORE) {
            const float c = p.scale * kLog2e;
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
                    wait(it);
                    if (!ok) break;
                    const uint32_t at = from + (uint32_t)((it & 1) * COLS);
                    if (q == 0) {
                        lin_tmem_load128(at, v);
                    } else {
#pragma unroll
                        for (int cc = 0; cc < 128 / 32; ++cc) lin_tmem_add(at + 32 * cc, v + 32 * cc);
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
                    float *o = p.part + (int64_t)(j.n0 / COLS) * p.rows_cap + m;
                    const int64_t plane = (int64_t)p.token_tiles * p.rows_cap;
                    o[0] = x.a;
                    o[plane] = x.s;
                    o[2 * plane] = x.t;
                }
            }
        } else {
            // 64 columns of the tile's rows to `x`, `y` of the result.  STAGED: by way of one of this half's two places in shared memory, which the
            // block before the last one has left.  (After a failed wait the barriers go on and nothing is stored.)
            const uint32_t out = smem_u32(ring) + (uint32_t)(STAGES * STAGE + mine * 2 * kLinBlock);
            const bool first = quarter == 0 && lane == 0;
            int place = 0;
            auto emit = [&](const uint32_t (&w)[32], int x, int y) {
                if constexpr (STAGED) {
                    const uint32_t to = out + place * kLinBlock + lrow * 128;
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + ((q ^ (lrow & 7)) << 4)), "r"(w[4 * q]), "r"(w[4 * q + 1]),
                                     "r"(w[4 * q + 2]), "r"(w[4 * q + 3])
                                     : "memory");
                    fence_proxy_async_smem();
                    if (first) lin_stores_read();  // (the other place is free)
                    __syncwarp();
                    named_bar_sync(1 + mine, 128);
                    if (first && ok && (MODE == LIN_DZ || y < p.V)) lin_store(&tmOut, out + place * kLinBlock, x, y);  // (rows behind the last are cut off)
                    place ^= 1;
                } else if (ok && (MODE == LIN_DZ || y + lrow < p.V)) {
                    uint16_t *o = p.out + (int64_t)(y + lrow) * p.out_stride + x;
                    const int left = MODE == LIN_DZ ? 64 : p.d - x;
                    if (p.wide && left >= 64) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float f[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[8 * q + e]);
                            st_global_v8(reinterpret_cast<float *>(o + 16 * q), f);
                        }
                    } else {
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (8 * q < left) *reinterpret_cast<uint4 *>(o + 8 * q) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
                    }
                }
            };
            // GRAD: the rows whose token is one of the tile's (`sorted` from `start` on), brought for the tiles behind this one step by step: where
            // they stand, which they are, then the first of them themselves, so that none of these loads is waited for
            struct Hits {
                int x0, n, row, tok;  // (row, tok, delta: lane e's entry e)
                float delta;
            };
            const int blocks = (live + kLinSort - 1) / kLinSort;
            auto where = [&](int i) {
                Hits h = {0, 0, 0, -1, 0.f};
                LinJob j;
                if (MODE == LIN_GRAD && i < work.count && work.job(p, i, j) && j.kind) {
                    const int bucket = (p.v0 + j.m0 + rank * kLinRows) / kLinRows;
                    if (bucket < p.buckets) {
                        h.x0 = p.start[bucket];
                        h.n = p.start[bucket + 1];
                    }
                }
                return h;
            };
            auto which = [&](Hits &h) {
                h.n -= h.x0;
                if (lane < min(h.n, kLinHits)) {
                    const int2 x = p.sorted[h.x0 + lane];
                    h.row = x.x;
                    h.tok = x.y;
                }
            };
            auto fetch = [&](Hits &h, int i, int buf) {
                if (lane < min(h.n, kLinHits)) h.delta = p.delta[h.row];
                if constexpr (MODE == LIN_GRAD) {
                    LinJob j;
                    if (h.n > 0 && work.job(p, i, j)) {
                        const int n = min(h.n, kLinHits), left = min(p.d - j.n0, j.n) - c0, x = 2 * quarter + lane / 16, at = lane % 16 * 8;
                        const int row = __shfl_sync(0xffffffffu, h.row, x);  // (a half warp a row)
                        if (x < n && at < left) cp_async16(smem_u32(&E.row[mine][buf][x][at]), p.low + (int64_t)row * p.d + j.n0 + c0 + at);
                    }
                }
                cp_async_commit();
            };
            Hits now = {0, 0, 0, -1, 0.f}, next = now, later = now, last = now;
            int buf = 0;
            if (MODE == LIN_GRAD && p.dw) {
                next = where(0);
                later = where(1);
                last = where(2);
                which(next);
                which(later);
                fetch(next, 0, 0);
            }
            auto move_on = [&](int i) {
                now = next;
                next = later;
                later = last;
                fetch(next, i + 1, buf ^ 1);
                which(later);
                last = where(i + 3);
            };
            const float k = MODE == LIN_GRAD ? p.scale * pow2f(-p.head->exp) : 0.f;
            int it = 0;  // accumulators
#pragma unroll 1
            for (int i = 0; i < work.count; ++i) {
                LinJob j;
                if (!work.job(p, i, j)) break;
                const int m = j.m0 + rank * kLinRows + lrow;
                float v[128];
                auto read = [&]() {
                    if (ok) wait(it);
                    lin_tmem_load128(from + (uint32_t)((it & 1) * COLS), v);
                    if (ok) give(it & 1);
                    ++it;
                    if constexpr (PARTED) {
#pragma unroll 1
                        for (int q = 1; q < (j.k1 - j.k0 + PART - 1) / PART && ok; ++q, ++it) {
                            wait(it);
                            if (!ok) break;
                            const uint32_t at = from + (uint32_t)((it & 1) * COLS);
#pragma unroll
                            for (int cc = 0; cc < 128 / 32; ++cc) lin_tmem_add(at + 32 * cc, v + 32 * cc);
                            give(it & 1);
                        }
                    }
                };
                if constexpr (MODE == LIN_DZ) {
                    // What the row wants, read while the MMAs run.  In base 2: with r = (max + log S) log2(e) as rounded and f what the rounding
                    // took, y = acc scale log2(e) - r, p = 2^y 2^f, dz = 2^y (a y + b) with a = -2^f g' ln 2, b = -2^f (g + g' (entropy + f ln 2)).
                    int tok = -1;
                    float r = 0.f, ga = 0.f, gb = 0.f, g = 0.f, mx = 0.f, ls = 0.f;
                    bool zero = true, wrong = false;
                    const float c = p.scale * kLog2e;
                    if (m < live) {
                        const int row = p.src[m];
                        tok = p.tokens ? p.tokens[row] : -1;
                        mx = p.stats[2 * (int64_t)row];
                        ls = p.stats[2 * (int64_t)row + 1];
                        float gh = 0.f, H = 0.f;
                        if (p.glp) g = p.glp[row];
                        if (p.gent) {
                            gh = p.gent[row];
                            H = p.entropy[row];
                        }
                        wrong = tok >= p.V;
                        zero = mx == -INFINITY && ls == 0.f && !wrong;
                        const float raise = wrong ? __int_as_float(0x7fc00000) : pow2f(p.kexp[row]);
                        const float p1 = mx * kLog2e, p2 = ls * kLog2e;
                        r = p1 + p2;
                        const float x = r - p1, f = ((p1 - (r - x)) + (p2 - x)) + (fmaf(mx, kLog2e, -p1) + fmaf(ls, kLog2e, -p2));  // exactly r + f
                        const float k = exp2_approx(fminf(fmaxf(-f, -100.f), 100.f)) * raise;
                        ga = -k * gh * kLn2;
                        gb = -k * fmaf(gh, fmaf(-f, kLn2, H), g);
                        g *= raise;
                    }
                    read();
                    const int left = p.cols - j.n0 - c0, at = tok - p.v0 - j.n0 - c0;
                    const uint64_t c2 = pack_f32x2(c, c), r2 = pack_f32x2(-r, -r), a2 = pack_f32x2(ga, ga), b2 = pack_f32x2(gb, gb);
#pragma unroll
                    for (int cc = 0; cc < 128; cc += 64) {
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 64; e += 2) {
                            // (2^-1000 is 0; its factor is to stay finite)
                            const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(v[cc + e], v[cc + e + 1]), c2, r2));
                            const float y0 = max_nan(y.x, -1000.f), y1 = max_nan(y.y, -1000.f);
                            const float2 f = unpack_f32x2(fma_f32x2(pack_f32x2(y0, y1), a2, b2));
                            w[e / 2] = pack_grad<TYPE>(exp2_approx(y0) * f.x, exp2_approx(y1) * f.y);
                        }
                        if (__any_sync(0xffffffffu, at >= cc && at < cc + 64)) {  // (seldom) the token's own
                            if (at >= cc && at < cc + 64 && m < live) {
                                float z = 0.f;
#pragma unroll
                                for (int e = 0; e < 64; ++e) z = cc + e == at ? v[cc + e] : z;
                                // 1 - p from the logarithm.  A token within the error of its logit's sums of the maximum (of either call's, whose parts may be
                                // others) is the maximum, or shares it, where 1 - p depends little on the difference.  (Each 16 products lose 2 steps of the part's sum at
                                // most.  1 - p = 1e-5 at a logit of 22 in bf16: off by 2.6 times itself without.  fp16 with the error of one sum over 4,096 dims, a token 1.4e-3
                                // below a maximum of 100: 1 - p off by 1.4e-3)
                                const int row = p.src[m];
                                float t = fmaf(z, p.scale, -mx);
                                constexpr int kSteps = TYPE == SARA_FP16 ? 8 * kLinK / 16 : kLinLongPart * kLinK / 16;
                                if (fabsf(t) <= (2 * min(p.d / 16, kSteps) + p.d / 512 + 8) * 0x1p-24f * fabsf(mx)) t = 0.f;
                                const float lp = max_nan(t - ls, -700.f), H = p.gent ? p.entropy[row] : 0.f, gh = p.gent ? p.gent[row] : 0.f;
                                const float x = (wrong ? __int_as_float(0x7fc00000) : pow2f(p.kexp[row])) *
                                                (-(p.glp ? p.glp[row] : 0.f) * expm1f(lp) - gh * expf(lp) * (lp + H));
                                const uint32_t h = pack_grad<TYPE>(x, x);
                                p.delta[m] = zero ? 0.f : x - unpack2<TYPE>(h).x;
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (cc + 2 * e == (at & ~1)) w[e] = at & 1 ? (w[e] & 0xffffu) | (h & 0xffff0000u) : (w[e] & 0xffff0000u) | (h & 0xffffu);
                            }
                        }
                        if (__any_sync(0xffffffffu, zero) || left < cc + 64) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                if (zero || cc + 2 * e >= left) w[e] = 0;
                                else if (cc + 2 * e + 1 >= left) w[e] &= 0xffffu;
                            }
                        }
                        emit(w, 0, (j.n0 + c0 + cc) / 64 * p.rows_cap + j.m0 + rank * kLinRows);
                    }
                } else if (j.kind) {
                    const int token = p.v0 + m, left = min(p.d - j.n0, j.n) - c0;
                    cp_async_wait<0>();
                    __syncwarp();
                    named_bar_sync(1 + mine, 128);  // (its rows have come; the tile before has left the other place)
                    move_on(i);
                    uint32_t match = 0;  // which of them are the row's
#pragma unroll
                    for (int x = 0; x < kLinHits; ++x) match |= (uint32_t)(__shfl_sync(0xffffffffu, now.tok, x) == token) << x;
                    read();
                    auto add = [&](float f, const uint16_t *h) {
#pragma unroll
                        for (int q = 0; q < 16; ++q) {
                            if (8 * q >= left) continue;
                            const uint4 y = *reinterpret_cast<const uint4 *>(h + 8 * q);
                            const uint32_t u[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float2 z = unpack2<TYPE>(u[e]);
                                v[8 * q + 2 * e] = fmaf(f, z.x, v[8 * q + 2 * e]);
                                v[8 * q + 2 * e + 1] = fmaf(f, z.y, v[8 * q + 2 * e + 1]);
                            }
                        }
                    };
                    if (__any_sync(0xffffffffu, match != 0)) {
#pragma unroll 1
                        for (int x = 0; x < min(now.n, kLinHits); ++x) {
                            const float f = __shfl_sync(0xffffffffu, now.delta, x);
                            if (match >> x & 1) add(f, E.row[mine][buf][x]);
                        }
                    }
                    // the others, in their order, each thread its token's (5,027 rows of 512 tokens, dW of 96 columns: 86 us, 422 with a look at all of the
                    // tile's; a warp together for a token's, 4 columns a lane, costs registers: 164, and 301 rows' dW 136 -> 146, while 4,096 rows of one token
                    // take 4.1 ms instead of 7.4)
                    if (now.n > kLinHits || blocks > 1) {
#pragma unroll 1
                        for (int b = 0; b < blocks; ++b) {
                            const int *start = p.start + (int64_t)b * (p.buckets + 1) + (p.v0 + j.m0 + rank * kLinRows) / kLinRows;
                            if (token >= p.V) break;
                            int x = start[0] + (b == 0 ? kLinHits : 0), end = start[1];
                            const int2 *sorted = p.sorted + (int64_t)b * kLinSort;
                            for (int high = end; x < high;) {  // the first of the token's
                                const int mid = (x + high) / 2;
                                if (sorted[mid].y < token) x = mid + 1;
                                else high = mid;
                            }
#pragma unroll 1
                            for (; x < end; ++x) {
                                const int2 r = sorted[x];
                                if (r.y != token) break;
                                add(p.delta[r.x], p.low + (int64_t)r.x * p.d + j.n0 + c0);
                            }
                        }
                    }
#pragma unroll
                    for (int cc = 0; cc < 128; cc += 64) {
                        if (cc >= left) continue;
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) w[e] = pack_grad<TYPE>(v[cc + 2 * e] * k, v[cc + 2 * e + 1] * k);
                        emit(w, j.n0 + c0 + cc, p.v0 + j.m0 + rank * kLinRows);
                    }
                    buf ^= 1;
                } else {
                    if (p.dw) {  // (the next tile may be one of dW's)
                        move_on(i);
                        buf ^= 1;
                    }
                    read();
                    const int left = min(p.d - j.n0, j.n) - c0;
                    float *acc = p.acc + ((int64_t)j.split * p.rows_cap + m) * p.d + j.n0 + c0;
                    if (m < live) {
#pragma unroll
                        for (int q = 0; q < 32; ++q) {
                            if (4 * q >= left) continue;
                            float4 *to = reinterpret_cast<float4 *>(acc + 4 * q);
                            float4 x = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
                            if (!p.first) {
                                const float4 y = *to;
                                x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                            }
                            *to = x;
                        }
                    }
                }
            }
            if (STAGED && first) lin_stores_done();
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
// The live rows' places, and in fp16 the power of two that each row's dZ is raised by, so that the largest is of some 2^13
// and p down to 2^-27 of it is not a subnormal number.  (|dZ| <= b = |g| + 16 |g'|, for p |log p + H| is below 16.)  bf16 has fp32's range.
struct LinRowParams {
    LinHeader *head;
    int R;
    const int32_t *tokens;
    const float *glp, *gent;  // null in the forward pass
    int *src, *pos, *kexp;    // [R]; kexp null in the forward pass
    int *tokc;                // the compact rows' tokens, or null
    bool raise;
};
// What a CTA that finds the rows for itself keeps of them
constexpr int kLinFew = 1024;
struct LinFew {
    int live;
    int src[kLinFew], kexp[kLinFew], tokc[kLinFew];
};
// A CTA of THREADS; write: for the kernels behind it; keep: for itself
template <int THREADS>
__device__ __forceinline__ void lin_rows(const LinRowParams &p, bool write, LinFew *keep) {
    __shared__ int s_warp[32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int base = 0;
    if (threadIdx.x < 32) s_warp[threadIdx.x] = 0;
#pragma unroll 1
    for (int r0 = 0; r0 < p.R; r0 += THREADS) {
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
        if (write && r < p.R) p.pos[r] = on ? at : -1;
        if (on) {
            const int tok = p.tokc && p.tokens ? p.tokens[r] : -1;
            if (write) p.src[at] = r;
            if (write && p.tokc) p.tokc[at] = tok;
            if (keep) {
                keep->src[at] = r;
                keep->tokc[at] = tok;
            }
        }
        if (p.kexp && r < p.R) {
            int k = 0;
            if (on && p.raise) {
                const float b = (p.glp ? fabsf(p.glp[r]) : 0.f) + 16.f * (p.gent ? fabsf(p.gent[r]) : 0.f);
                // 2^e > b >= 2^(e - 1) (a NaN or an infinity: 0)
                if (b < INFINITY) k = b > 0.f ? max(min(13 - (ilogbf(b) + 1), 120), -120) : 120;
            }
            if (write) p.kexp[r] = k;
            if (keep) keep->kexp[r] = k;
        }
    }
    if (threadIdx.x == 0) {
        if (write) {
            p.head->live = base;
            p.head->exp = 0;
        }
        if (keep) keep->live = base;
    }
    __syncthreads();
}
// One CTA, for more than kLinFew rows
__global__ void __launch_bounds__(1024) lin_rows_kernel(LinRowParams p) {
    pdl_allow_dependents();
    lin_rows<1024>(p, true, nullptr);
}

// The live rows side by side, zeros behind them up to a whole tile; in fp16, for dW, the power of two 2^E that its sums are raised by is found on the way:
// dW = 2^-E sum (2^k dZ) (2^(E - k) h), k what the row's dZ is raised by, E the largest for which no 2^(E - k) |h| passes 2^15.
// The CTAs behind those put the rows in the order of their tokens (and of the rows of one), `kLinSort` rows at a time, so that
// dW's epilogue finds a tile's: sorted[start[b] .. start[b + 1]) are those of tile b.  A row's place is the number of rows before it, counted
// by 8 lanes.
// FEW: each CTA finds the rows for itself, the first one for the kernels behind it too (a launch less: gradient of 32 x 128 x 512 through the binding 33 -> 29 us, on the device 24.7 -> 24.2).
constexpr int kLinUp = 512;  // (the least is 15 - 16 - 120, the greatest 15 + 23 + 120)
struct LinGatherParams {
    LinHeader *head;
    const uint16_t *h;
    int64_t stride;
    int d, tile;
    const int *src, *kexp;
    uint16_t *out;          // [rows_cap][d]
    bool raise;             // 2^E is wanted
    int row_ctas;           // along x; the others sort
    const int *tokc;
    int2 *sorted;           // [rows_cap]: row, token
    int *start;             // [rows_cap / kLinSort up][buckets + 1]
    int buckets;
};
template <bool FEW>
__global__ void __launch_bounds__(256) lin_gather_kernel(LinGatherParams p, LinRowParams rows) {
    __shared__ std::conditional_t<FEW, LinFew, LinNoSmem> s_few;
    pdl_allow_dependents();
    pdl_wait_prior_grids();
    int live;
    const int *src = p.src, *kexp = p.kexp, *tokc = p.tokc;
    if constexpr (FEW) {
        lin_rows<256>(rows, blockIdx.x == 0 && blockIdx.y == 0, &s_few);
        live = s_few.live;
        src = s_few.src;
        kexp = s_few.kexp;
        tokc = s_few.tokc;
    } else {
        live = p.head->live;
    }
    const int lane = threadIdx.x & 31;
    if ((int)blockIdx.x >= p.row_ctas) {
        if (blockIdx.y) return;
        const int blocks = max((live + kLinSort - 1) / kLinSort, 1), part = threadIdx.x & 7;
        const int64_t asks = (int64_t)blocks * (p.buckets + 1) + live, stride = (int64_t)(gridDim.x - p.row_ctas) * 32;
        __shared__ __align__(16) int s_key[2048];
        for (int64_t q0 = (int64_t)(blockIdx.x - p.row_ctas) * 32; q0 < asks; q0 += stride) {  // (whole CTAs)
            const int64_t q = q0 + threadIdx.x / 8;
            const bool row = q < live;
            const int64_t y = q - live;
            const int me = row ? (int)q : 0, block = row ? me / kLinSort : (int)min(y / (p.buckets + 1), (int64_t)(blocks - 1));
            const int token = row ? tokc[me] : 0;
            const int key = row ? min(token, kLinNoToken) : (int)(y - (int64_t)block * (p.buckets + 1)) * kLinRows;
            int before = 0;
            // (a CTA's asks may be of different blocks: all of the rows go by, those of others count as behind)
            const int first = (int)(q0 < live ? q0 / kLinSort : min((q0 - live) / (p.buckets + 1), (int64_t)(blocks - 1)));
            const int64_t q1 = min(q0 + 31, asks - 1);
            const int last = q1 < live ? (int)(q1 / kLinSort) : q0 < live ? blocks - 1 : (int)min((q1 - live) / (p.buckets + 1), (int64_t)(blocks - 1));
            const int r_first = q0 < live && q1 >= live ? 0 : first * kLinSort;
            for (int r0 = r_first; r0 < min(live, (last + 1) * kLinSort); r0 += 2048) {
                __syncthreads();
                for (int x = threadIdx.x; x < 2048; x += 256) s_key[x] = r0 + x < live ? min(tokc[r0 + x], kLinNoToken) : INT32_MAX;
                __syncthreads();
                if (r0 / kLinSort != block) continue;
#pragma unroll 8
                for (int x = 4 * part; x < 2048; x += 32) {
                    const int4 b = *reinterpret_cast<const int4 *>(s_key + x);
                    const int d = row ? me - r0 - x : 0;  // (of equal ones those before this row count)
                    before += (b.x < key + (d > 0)) + (b.y < key + (d > 1)) + (b.z < key + (d > 2)) + (b.w < key + (d > 3));
                }
            }
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) before += __shfl_xor_sync(0xffffffffu, before, d);
            if (part == 0 && q < asks) {
                if (row) p.sorted[block * kLinSort + before] = make_int2(me, token);
                else p.start[y] = before;
            }
        }
        return;
    }
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5), x0 = blockIdx.y * kLinGatherCols, x1 = min(p.d, x0 + kLinGatherCols);
    if (row >= max((live + p.tile - 1) / p.tile, 1) * p.tile) return;
    uint16_t *o = p.out + (int64_t)row * p.d;
    const int r = row < live ? src[row] : 0;
    const uint16_t *h = p.h + r * p.stride;
    uint32_t top = 0;
#pragma unroll 4
    for (int x = x0 + 8 * lane; x < x1; x += 256) {
        const uint4 v = row < live ? *reinterpret_cast<const uint4 *>(h + x) : make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(o + x) = v;
        top = __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
    }
    if (!p.raise || row >= live) return;
    const uint32_t most = __reduce_max_sync(0xffffffffu, max(top & 0xffff, top >> 16));
    if (lane || !most) return;
    // |h| < 2^e of these (an infinity or a NaN: as the largest number)
    const int e = most >= 1024 ? min((int)(most >> 10) - 14, 16) : 8 - __clz(most), up = kLinUp - (15 - e + kexp[r]);
    if (up > *(volatile int *)&p.head->up) atomicMax(&p.head->up, up);
}

// fp16: the rows as dW's product has them, 2^(E - k) h.  A row keeps all bits but of elements that come out below 2^-14: with |dZ| 2^k < 2^13 they are off by
// 2^-25 2^13 2^-E at most, 2^-38 of the largest b |h| of any row.  Where that is within 2^13, it is less than half of fp16's least step.
struct LinLowParams {
    LinHeader *head;
    int d, tile;
    const int *src, *kexp;
    const uint16_t *rows;
    uint16_t *low;
};
__global__ void __launch_bounds__(256) lin_low_kernel(LinLowParams p) {
    pdl_allow_dependents();
    pdl_wait_prior_grids();
    const int live = p.head->live, up = p.head->up, exp = up ? min(kLinUp - up, 126) : 0;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) p.head->exp = exp;
    const int lane = threadIdx.x & 31, row = blockIdx.x * 8 + (threadIdx.x >> 5), x0 = blockIdx.y * kLinGatherCols, x1 = min(p.d, x0 + kLinGatherCols);
    if (row >= max((live + p.tile - 1) / p.tile, 1) * p.tile) return;
    const float f = pow2f(row < live ? max(exp - p.kexp[p.src[row]], -126) : 0);  // (of zeros behind the rows: any)
#pragma unroll 4
    for (int x = x0 + 8 * lane; x < x1; x += 256) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p.rows + (int64_t)row * p.d + x);
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&w[e]));
            w[e] = pack_half2(y.x * f, y.y * f);
        }
        *reinterpret_cast<uint4 *>(p.low + (int64_t)row * p.d + x) = make_uint4(w[0], w[1], w[2], w[3]);
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
    pdl_wait_prior_grids();
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
    LinHeader *head;
    int R, d, splits, rows_cap;
    const int *pos, *kexp;
    const float *acc, *delta;
    const int32_t *tokens;
    int V;
    const uint16_t *w;
    int64_t w_stride;
    float scale;
    uint16_t *out;      // or null
    int64_t stride;
    uint16_t *dw;       // or null: made NaN after a failed wait, as out is
    int64_t dw_stride;
};
constexpr int kLinOutCols = 512;  // of a warp
template <int TYPE>
__global__ void __launch_bounds__(256) lin_out_kernel(LinOutParams p) {
    pdl_wait_prior_grids();
    const bool failed = p.head->err != 0;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) p.head->up = 0;
    const int lane = threadIdx.x & 31, r = blockIdx.x * 8 + (threadIdx.x >> 5), x0 = blockIdx.y * kLinOutCols, x1 = min(p.d, x0 + kLinOutCols);
    if (failed && p.dw)
        for (int64_t v = r; v < p.V; v += 8 * (int64_t)gridDim.x)
            for (int x = x0 + lane; x < x1; x += 32) p.dw[v * p.dw_stride + x] = 0x7fff;
    if (r >= p.R || !p.out) return;
    const int at = p.pos[r];
    const float k = failed ? __int_as_float(0x7fc00000) : p.scale * pow2f(-p.kexp[r]);
    uint16_t *o = p.out + r * p.stride;
    const int tok = p.tokens && at >= 0 ? p.tokens[r] : -1;
    const bool fix = tok >= 0 && tok < p.V;
    const float f = fix ? p.delta[at] : 0.f;
#pragma unroll 2
    for (int x = x0 + 8 * lane; x < x1; x += 256) {
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
#pragma unroll 4
            for (int s = 0; s < p.splits; ++s) {
                const float4 *q = reinterpret_cast<const float4 *>(p.acc + ((int64_t)s * p.rows_cap + at) * p.d + x);
                const float4 a = q[0], b = q[1];
                v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
                v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
            }
        }
        uint32_t h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = at >= 0 ? pack_grad<TYPE>(v[2 * e] * k, v[2 * e + 1] * k) : 0u;
        *reinterpret_cast<uint4 *>(o + x) = make_uint4(h[0], h[1], h[2], h[3]);
    }
}

// ------------------------------------------------------------------------------- host: sizes
inline int64_t lin_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// How a call's work is cut, and where its parts stand in the workspace
struct LinPlan {
    int ctas, rows_cap, tiles;        // CTAs of a tile; rows up to whole tiles; tiles of tokens
    bool gather;                      // the live rows are gathered
    int piece, splits, buckets;       // gradient: tokens of a piece, parts of its dH, tiles of 128 tokens
    size_t src, pos, kexp, tokc, sorted, start, delta, rows, low, part, ztok, dz, acc, bytes;
};
// Tokens of a piece.  76 tiles of 256 are as many as there are pairs of CTAs, so that whatever the rows' tiles the logits' come out even; dZ is kept to 384 MB
// (a piece costs some 36 us besides its products, while the last tiles end: 4,096 rows in 16 pieces 3.85 ms, in 8 3.56).  Up to 128 rows the piece's weights, which are read twice, have to stay in L2 besides.
inline int64_t lin_piece(int rows_cap, int d, int V, int ctas) {
    constexpr int64_t kEven = 76 * 256;
    const int64_t most = ((int64_t)384 << 20) / 2 / rows_cap;
    int64_t piece = ctas == 1 ? (d <= 1152 ? 2 * kEven : d <= 2304 ? kEven : kEven / 2) : most >= kEven ? most / kEven * kEven : most / 256 * 256;
    if (piece < 1024) piece = 1024;
    const int64_t all = lin_up(V, 256);
    return piece < all ? piece : all;
}
inline LinPlan lin_plan(int R, int d, int V, bool backward) {
    LinPlan q{};
    R = R > 1 ? R : 1;  // (no rows: a call has nothing to cut)
    q.ctas = R > kLinRows ? 2 : 1;
    const int tm = kLinRows * q.ctas, cols = kLinCols;
    q.rows_cap = (int)lin_up(R, tm);
    q.tiles = (int)lin_up(V, cols) / cols;
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
        q.buckets = (int)lin_up(V, kLinRows) / kLinRows;
        q.kexp = take((size_t)R * 4);
        q.tokc = take((size_t)q.rows_cap * 4);
        q.sorted = take((size_t)q.rows_cap * 8);
        q.start = take((size_t)(lin_up(R, kLinSort) / kLinSort) * (q.buckets + 1) * 4);
        q.delta = take((size_t)q.rows_cap * 4);
        q.low = take((size_t)q.rows_cap * d * 2);
        const int64_t workers = kLinWorkers / q.ctas, mt = q.rows_cap / tm, nt = lin_up(d, cols) / cols;
        q.piece = (int)lin_piece(q.rows_cap, d, V, q.ctas);
        const int64_t kc = lin_up(q.piece < V ? q.piece : V, kLinK) / kLinK, kr = lin_up(R, kLinK) / kLinK, jw = lin_up(q.piece, tm) / tm * nt;
        const int64_t load = (jw * lin_dw_cost((int)kr) + mt * nt * kc) / workers + 1;
        int64_t s = workers / (mt * nt);
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
