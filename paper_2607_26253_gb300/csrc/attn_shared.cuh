// Decode attention over the 8-bit paged cache for groups of sequences whose first positions are the same: the shared ones are
// computed once for all of a group's queries, each sequence's own by the decode attention, and the two are joined,
//     out = (2^(m1 - m) o1 + 2^(m2 - m) o2) / (2^(m1 - m) l1 + 2^(m2 - m) l2),   m = max(m1, m2).
// Bound by reading the shared positions once (2 hd bytes each) up to some 128 queries a KV head, by the tensor cores beyond.  What it comes to
// (us, 32 / 8 heads of 128 dims in e4m3): 8 groups of 64 with 32,768 positions in common and 128 each of their own 412, of which the prefix kernel
// 355 (a page of 128 queries 3,200 cycles; its products alone would take 1,000, its exponentials 1,024: each page is a chain of scores,
// maximum, exponentials and product whose parts wait for one another); 64 groups of 8 with 1,024 and 512: 172, of which the prefix kernel 70
// (27 pages of 3 or 4 units a CTA: 2,800 cycles a page, some 9,000 a change of units and 10,000 until the first page) and each
// sequence's own positions 89.
// Rows that save little by it attend by themselves (see the entry point).
//
// Prefix kernel: a unit is (group, KV head, 128 queries: rows times heads); its positions go by in pages of 128, and the pages of all
// units are cut into equal shares, one a CTA.  Four kinds of warps in a row:
//   - one brings a page's codes by bulk copies, two or three pages ahead;
//   - 3 and 3 turn keys and values into fp16 (which holds both formats exactly) in shared memory, swizzled as the tensor core reads them: the same image
//     is K-major for the scores and N-major for the values;
//   - one issues S = Q K^T (128 queries x 128 positions) and O += P V, both tcgen05, Q and P from tensor memory; the next page's scores are
//     made while this one's softmax goes on, two pages of scores in turn;
//   - 8 have the softmax, two threads a query with 64 positions each: maximum, exponentials, P back to tensor memory.
// 8 x 64, us, as they were found: codes made fp16 by the softmax's warps 543, by warps of their own 534, no waits for scales and maxima 491, masks only where a
// query has some 424, scales prepared once a page 414, queries read once 410; 412 with what makes any scale behind a mask safe (blocks looked at
// one by one as they are converted: 423).
// Scales: K's is a factor of the scores; V's of P, so P times V's scale, relative to the query's largest such product so far (2^R),
// is what enters the product, in fp16: 11 bits, or within 2^-31 of the largest.  m and R are raised only when a score or a product
// passes them by 2^8: most pages then need no rescaling of O.
#pragma once
#include <cstddef>

#include "attn_kv8.cuh"

namespace sara {

constexpr int kSharedQ = 128;                       // queries of a unit
constexpr int kSharedSoft = 8, kSharedConv = 3;     // warps of the softmax; that make fp16 of keys, and of values
constexpr int kSharedThreads = 32 * (kSharedSoft + 2 * kSharedConv + 2);
constexpr int kSharedSlots = 4;                     // K and V of two pages
__host__ __device__ constexpr int shared_tile(int hd) { return kSharedQ * 128 * ((hd + 63) / 64); }  // bytes of 128 rows in blocks of 64 dims
__host__ __device__ constexpr int shared_raw(int hd) { return kKv8Page * hd; }                       // of a page's keys or values in codes
__host__ __device__ constexpr int shared_raws(int hd, int v) { return hd == 128 ? 3 - v : 4; }       // of those: keys, values
__host__ __device__ constexpr int shared_smem(int hd) {
    return 1024 + kSharedSlots * shared_tile(hd) + (shared_raws(hd, 0) + shared_raws(hd, 1)) * shared_raw(hd);
}
// Floats of a query's state: outputs, maximum, sum, and two to whole 16 bytes
__host__ __device__ constexpr int shared_state(int hd) { return hd + 4; }
constexpr float kSharedShift = 6.f;                 // log2 of the products' scale
constexpr int kSharedMaxShares = 160;               // CTAs, one an SM
constexpr double kSharedAlone = 160 << 20;         // bytes that it does not pay to share
constexpr int kSharedWideJoin = 1216;               // queries up to which 8 warps join a query

struct SharedGroup {
    int row0, rows;      // its sequences
    int lo, hi;          // the shared positions that one of them attends to
    int page0, pages;
    int tiles;           // of queries, a KV head
    int entry0;          // pages of units before its first
};
struct SharedPlan {      // at the start of the workspace
    int err, entries, pad[62];
};

struct SharedParams {
    Kv8Cache c;
    const uint16_t *q;
    int64_t q_stride;
    const int32_t *ctx, *first, *start, *prefix;
    int n, groups, H, type;
    float scale_log2;
    int32_t *status;
    SharedPlan *plan;
    SharedGroup *group;
    int *row_group, *row_first, *row_prefix;  // [n]: group (-1: none), first own position, shared ones
    float *whole;      // [n][H] states: sums of a unit that one share holds
    float *part;       // [share][2][128] states: of a unit that begins before the share, or in it
    int max_shares;
    // join
    const float *own, *own_lse;  // [n][H][hd], [n][H]
    uint16_t *out;
    float *lse;
};

// ------------------------------------------------------------------------------- plan
// One CTA.  Groups with one sequence, and sequences of no group, are left to the decode attention alone.
__global__ void __launch_bounds__(1024) shared_plan_kernel(SharedParams p) {
    __shared__ int s_warp[32];
    __shared__ int s_bad;
    pdl_allow_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t most = (int64_t)p.c.max_blocks * kKv8Page;
    if (threadIdx.x == 0) {
        s_bad = 0;
        p.plan->err = 0;
    }
    __syncthreads();
    for (int g = threadIdx.x; g < p.groups; g += 1024) {
        const int a = p.start[g], b = p.start[g + 1];
        if (a < 0 || b < a || b > p.n) s_bad = 1;
        SharedGroup x{};
        x.row0 = a;
        x.rows = b - a;
        x.lo = INT32_MAX;
        p.group[g] = x;
    }
    __syncthreads();
    const bool bad = s_bad != 0;
    for (int i = threadIdx.x; i < p.n; i += 1024) {
        int lo = 0, hi = p.groups;  // the last group that begins at i or before
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (p.start[mid] <= i) lo = mid + 1;
            else hi = mid;
        }
        const int g = lo - 1;
        const bool in = !bad && g >= 0 && i < p.start[g + 1];
        const int first = p.first ? p.first[i] : 0, ctx = p.ctx[i], shared = in ? p.prefix[g] : 0;
        const bool wrong = bad || (in && (shared < 0 || shared > most));
        const bool live = in && !wrong && p.start[g + 1] - p.start[g] > 1 && ctx >= 0 && ctx <= most && first >= 0 && min(ctx, shared) > first;
        p.row_group[i] = live ? g : -1;
        p.row_prefix[i] = live ? shared : 0;
        p.row_first[i] = wrong ? -1 : live ? max(first, shared) : first;
        if (live) {
            atomicMin(&p.group[g].lo, first);
            atomicMax(&p.group[g].hi, min(ctx, shared));
        }
    }
    __syncthreads();
    int base = 0;
    for (int g0 = 0; g0 < p.groups; g0 += 1024) {
        const int g = g0 + threadIdx.x;
        int entries = 0;
        SharedGroup x{};
        if (g < p.groups) {
            x = p.group[g];
            x.lo = __ldcg(&p.group[g].lo);
            x.hi = __ldcg(&p.group[g].hi);
            if (bad || x.hi <= x.lo) x.lo = x.hi = 0;
            x.page0 = x.lo / kKv8Page;
            x.pages = x.hi > x.lo ? (x.hi - 1) / kKv8Page - x.page0 + 1 : 0;
            x.tiles = (int)(((int64_t)x.rows * (p.H / p.c.KVH) + kSharedQ - 1) / kSharedQ);
            entries = x.pages * x.tiles * p.c.KVH;
        }
        int end = entries;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, end, d);
            if (lane >= d) end += y;
        }
        __syncthreads();
        if (lane == 31) s_warp[warp] = end;
        __syncthreads();
        const int t = s_warp[lane];
        const int before = __reduce_add_sync(0xffffffffu, lane < warp ? t : 0), all = __reduce_add_sync(0xffffffffu, t);
        if (g < p.groups) {
            x.entry0 = base + before + end - entries;
            p.group[g] = x;
        }
        base += all;
    }
    if (threadIdx.x == 0) {
        p.plan->entries = base;
        if (bad) kv8_report(p.status);
    }
}

// The shares of `entries` over `most` CTAs, and whose an entry is
struct SharedShares {
    int n, each, more;
    __device__ __forceinline__ SharedShares(int entries, int most) {
        n = max(min(most, entries), 1);
        each = entries / n;
        more = entries - each * n;
    }
    __device__ __forceinline__ int begin(int c) const { return c * each + min(c, more); }
    __device__ __forceinline__ int of(int x) const {
        const int big = more * (each + 1);
        return x < big ? x / (each + 1) : more + (x - big) / each;
    }
};

// A share's pages of a unit
struct SharedSegment {
    int count;                  // pages
    int row0, h, q0, queries;   // the group's first row; KV head; first query and number of the unit's queries
    int lo, hi, page;           // the group's positions; the first page
    bool begins, whole;
};
// A warp's way through its share: kept in shared memory, since it is wanted between segments only.
struct SharedWalk {
    int g, e, end, entry1;  // group, next entry, the share's end; the next group's first entry
    SharedGroup x;
    SharedSegment s;        // the present segment
    __device__ __forceinline__ void load(const SharedParams &p) {
        const int4 a = __ldg(reinterpret_cast<const int4 *>(p.group + g)), b = __ldg(reinterpret_cast<const int4 *>(p.group + g) + 1);
        x = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        entry1 = x.entry0 + x.pages * x.tiles * p.c.KVH;
    }
    // (one lane)
    __device__ __forceinline__ void begin(const SharedParams &p, int from, int to) {
        int lo = 0, hi = p.groups;  // the last group that begins at `from` or before
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (__ldg(&p.group[mid].entry0) <= from) lo = mid + 1;
            else hi = mid;
        }
        g = max(lo - 1, 0);
        e = from;
        end = to;
        load(p);
    }
    __device__ __forceinline__ bool advance(const SharedParams &p) {
        if (e >= end) return false;
        while (e >= entry1 && g + 1 < p.groups) {
            ++g;
            load(p);
        }
        const int off = e - x.entry0, unit = off / x.pages, at = off - unit * x.pages, t = unit % x.tiles;
        s.count = min(x.pages - at, end - e);
        s.row0 = x.row0;
        s.h = unit / x.tiles;
        s.q0 = t * kSharedQ;
        s.queries = min(kSharedQ, x.rows * (p.H / p.c.KVH) - s.q0);
        s.lo = x.lo;
        s.hi = x.hi;
        s.page = x.page0 + at;
        s.begins = at == 0;
        s.whole = at == 0 && s.count == x.pages;
        e += s.count;
        return true;
    }
    // The next segment, or false behind the last (a warp)
    __device__ __forceinline__ bool next(const SharedParams &p) {
        __syncwarp();
        bool more = false;
        if ((threadIdx.x & 31) == 0) more = advance(p);
        return __shfl_sync(0xffffffffu, more, 0);  // (orders what lane 0 wrote)
    }
};

// ------------------------------------------------------------------------------- prefix
struct SharedSmem {
    uint64_t raw_full[2][4], raw_empty[2][4], full[kSharedSlots], empty[kSharedSlots], q_full, s_full[2], p_full[2], pv_done;
    float scale[8][3][4];          // of a page's blocks: K's scale, V's as 2^e and what is left, e
    float raw_scale[4][8];         // the same, as they come with the keys
    alignas(16) uint32_t nan[8][2][4];  // blocks of a page in which a warp met a NaN among K's, V's codes, and ([0][3]) those whose scales are none (16: the page itself is none)
    float2 top[2][kSharedQ];       // a query's largest score and product, of either half of a page
    float sum[kSharedQ];           // of the second half's probabilities
    uint32_t size[2][kSharedQ];    // of a query's halves, the largest element in bits
    int block[2][4];               // of a page of codes
    uint32_t tmem_base;
    SharedWalk walk[kSharedThreads / 32];
};

__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 64 or 16 columns of a lane; the wait is part of the instruction, so that nothing uses the values before it
__device__ __forceinline__ void tmem_load64(uint32_t taddr, float (&v)[64]) {
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
        "%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), 
          "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), 
          "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]), "=f"(v[32]), "=f"(v[33]), 
          "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]), "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), 
          "=f"(v[45]), "=f"(v[46]), "=f"(v[47]), "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]), 
          "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t (&r)[16]) {
    __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_store4(uint32_t taddr, const uint4 &x) {
    __syncwarp();
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 columns, waited for with every store before
__device__ __forceinline__ void tmem_store32(uint32_t taddr, const uint32_t (&r)[32]) {
    __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), 
          "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), 
          "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
// Arrive on `bar` when this thread's asynchronous copies so far have come (none: at once)
__device__ __forceinline__ void cp_async_arrive(uint64_t *bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// (bulk_load to a shared-memory address)
__device__ __forceinline__ void bulk_load_at(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
                 "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ uint64_t sdesc_128(uint32_t addr, uint32_t lbo) {  // 128-byte swizzle, 8 rows after 1,024 bytes
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Whether any of the barrier's threads says so
__device__ __forceinline__ bool named_bar_or(int id, int nthreads, bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, %2, %3, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)x), "r"(id), "r"(nthreads)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ float max3(float a, float b, float c) {  // a NaN gives way
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
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
__device__ __forceinline__ void st_shared_v4(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

template <int HD, int FMT>
__global__ void __launch_bounds__(kSharedThreads, 1) shared_prefix_kernel(SharedParams p) {
    constexpr int TILE = shared_tile(HD), RAW = shared_raw(HD), RAWS[2] = {shared_raws(HD, 0), shared_raws(HD, 1)};
    constexpr int CHUNKS = HD / 16, STEP = 32 * kSharedConv / CHUNKS;  // 16-byte pieces of a row; rows that the warps of a tile cover at a time
    constexpr int BATCH = 4;  // of them
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) SharedSmem S;
    const uint32_t ring = (smem_u32(smem_raw) + 1023) & ~1023u, raw = ring + kSharedSlots * TILE;
    constexpr uint32_t O_AT = 256, Q_AT = 384, P_AT = 448;  // tensor memory: two pages' scores, outputs, queries, probabilities
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = p.H / p.c.KVH;
    int *err = &p.plan->err;
    if (threadIdx.x == 0) {
        for (int s = 0; s < 4; ++s) {
            for (int v = 0; v < 2; ++v) {
                mbar_init(&S.raw_full[v][s], v ? 1 : 9);  // (keys come with eight scales)
                mbar_init(&S.raw_empty[v][s], kSharedConv);
            }
            mbar_init(&S.full[s], kSharedConv);
            mbar_init(&S.empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&S.s_full[s], 1);
            mbar_init(&S.p_full[s], kSharedSoft);
        }
        mbar_init(&S.q_full, kSharedSoft);
        mbar_init(&S.pv_done, 1);
        for (int s = 0; s < 8; ++s)
            for (int k = 0; k < 8; ++k) S.nan[s][k / 4][k % 4] = 0;
        fence_mbar_init();
    }
    constexpr int MMA_WARP = kSharedSoft + 2 * kSharedConv, LOAD_WARP = MMA_WARP + 1;
    if (warp == MMA_WARP) {
        tmem_alloc(&S.tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait_prior_grids();
    const uint32_t tmem = S.tmem_base;
    const SharedShares shares(p.plan->entries, min((int)gridDim.x, p.max_shares));
    const int c = blockIdx.x, from = c < shares.n ? shares.begin(c) : 0, to = c < shares.n ? shares.begin(c + 1) : 0;
    SharedWalk &w = S.walk[warp];
    const SharedSegment &s = w.s;
    if (from < to && lane == 0) w.begin(p, from, to);
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity & 1, err)); };

    if (from >= to) {
    } else if (warp == LOAD_WARP) {
        // ------------------------------------------------------------ codes
        uint32_t got[2] = {};  // pages asked for
        // keys, then the values of the page before: keys are wanted earlier, and have more room
        auto bring = [&](auto value, int block, int h) {
            constexpr int v = decltype(value)::value;
            const uint32_t j = got[v], st = j % RAWS[v];
            if (j >= (uint32_t)RAWS[v]) wait(&S.raw_empty[v][st], j / RAWS[v] - 1);
            if (!ok) return;
            if (lane == 0) {
                S.block[v][st] = block;
                if (block >= 0) {
                    mbar_arrive_expect_tx(&S.raw_full[v][st], RAW);
                    bulk_load_at(raw + (v * RAWS[0] + st) * RAW, p.c.codes + kv8_tile(p.c, block, v, h) * (kKv8Page * HD), RAW, &S.raw_full[v][st]);
                } else {
                    mbar_arrive(&S.raw_full[v][st]);
                }
            }
            if (v == 0 && lane < 8) {
                if (block >= 0)
                    cp_async4(smem_u32(&S.raw_scale[st][lane]), p.c.scales + (((int64_t)block * 2 + lane / 4) * p.c.KVH + h) * kKv8PageBlocks + lane % 4);
                cp_async_arrive(&S.raw_full[0][st]);
            }
            __syncwarp();
            ++got[v];
        };
        int last = 0, last_h = -1;  // the page before
        while (ok && w.next(p)) {
            int ids = 0, idbase = -64;
#pragma unroll 1
            for (int x = 0; x < s.count && ok; ++x) {
                const int page = s.page + x;
                if ((unsigned)(page - idbase) >= 32u) {
                    idbase = page;
                    ids = page + lane <= (s.hi - 1) / kKv8Page ? __ldg(p.c.table + s.row0 * p.c.table_stride + page + lane) : 0;
                    if (ids >= p.c.n_blocks) ids = -1;  // (any negative one: none.  Rows that attend to it report it)
                }
                const int block = __shfl_sync(0xffffffffu, ids, page - idbase);
                bring(std::integral_constant<int, 0>(), block, s.h);
                if (last_h >= 0 && ok) bring(std::integral_constant<int, 1>(), last, last_h);
                last = block;
                last_h = s.h;
            }
        }
        if (last_h >= 0 && ok) bring(std::integral_constant<int, 1>(), last, last_h);
        // every copy lands before the CTA ends
        for (int v = 0; v < 2; ++v)
            for (uint32_t q = 1; q <= (uint32_t)RAWS[v] && q <= got[v]; ++q) mbar_wait(&S.raw_full[v][(got[v] - q) % RAWS[v]], ((got[v] - q) / RAWS[v]) & 1, err);
    } else if (warp >= kSharedSoft && warp < MMA_WARP) {
        // ------------------------------------------------------------ codes to fp16
        const int cw = (warp - kSharedSoft) % kSharedConv, ct = cw * 32 + lane;
        const bool value = warp >= kSharedSoft + kSharedConv;
        const uint32_t raws = value ? RAWS[1] : RAWS[0];
        // this thread's row and 16 dims of the first STEP rows (128 dims: 8 lanes have pieces of different halves of two rows, whose places meet
        // all banks)
        const int row = HD == 128 ? ct / 16 * 2 + (ct / 4 & 1) : ct / CHUNKS, d = HD == 128 ? (ct & 3) + 4 * ((ct / 4 ^ ct / 8) & 1) : ct % CHUNKS;
        uint32_t j = 0;
        while (ok && w.next(p)) {
#pragma unroll 1
            for (int x = 0; x < s.count && ok; ++x, ++j) {
                const uint32_t st = j % raws, at = 2 * (j & 1) + value;
                wait(&S.raw_full[value][st], j / raws);
                if (!ok) break;
                const int block = S.block[value][st], p0 = (s.page + x) * kKv8Page;
                const bool cut = block < 0 || p0 < s.lo || p0 + kKv8Page > s.hi;  // positions that nobody attends to are 0: what they hold does not matter
                // (eight places: the page three before has its scores, so that the softmax is done with the one five before, and a page's flags are read in the one
                // behind it, or when the next unit's first scores may have been made)
                // (the warp with the fewest rows.  A block whose scale is NaN or infinite, or negative among keys, reads as NaN: it goes in as 0 with a scale of 1, and is
                // flagged, which reaches the rows that attend to it alone.  So whatever the memory of a block holds that nobody has written does not matter)
                if (!value && cw == kSharedConv - 1) {
                    float k = 1.f, f = 0.f;
                    if (block >= 0 && lane < 4) {
                        k = S.raw_scale[st][lane];
                        f = S.raw_scale[st][4 + lane];
                    }
                    const bool bad = block < 0 || max(__float_as_uint(k), __float_as_uint(f) & 0x7fffffffu) >= 0x7f800000u;
                    const int e = min(max(scale_exp(bad ? 0.f : f), -126), 126);
                    const uint32_t flag = __ballot_sync(0xffffffffu, bad) & 15;
                    if (lane < 4) {
                        S.scale[j & 7][0][lane] = bad ? 1.f : k;
                        S.scale[j & 7][1][lane] = bad ? 0.f : f * pow2f(-e);
                        S.scale[j & 7][2][lane] = (float)e;
                    }
                    if (lane == 0) S.nan[j & 7][0][3] = flag | (block < 0 ? 16u : 0u);
                }
                if (j >= 2) wait(&S.empty[at], (j >> 1) - 1);
                if (!ok) break;
                const uint32_t src = raw + ((value ? RAWS[0] : 0) + st) * RAW + row * HD + 16 * d, slot = ring + at * TILE;
                // the places of dims 16 d .. in the row, as the tensor core reads it; STEP rows on they are the same ones or change sides
                const uint32_t to = slot + (d / 4) * (kSharedQ * 128) + row * 128, place = ((d % 4 * 2) ^ (row & 7)) << 4;
                const uint32_t even[2] = {to + place, to + (place ^ 16)}, odd[2] = {to + (place ^ (STEP % 8 * 16)), to + (place ^ (STEP % 8 * 16) ^ 16)};
                static_assert(STEP % 8 == 0 || STEP % 8 == 4, "an exclusive or is then the sum");
                uint32_t nan = 0;
                __half2 seen = __floats2half2_rn(0.f, 0.f);
                // (not unrolled further: the warps' different parts share the instruction cache)
#pragma unroll 1
                for (int at_row = row, off = 0; at_row < kKv8Page; at_row += BATCH * STEP, off += BATCH * STEP * 128) {
                    uint32_t r[BATCH][4];
#pragma unroll
                    for (int i = 0; i < BATCH; ++i)
                        if (at_row + i * STEP < kKv8Page) load_codes<4>(src + (at_row - row + i * STEP) * HD, r[i]);
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                        const int x = at_row + i * STEP;
                        if (x >= kKv8Page) continue;
                        uint32_t h[8];
                        if (cut) {
                            if (block < 0 || p0 + x < s.lo || p0 + x >= s.hi) r[i][0] = r[i][1] = r[i][2] = r[i][3] = 0;
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) decode4_half<FMT>(r[i][e], h[2 * e], h[2 * e + 1]);
                        if (FMT == SARA_KV8_E4M3) {  // (0, or NaN from a code's on)
#pragma unroll
                            for (int e = 0; e < 8; ++e) seen = __hfma2(*reinterpret_cast<const __half2 *>(&h[e]), __floats2half2_rn(0.f, 0.f), seen);
                        }
                        const uint32_t(&o)[2] = i % 2 ? odd : even;
                        st_shared_v4(o[0] + off + i * STEP * 128, h[0], h[1], h[2], h[3]);
                        st_shared_v4(o[1] + off + i * STEP * 128, h[4], h[5], h[6], h[7]);
                    }
                }
                if (FMT == SARA_KV8_E4M3 && __any_sync(0xffffffffu, __hisnan(__low2half(seen)) || __hisnan(__high2half(seen)))) {
                    // codes 0x7f and 0xff (none that kv8_write writes): their block reads as NaN, and nothing else is to be
#pragma unroll 1
                    for (int x = row; x < kKv8Page; x += STEP) {
                        uint32_t r[4], any = 0;
                        load_codes<4>(src + (x - row) * HD, r);
#pragma unroll
                        for (int e = 0; e < 4; ++e) any |= (r[e] & 0x7f7f7f7fu) + 0x01010101u;
                        if (!(any & 0x80808080u) || p0 + x < s.lo || p0 + x >= s.hi) continue;
                        nan |= 1u << (x / kKv8Block);
                        const uint32_t(&o)[2] = (x - row) / STEP % 2 ? odd : even;
                        st_shared_v4(o[0] + (x - row) * 128, 0, 0, 0, 0);
                        st_shared_v4(o[1] + (x - row) * 128, 0, 0, 0, 0);
                    }
                }
                if (FMT == SARA_KV8_E4M3) {
                    nan = __reduce_or_sync(0xffffffffu, nan);
                    if (lane == 0) S.nan[j & 7][value][cw] = nan;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&S.full[at]);
                    mbar_arrive(&S.raw_empty[value][st]);
                }
            }
        }
    } else if (warp == MMA_WARP) {
        // ------------------------------------------------------------ MMAs
        constexpr uint32_t idesc_s = 1u << 4 | (128u >> 3) << 17 | (128u >> 4) << 24;
        constexpr uint32_t idesc_o = 1u << 4 | 1u << 16 | ((uint32_t)HD >> 3) << 17 | (128u >> 4) << 24;  // values: N-major
        uint32_t j0 = 0, unit = 0, done = 0;  // pages before, units, products issued
        auto scores = [&](uint32_t j) {
            const uint32_t sk = 2 * (j & 1);
            wait(&S.full[sk], j >> 1);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t b = ring + sk * TILE;
#pragma unroll
                for (int k = 0; k < HD / 16; ++k)
                    tc_mma_ts(tmem + (j & 1) * 128, tmem + Q_AT + k * 8, sdesc_128(b + k / 4 * (kSharedQ * 128) + k % 4 * 32, 16), idesc_s, k > 0);
                tc_commit(&S.s_full[j & 1]);
                tc_commit(&S.empty[sk]);
            }
            __syncwarp();
        };
        while (ok && w.next(p)) {
            wait(&S.q_full, unit++);
            if (ok) scores(j0);
            if (ok && s.count > 1) scores(j0 + 1);
#pragma unroll 1
            for (uint32_t x = 0; x < (uint32_t)s.count && ok; ++x) {
                const uint32_t j = j0 + x, sv = 2 * (j & 1) + 1;
                wait(&S.full[sv], j >> 1);
                wait(&S.p_full[j & 1], j >> 1);  // (and the page's scores have been read)
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t b = ring + sv * TILE;
#pragma unroll
                    for (int k = 0; k < 8; ++k) tc_mma_ts(tmem + O_AT, tmem + P_AT + k * 8, sdesc_128(b + k * 2048, kSharedQ * 128), idesc_o, x > 0 || k > 0);
                    tc_commit(&S.pv_done);
                    tc_commit(&S.empty[sv]);
                }
                __syncwarp();
                ++done;
                if (x + 2 < (uint32_t)s.count) scores(j + 2);
            }
            j0 += s.count;
        }
        if (done > 0) mbar_wait(&S.pv_done, (done - 1) & 1, err);  // every MMA has retired before tensor memory is released
    } else if (warp < kSharedSoft) {
        // ------------------------------------------------------------ softmax: a query's first or second 64 positions a thread
        const int quarter = warp & 3, half = warp >> 2, lrow = quarter * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), o_at = lanes + O_AT + half * (HD / 2);
        uint32_t j0 = 0;
        // A unit's query as fp16, one half of it, into tensor memory (the scores of the unit before have been made): its outputs' place, its positions
        // and the factor that brings scores to base-2 exponents
        struct Query {
            float *out;
            float mul;
            int lo, hi;
            bool live, any;
        };
        auto begin = [&]() {
            Query y;
            const int at = s.q0 + lrow;  // among the group's queries
            y.live = lrow < s.queries;
            y.any = __any_sync(0xffffffffu, y.live);
            const int row = s.row0 + (y.live ? at / G : 0), head = s.h * G + (y.live ? at % G : 0);
            y.out = s.whole ? p.whole + ((int64_t)row * p.H + head) * shared_state(HD)
                            : p.part + (((int64_t)c * 2 + s.begins) * kSharedQ + lrow) * shared_state(HD);
            y.mul = p.scale_log2;
            y.lo = y.hi = 0;
            if (y.any) {
                const uint4 *src = reinterpret_cast<const uint4 *>(p.q + row * p.q_stride + (int64_t)head * HD);
                const int first = p.first ? p.first[row] : 0, end = min(p.ctx[row], p.row_prefix[row]), group = p.row_group[row];
                uint4 x[HD / 16];
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) x[i] = __ldg(src + half * (HD / 16) + i);
                float f = 1.f;
                if (p.type == SARA_BF16) {
                    uint32_t top = 0;
#pragma unroll
                    for (int i = 0; i < HD / 16; ++i)
                        top = __vmaxu2(top, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu), __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
                    S.size[half][lrow] = max(top & 0xffff, top >> 16);
                    named_bar_sync(1 + quarter, 64);
                    top = max(S.size[0][lrow], S.size[1][lrow]);
                    const int e = max(min(14 - ((int)(top >> 7) - 127), 126), -113);  // brings the largest magnitude's power of two to 2^14
                    f = pow2f(e);
                    y.mul *= pow2f(-e);
                }
#pragma unroll
                for (int i = 0; i < HD / 16; ++i) {
                    uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                    if (p.type == SARA_BF16) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 g = unpack2<SARA_BF16>(u[e]);
                            u[e] = pack_half2(g.x * f, g.y * f);
                        }
                    }
                    tmem_store4(lanes + Q_AT + (half * (HD / 16) + i) * 4, make_uint4(u[0], u[1], u[2], u[3]));
                }
                if (y.live && group >= 0) {
                    y.lo = first;
                    y.hi = end;
                }
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&S.q_full);
            return y;
        };
        // (after a failed wait the barriers go on, so that no warp is left in one)
        bool more = w.next(p);
        Query next = begin();
        while (more) {
            const Query now = next;
            const bool any = now.any;
            const int lo = now.lo, hi = now.hi, count = s.count, page0 = s.page;
            const float mul = now.mul;
            float m = -3.4028235e38f, R = m, l = 0.f;
            // a block that reads as NaN (bit b: of this half's) makes the sums of those that attend to it NaN, and leaves the others alone
            auto poison = [&](int page, uint32_t bad) {
                const int p0 = page * kKv8Page + 64 * half;
                if ((bad << (2 * half) & 16) && lo < p0 + 64 && hi > p0) kv8_report(p.status);
                if ((bad & 1) && lo < p0 + 32 && hi > p0) l = __int_as_float(0x7fc00000);
                if ((bad & 2) && lo < p0 + 64 && hi > p0 + 32) l = __int_as_float(0x7fc00000);
            };
            // the flags of codes that have gone into a product: a page's when the next one's is asked for
            auto flags = [&](uint32_t j, int page) {
                static_assert(kSharedConv == 3 && offsetof(SharedSmem, nan) % 16 == 0, "a word a warp, read at once");
                uint32_t bad = S.nan[j & 7][0][3];
                if constexpr (FMT == SARA_KV8_E4M3) {
                    const uint4 a = *reinterpret_cast<const uint4 *>(&S.nan[j & 7][0][0]), b = *reinterpret_cast<const uint4 *>(&S.nan[j & 7][1][0]);
                    bad = a.x | a.y | a.z | a.w | b.x | b.y | b.z;
                }
                if (bad >> (2 * half) & 3) poison(page, bad >> (2 * half));
            };
#pragma unroll 1
            for (int x = 0; x < count; ++x) {
                const uint32_t j = j0 + x, s_at = lanes + (j & 1) * 128 + half * 64;
                // the product before this page's has been taken (every page waits for it once: a phase later its parity would not tell)
                bool waited = j == 0;
                auto before = [&]() {
                    if (!waited) {
                        wait(&S.pv_done, j - 1);
                        tc_fence_after();
                    }
                    waited = true;
                };
                wait(&S.s_full[j & 1], j >> 1);  // (the page's scales were there before its keys)
                if (any) {
                    tc_fence_after();
                    const int p0 = (page0 + x) * kKv8Page + 64 * half;
                    // its positions from `skip` on, `take` of them; a query that attends to none has all of them, and exponents of -1e30
                    const bool none = lo >= p0 + 64 || hi <= p0;
                    const int skip = none ? 0 : max(lo - p0, 0), take = none ? 64 : min(hi - p0, 64) - skip;
                    float v[64], ks[2], F[2], ev[2];
                    tmem_load64(s_at, v);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        // (a masked product is -inf times this, which may not be 0 then.  A factor below 2^-126, of a query or keys of zeros, counts as that: |q k| <= 2^32
                        // here, so the scores stay 0 beside any that counts)
                        ks[b] = fmaxf(S.scale[j & 7][0][2 * half + b] * mul, 0x1p-126f);
                        F[b] = S.scale[j & 7][1][2 * half + b];
                        ev[b] = S.scale[j & 7][2][2 * half + b];
                    }
                    if (__any_sync(0xffffffffu, take < 64)) {
#pragma unroll
                        for (int e = 0; e < 64; ++e) v[e] = (unsigned)(e - skip) < (unsigned)take ? v[e] : -INFINITY;
                    }
                    float2 top = make_float2(-INFINITY, -INFINITY);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        float n = fmaxf(v[32 * b], v[32 * b + 1]), n1 = fmaxf(v[32 * b + 2], v[32 * b + 3]);
#pragma unroll
                        for (int e = 4; e < 32; e += 4) {
                            n = max3(n, v[32 * b + e], v[32 * b + e + 1]);
                            n1 = max3(n1, v[32 * b + e + 2], v[32 * b + e + 3]);
                        }
                        n = fmaxf(n, n1);
                        n *= ks[b];
                        top.x = fmaxf(top.x, n);
                        top.y = fmaxf(top.y, n + ev[b]);
                    }
                    if (none) top = make_float2(-INFINITY, -INFINITY);
                    if (named_bar_or(1 + quarter, 64, top.x > m + 8.f || top.y > R + 8.f)) {  // of either half: both raise the same
                        S.top[half][lrow] = top;
                        named_bar_sync(1 + quarter, 64);
                        const float2 other = S.top[half ^ 1][lrow];
                        top.x = fmaxf(top.x, other.x);
                        top.y = fmaxf(top.y, other.y);
                        const bool raise = top.x > m + 8.f || top.y > R + 8.f;
                        const float m1 = raise ? fmaxf(m, top.x) : m, R1 = raise ? fmaxf(R, top.y) : R;
                        l *= ex2(fmaxf(m - m1, -1e4f));
                        const float f = ex2(fmaxf(R - R1, -1e4f));
                        m = m1;
                        R = R1;
                        if (x > 0) {
                            before();
#pragma unroll 1
                            for (int d = 0; d < HD / 2; d += 16) {
                                float o[16];
                                tmem_load16(o_at + d, o);
                                uint32_t y[16];
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(o[e] * f);
                                tmem_st_x16(o_at + d, y);
                            }
                        }
                    }
                    uint64_t l2 = 0;  // two sums
                    uint32_t h[32];
                    const float off = none ? -1e30f : -m;
                    const uint64_t m2 = pack_f32x2(off, off);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const float f = F[b] * ex2(fminf(m - R + ev[b] + kSharedShift, 126.f));
                        const float k = none ? 0.f : ks[b];
                        const uint64_t k2 = pack_f32x2(k, k), f2 = pack_f32x2(f, f);
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const float2 y = unpack_f32x2(fma_f32x2(pack_f32x2(v[32 * b + e], v[32 * b + e + 1]), k2, m2));
                            const uint64_t a = pack_f32x2(ex2(y.x), ex2(y.y));
                            l2 = add_f32x2(l2, a);
                            const float2 w = unpack_f32x2(mul_f32x2(a, f2));
                            h[16 * b + e / 2] = pack_half2(w.x, w.y);
                        }
                    }
                    l += unpack_f32x2(l2).x + unpack_f32x2(l2).y;
                    before();
                    tmem_store32(lanes + P_AT + half * 32, h);
                    if (x > 0) flags(j - 1, page0 + x - 1);
                }
                before();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.p_full[j & 1]);
            }
            // the next unit's queries go in before this one's outputs come out, so that its scores are made meanwhile
            more = w.next(p);
            if (more) next = begin();
            wait(&S.pv_done, j0 + count - 1);
            if (any) {
                flags(j0 + count - 1, page0 + count - 1);
                if (half) S.sum[lrow] = l;
                named_bar_sync(1 + quarter, 64);
                tc_fence_after();
                const float f = ex2(fminf(fmaxf(R - m - kSharedShift, -1e4f), 126.f));
#pragma unroll 1
                for (int d = 0; d < HD / 2; d += 16) {
                    float y[16];
                    tmem_load16(o_at + d, y);
                    if (now.live) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4)
                            *reinterpret_cast<float4 *>(now.out + half * (HD / 2) + d + e) = make_float4(y[e] * f, y[e + 1] * f, y[e + 2] * f, y[e + 3] * f);
                    }
                }
                if (now.live && !half) *reinterpret_cast<float2 *>(now.out + HD) = make_float2(m, l + S.sum[lrow]);
                named_bar_sync(1 + quarter, 64);  // (the sums have been read)
            }
            tc_fence_before();
            j0 += count;
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == MMA_WARP) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------------------- join
template <int N>
__device__ __forceinline__ void vec_load(const float *p, float (&y)[N]) {
    if constexpr (N == 4) {
        const float4 x = *reinterpret_cast<const float4 *>(p);
        y[0] = x.x, y[1] = x.y, y[2] = x.z, y[3] = x.w;
    } else if constexpr (N == 2) {
        const float2 x = *reinterpret_cast<const float2 *>(p);
        y[0] = x.x, y[1] = x.y;
    } else {
        y[0] = *p;
    }
}
// A query's state of its own positions and those of its shared ones, W warps to a query; D neighbouring dims a lane
template <int HD, int W>
__global__ void __launch_bounds__(256) shared_join_kernel(SharedParams p, int shares_most) {
    constexpr int D = HD / 32;
    __shared__ float s_m[8], s_l[8];
    __shared__ __align__(16) float s_o[8][HD];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = W == 1 ? 0 : warp;
    const int64_t x = W == 1 ? (int64_t)blockIdx.x * 8 + warp : blockIdx.x;
    if (x >= (int64_t)p.n * p.H) return;
    const int row = (int)(x / p.H), head = (int)(x - (int64_t)row * p.H), G = p.H / p.c.KVH;
    float m = -3.4028235e38f, l = 0.f, o[D] = {};
    auto add = [&](float m1, float l1, const float *src) {
        float y[D];
        vec_load<D>(src + D * lane, y);
        const float n = fmaxf(m, m1), a = ex2(fmaxf(m - n, -1e4f)), down = m1 - n, b = ex2(down < -1e4f ? -1e4f : down);  // (a NaN stays)
        m = n;
        l = fmaf(l1, b, l * a);
#pragma unroll
        for (int d = 0; d < D; ++d) o[d] = fmaf(y[d], b, o[d] * a);
    };
    const int g = p.row_group[row];
    if (part == 0) {  // (of no position: -inf; a NaN stays)
        const float own = p.own_lse[x];
        if (!(own == -INFINITY)) add(own * 1.44269504f, 1.f, p.own + x * HD);
    }
    if (g >= 0) {
        const SharedGroup y = p.group[g];
        const SharedShares shares(p.plan->entries, shares_most);
        const int at = (row - y.row0) * G + head % G, e0 = y.entry0 + (head / G * y.tiles + at / kSharedQ) * y.pages;
        const int c0 = shares.of(e0), c1 = shares.of(e0 + y.pages - 1);
        if (c0 == c1) {
            const float *s = p.whole + x * shared_state(HD);
            if (part == 0) add(s[HD], s[HD + 1], s);
        } else {
#pragma unroll 4
            for (int c = c0 + part; c <= c1; c += W) {
                const float *s = p.part + (((int64_t)c * 2 + (c == c0)) * kSharedQ + at % kSharedQ) * shared_state(HD);
                add(s[HD], s[HD + 1], s);
            }
        }
    }
    if constexpr (W > 1) {
        if (lane == 0) {
            s_m[warp] = m;
            s_l[warp] = l;
        }
#pragma unroll
        for (int d = 0; d < D; ++d) s_o[warp][D * lane + d] = o[d];
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int k = 1; k < W; ++k) add(s_m[k], s_l[k], s_o[k]);
    }
    // (nothing anywhere: 0 and -inf.  A failed wait: NaN)
    const bool none = l == 0.f;
    const float inv = p.plan->err ? __int_as_float(0x7fc00000) : none ? 0.f : 1.f / l;
    uint16_t *out = p.out + x * HD + D * lane;
    if constexpr (D == 1) {
        *out = p.type == SARA_BF16 ? f32_to_bf16(o[0] * inv) : __half_as_ushort(__float2half_rn(o[0] * inv));
    } else {
        uint32_t y[D / 2];
#pragma unroll
        for (int d = 0; d < D; d += 2)
            y[d / 2] = p.type == SARA_BF16 ? pack2<SARA_BF16>(o[d] * inv, o[d + 1] * inv) : pack2<SARA_FP16>(o[d] * inv, o[d + 1] * inv);
        if constexpr (D == 4) *reinterpret_cast<uint2 *>(out) = make_uint2(y[0], y[1]);
        else *reinterpret_cast<uint32_t *>(out) = y[0];
    }
    if (p.lse && lane == 0) p.lse[x] = none ? -INFINITY : (m + log2f(l)) * 0.69314718f;
}

}  // namespace sara
