// Decode attention over the 8-bit paged cache for groups of sequences whose first positions are the same: the shared ones are
// computed once for all of a group's queries, each sequence's own by the decode attention, and the two are joined,
//     out = (2^(m1 - m) o1 + 2^(m2 - m) o2) / (2^(m1 - m) l1 + 2^(m2 - m) l2),   m = max(m1, m2).
// Bound by reading the shared positions once (2 hd bytes each) up to some 128 queries a KV head, by the tensor cores beyond.
//
// Prefix kernel: a unit is (group, KV head, 128 QT queries: rows times heads); its positions go by in pages of 128, and the pages of
// all units are cut into equal shares, one a CTA.  Three kinds of warps in a row:
//   - 8 warps bring codes, by plain loads a page or two ahead, and leave them in shared memory as fp16 (which holds both formats exactly), swizzled
//     as the tensor core reads them: the same image is K-major for the scores and N-major for the values;
//   - one issues S = Q K^T (128 queries x 128 positions) and O += P V, P from tensor memory, both tcgen05;
//   - 4 warps per 128 queries, a query a thread: maximum, exponentials, P back to tensor memory in the place of S.
// Scales: K's is a factor of the scores; V's of P, so P times V's scale, relative to the query's largest such product so far (2^R),
// is what enters the product, in fp16: 11 bits, or within 2^-31 of the largest.  m and R are raised only when a score or a product
// passes them by 2^8: most pages then need no rescaling of O.
#pragma once
#include "attn_kv8.cuh"

namespace sara {

constexpr int kSharedQ = 128, kSharedConv = 8;      // queries of a tile; warps that bring codes
constexpr int kSharedSlots = 4;                     // K and V of two pages
constexpr float kSharedShift = 6.f;                 // log2 of the products' scale
constexpr int kSharedMaxShares = 160;               // CTAs, one an SM
constexpr int kSharedWideJoin = 1216;               // queries up to which 8 warps join a query
__host__ __device__ constexpr int shared_warps(int qt) { return 4 * qt + kSharedConv + 1; }
__host__ __device__ constexpr int shared_threads(int qt) { return 32 * shared_warps(qt); }
__host__ __device__ constexpr int shared_tile(int hd) { return kSharedQ * 128 * ((hd + 63) / 64); }  // bytes of 128 rows in blocks of 64 dims
__host__ __device__ constexpr int shared_smem(int hd, int qt) { return 1024 + (qt + kSharedSlots) * shared_tile(hd); }

struct SharedGroup {
    int row0, rows;      // its sequences
    int lo, hi;          // the shared positions that one of them attends to
    int page0, pages;
    int tiles;           // of queries, a KV head
    int entry0;          // pages of units before its first
};
struct SharedPlan {      // at the start of the workspace
    int err, entries, bad, pad[61];
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
    float *whole;      // [n][H][hd + 2]: sums of a unit that one share holds: maximum, sum, outputs
    float *part;       // [share][2][128 QT][hd + 2]: of a unit that begins before the share, or in it
    int max_shares;
    // join
    const float *own, *own_lse;  // [n][H][hd], [n][H]
    uint16_t *out;
    float *lse;
};

// ------------------------------------------------------------------------------- plan
// One CTA.  Groups with one sequence, and sequences of no group, are left to the decode attention alone.
template <int TQ>
__global__ void __launch_bounds__(1024) shared_plan_kernel(SharedParams p) {
    __shared__ int s_warp[32];
    __shared__ int s_bad;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t most = (int64_t)p.c.max_blocks * kKv8Page;
    if (threadIdx.x == 0) s_bad = 0;
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
            x.tiles = (int)(((int64_t)x.rows * (p.H / p.c.KVH) + TQ - 1) / TQ);
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
    int e, count;               // first entry, pages
    int row0, h, q0, queries;   // the group's first row; KV head; first query and number of the unit's queries
    int lo, hi, page;           // the group's positions; the first page
    bool begins, whole;
};
struct SharedWalk {
    const SharedParams &p;
    int g, e, end;
    SharedGroup x;
    int entry1;  // of the next group
    __device__ __forceinline__ SharedWalk(const SharedParams &p_, int from, int to) : p(p_), g(0), e(from), end(to) {
        int hi = p.groups;  // the last group that begins at `from` or before
        while (g < hi) {
            const int mid = (g + hi) / 2;
            if (__ldg(&p.group[mid].entry0) <= from) g = mid + 1;
            else hi = mid;
        }
        g = max(g - 1, 0);
        load();
    }
    __device__ __forceinline__ void load() {
        const int4 a = __ldg(reinterpret_cast<const int4 *>(p.group + g)), b = __ldg(reinterpret_cast<const int4 *>(p.group + g) + 1);
        x = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        entry1 = x.entry0 + x.pages * x.tiles * p.c.KVH;
    }
    template <int TQ>
    __device__ __forceinline__ bool next(SharedSegment &s) {
        if (e >= end) return false;
        while (e >= entry1 && g + 1 < p.groups) {
            ++g;
            load();
        }
        const int off = e - x.entry0, unit = off / x.pages, at = off - unit * x.pages, t = unit % x.tiles;
        s.e = e;
        s.count = min(x.pages - at, end - e);
        s.row0 = x.row0;
        s.h = unit / x.tiles;
        s.q0 = t * TQ;
        s.queries = min(TQ, x.rows * (p.H / p.c.KVH) - s.q0);
        s.lo = x.lo;
        s.hi = x.hi;
        s.page = x.page0 + at;
        s.begins = at == 0;
        s.whole = at == 0 && s.count == x.pages;
        e += s.count;
        return true;
    }
};

// ------------------------------------------------------------------------------- prefix
struct SharedSmem {
    uint64_t full[kSharedSlots], empty[kSharedSlots], scales[4], q_full[2], s_full[2], p_full[2], pv_done[2], o_full[2];
    float scale[4][8];       // of a page: K's four, V's four
    uint32_t nan[4][kSharedConv];  // blocks of a page in which a warp met a NaN among V's codes
    uint32_t tmem_base;
    int abort;
};

__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 32 or 16 columns of a lane; the wait is part of the instruction, so that nothing uses the values before it
__device__ __forceinline__ void tmem_load32(uint32_t taddr, float (&v)[32]) {
    uint32_t r[32];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
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
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint64_t sdesc_128(uint32_t addr, uint32_t lbo) {  // 128-byte swizzle, 8 rows after 1,024 bytes
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void st_shared_v4(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// QT: tiles of 128 queries that share a page
template <int HD, int FMT, int QT>
__global__ void __launch_bounds__(shared_threads(QT), 1) shared_prefix_kernel(SharedParams p) {
    constexpr int TILE = shared_tile(HD), TQ = kSharedQ * QT;
    constexpr int CHUNKS = HD / 16, LOADS = kKv8Page * CHUNKS / (32 * kSharedConv);  // 16-byte pieces of a row, of a thread
    constexpr int AHEAD = QT == 1 ? 2 : 1;  // pages on their way
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) SharedSmem S;
    const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;  // queries, then the slots
    const uint32_t ring = base + QT * TILE;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = p.H / p.c.KVH;
    int *err = &p.plan->err;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kSharedSlots; ++s) {
            mbar_init(&S.full[s], kSharedConv);
            mbar_init(&S.empty[s], 1);
            mbar_init(&S.scales[s], kSharedConv);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&S.q_full[s], 4);
            mbar_init(&S.s_full[s], 1);
            mbar_init(&S.p_full[s], 4);
            mbar_init(&S.pv_done[s], 1);
            mbar_init(&S.o_full[s], 1);
        }
        S.abort = 0;
        fence_mbar_init();
    }
    constexpr int MMA_WARP = 4 * QT + kSharedConv;
    if (warp == MMA_WARP) {
        tmem_alloc(&S.tmem_base, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = S.tmem_base;
    volatile int *ab = &S.abort;
    const SharedShares shares(p.plan->entries, min((int)gridDim.x, p.max_shares));
    const int c = blockIdx.x, from = c < shares.n ? shares.begin(c) : 0, to = c < shares.n ? shares.begin(c + 1) : 0;

    if (from >= to) {
    } else if (warp >= 4 * QT && warp < MMA_WARP) {
        // ------------------------------------------------------------ codes to fp16
        const int cw = warp - 4 * QT, ct = cw * 32 + lane;
        // the pages that are loaded run ahead of those that are stored
        SharedWalk lw(p, from, to), sw(p, from, to);
        SharedSegment ls, ss;
        int l_at = 0, s_at = 0, ids = 0, idbase = -64;
        bool wrong = false, more = lw.next<TQ>(ls);
        uint4 kr[AHEAD][LOADS], vr[AHEAD][LOADS];
        int valid[AHEAD];  // whether the page's id is right
        // pieces ct, ct + 256, ... of the page's 128 CHUNKS
        auto load = [&](int a) {
            if (more && l_at == ls.count) {
                more = lw.next<TQ>(ls);
                l_at = 0;
                idbase = -64;
            }
            if (!more) return;
            const int page = ls.page + l_at;
            if ((unsigned)(page - idbase) >= 32u) {
                idbase = page;
                ids = page + lane <= (ls.hi - 1) / kKv8Page ? __ldg(p.c.table + ls.row0 * p.c.table_stride + page + lane) : 0;
                if (ids < 0 || ids >= p.c.n_blocks) {
                    wrong = true;
                    ids = -1;
                }
            }
            const int block = __shfl_sync(0xffffffffu, ids, page - idbase);
            valid[a] = block;
            const int p0 = page * kKv8Page;
            const uint8_t *k = p.c.codes + kv8_tile(p.c, max(block, 0), 0, ls.h) * (kKv8Page * HD) + 16 * ct;
            const uint8_t *v = k + (int64_t)p.c.KVH * (kKv8Page * HD);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {  // (positions that nobody attends to are not read)
                const int at = p0 + (ct + 32 * kSharedConv * i) / CHUNKS;
                const bool on = block >= 0 && at >= ls.lo && at < ls.hi;
                kr[a][i] = on ? __ldg(reinterpret_cast<const uint4 *>(k + 16 * 32 * kSharedConv * i)) : make_uint4(0, 0, 0, 0);
                vr[a][i] = on ? __ldg(reinterpret_cast<const uint4 *>(v + 16 * 32 * kSharedConv * i)) : make_uint4(0, 0, 0, 0);
            }
            ++l_at;
        };
        auto store = [&](uint32_t slot, const uint4 (&x)[LOADS]) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int piece = ct + 32 * kSharedConv * i, row = piece / CHUNKS, d = piece % CHUNKS;  // dims 16 d ..
                uint32_t h[8];
                decode4_half<FMT>(x[i].x, h[0], h[1]);
                decode4_half<FMT>(x[i].y, h[2], h[3]);
                decode4_half<FMT>(x[i].z, h[4], h[5]);
                decode4_half<FMT>(x[i].w, h[6], h[7]);
                const uint32_t at = slot + (d / 4) * (kSharedQ * 128) + row * 128, c0 = d % 4 * 2;
                // (the second 64 dims' pieces the other way round, so that lanes of a row meet all banks)
                const bool turn = d >= 4;
                const uint32_t a0 = at + (((c0 + turn) ^ (row & 7)) << 4), a1 = at + (((c0 + !turn) ^ (row & 7)) << 4);
                st_shared_v4(a0, turn ? h[4] : h[0], turn ? h[5] : h[1], turn ? h[6] : h[2], turn ? h[7] : h[3]);
                st_shared_v4(a1, turn ? h[0] : h[4], turn ? h[1] : h[5], turn ? h[2] : h[6], turn ? h[3] : h[7]);
            }
        };
        auto give = [&](uint64_t *bar) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        bool ok = true;
        uint32_t j = 0;  // pages stored
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) load(a);
        int a = 0;
        for (bool live = sw.next<TQ>(ss); live && ok; live = sw.next<TQ>(ss)) {
            const int64_t tiles = (int64_t)ss.h;
            for (s_at = 0; s_at < ss.count && ok; ++s_at, ++j) {
                auto step = [&](auto slot_of) {
                    constexpr int A = decltype(slot_of)::value;
                    const uint32_t sk = 2 * (j & 1), sv = sk + 1, ph = ((j >> 1) & 1) ^ 1;
                    const int block = valid[A];
                    if (cw == 0 && lane < 8) {  // (slot j & 3: read long ago when page j - 4's went)
                        float f = __int_as_float(0x7fc00000);
                        if (block >= 0) f = __ldg(p.c.scales + (((int64_t)block * 2 + lane / 4) * p.c.KVH + tiles) * kKv8PageBlocks + lane % 4);
                        S.scale[j & 3][lane] = f;
                    }
                    if (j >= 2) ok = __all_sync(0xffffffffu, mbar_wait(&S.empty[sk], ph, err) && !*ab);
                    if (!ok) return;
                    store(ring + sk * TILE, kr[A]);
                    give(&S.full[sk]);
                    uint32_t nan = 0;
                    if constexpr (FMT == SARA_KV8_E4M3) {  // codes 0x7f and 0xff: their block reads as NaN, and 0 times them must not
#pragma unroll
                        for (int i = 0; i < LOADS; ++i) {
                            const uint32_t w[4] = {vr[A][i].x, vr[A][i].y, vr[A][i].z, vr[A][i].w};
                            uint32_t any = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) any |= ((w[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                            if (any) {
                                nan |= 1u << ((ct + 32 * kSharedConv * i) / CHUNKS / kKv8Block);
                                vr[A][i] = make_uint4(0, 0, 0, 0);
                            }
                        }
                        nan = __reduce_or_sync(0xffffffffu, nan);
                    }
                    if (j >= 2) ok = __all_sync(0xffffffffu, mbar_wait(&S.empty[sv], ph, err) && !*ab);
                    if (!ok) return;
                    store(ring + sv * TILE, vr[A]);
                    if (lane == 0) S.nan[j & 3][cw] = nan;
                    give(&S.full[sv]);
                    if (lane == 0) mbar_arrive(&S.scales[j & 3]);
                    load(A);
                };
                if (AHEAD == 1 || a == 0) step(std::integral_constant<int, 0>());
                else step(std::integral_constant<int, AHEAD - 1>());
                a = a + 1 == AHEAD ? 0 : a + 1;
            }
        }
        if (!ok) *ab = 1;
        if (wrong) kv8_report(p.status);
    } else if (warp == MMA_WARP) {
        // ------------------------------------------------------------ MMAs
        constexpr uint32_t idesc_s = 1u << 4 | (128u >> 3) << 17 | (128u >> 4) << 24;
        constexpr uint32_t idesc_o = 1u << 4 | 1u << 16 | ((uint32_t)HD >> 3) << 17 | (128u >> 4) << 24;  // values: N-major
        SharedWalk w(p, from, to);
        SharedSegment s;
        uint32_t j0 = 0, unit[2] = {}, done[2] = {};  // pages before; per tile of queries: units, products issued
        bool ok = true;
        auto wait = [&](uint64_t *bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity & 1, err) && !*ab); };
        while (ok && w.next<TQ>(s)) {
            const int nq = QT == 1 ? 1 : (s.queries + kSharedQ - 1) / kSharedQ;
            auto scores = [&](int q, uint32_t x) {  // of the segment's page x
                const uint32_t j = j0 + x, sk = 2 * (j & 1);
                if (q == 0) wait(&S.full[sk], j >> 1);
                const uint32_t buf = QT == 1 ? j & 1 : (uint32_t)q;
                // its place holds the probabilities of an earlier page until their product is done
                if (done[q] > 0) wait(&S.pv_done[q], done[q] - 1);
                if (!ok) return;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t a = base + q * TILE, b = ring + sk * TILE;
#pragma unroll
                    for (int k = 0; k < HD / 16; ++k)
                        tc_mma_bf16(tmem + buf * 128, sdesc_128(a + k / 4 * (kSharedQ * 128) + k % 4 * 32, 16),
                                    sdesc_128(b + k / 4 * (kSharedQ * 128) + k % 4 * 32, 16), idesc_s, k > 0);
                    if (q == nq - 1) tc_commit(&S.empty[sk]);
                    tc_commit(&S.s_full[buf]);
                }
                __syncwarp();
            };
            auto values = [&](int q, uint32_t x) {
                const uint32_t j = j0 + x, sv = 2 * (j & 1) + 1, buf = QT == 1 ? j & 1 : (uint32_t)q;
                if (q == 0) wait(&S.full[sv], j >> 1);
                wait(&S.p_full[buf], QT == 1 ? j >> 1 : done[q]);
                if (!ok) return;
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t b = ring + sv * TILE;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        tc_mma_ts(tmem + 256 + q * 128, tmem + buf * 128 + k * 8, sdesc_128(b + k * 2048, kSharedQ * 128), idesc_o, x > 0 || k > 0);
                    if (q == nq - 1) tc_commit(&S.empty[sv]);
                    tc_commit(&S.pv_done[q]);
                    if (x + 1 == (uint32_t)s.count) tc_commit(&S.o_full[q]);
                }
                __syncwarp();
                ++done[q];
            };
            for (int q = 0; q < nq; ++q) wait(&S.q_full[q], unit[q]++);
            for (int q = 0; q < nq && ok; ++q) scores(q, 0);
#pragma unroll 1
            for (uint32_t x = 0; x < (uint32_t)s.count && ok; ++x) {
                if (QT == 1) {
                    if (x + 1 < (uint32_t)s.count) scores(0, x + 1);
                    if (ok) values(0, x);
                } else {
                    for (int q = 0; q < nq && ok; ++q) values(q, x);
                    for (int q = 0; q < nq && ok && x + 1 < (uint32_t)s.count; ++q) scores(q, x + 1);
                }
            }
            j0 += s.count;
        }
        if (!ok) *ab = 1;
        // every MMA has retired before tensor memory is released: the last commits
        for (int q = 0; q < QT; ++q)
            if (done[q] > 0) mbar_wait(&S.pv_done[q], (done[q] - 1) & 1, err);
    } else if (warp < 4 * QT) {
        // ------------------------------------------------------------ softmax, a query a thread
        const int qt = warp >> 2, lrow = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), o_at = lanes + 256 + qt * 128;
        SharedWalk w(p, from, to);
        SharedSegment s;
        uint32_t j0 = 0, tile = 0, unit = 0;  // pages before; pages and units of this tile of queries
        bool ok = true;
        auto wait = [&](uint64_t *bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity & 1, err) && !*ab); };
        while (ok && w.next<TQ>(s)) {
            if (QT == 2 && qt * kSharedQ >= s.queries) {  // (no query of this tile)
                j0 += s.count;
                continue;
            }
            const int at = s.q0 + qt * kSharedQ + lrow;  // among the group's queries
            const bool live = qt * kSharedQ + lrow < s.queries;
            const int row = s.row0 + (live ? at / G : 0), head = s.h * G + (live ? at % G : 0);
            const bool any = __any_sync(0xffffffffu, live);
            // the query, as fp16
            float mul = p.scale_log2;
            int lo = 0, hi = 0;
            {
                const uint4 *src = reinterpret_cast<const uint4 *>(p.q + row * p.q_stride + (int64_t)head * HD);
                uint32_t top = 0;
                float f = 1.f;
                if (live && p.type == SARA_BF16) {
#pragma unroll
                    for (int i = 0; i < HD / 8; ++i) {
                        const uint4 x = __ldg(src + i);
                        top = __vmaxu2(top, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
                    }
                    top = max(top & 0xffff, top >> 16);
                    const int e = max(min(14 - ((int)(top >> 7) - 127), 126), -113);  // brings the largest magnitude's power of two to 2^14
                    f = pow2f(e);
                    mul *= pow2f(-e);
                }
                const uint32_t to = base + qt * TILE + lrow * 128;
#pragma unroll
                for (int i = 0; i < HD / 8; ++i) {
                    uint4 x = live ? __ldg(src + i) : make_uint4(0, 0, 0, 0);
                    if (p.type == SARA_BF16) {
                        uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 z = unpack2<SARA_BF16>(y[e]);
                            y[e] = pack_half2(z.x * f, z.y * f);
                        }
                        x = make_uint4(y[0], y[1], y[2], y[3]);
                    }
                    st_shared_v4(to + i / 8 * (kSharedQ * 128) + (((i % 8) ^ (lrow & 7)) << 4), x.x, x.y, x.z, x.w);
                }
                if (live && p.row_group[row] >= 0) {
                    lo = p.first ? p.first[row] : 0;
                    hi = min(p.ctx[row], p.row_prefix[row]);
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&S.q_full[qt]);

            float m = -3.4028235e38f, R = m, l = 0.f;
#pragma unroll 1
            for (int x = 0; x < s.count && ok; ++x, ++tile) {
                const uint32_t j = j0 + x, buf = QT == 1 ? j & 1 : (uint32_t)qt;
                const uint32_t s_at = lanes + buf * 128;
                wait(&S.s_full[buf], QT == 1 ? j >> 1 : tile);
                wait(&S.scales[j & 3], j >> 2);
                if (!ok) break;
                tc_fence_after();
                if (any) {
                    float ks[4], vs[4], ev[4];
                    uint32_t bad = 0;
                    if constexpr (FMT == SARA_KV8_E4M3) {
                        const uint4 b0 = *reinterpret_cast<const uint4 *>(&S.nan[j & 3][0]), b1 = *reinterpret_cast<const uint4 *>(&S.nan[j & 3][4]);
                        bad = b0.x | b0.y | b0.z | b0.w | b1.x | b1.y | b1.z | b1.w;
                    }
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        ks[b] = S.scale[j & 3][b] * mul;
                        vs[b] = bad >> b & 1 ? __int_as_float(0x7fc00000) : S.scale[j & 3][4 + b];
                        ev[b] = (float)min(max(scale_exp(vs[b]), -126), 126);
                    }
                    const int p0 = (s.page + x) * kKv8Page;
                    const bool masked = __any_sync(0xffffffffu, lo > p0 || hi < p0 + kKv8Page);
                    float most = -INFINITY, product = -INFINITY;
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        float v[32];
                        tmem_load32(s_at + 32 * b, v);
                        if (masked) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = p0 + 32 * b + e >= lo && p0 + 32 * b + e < hi ? v[e] : -INFINITY;
                        }
                        float n = fmaxf(v[0], v[1]);
#pragma unroll
                        for (int e = 2; e < 32; ++e) n = fmaxf(n, v[e]);
                        n *= ks[b];
                        most = fmaxf(most, n);
                        product = fmaxf(product, n + ev[b]);
                    }
                    const bool raise = most > m + 8.f || product > R + 8.f;
                    if (__any_sync(0xffffffffu, raise)) {
                        const float m1 = raise ? fmaxf(m, most) : m, R1 = raise ? fmaxf(R, product) : R;
                        l *= ex2(fmaxf(m - m1, -1e4f));
                        const float f = ex2(fmaxf(R - R1, -1e4f));
                        m = m1;
                        R = R1;
                        if (x > 0) {
                            wait(&S.pv_done[qt], tile - 1);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int d = 0; d < HD; d += 16) {
                                float o[16];
                                tmem_load16(o_at + d, o);
                                uint32_t y[16];
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(o[e] * f);
                                tmem_st_x16(o_at + d, y);
                            }
                            tmem_wait_st();
                        }
                    }
                    float l0 = 0.f, l1 = 0.f;
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        float v[32];
                        tmem_load32(s_at + 32 * b, v);
                        const float F = ex2(fminf(m - R + ev[b] + kSharedShift, 126.f)) * (vs[b] * pow2f(-(int)ev[b]));
                        uint32_t h[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float a0 = ex2(fmaf(v[e], ks[b], -m)), a1 = ex2(fmaf(v[e + 1], ks[b], -m));
                            float w0 = a0 * F, w1 = a1 * F;
                            if (masked) {
                                const int at0 = p0 + 32 * b + e;
                                const bool on0 = at0 >= lo && at0 < hi, on1 = at0 + 1 >= lo && at0 + 1 < hi;
                                a0 = on0 ? a0 : 0.f;
                                a1 = on1 ? a1 : 0.f;
                                w0 = on0 ? w0 : 0.f;
                                w1 = on1 ? w1 : 0.f;
                            }
                            l0 += a0;
                            l1 += a1;
                            h[e / 2] = pack_half2(w0, w1);
                        }
                        tmem_st_x16(s_at + 16 * b, h);
                    }
                    l += l0 + l1;
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&S.p_full[buf]);
            }
            // (not pv_done, which may be two pages behind a warp that has just left the last: its parity would not tell)
            wait(&S.o_full[qt], unit++);
            if (!ok) break;
            tc_fence_after();
            if (any) {
                float *o = s.whole ? p.whole + ((int64_t)row * p.H + head) * (HD + 2)
                                   : p.part + (((int64_t)c * 2 + s.begins) * TQ + qt * kSharedQ + lrow) * (HD + 2);
                const float f = ex2(fminf(fmaxf(R - m - kSharedShift, -1e4f), 126.f));
#pragma unroll 1
                for (int d = 0; d < HD; d += 16) {
                    float y[16];
                    tmem_load16(o_at + d, y);
                    if (live) {
#pragma unroll
                        for (int e = 0; e < 16; e += 2) *reinterpret_cast<float2 *>(o + 2 + d + e) = make_float2(y[e] * f, y[e + 1] * f);
                    }
                }
                if (live) *reinterpret_cast<float2 *>(o) = make_float2(m, l);
            }
            tc_fence_before();
            j0 += s.count;
        }
        if (!ok) *ab = 1;
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == MMA_WARP) tmem_dealloc(tmem, 512);
}

// ------------------------------------------------------------------------------- join
// A query's state of its own positions and those of its shared ones, W warps to a query
template <int HD, int TQ, int W>
__global__ void __launch_bounds__(256) shared_join_kernel(SharedParams p, int shares_most) {
    constexpr int D = HD / 32;
    __shared__ float s_m[8], s_l[8], s_o[8][HD];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = W == 1 ? 0 : warp;
    const int64_t x = W == 1 ? (int64_t)blockIdx.x * 8 + warp : blockIdx.x;
    if (x >= (int64_t)p.n * p.H) return;
    const int row = (int)(x / p.H), head = (int)(x - (int64_t)row * p.H), G = p.H / p.c.KVH;
    float m = -3.4028235e38f, l = 0.f, o[D] = {};
    auto add = [&](float m1, float l1, const float *src) {
        float y[D];
#pragma unroll
        for (int d = 0; d < D; ++d) y[d] = src[lane + 32 * d];
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
        const int at = (row - y.row0) * G + head % G, e0 = y.entry0 + (head / G * y.tiles + at / TQ) * y.pages;
        const int c0 = shares.of(e0), c1 = shares.of(e0 + y.pages - 1);
        if (c0 == c1) {
            const float *s = p.whole + x * (HD + 2);
            if (part == 0) add(s[0], s[1], s + 2);
        } else {
#pragma unroll 4
            for (int c = c0 + part; c <= c1; c += W) {
                const float *s = p.part + (((int64_t)c * 2 + (c == c0)) * TQ + at % TQ) * (HD + 2);
                add(s[0], s[1], s + 2);
            }
        }
    }
    if constexpr (W > 1) {
        if (lane == 0) {
            s_m[warp] = m;
            s_l[warp] = l;
        }
#pragma unroll
        for (int d = 0; d < D; ++d) s_o[warp][lane + 32 * d] = o[d];
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int k = 1; k < W; ++k) add(s_m[k], s_l[k], s_o[k]);
    }
    // (nothing anywhere: 0 and -inf.  A failed wait: NaN)
    const bool none = l == 0.f;
    const float inv = p.plan->err ? __int_as_float(0x7fc00000) : none ? 0.f : 1.f / l;
#pragma unroll
    for (int d = 0; d < D; ++d) {
        const float y = o[d] * inv;
        p.out[x * HD + lane + 32 * d] = p.type == SARA_BF16 ? f32_to_bf16(y) : __half_as_ushort(__float2half_rn(y));
    }
    if (p.lse && lane == 0) p.lse[x] = none ? -INFINITY : (m + log2f(l)) * 0.69314718f;
}

}  // namespace sara
