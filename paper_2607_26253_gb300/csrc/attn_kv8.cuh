// Decode attention over the 8-bit paged KV cache: one query row per sequence,
//     out[i, h] = softmax(q[i, h] . K[first_i .. ctx_i)^T / sqrt(hd)) V[first_i .. ctx_i)
// Bound by reading the codes once (2 hd bytes a position and KV head), so every byte goes from memory to registers in
// the order in which the warp-level MMAs want it, 16 bytes a lane, and becomes fp16 there, which both
// formats fit exactly; a warp takes 16 positions at a time (32 below 128 dims).
//   - Scores: A = K (rows: positions), B = q^T (columns: the group's query heads, at most 8).  Lane (g, t) loads
//     16 consecutive dims of positions g and g + 8; which dims meet in a k-step does not matter as long as q is laid out
//     alike.  bf16 queries enter as fp16 after a power of two has brought the row's largest to 2^14.
//   - Output: A = V^T (rows: dims, lane (g, t) holds hd / 8 dims of 4 positions, byte permutes pair the positions),
//     B = P^T, the scores' own registers transposed by movmatrix.  P enters as an fp16 pair, hi + lo: 22 bits, and
//     multiples of 2^-31 of the maximum (probabilities are scaled by 2^7).
//   - A scale covers all of a warp's positions: K's is a factor of the scores, V's of P, relative to the largest so far
//     (vref), so that neither costs a multiplication per code.
// Online softmax in fp32 per warp; the maximum is re-based only when a probability would pass 2^8, so most steps
// skip the column maximum and the rescale.  A step's values are asked for before its scores are taken, the next step's keys
// over the used ones right after: 64 KB an SM are on their way (both ahead of a whole step: 179 us for 174 below).
// Work: the (row, KV head, 64 or 128 positions) triples in one list, cut into equal shares, one per CTA of 4 warps (4 an SM:
// 8-warp CTAs on whole pages took 212 us for 174, since fewer units overlap where one ends); a unit's first loads are
// under way while the one before is put together.  A (row, KV head) that several CTAs share is joined by the last of them
// to finish, in the list's order (so results repeat bit for bit), in two levels where there are many.
// Measured (kernel in a graph): 64 rows x 8,192 positions, 32 / 8 heads of 128: 171 us, 6.3 TB/s; 2 x 200,000, 16 / 2 heads: 48 us
// (the steps end after 33 to 37, the two levels of joins take 10); 26 ragged rows of mean 758, 12 / 2 heads: 12 us and one row 7.6,
// chains of latencies: share 0.7 us, first keys 1.1, step 0.5, state 0.9, arrival 0.7, join 2.5.
#pragma once
#include "kv8.cuh"

namespace sara {

constexpr int kAttnKv8Warps = 4;
constexpr int kAttnKv8Threads = 32 * kAttnKv8Warps;
// Positions that a warp takes at a time: as many bytes in flight at 64 dims as at 128; 32 is a scale's block
__host__ __device__ constexpr int attn_kv8_positions(int hd) { return hd == 128 ? 16 : 32; }
__host__ __device__ constexpr int attn_kv8_step(int hd) { return attn_kv8_positions(hd) * kAttnKv8Warps; }  // positions of an entry of the list
constexpr int kAttnKv8SmCtas = 16 / kAttnKv8Warps;
constexpr int kAttnKv8MaxCtas = 160 * kAttnKv8SmCtas;
constexpr int kAttnKv8Group = 16;                               // states joined at a time (2 x 200,000: 48.0 us; 8 49.0, 32 49.5, 64 53.2)
constexpr int kAttnKv8Batch = 4;                                // of them to a copy, two copies in shared memory
constexpr float kAttnKv8Shift = 7.f;                            // log2 of the probabilities' scale

// Floats of a state: max and sum of 8 heads, then their outputs
__host__ __device__ constexpr int attn_kv8_state(int hd) { return 8 * (hd + 2); }

struct AttnKv8Params {
    Kv8Cache c;
    const uint16_t *q;
    int64_t q_stride;
    const int32_t *ctx, *first;
    uint16_t *out;
    float *lse;
    int32_t *status;
    int *count;   // [CTA][2][2] arrivals at the two levels of a join, kept at its first state; left zero
    float *part;  // [CTA][2] states
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

// A row's positions, and the steps of the list that hold them
struct AttnKv8Row {
    int first, ctx, step0, steps;
    bool bad;
};
template <int STEP>
__device__ __forceinline__ AttnKv8Row attn_kv8_row(const AttnKv8Params &p, int i) {
    AttnKv8Row r;
    r.ctx = __ldg(p.ctx + i);
    r.first = p.first ? min(__ldg(p.first + i), r.ctx) : 0;  // (past the end: no position)
    r.bad = r.ctx < 0 || r.first < 0 || r.ctx > (int64_t)p.c.max_blocks * kKv8Page;
    r.step0 = r.first / STEP;
    r.steps = r.bad || r.ctx <= r.first ? 0 : (r.ctx - 1) / STEP - r.step0 + 1;
    return r;
}

// Two neighbouring outputs, at place i of a state
template <int HD>
__device__ __forceinline__ void attn_kv8_put(const AttnKv8Params &p, int row, int head, int i, float y0, float y1) {
    const int dim = HD / 8 * (i % 16 / 2) + i / 16 * 2;
    *reinterpret_cast<uint32_t *>(p.out + ((int64_t)row * p.H + head) * HD + dim) =
        p.type == SARA_BF16 ? pack2<SARA_BF16>(y0, y1) : pack2<SARA_FP16>(y0, y1);
}

// A (row, KV head) that CTAs c0 .. c1 share, as CTA c sees it: its states, or where there are more than a group's those
// of its group, whose result takes the place of the first; then the groups' results.
struct AttnKv8Join {
    int row, h, c0, c1;  // row < 0: nothing
};
template <int HD>
struct AttnKv8Group {
    const AttnKv8Params &p;
    const AttnKv8Join j;
    int from, n, pace;
    __device__ __forceinline__ AttnKv8Group(const AttnKv8Params &p_, const AttnKv8Join &j_, int c) : p(p_), j(j_), from(j_.c0), n(j_.c1 - j_.c0 + 1), pace(1) {
        if (two()) {
            from = max(j.c0, c & ~(kAttnKv8Group - 1));
            n = min(j.c1, c | (kAttnKv8Group - 1)) - from + 1;
        }
    }
    __device__ __forceinline__ bool two() const { return j.c1 - j.c0 >= kAttnKv8Group; }
    __device__ __forceinline__ void groups() {
        from = j.c0;
        n = j.c1 / kAttnKv8Group - j.c0 / kAttnKv8Group + 1;
        pace = kAttnKv8Group;
    }
    __device__ __forceinline__ float *state(int k) const {
        const int x = pace == 1 ? from + k : k == 0 ? j.c0 : (j.c0 & ~(kAttnKv8Group - 1)) + k * kAttnKv8Group;
        return p.part + (x * 2 + (x == j.c0)) * attn_kv8_state(HD);
    }
    // One thread, after a barrier: whether the CTA is the last of the group to come
    __device__ __forceinline__ bool arrive() const {
        int *arrived = p.count + (from * 2 + (from == j.c0)) * 2 + (pace > 1);
        const bool last = atom_add_acq_rel_gpu(arrived, 1) == n - 1;  // (orders the CTA's stores before it, its loads behind)
        if (last) *arrived = 0;
        return last;
    }
};

// The last CTA of a group joins its states, and so on up, by way of shared memory (whose copies leave the main loop its
// registers): 16 threads a head, two batches of states on their way at a time.  Whole CTAs; room: of both batches.
template <int HD>
__device__ __forceinline__ void attn_kv8_join(AttnKv8Group<HD> u, float *room, int *s_last) {
    constexpr int B = kAttnKv8Batch, STATE = attn_kv8_state(HD), NF = HD / 16, W = NF < 4 ? NF : 4;
    const AttnKv8Params &p = u.p;
    const int tid = threadIdx.x, G = p.H / p.c.KVH, hh = tid / 16, i0 = tid % 16 * W;
    auto fetch = [&](int k0) {  // the batch from state k0 on, if there is one
        const uint32_t to = smem_u32(room + (k0 / B & 1) * (B * STATE));
#pragma unroll
        for (int k = 0; k < B; ++k) {
            if (k >= u.n - k0) continue;
            const float *src = u.state(k0 + k);
#pragma unroll
            for (int e = 0; e < STATE / 4; e += kAttnKv8Threads)
                if (e + tid < STATE / 4) cp_async16(to + (k * STATE + 4 * (e + tid)) * 4, src + 4 * (e + tid));
        }
        cp_async_commit();
    };
#pragma unroll 1
    for (;;) {
        float M = -3.4028235e38f, L = 0.f, y[NF];
#pragma unroll
        for (int i = 0; i < NF; ++i) y[i] = 0.f;
        fetch(0);
        fetch(B);
#pragma unroll 1
        for (int k0 = 0; k0 < u.n; k0 += B) {
            cp_async_wait<1>();
            __syncthreads();
            const float *batch = room + (k0 / B & 1) * (B * STATE);
            float N = M, m[B];
#pragma unroll
            for (int k = 0; k < B; ++k) {  // (behind the last state: nothing)
                m[k] = k < u.n - k0 ? batch[k * STATE + hh] : -INFINITY;
                N = fmaxf(N, m[k]);
            }
            const float old = ex2(M - N);
            M = N;
            L *= old;
#pragma unroll
            for (int i = 0; i < NF; ++i) y[i] *= old;
#pragma unroll
            for (int k = 0; k < B; ++k) {
                if (k >= u.n - k0) continue;
                const float *x = batch + k * STATE;
                const float f = ex2(m[k] - N);
                L += f * x[8 + hh];
#pragma unroll
                for (int i = 0; i < NF; ++i) y[i] += f * x[16 + hh * HD + i0 + i / W * 64 + i % W];
            }
            __syncthreads();
            fetch(k0 + 2 * B);
        }
        const bool final = !u.two() || u.pace > 1;
        if (hh < G) {
            const float inv = 1.f / L;
            float *x = u.state(0);
#pragma unroll
            for (int i = 0; i < NF; i += 2) {
                const int at = i0 + i / W * 64 + i % W;
                if (final) attn_kv8_put<HD>(p, u.j.row, u.j.h * G + hh, at, y[i] * inv, y[i + 1] * inv);
                else *reinterpret_cast<float2 *>(x + 16 + hh * HD + at) = make_float2(y[i], y[i + 1]);
            }
            if (tid % 16 == 0) {
                if (!final) {
                    x[hh] = M;
                    x[8 + hh] = L;
                } else if (p.lse) {
                    p.lse[(int64_t)u.j.row * p.H + u.j.h * G + hh] = (M - kAttnKv8Shift + log2f(L)) * 0.69314718f;
                }
            }
        }
        if (final) return;
        u.groups();
        __syncthreads();
        if (tid == 0) *s_last = u.arrive();
        __syncthreads();
        if (!*s_last) return;
    }
}

template <int HD, int FMT>
__global__ void __launch_bounds__(kAttnKv8Threads, kAttnKv8SmCtas) attn_kv8_kernel(AttnKv8Params p) {
    constexpr int KW = HD / 16, VW = HD / 32, NT = HD / 16;  // words a lane of a key row, of a value row; output tiles
    constexpr int KL = KW < 4 ? KW : 4;                      // words a load
    // Steps at a time: 32 dims leave registers for two (64 rows x 16,384: 121 -> 105 us, int8 131 -> 115; 512 positions 12.3 -> 12.7)
    constexpr int SUB = HD == 32 ? 2 : 1;
    constexpr int POS = attn_kv8_positions(HD), NG = POS / 16, STEP = attn_kv8_step(HD), PS = kKv8Page / STEP;
    constexpr int PITCH = HD + 4;                            // (conflict-free 8-byte stores)
    constexpr int STATE = attn_kv8_state(HD);
    __shared__ __align__(16) union {
        float o[kAttnKv8Warps][8][PITCH];     // the warps' outputs
        float room[2 * kAttnKv8Batch * STATE];  // states that are joined
    } sm;
    auto &s_o = sm.o;
    __shared__ float s_m[kAttnKv8Warps][8], s_l[kAttnKv8Warps][8];
    __shared__ AttnKv8Join s_join[2];
    __shared__ int s_last[2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int KVH = p.c.KVH, G = p.H / KVH;
    const float nan = __int_as_float(0x7fc00000);

    // this CTA's share lo .. hi of the list, and the row in which it begins: every warp for itself, 32 rows at a time
    int steps = 0, total = 0;
    bool idle = false;  // a row without a position (or a wrong one) that is this CTA's to write
#pragma unroll 4
    for (int i = lane; i - lane < p.n; i += 32) {
        steps = i < p.n ? attn_kv8_row<STEP>(p, i).steps : 0;
        if (i < p.n && steps == 0) idle = idle || (unsigned)i % gridDim.x == blockIdx.x;
        total += __reduce_add_sync(0xffffffffu, steps);
    }
    if (__any_sync(0xffffffffu, idle)) {
        for (int i = blockIdx.x; i < p.n; i += gridDim.x) {
            const AttnKv8Row r = attn_kv8_row<STEP>(p, i);
            if (r.steps) continue;
            const float y = r.bad ? nan : 0.f;
            const uint32_t y2 = p.type == SARA_BF16 ? pack2<SARA_BF16>(y, y) : pack2<SARA_FP16>(y, y);
            uint32_t *o = reinterpret_cast<uint32_t *>(p.out + (int64_t)i * p.H * HD);
            for (int e = tid; e < p.H * HD / 2; e += kAttnKv8Threads) o[e] = y2;
            if (p.lse)
                for (int e = tid; e < p.H; e += kAttnKv8Threads) p.lse[(int64_t)i * p.H + e] = r.bad ? nan : -INFINITY;
            if (r.bad && tid == 0) kv8_report(p.status);
        }
    }
    total *= KVH;
    const int ctas = min((int)gridDim.x, total), c = blockIdx.x;
    if (c >= ctas) return;
    const int share = total / ctas, more = total - share * ctas;  // the first `more` CTAs have one entry more
    const int lo = c * share + min(c, more), hi = lo + share + (c < more);
    int row = 0, base = 0;  // base: of the row's first entry
    for (int i = lane, before = 0;; i += 32) {
        if (p.n > 32) steps = i < p.n ? attn_kv8_row<STEP>(p, i).steps : 0;
        int end = steps;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, end, d);
            if (lane >= d) end += y;
        }
        const uint32_t behind = __ballot_sync(0xffffffffu, (before + end) * KVH > lo);
        if (behind) {  // (lo < total: some row holds it)
            row = i - lane + __ffs(behind) - 1;
            base = (before + __shfl_sync(0xffffffffu, end - steps, __ffs(behind) - 1)) * KVH;
            break;
        }
        before += __shfl_sync(0xffffffffu, end, 31);
    }
    if (tid < 2) s_join[tid].row = -1;
    auto cta_of = [&](int x) {  // whose share entry x is
        const int big = more * (share + 1);
        return x < big ? x / (share + 1) : more + (x - big) / share;
    };

    AttnKv8Row r = attn_kv8_row<STEP>(p, row);
    int h = 0, a = 0, b = 0, unit = 0, xa = 0, xb = 0;  // entries unit + a .. unit + b: of the row, for KV head h
    const int32_t *tab = nullptr;
    int ids = 0, idbase = 0;  // this lane's entry of the 32 table entries from idbase on
    bool wrong = false;
    auto block_of = [&](int x, bool begin) {
        const int page = x / PS;
        if (begin || page - idbase >= 32) {
            idbase = page;
            ids = (page + lane) * PS < xb ? __ldg(tab + page + lane) : 0;
            const bool out = ids < 0 || ids >= p.c.n_blocks;
            wrong = wrong || out;
            ids = out ? -1 : ids;
        }
        return __shfl_sync(0xffffffffu, ids, page - idbase);
    };
    const int lane_k = (KW == 8 ? 16 : HD / 4) * t, lane_v = HD / 8 * g;
    auto step_of = [&](int x, int u) { return u == 0 ? x : min(x + u, xb - 1); };  // (behind the last step that step again, masked)
    auto edge = [&](int x) {  // whether some of its positions are masked
        const int p0 = x * STEP + POS * warp;
        return p0 < r.first || p0 > r.ctx - POS;
    };
    auto slot_of = [&](int x, int e) {  // (masked positions stand for the nearest that is not: their probability is 0)
        return min(max(x * STEP + POS * warp + e, r.first), r.ctx - 1) & (kKv8Page - 1);
    };
    auto block_in_page = [&](int x) { return (x % PS * STEP + POS * warp) / kKv8Block; };
    uint32_t kr[SUB][2 * NG][KW], vr[SUB][4 * NG][VW];  // positions g + 8 e; 2 t + (e & 1) + 8 (e >> 1)
    float ks[SUB], vs[SUB];
    int blk[SUB] = {};
    auto load_k = [&](int x, int u) {
        const int64_t tile = kv8_tile(p.c, max(blk[u], 0), 0, h);
        ks[u] = blk[u] < 0 ? nan : __ldg(p.c.scales + tile * kKv8PageBlocks + block_in_page(x));
        const uint8_t *k = p.c.codes + tile * (kKv8Page * HD) + lane_k;
        if (!edge(x)) {
            k += (x % PS * STEP + POS * warp + g) * HD;
#pragma unroll
            for (int e = 0; e < 2 * NG; ++e)
#pragma unroll
                for (int i = 0; i < KW / KL; ++i) load_codes<KL>(k + 8 * e * HD + 64 * i, &kr[u][e][4 * i]);
        } else {
#pragma unroll
            for (int e = 0; e < 2 * NG; ++e)
#pragma unroll
                for (int i = 0; i < KW / KL; ++i) load_codes<KL>(k + slot_of(x, g + 8 * e) * HD + 64 * i, &kr[u][e][4 * i]);
        }
    };
    auto load_v = [&](int x, int u) {
        const int64_t tile = kv8_tile(p.c, max(blk[u], 0), 1, h);
        vs[u] = __ldg(p.c.scales + tile * kKv8PageBlocks + block_in_page(x));
        const uint8_t *v = p.c.codes + tile * (kKv8Page * HD) + lane_v;
        if (!edge(x)) {
            v += (x % PS * STEP + POS * warp + 2 * t) * HD;
#pragma unroll
            for (int e = 0; e < 4 * NG; ++e) load_codes<VW>(v + ((e & 1) + 8 * (e >> 1)) * HD, vr[u][e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4 * NG; ++e) load_codes<VW>(v + slot_of(x, 2 * t + (e & 1) + 8 * (e >> 1)) * HD, vr[u][e]);
        }
    };
    // queries: head g of the group, the dims of this lane's key words
    uint32_t qb[KW][2];
    auto begin = [&](int at) {  // the unit of entry `at`; its first keys and its queries are on their way
        h = (at - base) / r.steps;
        unit = base + h * r.steps;
        a = at - unit;
        b = min(r.steps, hi - unit);
        // this warp's positions of step x: STEP x + POS warp .. + POS - 1; the row's first and last step may have none
        xa = r.step0 + a;
        xb = r.step0 + b;
        if (xa * STEP + POS * (warp + 1) <= r.first) ++xa;
        if ((xb - 1) * STEP + POS * warp >= r.ctx) --xb;
        tab = p.c.table + row * p.c.table_stride;
        if (xa < xb) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                blk[u] = block_of(step_of(xa, u), u == 0);
                load_k(step_of(xa, u), u);
            }
        }
        const uint16_t *qp = p.q + row * p.q_stride + (int64_t)(h * G + min(g, G - 1)) * HD;
#pragma unroll
        for (int s = 0; s < KW; ++s) {
            const int d = KW == 8 ? 64 * (s / 4) + 16 * t + 4 * (s % 4) : HD / 4 * t + 4 * s;
            const uint2 x = __ldg(reinterpret_cast<const uint2 *>(qp + d));
            qb[s][0] = x.x;
            qb[s][1] = x.y;
        }
    };

    begin(lo);
    for (int at = lo;;) {
        float mul0, mul1;  // from MMA sums to base-2 exponents, heads 2 t and 2 t + 1
        {
#pragma unroll
            for (int s = 0; s < KW; ++s) qb[s][0] = g < G ? qb[s][0] : 0, qb[s][1] = g < G ? qb[s][1] : 0;
            float mul = p.scale_log2;
            if (p.type == SARA_BF16) {
                uint32_t top = 0;
#pragma unroll
                for (int s = 0; s < KW; ++s)
                    top = __vmaxu2(top, __vmaxu2(qb[s][0] & 0x7fff7fffu, qb[s][1] & 0x7fff7fffu));
                top = max(top & 0xffff, top >> 16);
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // 2^e brings the largest magnitude's power of two to 2^14
                const int e = max(min(14 - ((int)(top >> 7) - 127), 126), -113);
                const float f = pow2f(e);
#pragma unroll
                for (int s = 0; s < KW; ++s)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 x = unpack2<SARA_BF16>(qb[s][i]);
                        qb[s][i] = pack_half2(x.x * f, x.y * f);
                    }
                mul *= pow2f(-e);
            }
            mul0 = __shfl_sync(0xffffffffu, mul, 8 * t);
            mul1 = __shfl_sync(0xffffffffu, mul, 8 * t + 4);
        }

        float m0 = -3.4028235e38f, m1 = m0, l0 = 0.f, l1 = 0.f, vref = 0.f, vinv = 0.f, o[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
#pragma unroll 1
        for (int x = xa; x < xb; x += SUB) {
            // these steps' values come while their scores are taken, the next ones' keys after that
#pragma unroll
            for (int u = 0; u < SUB; ++u) load_v(step_of(x, u), u);
            float s[SUB][NG][4];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const float f0 = ks[u] * mul0, f1 = ks[u] * mul1;
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    float s2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][n][e] = 0.f;
#pragma unroll
                    for (int i = 0; i < KW; ++i) {
                        uint32_t f[4];
                        decode4_half<FMT>(kr[u][2 * n][i], f[0], f[2]);
                        decode4_half<FMT>(kr[u][2 * n + 1][i], f[1], f[3]);
                        mma_f16_16816(i & 1 ? s2 : s[u][n], f, qb[i][0], qb[i][1]);
                    }
                    // s[u][n][0], [1]: position 16 n + g, heads 2 t and 2 t + 1; [2], [3]: position 16 n + g + 8
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[u][n][e] = (s[u][n][e] + s2[e]) * (e & 1 ? f1 : f0);
                }
            }
            float vsc[SUB];
            bool cut[SUB];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                vsc[u] = vs[u];
                cut[u] = edge(x + u);
            }
            if (x + SUB < xb) {
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    blk[u] = block_of(step_of(x + SUB, u), false);
                    load_k(step_of(x + SUB, u), u);
                }
            }
            float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const bool none = u > 0 && x + u >= xb;
                if (none || cut[u]) {
#pragma unroll
                    for (int n = 0; n < NG; ++n) {
                        const int p0 = (x + u) * STEP + POS * warp + 16 * n + g;
                        if (none || p0 < r.first || p0 >= r.ctx) s[u][n][0] = s[u][n][1] = -INFINITY;
                        if (none || p0 + 8 < r.first || p0 + 8 >= r.ctx) s[u][n][2] = s[u][n][3] = -INFINITY;
                    }
                }
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    t0 = fmaxf(t0, fmaxf(s[u][n][0], s[u][n][2]));
                    t1 = fmaxf(t1, fmaxf(s[u][n][1], s[u][n][3]));
                }
            }
            if (__any_sync(0xffffffffu, t0 > m0 + 8.f || t1 > m1 + 8.f)) {
                float n0 = fmaxf(m0, t0), n1 = fmaxf(m1, t1);
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
            const float c0 = m0 - kAttnKv8Shift, c1 = m1 - kAttnKv8Shift;
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                if (!(vsc[u] <= vref)) {  // the largest scale so far (or NaN)
                    const float inv = 1.f / vsc[u], f = vref * inv;
                    vref = vsc[u];
                    vinv = inv;
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[j][e] *= f;
                }
                const float vf = vsc[u] * vinv;
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    float w0 = ex2(s[u][n][0] - c0), w1 = ex2(s[u][n][1] - c1), w2 = ex2(s[u][n][2] - c0), w3 = ex2(s[u][n][3] - c1);
                    l0 += w0 + w2;
                    l1 += w1 + w3;
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
                        uint32_t v0[4], v1[4];  // dims 4 i, 4 i + 1 and 4 i + 2, 4 i + 3 of the lane's
                        const uint32_t a = vr[u][4 * n][i], b = vr[u][4 * n + 1][i], c = vr[u][4 * n + 2][i], d = vr[u][4 * n + 3][i];
                        decode4_half<FMT>(__byte_perm(a, b, 0x5140), v0[0], v0[1]);
                        decode4_half<FMT>(__byte_perm(c, d, 0x5140), v0[2], v0[3]);
                        decode4_half<FMT>(__byte_perm(a, b, 0x7362), v1[0], v1[1]);
                        decode4_half<FMT>(__byte_perm(c, d, 0x7362), v1[2], v1[3]);
                        mma_f16_16816(o[2 * i], v0, ph[0], ph[1]);
                        mma_f16_16816(o[2 * i + 1], v1, ph[0], ph[1]);
                        mma_f16_16816(o[2 * i], v0, pl[0], pl[1]);
                        mma_f16_16816(o[2 * i + 1], v1, pl[0], pl[1]);
                    }
                }
            }
        }

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
        const AttnKv8Join me = {row, h, unit, unit + r.steps - 1};
        const bool begins = a == 0, whole = begins && b == r.steps;
        at = unit + b;
        if (at < hi) {  // the next unit's loads, while this one is put together
            if (h == KVH - 1) {
                base += KVH * r.steps;
                do r = attn_kv8_row<STEP>(p, ++row);
                while (r.steps == 0);
            }
            begin(at);
        }
        __syncthreads();
        float *mine = p.part + (c * 2 + begins) * STATE;  // (a share begins in at most one unit that it does not begin)
        for (int e = tid; e < G * HD / 2; e += kAttnKv8Threads) {
            const int hh = e / (HD / 2), i = e % (HD / 2) * 2;
            float M = s_m[0][hh], L = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
            for (int w = 1; w < kAttnKv8Warps; ++w) M = fmaxf(M, s_m[w][hh]);
#pragma unroll
            for (int w = 0; w < kAttnKv8Warps; ++w) {
                const float2 y = *reinterpret_cast<const float2 *>(&s_o[w][hh][i]);
                const float f = ex2(s_m[w][hh] - M);
                L += f * s_l[w][hh];
                y0 += f * y.x;
                y1 += f * y.y;
            }
            if (whole) {
                const float inv = 1.f / L;
                attn_kv8_put<HD>(p, me.row, me.h * G + hh, i, y0 * inv, y1 * inv);
                if (p.lse && i == 0) p.lse[(int64_t)me.row * p.H + me.h * G + hh] = (M - kAttnKv8Shift + log2f(L)) * 0.69314718f;
            } else {
                *reinterpret_cast<float2 *>(mine + 16 + hh * HD + i) = make_float2(y0, y1);
                if (i == 0) {
                    mine[hh] = M;
                    mine[8 + hh] = L;
                }
            }
        }
        if (!whole && tid == 0) s_join[begins] = {me.row, me.h, cta_of(me.c0), cta_of(me.c1)};
        __syncthreads();  // (shared memory is the next unit's)
        if (at >= hi) break;
    }
    if (wrong) kv8_report(p.status);

    // the units that other CTAs share: at most the one in which the share begins and the one in which it ends
    if ((tid == 0 || tid == 32) && s_join[tid / 32].row >= 0) s_last[tid / 32] = AttnKv8Group<HD>(p, s_join[tid / 32], c).arrive();
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < 2; ++i)
        if (s_join[i].row >= 0 && s_last[i]) attn_kv8_join<HD>({p, s_join[i], c}, sm.room, &s_last[i]);
}

inline size_t attn_kv8_count_bytes() { return kAttnKv8MaxCtas * 4 * sizeof(int); }
inline size_t attn_kv8_workspace(int hd) { return attn_kv8_count_bytes() + (size_t)kAttnKv8MaxCtas * 2 * attn_kv8_state(hd) * sizeof(float); }

}  // namespace sara
