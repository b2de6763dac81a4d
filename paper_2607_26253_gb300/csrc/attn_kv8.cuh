// Decode attention over the 8-bit paged KV cache: one query row per sequence,
//     out[i, h] = softmax(q[i, h] . K[first_i .. ctx_i)^T / sqrt(hd)) V[first_i .. ctx_i)
// Bound by reading the codes once (2 hd bytes a position and KV head).  They come by asynchronous copies into a ring in shared
// memory, a warp's own, and become fp16 in registers, which both formats fit exactly; a warp takes 16 positions at a time (32 below
// 128 dims).
//   - Scores: A = K (rows: positions), B = q^T (columns: the group's query heads, at most 8).  Lane (g, t) takes
//     16-byte pieces of positions g and g + 8; which dims meet in a k-step does not matter as long as q is laid out
//     alike.  bf16 queries enter as fp16 after a power of two has brought the head's largest to 2^14: exact down to 2^-31 of it,
//     within 2^-39 of it below, so scores are off by 2^-39 max |q| sum |k| at most (a second, low half would cost as many MMAs again).
//   - Output: A = V^T (rows: dims, lane (g, t) holds hd / 8 dims of 4 positions, byte permutes pair the positions),
//     B = P^T, the scores' own registers transposed by movmatrix.
//   - A scale covers all of a warp's positions: K's is a factor of the scores, V's of P, so that neither costs a multiplication
//     per code.  P times V's scale enters as an fp16 pair, hi + lo: 22 bits, or within 2^-31 of the largest such product of the head
//     so far.  A power of two of the head's own, r, brings that one to 2^6 .. 2^7, so that a block of large values without weight does not
//     push out the small values that have it.
// Online softmax in fp32 per warp; the maximum and r are re-based only when a probability or a product would pass 2^8 of them, so most
// steps skip the column maximum and the rescale.
// The next step's copies are under way while a step is computed, across the ends of units: 64 KB an SM, which is enough, and more
// is worse (64 x 8,192 positions: 166 us, with two steps ahead 177; a step in registers instead, its values asked for with its scores,
// the next one's keys after them: 174, in int8 188 for 168).  Five CTAs an SM, whose 96 registers spill: 182; four's 128 spill
// 28 bytes at most, at 128 dims in e4m3 (<128, e4m3, 1>: 16 stored, 28 loaded), others none.
// Work: the (row, KV head, positions) triples in one list, cut into equal shares, one per CTA of 4 warps (4 an SM), or per warp
// where there are many rows (kAttnKv8Units).  A (row, KV head) that several shares hold is joined by the last of them to finish,
// in the list's order (so results repeat bit for bit), by levels where there are many.
// Measured (kernel in a graph): 64 rows x 8,192 positions, 32 / 8 heads of 128: 167 us, 6.4 TB/s (350 x 4,000: 6.7); 2 x 200,000, 16 / 2
// heads: 45 (the joins take 10); 26 ragged rows of mean 758, 12 / 2 heads: 12 us and one row 7.7, chains of latencies: share 0.7
// us, first keys 1.1, step 0.5, state 0.9, arrival 0.7, join 2.5.  700 ragged rows of mean 200, 32 / 8 heads: 65 us (44 at the copy's
// rate: 8 us until the first step and 5 of joins).
#pragma once
#include "kv8.cuh"

namespace sara {

constexpr int kAttnKv8Warps = 4;
constexpr int kAttnKv8Threads = 32 * kAttnKv8Warps;
// Positions that a warp takes at a time: as many bytes in flight at 64 dims as at 128; 32 is a scale's block
__host__ __device__ constexpr int attn_kv8_positions(int hd) { return hd == 128 ? 16 : 32; }
__host__ __device__ constexpr int attn_kv8_step(int hd, int warps) { return attn_kv8_positions(hd) * warps; }  // positions of an entry of the list
constexpr int kAttnKv8SmCtas = 16 / kAttnKv8Warps;
constexpr int kAttnKv8MaxCtas = 160 * kAttnKv8SmCtas;
constexpr int kAttnKv8MaxShares = kAttnKv8MaxCtas * kAttnKv8Warps;
// (row, KV head) pairs from which each warp has a share of its own: nothing is put together between warps, but there are
// four times the states to join.  8 KV heads of 128, us with a CTA's shares and a warp's: 1,040 pairs of 200 positions 23.7, 28.7 (of
// 4,000: 170, 172); 1,400: 29.4, 28.1 (223, 225); 2,000: 37.0, 33.4 (313, 313); 5,600: 87.6, 64.8 (847, 842); 64 and 32 dims alike
constexpr int kAttnKv8Units = 1600;
constexpr int kAttnKv8Levels = 3;                               // of joins
constexpr int kAttnKv8Group = 16;                               // states joined at a time (2 x 200,000: 48.0 us at the time; 8 49.0, 32 49.5, 64 53.2)
constexpr int kAttnKv8Batch = 4;                                // of them to a copy, two copies in shared memory
// Stages of a warp's ring (32 dims, whose stages are half as large, 64 rows x 16,384: 98 us, 106 with two)
__host__ __device__ constexpr int attn_kv8_stages(int hd) { return hd == 32 ? 3 : 2; }
constexpr float kAttnKv8Shift = 7.f;                            // log2 of the probabilities' scale

// Floats of a state: max and sum of 8 heads, then their outputs
__host__ __device__ constexpr int attn_kv8_state(int hd) { return 8 * (hd + 2); }

// Bytes of a warp's ring of keys and values, which is also its part of the joins' room, and of a CTA's with their scales
__host__ __device__ constexpr int attn_kv8_ring(int hd) {
    const int ring = attn_kv8_stages(hd) * 2 * attn_kv8_positions(hd) * hd, room = 2 * kAttnKv8Batch / kAttnKv8Warps * attn_kv8_state(hd) * 4;
    return ring > room ? ring : room;
}
__host__ __device__ constexpr int attn_kv8_smem(int hd) { return kAttnKv8Warps * (attn_kv8_ring(hd) + attn_kv8_stages(hd) * 16); }

struct AttnKv8Params {
    Kv8Cache c;
    const uint16_t *q;
    int64_t q_stride;
    const int32_t *ctx, *first;
    uint16_t *out;
    float *lse;
    int32_t *status;
    int *count;   // [share][2][levels] arrivals at a join, kept at its first state; left zero
    float *part;  // [share][2] states
    int n, H, type;
    float scale_log2;  // log2(e) / sqrt(hd)
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {  // the smaller; a NaN stays
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
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
__device__ __forceinline__ void load_codes(uint32_t p, uint32_t *r) {  // from shared memory
    if constexpr (WORDS == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(p) : "memory");
    else if constexpr (WORDS == 2)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(p) : "memory");
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r[0]) : "r"(p) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
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

// A (row, KV head) that shares c0 .. c1 hold together, as share c sees it: its states, or where there are more than a
// group's those of its group, whose result takes the place of the first; then the groups' results, and so on up (for the
// shares of CTAs, whose number is smaller, two levels at most: a level costs them more than a longer group).
struct AttnKv8Join {
    int row, h, c0, c1;  // row < 0: nothing
};
template <int HD, int W>
struct AttnKv8Group {
    const AttnKv8Params &p;
    const AttnKv8Join j;
    const int c;
    int level, pace, from, n;
    bool whole;
    __device__ __forceinline__ AttnKv8Group(const AttnKv8Params &p_, const AttnKv8Join &j_, int c_) : p(p_), j(j_), c(c_), level(0), pace(1) { set(); }
    __device__ __forceinline__ void set() {
        const int wide = pace * kAttnKv8Group, of = j.c1 / pace - j.c0 / pace + 1;
        whole = of <= kAttnKv8Group || level == (W == 1 ? kAttnKv8Levels : 2) - 1;
        from = whole ? j.c0 : max(j.c0, c & ~(wide - 1));
        n = whole ? of : min(j.c1, c | (wide - 1)) / pace - from / pace + 1;
    }
    __device__ __forceinline__ void up() {
        ++level;
        pace *= kAttnKv8Group;
        set();
    }
    __device__ __forceinline__ float *state(int k) const {
        const int x = k == 0 ? from : (from & ~(pace - 1)) + k * pace;
        return p.part + (x * 2 + (x == j.c0)) * attn_kv8_state(HD);
    }
    // One thread, after a barrier: whether the share is the last of the group to come
    __device__ __forceinline__ bool arrive() const {
        int *arrived = p.count + (from * 2 + (from == j.c0)) * kAttnKv8Levels + level;
        const bool last = atom_add_acq_rel_gpu(arrived, 1) == n - 1;  // (orders the share's stores before it, its loads behind)
        if (last) *arrived = 0;
        return last;
    }
};
template <int W>
__device__ __forceinline__ void attn_kv8_sync() {  // of a share's threads
    if constexpr (W == 1) __syncwarp();
    else __syncthreads();
}

// The last share of a group joins its states, and so on up, by way of shared memory (whose copies leave the main loop its
// registers): 4 threads a head and warp, two batches of states on their way at a time.  tid: of the share's W warps; room: of both
// batches.
template <int HD, int W>
__device__ __forceinline__ void attn_kv8_join(AttnKv8Group<HD, W> u, float *room, int *s_last, int tid) {
    constexpr int T = 4 * W, B = kAttnKv8Batch * W / kAttnKv8Warps, STATE = attn_kv8_state(HD), NF = HD / T, V = NF < 4 ? NF : 4;
    const AttnKv8Params &p = u.p;
    const int G = p.H / p.c.KVH, hh = tid / T, i0 = tid % T * V;
    auto fetch = [&](int k0) {  // the batch from state k0 on, if there is one
        const uint32_t to = smem_u32(room + (k0 / B & 1) * (B * STATE));
#pragma unroll
        for (int k = 0; k < B; ++k) {
            if (k >= u.n - k0) continue;
            const float *src = u.state(k0 + k);
#pragma unroll
            for (int e = 0; e < STATE / 4; e += 32 * W)
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
            attn_kv8_sync<W>();
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
                for (int i = 0; i < NF; ++i) y[i] += f * x[16 + hh * HD + i0 + i / V * (T * V) + i % V];
            }
            attn_kv8_sync<W>();
            fetch(k0 + 2 * B);
        }
        if (hh < G) {
            const float inv = 1.f / L;
            float *x = u.state(0);
#pragma unroll
            for (int i = 0; i < NF; i += 2) {
                const int at = i0 + i / V * (T * V) + i % V;
                if (u.whole) attn_kv8_put<HD>(p, u.j.row, u.j.h * G + hh, at, y[i] * inv, y[i + 1] * inv);
                else *reinterpret_cast<float2 *>(x + 16 + hh * HD + at) = make_float2(y[i], y[i + 1]);
            }
            if (tid % T == 0) {
                if (!u.whole) {
                    x[hh] = M;
                    x[8 + hh] = L;
                } else if (p.lse) {
                    p.lse[(int64_t)u.j.row * p.H + u.j.h * G + hh] = (M - kAttnKv8Shift + log2f(L)) * 0.69314718f;
                }
            }
        }
        if (u.whole) return;
        u.up();
        attn_kv8_sync<W>();
        if (tid == 0) *s_last = u.arrive();
        attn_kv8_sync<W>();
        if (!*s_last) return;
    }
}

// W: warps of a share
template <int HD, int FMT, int W>
__global__ void __launch_bounds__(kAttnKv8Threads, kAttnKv8SmCtas) attn_kv8_kernel(AttnKv8Params p) {
    constexpr int KW = HD / 16, VW = HD / 32, NT = HD / 16;  // words a lane of a key row, of a value row; output tiles
    constexpr int KL = KW < 4 ? KW : 4;                      // words a load
    constexpr int POS = attn_kv8_positions(HD), NG = POS / 16, STEP = attn_kv8_step(HD, W), PS = kKv8Page / STEP;
    constexpr int STATE = attn_kv8_state(HD);
    __shared__ int s_free[kAttnKv8Warps];
    __shared__ float s_m[kAttnKv8Warps][8], s_l[kAttnKv8Warps][8];
    constexpr int SHARES = kAttnKv8Warps / W;                // of a CTA
    __shared__ AttnKv8Join s_joins[SHARES][2];
    __shared__ int s_lasts[SHARES][2];
    const int tid = threadIdx.x, warp = (tid >> 5) % W, mine = (tid >> 5) / W, lane = tid & 31, g = lane >> 2, t = lane & 3;
    auto &s_join = s_joins[mine];
    auto &s_last = s_lasts[mine];
    const int KVH = p.c.KVH, G = p.H / KVH;
    const float nan = __int_as_float(0x7fc00000);

    // this share lo .. hi of the list, and the row in which it begins: up to 32 rows by every warp for itself, more in 32 parts,
    // 8 a warp (every warp all by itself took 94 us for 88 at 700 rows)
    const bool many = p.n > 32;
    const int deep = (p.n + 1023) / 1024;  // rows of a part / 32
    __shared__ int s_part[32];
    int steps = 0, total = 0;
    bool idle = false;  // a row without a position (or a wrong one) that is this CTA's to write
    auto steps_of = [&](int i) {
        const int y = i < p.n ? attn_kv8_row<STEP>(p, i).steps : 0;
        idle = idle || (i < p.n && y == 0 && (unsigned)i % gridDim.x == blockIdx.x);
        return y;
    };
    if (many) {
        int sums[8] = {};
        const int at = (tid >> 5) * 8;
        for (int d = 0; d < deep; ++d)
#pragma unroll
            for (int k = 0; k < 8; ++k) sums[k] += steps_of(((at + k) * deep + d) * 32 + lane);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            sums[k] = __reduce_add_sync(0xffffffffu, sums[k]);
            if (lane == 0) s_part[at + k] = sums[k];
        }
        idle = __syncthreads_or(idle);
        total = s_part[lane];
    } else {
        total = steps = steps_of(lane);
        idle = __any_sync(0xffffffffu, idle);
    }
    const int part = total;
    total = __reduce_add_sync(0xffffffffu, total);
    if (idle) {
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
    const int shares = min((int)gridDim.x * SHARES, total), c = blockIdx.x * SHARES + mine;
    if (c >= shares) return;
    const int share = total / shares, more = total - share * shares;  // the first `more` shares have one entry more
    const int lo = c * share + min(c, more), hi = lo + share + (c < more);
    int row = 0, base = 0;  // base: of the row's first entry
    auto find = [&](int y) {  // the first lane whose end is behind lo (there is one); base: entries before it
        int end = y;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int z = __shfl_up_sync(0xffffffffu, end, d);
            if (lane >= d) end += z;
        }
        const uint32_t behind = __ballot_sync(0xffffffffu, (base + end) * KVH > lo);
        const int k = behind ? __ffs(behind) - 1 : 32;
        base += __shfl_sync(0xffffffffu, behind ? end - y : end, behind ? k : 31);
        return k;
    };
    if (many) {
        row = find(part) * deep * 32;
        for (int k = 32; k == 32; row += k) k = find(row + lane < p.n ? attn_kv8_row<STEP>(p, row + lane).steps : 0);
    } else {
        row = find(steps);
    }
    base *= KVH;
    if (warp == 0 && lane == 0) s_join[0].row = s_join[1].row = -1;
    auto share_of = [&](int x) {  // whose share entry x is
        const int big = more * (share + 1);
        return x < big ? x / (share + 1) : more + (x - big) / share;
    };

    // This warp's ring, and what its loads, which run ahead of the sums, are about
    constexpr int S = attn_kv8_stages(HD), TILE = POS * HD, CHUNKS = HD / 16, LC = TILE / 16 / 32, RING = attn_kv8_ring(HD);
    extern __shared__ __align__(128) uint8_t s_ring[];
    static_assert(2 * TILE >= 8 * HD * 4, "a stage holds a warp's sums");
    static_assert(RING % 128 == 0, "lines");
    const uint32_t ring = smem_u32(s_ring) + (tid >> 5) * RING;
    const uint32_t ring_s = smem_u32(s_ring) + kAttnKv8Warps * RING + (tid >> 5) * (S * 16);
    AttnKv8Row r = attn_kv8_row<STEP>(p, row), lr = r;
    int h = (lo - base) / r.steps, unit = base + h * r.steps;  // KV head; the first entry of the (row, KV head)
    int l_row = row, l_h = h - 1, l_unit = unit - r.steps, l_x = 0, l_end = 0, fill = 0;
    // this warp's steps of a unit in this share, x .. end: of a step x it has positions STEP x + POS warp .. + POS - 1, the row's
    // first and last step may have none of them
    auto range = [&](const AttnKv8Row &r, int unit, int &x, int &end) {
        x = r.step0 + max(lo - unit, 0);
        end = r.step0 + min(r.steps, hi - unit);
        if (r.first - x * STEP >= POS * (warp + 1)) ++x;
        if ((end - 1) * STEP + POS * warp >= r.ctx) --end;
    };
    int ids = 0, idbase = -32;  // this lane's entry of the 32 table entries from idbase on
    bool wrong = false;
    // Where 16 bytes of a tile stand: rows fill lines of 128 bytes, whose eight pieces are exchanged so that the lanes that read at a time
    // meet all banks
    auto place = [&](int pos, int chunk, bool value) {
        const int line = pos * CHUNKS / 8, piece = pos * CHUNKS % 8 + chunk;
        const int x = HD == 128 ? (value ? line & 6 : (line & 1) * 4) : HD == 64 ? (line & 3) * 2 : (line & 1) * 2;
        return line * 128 + (piece ^ x) * 16;
    };
    // this lane's 16 bytes, and those 512 bytes further on, of keys and values (whose places change sides from row 4 to row 4 at 128 dims)
    const uint32_t put = place(lane / CHUNKS, lane % CHUNKS, false), put_v = TILE + place(lane / CHUNKS, lane % CHUNKS, true);
    const int64_t v_behind = (int64_t)KVH * (kKv8Page * HD);
    auto load = [&]() {
        while (l_x >= l_end && l_unit + lr.steps < hi) {  // the next unit that has something for this warp
            l_unit += lr.steps;
            if (++l_h == KVH) {
                l_h = 0;
                do lr = attn_kv8_row<STEP>(p, ++l_row);
                while (lr.steps == 0);
                idbase = -32;
            }
            range(lr, l_unit, l_x, l_end);
        }
        if (l_x < l_end) {
            const int page = l_x / PS;
            if ((unsigned)(page - idbase) >= 32u) {  // (a row's next head finds them here where there are not many)
                idbase = page;
                ids = (page + lane) * PS < lr.step0 + lr.steps ? __ldg(p.c.table + l_row * p.c.table_stride + page + lane) : 0;
                const bool out = ids < 0 || ids >= p.c.n_blocks;
                wrong = wrong || out;
                ids = out ? -1 : ids;
            }
            const int block = __shfl_sync(0xffffffffu, ids, page - idbase), p0 = l_x * STEP + POS * warp;
            const uint32_t to = ring + put + fill * (2 * TILE), to_v = ring + put_v + fill * (2 * TILE), to_s = ring_s + fill * 16;
            const uint32_t to_v1 = HD == 128 ? to_v ^ 64 : to_v;
            if (block >= 0) {
                const int64_t tile = kv8_tile(p.c, block, 0, l_h);
                const uint8_t *src = p.c.codes + (tile * kKv8Page + (p0 & (kKv8Page - 1))) * HD + 16 * lane, *src_v = src + v_behind;
                if (p0 >= lr.first && p0 <= lr.ctx - POS) {
#pragma unroll
                    for (int i = 0; i < LC; ++i) {
                        cp_async16(to + 512 * i, src + 512 * i);
                        cp_async16(i & 1 ? to_v1 + 512 * i : to_v + 512 * i, src_v + 512 * i);
                    }
                } else {  // masked positions stand for the nearest that is not: their probability is 0
#pragma unroll 1
                    for (int i = 0; i < LC; ++i) {
                        const int at = lane / CHUNKS + i * (32 / CHUNKS), off = (min(max(p0 + at, lr.first), lr.ctx - 1) - p0 - lane / CHUNKS) * HD;
                        cp_async16(to + 512 * i, src + off);
                        cp_async16(i & 1 ? to_v1 + 512 * i : to_v + 512 * i, src_v + off);
                    }
                }
                if (lane < 2) cp_async4(to_s + 4 * lane, p.c.scales + (tile + lane * KVH) * kKv8PageBlocks + (p0 & (kKv8Page - 1)) / kKv8Block);
            } else if (lane < 2) {
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(to_s + 4 * lane), "f"(nan) : "memory");
            }
            ++l_x;
        }
        cp_async_commit();
        fill = fill == S - 1 ? 0 : fill + 1;
    };
    int xa = 0, xb = 0, take = 0;
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) load();
    uint32_t at_k[2], at_v[2];  // this lane's places in a tile
    at_k[0] = place(g, KW == 2 ? t / 2 : t, false) + (KW == 2 ? t % 2 * 8 : 0);
    at_k[1] = at_k[0] ^ 64;  // (128 dims: the dims from 64 on)
    at_v[0] = place(2 * t, HD == 128 ? g : HD == 64 ? g / 2 : g / 4, true) + (HD == 128 ? 0 : HD == 64 ? g % 2 * 8 : g % 4 * 4);
    at_v[1] = HD == 128 ? at_v[0] + 128 : HD == 64 ? at_v[0] ^ 64 : at_v[0] ^ 32;
    // queries: head g of the group, the dims of this lane's key words
    uint32_t qb[KW][2];
    auto begin = [&]() {
        range(r, unit, xa, xb);
        const uint16_t *qp = p.q + row * p.q_stride + (int64_t)(h * G + min(g, G - 1)) * HD;
#pragma unroll
        for (int s = 0; s < KW; ++s) {
            const int d = KW == 8 ? 64 * (s / 4) + 16 * t + 4 * (s % 4) : HD / 4 * t + 4 * s;
            const uint2 x = __ldg(reinterpret_cast<const uint2 *>(qp + d));
            qb[s][0] = x.x;
            qb[s][1] = x.y;
        }
    };

    begin();
    for (;;) {
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

        // o: sums of probability times scale times r times code
        float m0 = -3.4028235e38f, m1 = m0, l0 = 0.f, l1 = 0.f, r0 = 1.f, r1 = 1.f, o[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
#pragma unroll 1
        for (int x = xa; x < xb; ++x) {
            cp_async_wait<S - 2>();
            __syncwarp();  // (every lane's copies have come, and every lane has left the stage that is filled next)
            load();
            const uint32_t from = ring + take * (2 * TILE), from_s = ring_s + take * 16;
            take = take == S - 1 ? 0 : take + 1;
            float ks, vsc;
            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(ks), "=f"(vsc) : "r"(from_s) : "memory");
            uint32_t kr[2 * NG][KW];  // positions g + 8 e
#pragma unroll
            for (int e = 0; e < 2 * NG; ++e)
#pragma unroll
                for (int i = 0; i < KW / KL; ++i) load_codes<KL>(from + at_k[i] + 8 * e * HD, &kr[e][4 * i]);
            uint32_t vr[4 * NG][VW];  // positions 2 t + (e & 1) + 8 (e >> 1)
#pragma unroll
            for (int e = 0; e < 4 * NG; ++e) load_codes<VW>(from + TILE + at_v[e & 1] + 8 * (e >> 1) * HD, vr[e]);
            float s[NG][4];
            const float f0 = ks * mul0, f1 = ks * mul1;
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                float s2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
                for (int i = 0; i < KW; ++i) {
                    uint32_t f[4];
                    decode4_half<FMT>(kr[2 * n][i], f[0], f[2]);
                    decode4_half<FMT>(kr[2 * n + 1][i], f[1], f[3]);
                    mma_f16_16816(i & 1 ? s2 : s[n], f, qb[i][0], qb[i][1]);
                }
                // s[n][0], s[n][1]: position 16 n + g, heads 2 t and 2 t + 1; s[n][2], s[n][3]: position 16 n + g + 8
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] = (s[n][e] + s2[e]) * (e & 1 ? f1 : f0);
            }
            const int p0 = x * STEP + POS * warp;
            if (p0 < r.first || p0 > r.ctx - POS) {  // some are masked
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    const int at = p0 + 16 * n + g;
                    if (at < r.first || at >= r.ctx) s[n][0] = s[n][1] = -INFINITY;
                    if (at + 8 < r.first || at + 8 >= r.ctx) s[n][2] = s[n][3] = -INFINITY;
                }
            }
            float w[NG][4], t0 = 0.f, t1 = 0.f;
            auto probabilities = [&]() {
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[n][e] = ex2(s[n][e] - ((e & 1 ? m1 : m0) - kAttnKv8Shift));
            };
            probabilities();
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                t0 = fmaxf(t0, fmaxf(w[n][0], w[n][2]));
                t1 = fmaxf(t1, fmaxf(w[n][1], w[n][3]));
            }
            float g0 = vsc * r0, g1 = vsc * r1;
            constexpr float kMost = (float)(1 << (int)(kAttnKv8Shift + 8.f));
            if (__any_sync(0xffffffffu, t0 * fmaxf(fabsf(g0), 1.f) > kMost || t1 * fmaxf(fabsf(g1), 1.f) > kMost)) {
                float n0 = s[0][0], n1 = s[0][1];
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    n0 = fmaxf(n0, fmaxf(s[n][0], s[n][2]));
                    n1 = fmaxf(n1, fmaxf(s[n][1], s[n][3]));
                }
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, d));
                    n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, d));
                }
                // to the larger maximum, and to the larger of the step's products and those so far, whose logarithm -log2(r) is
                const float v = (float)scale_exp(vsc);
                auto rebase = [&](float n, float &m, float &r, float &l) {
                    const float up = fmaxf(m, n), down = m - up, was = (float)-scale_exp(r) + down;
                    const float k = fminf(fmaxf(ceilf(fmaxf(was, n - up + v)), -126.f), 126.f);
                    m = up;
                    r = pow2f(-(int)k);
                    l *= ex2(down);
                    return ex2(was - k);
                };
                const float a0 = rebase(n0, m0, r0, l0), a1 = rebase(n1, m1, r1, l1);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    o[j][0] *= a0;
                    o[j][1] *= a1;
                    o[j][2] *= a0;
                    o[j][3] *= a1;
                }
                probabilities();
                g0 = vsc * r0;
                g1 = vsc * r1;
            }
            // (an infinite factor, which only probabilities of 0 have left here, is to leave them 0; a NaN stays)
            g0 = min_nan(g0, 3.4028235e38f);
            g1 = min_nan(g1, 3.4028235e38f);
#pragma unroll
            for (int n = 0; n < NG; ++n) {
                l0 += w[n][0] + w[n][2];
                l1 += w[n][1] + w[n][3];
                const float w0 = w[n][0] * g0, w1 = w[n][1] * g1, w2 = w[n][2] * g0, w3 = w[n][3] * g1;
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
                    const uint32_t a = vr[4 * n][i], b = vr[4 * n + 1][i], c = vr[4 * n + 2][i], d = vr[4 * n + 3][i];
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

        // this warp's state: o[j][e], o[j][2 + e]: head 2 t + e, dims hd / 8 g + 2 j and + 1, at place 16 j + 2 g
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, d);
            l1 += __shfl_xor_sync(0xffffffffu, l1, d);
        }
        if (W > 1 && g == 0) {
            s_m[warp][2 * t] = m0;
            s_m[warp][2 * t + 1] = m1;
            s_l[warp][2 * t] = l0;
            s_l[warp][2 * t + 1] = l1;
            if (t == 0) s_free[warp] = fill;
        }
        const AttnKv8Join me = {row, h, unit, unit + r.steps - 1};
        const bool begins = unit >= lo, last = unit + r.steps >= hi, whole = begins && unit + r.steps <= hi;
        if (!last) {  // the next unit's queries come while this one is put together
            unit += r.steps;
            if (++h == KVH) {
                h = 0;
                do r = attn_kv8_row<STEP>(p, ++row);
                while (r.steps == 0);
            }
            begin();
        }
        const float u0 = pow2f(-scale_exp(r0)), u1 = pow2f(-scale_exp(r1));  // 1 / r
        float *state = p.part + (c * 2 + begins) * STATE;  // (a share begins in at most one unit that it does not begin)
        if constexpr (W == 1) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int hh = 2 * t + e;
                const float M = e ? m1 : m0, L = e ? l1 : l0, u = e ? u1 : u0, inv = 1.f / L;
                if (hh >= G) continue;
                if (whole) {
                    uint32_t y[NT];
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        y[j] = p.type == SARA_BF16 ? pack2<SARA_BF16>(o[j][e] * u * inv, o[j][2 + e] * u * inv)
                                                   : pack2<SARA_FP16>(o[j][e] * u * inv, o[j][2 + e] * u * inv);
                    uint32_t *out = reinterpret_cast<uint32_t *>(p.out + ((int64_t)me.row * p.H + me.h * G + hh) * HD + HD / 8 * g);
#pragma unroll
                    for (int j = 0; j < NT; j += 2) *reinterpret_cast<uint2 *>(out + j) = make_uint2(y[j], y[j + 1]);
                    if (p.lse && g == 0) p.lse[(int64_t)me.row * p.H + me.h * G + hh] = (M - kAttnKv8Shift + log2f(L)) * 0.69314718f;
                } else {
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        *reinterpret_cast<float2 *>(state + 16 + hh * HD + 16 * j + 2 * g) = make_float2(o[j][e] * u, o[j][2 + e] * u);
                    if (g == 0) {
                        state[hh] = M;
                        state[8 + hh] = L;
                    }
                }
            }
        } else {
            // put together by way of the warps' free stages, [8 heads][hd places]: conflict-free with places exchanged by eights
            auto at_of = [&](int w, int stage, int hh, int i) {
                return reinterpret_cast<float2 *>(s_ring + w * RING + stage * (2 * TILE)) + (hh * HD + (i ^ (hh / 2 * 8))) / 2;
            };
            __syncwarp();  // (every lane has left the stage)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                *at_of(warp, fill, 2 * t, 16 * j + 2 * g) = make_float2(o[j][0] * u0, o[j][2] * u0);
                *at_of(warp, fill, 2 * t + 1, 16 * j + 2 * g) = make_float2(o[j][1] * u1, o[j][3] * u1);
            }
            __syncthreads();
            int stage[kAttnKv8Warps];
#pragma unroll
            for (int w = 0; w < kAttnKv8Warps; ++w) stage[w] = s_free[w];
            for (int e = tid; e < G * HD / 2; e += kAttnKv8Threads) {
                const int hh = e / (HD / 2), i = e % (HD / 2) * 2;
                float M = s_m[0][hh], L = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
                for (int w = 1; w < kAttnKv8Warps; ++w) M = fmaxf(M, s_m[w][hh]);
#pragma unroll
                for (int w = 0; w < kAttnKv8Warps; ++w) {
                    const float2 y = *at_of(w, stage[w], hh, i);
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
                    *reinterpret_cast<float2 *>(state + 16 + hh * HD + i) = make_float2(y0, y1);
                    if (i == 0) {
                        state[hh] = M;
                        state[8 + hh] = L;
                    }
                }
            }
        }
        if (!whole && lane == 0 && warp == 0) s_join[begins] = {me.row, me.h, share_of(me.c0), share_of(me.c1)};
        attn_kv8_sync<W>();  // (shared memory is the next unit's)
        if (last) break;
    }
    if (wrong) kv8_report(p.status);

    // the units that other shares hold too: at most the one in which the share begins and the one in which it ends
    const int who = W == 1 ? lane : lane == 0 ? warp : 2;
    if (who < 2 && s_join[who].row >= 0) s_last[who] = AttnKv8Group<HD, W>(p, s_join[who], c).arrive();
    attn_kv8_sync<W>();
#pragma unroll 1
    for (int i = 0; i < 2; ++i)
        if (s_join[i].row >= 0 && s_last[i])
            attn_kv8_join<HD, W>({p, s_join[i], c}, reinterpret_cast<float *>(s_ring + mine * RING), &s_last[i], 32 * warp + lane);
}

inline int64_t attn_kv8_entries(int n, int kvh, int max_blocks, int step) { return (int64_t)n * kvh * max_blocks * (kKv8Page / step); }
inline int attn_kv8_warps(int n, int kvh, int hd, int max_blocks) {
    return (int64_t)n * kvh >= kAttnKv8Units && attn_kv8_entries(n, kvh, max_blocks, attn_kv8_step(hd, 1)) <= INT32_MAX ? 1 : kAttnKv8Warps;
}
inline size_t attn_kv8_count_bytes() { return kAttnKv8MaxShares * 2 * kAttnKv8Levels * sizeof(int); }
inline size_t attn_kv8_workspace(int hd, int warps) {
    return attn_kv8_count_bytes() + (size_t)kAttnKv8MaxShares / warps * 2 * attn_kv8_state(hd) * sizeof(float);
}

}  // namespace sara
