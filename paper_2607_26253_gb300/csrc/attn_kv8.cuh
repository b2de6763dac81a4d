// Decode attention over the 8-bit paged KV cache: one query row per sequence,
//     out[i, h] = softmax(q[i, h] . K[first_i .. ctx_i)^T / sqrt(hd)) V[first_i .. ctx_i)
#pragma once
#include "kv8.cuh"

namespace sara {

struct AttnKv8Params {
    Kv8Cache c;
    const uint16_t *q;
    int64_t q_stride;
    const int32_t *ctx, *first;
    uint16_t *out;
    float *lse;
    int32_t *status;
    int n, H;
    float scale_log2;  // log2(e) / sqrt(hd)
};

// One CTA per row and query head, a warp per position, the warps' states joined in shared memory.
template <int HD, int FMT, int TYPE>
__global__ void __launch_bounds__(128) attn_kv8_kernel(AttnKv8Params p) {
    constexpr int PD = HD / 32;  // dims a lane
    __shared__ float s_m[4], s_l[4], s_o[4][HD];
    const int row = blockIdx.x / p.H, head = blockIdx.x % p.H, G = p.H / p.c.KVH, h = head / G;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t at = (int64_t)row * p.H + head;
    const int ctx = p.ctx[row], first = p.first ? min(p.first[row], ctx) : 0;  // (past the end: no position)
    bool bad = ctx < 0 || first < 0 || ctx > (int64_t)p.c.max_blocks * kKv8Page;
    float q[PD], o[PD], m = -3.4028235e38f, l = 0.f;
#pragma unroll
    for (int i = 0; i < PD; ++i) {
        q[i] = unpack2<TYPE>(p.q[row * p.q_stride + head * HD + lane * PD + i]).x * p.scale_log2;
        o[i] = 0.f;
    }
    for (int x = first + warp; x < ctx && !bad; x += 4) {
        const int block = p.c.table[row * p.c.table_stride + x / kKv8Page];
        if (block < 0 || block >= p.c.n_blocks) {
            bad = true;
            break;
        }
        const int64_t tk = kv8_tile(p.c, block, 0, h), tv = kv8_tile(p.c, block, 1, h);
        const int part = x % kKv8Page / kKv8Block;
        const uint8_t *k = p.c.codes + (tk * kKv8Page + x % kKv8Page) * HD + lane * PD;
        const uint8_t *v = p.c.codes + (tv * kKv8Page + x % kKv8Page) * HD + lane * PD;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < PD; ++i) s = fmaf(q[i], decode2<FMT>(k[i]).x, s);
        s = warp_sum(s) * p.c.scales[tk * kKv8PageBlocks + part];
        if (s > m) {
            const float a = exp2f(m - s);
            l *= a;
#pragma unroll
            for (int i = 0; i < PD; ++i) o[i] *= a;
            m = s;
        }
        const float w = exp2f(s - m);
        l += w;
#pragma unroll
        for (int i = 0; i < PD; ++i) o[i] = fmaf(w * p.c.scales[tv * kKv8PageBlocks + part], decode2<FMT>(v[i]).x, o[i]);
    }
    if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
    }
#pragma unroll
    for (int i = 0; i < PD; ++i) s_o[warp][lane * PD + i] = o[i];
    bad = __syncthreads_or(bad);
    if (bad && threadIdx.x == 0) kv8_report(p.status);
    float M = s_m[0], L = 0.f;
    for (int w = 1; w < 4; ++w) M = fmaxf(M, s_m[w]);
    for (int w = 0; w < 4; ++w) L += s_l[w] * exp2f(s_m[w] - M);
    const bool empty = ctx <= first;
    if (threadIdx.x < HD) {
        float y = 0.f;
        for (int w = 0; w < 4; ++w) y += s_o[w][threadIdx.x] * exp2f(s_m[w] - M);
        y = bad ? __int_as_float(0x7fc00000) : empty ? 0.f : y / L;
        p.out[at * HD + threadIdx.x] = (uint16_t)pack2<TYPE>(y, 0.f);
    }
    if (p.lse && threadIdx.x == 0)
        p.lse[at] = bad ? __int_as_float(0x7fc00000) : empty ? -INFINITY : (M + log2f(L)) * 0.69314718f;
}

inline size_t attn_kv8_workspace(int n, int KVH) { return ((size_t)n * KVH * sizeof(int) + 255) / 256 * 256; }

}  // namespace sara
