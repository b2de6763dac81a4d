// Log-probabilities of given tokens under softmax(logits), with entropy and top alternatives, and the gradient of both.
//   m = max z, S = sum e^(z - m), T = sum e^(z - m) (z - m)
//   logprob = z[token] - m - log S,   entropy = log S - T / S
//   dz_v = g (1[v = token] - p_v) - g' p_v (log p_v + entropy)
#pragma once
#include "device_common.cuh"
#include "host_util.h"

namespace sara {

constexpr int kScoreMaxTop = 32;

template <int TYPE>
__device__ __forceinline__ float load_logit(const void *z, int64_t i) {
    if constexpr (TYPE == SARA_FP32) return __ldg(static_cast<const float *>(z) + i);
    else if constexpr (TYPE == SARA_BF16) return bf16_to_f32(__ldg(static_cast<const uint16_t *>(z) + i));
    else return f16_to_f32(__ldg(static_cast<const uint16_t *>(z) + i));
}

struct ScoreParams {
    const void *z;
    int64_t stride;
    int R, V, top;
    const int32_t *tokens;
    float *logprob, *entropy, *stats;
    int32_t *top_token;
    float *top_logprob;
};

// A logit's place in the order of the alternatives: by value, then the lower token; 0 for one that is not listed.
__device__ __forceinline__ uint64_t score_key(float z, int v) {
    if (!(z > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(z + 0.f);  // (-0 as 0)
    return ((uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32) | (uint32_t)(0x7fffffff - v);
}
__device__ __forceinline__ float score_key_value(uint64_t k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int score_key_token(uint64_t k) { return 0x7fffffff - (int)(uint32_t)k; }

template <typename T, typename F>
__device__ __forceinline__ T block_reduce256(T x, T *room, F f) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = f(x, __shfl_xor_sync(0xffffffffu, x, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = x;
    __syncthreads();
    x = room[0];
    for (int w = 1; w < 8; ++w) x = f(x, room[w]);
    return x;
}

// One CTA per row: the maximum, the sums against it, and one pass for each alternative.
template <int TYPE>
__global__ void __launch_bounds__(256) score_kernel(ScoreParams p) {
    __shared__ float room[8];
    __shared__ uint64_t kroom[8];
    const int r = blockIdx.x, tok = p.tokens ? p.tokens[r] : 0;
    const int64_t row = r * p.stride;
    const float nan = __int_as_float(0x7fc00000);
    if (tok < 0) {
        if (threadIdx.x == 0) {
            if (p.logprob) p.logprob[r] = 0.f;
            if (p.entropy) p.entropy[r] = 0.f;
            if (p.stats) p.stats[2 * (int64_t)r] = p.stats[2 * (int64_t)r + 1] = 0.f;
        }
        for (int j = threadIdx.x; j < p.top; j += 256) {
            p.top_token[(int64_t)r * p.top + j] = -1;
            p.top_logprob[(int64_t)r * p.top + j] = -INFINITY;
        }
        return;
    }
    float m = -INFINITY;
    for (int64_t v = threadIdx.x; v < p.V; v += 256) m = fmaxf(m, load_logit<TYPE>(p.z, row + v));
    m = block_reduce256(m, room, [](float a, float b) { return fmaxf(a, b); });
    float S = 0.f, T = 0.f;
    for (int64_t v = threadIdx.x; v < p.V; v += 256) {
        const float z = load_logit<TYPE>(p.z, row + v);
        if (z == -INFINITY) continue;
        const float d = z - m, e = expf(d);
        S += e;
        T += e > 0.f ? e * d : e;
    }
    S = block_reduce256(S, room, [](float a, float b) { return a + b; });
    T = block_reduce256(T, room, [](float a, float b) { return a + b; });
    const bool none = S == 0.f;  // every logit is -inf
    const float ls = none ? 0.f : logf(S);
    if (threadIdx.x == 0) {
        const float z = tok < p.V ? load_logit<TYPE>(p.z, row + tok) : nan;
        if (p.logprob) p.logprob[r] = none && tok < p.V ? -INFINITY : z - m - ls;
        if (p.entropy) p.entropy[r] = none ? 0.f : ls - T / S;
        if (p.stats) {
            p.stats[2 * (int64_t)r] = m;
            p.stats[2 * (int64_t)r + 1] = ls;
        }
    }
    uint64_t last = ~0ull;
    for (int j = 0; j < p.top; ++j) {
        uint64_t best = 0;
        for (int64_t v = threadIdx.x; v < p.V; v += 256) {
            const uint64_t k = score_key(load_logit<TYPE>(p.z, row + v), (int)v);
            if (k < last && k > best) best = k;
        }
        best = block_reduce256(best, kroom, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        last = best;
        if (threadIdx.x == 0) {
            p.top_token[(int64_t)r * p.top + j] = best ? score_key_token(best) : -1;
            p.top_logprob[(int64_t)r * p.top + j] = best ? score_key_value(best) - m - ls : -INFINITY;
        }
    }
}

struct ScoreGradParams {
    const void *z;
    int64_t stride;
    int R, V;
    const int32_t *tokens;
    const float *stats, *entropy, *glp, *gent;
    void *out;
    int64_t out_stride;
};

// One CTA per row.  (Not __ldg: the gradient may take the logits' place.)
template <int TYPE>
__global__ void __launch_bounds__(256) score_grad_kernel(ScoreGradParams p) {
    const int r = blockIdx.x, tok = p.tokens ? p.tokens[r] : 0;
    const int64_t row = r * p.stride, orow = r * p.out_stride;
    const float m = p.stats[2 * (int64_t)r], ls = p.stats[2 * (int64_t)r + 1];
    const float g = p.glp ? p.glp[r] : 0.f, gh = p.gent ? p.gent[r] : 0.f, H = p.gent ? p.entropy[r] : 0.f;
    const bool zero = tok < 0 || (m == -INFINITY && ls == 0.f), wrong = tok >= p.V;
    for (int64_t v = threadIdx.x; v < p.V; v += 256) {
        float y = 0.f;
        if (wrong) {
            y = __int_as_float(0x7fc00000);
        } else if (!zero) {
            float z;
            if constexpr (TYPE == SARA_FP32) z = static_cast<const float *>(p.z)[row + v];
            else if constexpr (TYPE == SARA_BF16) z = bf16_to_f32(static_cast<const uint16_t *>(p.z)[row + v]);
            else z = f16_to_f32(static_cast<const uint16_t *>(p.z)[row + v]);
            const float lp = z - m - ls, q = expf(lp);
            y = g * ((v == tok ? 1.f : 0.f) - q) - (q == 0.f ? 0.f : gh * q * (lp + H));
        }
        if constexpr (TYPE == SARA_FP32) static_cast<float *>(p.out)[orow + v] = y;
        else if constexpr (TYPE == SARA_BF16) static_cast<uint16_t *>(p.out)[orow + v] = f32_to_bf16(y);
        else static_cast<uint16_t *>(p.out)[orow + v] = __half_as_ushort(__float2half_rn(y));
    }
}

}  // namespace sara
