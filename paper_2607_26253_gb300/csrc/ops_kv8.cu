// Entry points of the 8-bit paged KV cache: sara_kv8_write, sara_kv8_read, sara_attention_decode_kv8.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/sara.h"
#include "attn_kv8.cuh"
#include "host_util.h"
#include "kv8.cuh"
#include "kv8_host.h"

using namespace sara;

namespace {

// Rows of n_kv_heads * head_dim elements of `size` bytes, `stride` elements apart
bool rows_ok(const sara_kv8_cache *c, const void *p, int64_t stride, int total) {
    return p && !misaligned(p, 16) && stride % 8 == 0 && (total <= 1 || stride >= (int64_t)c->n_kv_heads * c->head_dim);
}

unsigned warp_ctas(int64_t warps) {
    const int64_t ctas = (warps + 3) / 4;
    if (ctas > INT32_MAX) throw SaraError(SARA_EINVAL, "too many tokens");
    return (unsigned)ctas;
}

}  // namespace

// (declared in attn_kv8.cuh)
void sara::attn_kv8_launch(const sara_kv8_cache *cache, const AttnKv8Params &p, int warps, cudaStream_t s) {
    // as many CTAs as fit, fewer where there are not as many entries
    const int64_t entries = attn_kv8_entries(p.n, cache->n_kv_heads, cache->max_blocks, attn_kv8_step(cache->head_dim, warps));
    const unsigned ctas = (unsigned)std::min<int64_t>(std::min(kAttnKv8SmCtas * sm_count(), kAttnKv8MaxCtas), (entries + kAttnKv8Warps / warps - 1) / (kAttnKv8Warps / warps));
    by_shape(cache, [&](auto hd, auto fmt) {
        const auto kern = p.groups ? attn_kv8_kernel<hd.value, fmt.value, kAttnKv8Warps, true>
                          : warps == 1 ? attn_kv8_kernel<hd.value, fmt.value, 1> : attn_kv8_kernel<hd.value, fmt.value, kAttnKv8Warps>;
        static_assert(attn_kv8_smem(hd.value) <= 48 * 1024, "more would have to be asked for");
        kern<<<ctas, kAttnKv8Threads, attn_kv8_smem(hd.value), s>>>(p);
    });
    CK(cudaGetLastError());
}

extern "C" {

int sara_kv8_write(const sara_kv8_cache *cache, int32_t n_seq, const int32_t *pos0, const int32_t *seq_start, int32_t total,
                   const void *k, int64_t k_stride, const void *v, int64_t v_stride, int32_t type, int32_t *status,
                   void *stream) {
    if (!cache_ok(cache, n_seq) || n_seq < 0 || n_seq > kKv8MaxSeqs || total < 0 || (type != SARA_BF16 && type != SARA_FP16)) return SARA_EINVAL;
    if (n_seq == 0 || total == 0) return SARA_OK;
    if (!pos0 || !seq_start || !rows_ok(cache, k, k_stride, total) || !rows_ok(cache, v, v_stride, total)) return SARA_EINVAL;
    return op_guard([&] {
        const int64_t warps = kv8_units(total, n_seq) * cache->n_kv_heads * 2;
        const unsigned ctas = warp_ctas(warps);
        const Kv8Range r{pos0, seq_start, n_seq, total};
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        by_shape(cache, [&](auto hd, auto fmt) {
            const auto kern = type == SARA_BF16 ? kv8_write_kernel<hd.value, fmt.value, SARA_BF16>
                                                : kv8_write_kernel<hd.value, fmt.value, SARA_FP16>;
            kern<<<ctas, 128, 0, s>>>(device_cache(cache), r, static_cast<const uint16_t *>(k), k_stride,
                                      static_cast<const uint16_t *>(v), v_stride, warps, status);
        });
        CK(cudaGetLastError());
    });
}

int sara_kv8_read(const sara_kv8_cache *cache, int32_t n_seq, const int32_t *pos0, const int32_t *seq_start, int32_t total,
                  void *k, int64_t k_stride, void *v, int64_t v_stride, int32_t type, int32_t *status, void *stream) {
    if (!cache_ok(cache, n_seq) || n_seq < 0 || n_seq > kKv8MaxSeqs || total < 0 || type < SARA_BF16 || type > SARA_FP32) return SARA_EINVAL;
    if (n_seq == 0 || total == 0) return SARA_OK;
    if (!pos0 || !seq_start || !rows_ok(cache, k, k_stride, total) || !rows_ok(cache, v, v_stride, total)) return SARA_EINVAL;
    return op_guard([&] {
        const int64_t warps = kv8_units(total, n_seq) * cache->n_kv_heads * 2;
        const unsigned ctas = warp_ctas(warps);
        const Kv8Range r{pos0, seq_start, n_seq, total};
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        by_shape(cache, [&](auto hd, auto fmt) {
            const auto kern = type == SARA_BF16   ? kv8_read_kernel<hd.value, fmt.value, SARA_BF16>
                              : type == SARA_FP16 ? kv8_read_kernel<hd.value, fmt.value, SARA_FP16>
                                                  : kv8_read_kernel<hd.value, fmt.value, SARA_FP32>;
            kern<<<ctas, 128, 0, s>>>(device_cache(cache), r, static_cast<uint8_t *>(k), k_stride, static_cast<uint8_t *>(v), v_stride,
                                      warps, status);
        });
        CK(cudaGetLastError());
    });
}

size_t sara_attention_kv8_workspace_bytes(int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (n_seq < 1 || n_heads < 1 || n_kv_heads < 1 || head_dim < 1) return 0;
    return attn_kv8_workspace(head_dim, attn_kv8_warps(n_seq, n_kv_heads, head_dim, 1));
}

int sara_attention_decode_kv8(const sara_kv8_cache *cache, int32_t n_seq, int32_t n_heads, const void *q, int64_t q_stride,
                              const int32_t *ctx, const int32_t *first, void *out, float *lse, int32_t type, int32_t *status,
                              void *workspace, size_t workspace_bytes, void *stream) {
    if (!cache_ok(cache, n_seq) || n_seq < 0 || n_heads < 1 || (type != SARA_BF16 && type != SARA_FP16)) return SARA_EINVAL;
    if (n_heads % cache->n_kv_heads || n_heads / cache->n_kv_heads > 8) return SARA_EINVAL;
    if (n_seq == 0) return SARA_OK;
    if (!q || !ctx || !out || !workspace || misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 16)) return SARA_EINVAL;
    if (q_stride % 8 || (n_seq > 1 && q_stride < (int64_t)n_heads * cache->head_dim)) return SARA_EINVAL;
    if ((int64_t)n_seq * n_heads > INT32_MAX) return SARA_EINVAL;
    return op_guard([&] {
        // (counts of entries, at most two a block and CTA, in 32 bits)
        if ((int64_t)n_seq * cache->n_kv_heads > (((int64_t)1 << 30) - 1) / cache->max_blocks) throw SaraError(SARA_EINVAL, "too many blocks");
        const int hd = cache->head_dim, warps = attn_kv8_warps(n_seq, cache->n_kv_heads, hd, cache->max_blocks);
        if (workspace_bytes < attn_kv8_workspace(hd, warps)) throw SaraError(SARA_EINVAL, "workspace too small");
        AttnKv8Params p{};
        p.c = device_cache(cache);
        p.q = static_cast<const uint16_t *>(q);
        p.q_stride = q_stride;
        p.ctx = ctx;
        p.first = first;
        p.out = static_cast<uint16_t *>(out);
        p.lse = lse;
        p.status = status;
        p.n = n_seq;
        p.H = n_heads;
        p.type = type;
        p.count = static_cast<int *>(workspace);
        p.part = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + attn_kv8_count_bytes());
        p.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)cache->head_dim));
        attn_kv8_launch(cache, p, warps, static_cast<cudaStream_t>(stream));
    });
}

}  // extern "C"
