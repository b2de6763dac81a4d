// Entry point of the attention of groups behind a common prefix: sara_attention_shared_kv8.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/sara.h"
#include "attn_shared.cuh"
#include "host_util.h"
#include "kv8_host.h"

using namespace sara;

namespace {

// Where a call's parts stand in the workspace.  What has to be zero comes first, at the same place whatever the sizes.
struct SharedLayout {
    size_t own, group, row_group, row_first, row_prefix, out32, lse, whole, part, bytes;
};
SharedLayout shared_layout(int n, int groups, int H, int kvh, int hd) {
    SharedLayout w{};
    size_t at = sizeof(SharedPlan);
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += (bytes + 255) / 256 * 256;
        return was;
    };
    const size_t rows = (size_t)n, states = rows * H;
    w.own = take(attn_kv8_workspace(hd, attn_kv8_warps(n, kvh, hd, 1)));
    w.group = take((size_t)groups * sizeof(SharedGroup));
    w.row_group = take(rows * 4);
    w.row_first = take(rows * 4);
    w.row_prefix = take(rows * 4);
    w.out32 = take(states * hd * 4);
    w.lse = take(states * 4);
    w.whole = take(states * shared_state(hd) * 4);
    w.part = take((size_t)kSharedMaxShares * 2 * kSharedQ * shared_state(hd) * 4);
    w.bytes = at;
    return w;
}

template <typename T>
T *at(void *ws, size_t off) {
    return reinterpret_cast<T *>(static_cast<uint8_t *>(ws) + off);
}

// Whether each row reads all of its positions by itself, in one launch of the decode attention.  Four launches cost some 15 us more, and the
// prefix kernel takes a page in twice the time that reading it takes: with k rows to a group, of which a share f is common, it saves
// f (1 - 2 / k) of the bytes' time, nothing for pairs.  The lengths are on the device: the bytes are those that the table's rows have room
// for.  us alone and shared, half of all positions common (where two are given: and 9 of 10), 128 dims: k = 2, 512 MB 102, 119 (2 GB: 324,
// 352); k = 3, 384 MB 72, 86 (79), 768 MB 130, 136 (120); k = 4, 256 MB 57, 66 (56), 512 MB 94, 97 (83); k = 8, 64 MB 24, 35 (34), 128 MB
// 33, 42 (36); k = 16, 128 MB 32, 37 (34), 256 MB 50, 56 (40); k = 64, 128 MB 32, 41 (33), 256 MB 50, 57 (39); alike in 64 and 32 dims.
bool shared_alone(int n, int groups, int kvh, int hd, int max_blocks) {
    const int64_t blocks = (int64_t)n * kvh * max_blocks;
    if (blocks > 1 << 28) return false;  // (steps are counted in 32 bits)
    return n <= 2 * (int64_t)groups || groups == 0 || (double)blocks * (kKv8Page * 2 * hd) * (1. - 2. * groups / n) <= kSharedAlone;
}

template <int HD, int FMT>
void shared_launch(const SharedParams &p, int shares, cudaStream_t s) {
    const auto kern = shared_prefix_kernel<HD, FMT>;
    static SmemOnce smem;
    smem.ask(kern, shared_smem(HD));
    launch_cluster(s, true, dim3((unsigned)shares), dim3(kSharedThreads), shared_smem(HD), 1, kern, p);
}
template <int HD>
void shared_join(const SharedParams &p, int shares, cudaStream_t s) {
    const int64_t states = (int64_t)p.n * p.H;
    if (states <= kSharedWideJoin) shared_join_kernel<HD, 8><<<(unsigned)states, 256, 0, s>>>(p, shares);
    else shared_join_kernel<HD, 1><<<(unsigned)((states + 7) / 8), 256, 0, s>>>(p, shares);
    CK(cudaGetLastError());
}

}  // namespace

extern "C" {

size_t sara_attention_shared_kv8_workspace_bytes(int32_t n_seq, int32_t n_groups, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (n_seq < 1 || n_groups < 0 || n_heads < 1 || n_kv_heads < 1 || head_dim < 1 || (int64_t)n_seq * n_heads > INT32_MAX) return 0;
    return shared_layout(n_seq, n_groups, n_heads, n_kv_heads, head_dim).bytes;
}

int sara_attention_shared_kv8(const sara_kv8_cache *cache, int32_t n_seq, int32_t n_heads, const void *q, int64_t q_stride,
                              const int32_t *ctx, const int32_t *first, int32_t n_groups, const int32_t *group_start,
                              const int32_t *prefix, void *out, float *lse, int32_t type, int32_t *status, void *workspace,
                              size_t workspace_bytes, void *stream) {
    if (!cache_ok(cache, n_seq) || n_seq < 0 || n_groups < 0 || n_heads < 1 || (type != SARA_BF16 && type != SARA_FP16)) return SARA_EINVAL;
    if (n_heads % cache->n_kv_heads || n_heads / cache->n_kv_heads > 8) return SARA_EINVAL;
    if (n_seq == 0) return SARA_OK;
    if (!q || !ctx || !out || !workspace || (n_groups > 0 && (!group_start || !prefix))) return SARA_EINVAL;
    if (misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 256)) return SARA_EINVAL;
    if (q_stride % 8 || (n_seq > 1 && q_stride < (int64_t)n_heads * cache->head_dim)) return SARA_EINVAL;
    if ((int64_t)n_seq * n_heads > INT32_MAX || n_groups > n_seq) return SARA_EINVAL;
    return op_guard([&] {
        if ((int64_t)n_seq * cache->n_kv_heads > (((int64_t)1 << 30) - 1) / cache->max_blocks) throw SaraError(SARA_EINVAL, "too many blocks");
        const int hd = cache->head_dim, warps = attn_kv8_warps(n_seq, cache->n_kv_heads, hd, cache->max_blocks);
        const SharedLayout w = shared_layout(n_seq, n_groups, n_heads, cache->n_kv_heads, hd);
        if (workspace_bytes < w.bytes) throw SaraError(SARA_EINVAL, "workspace too small");
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        AttnKv8Params a{};
        a.c = device_cache(cache);
        a.q = static_cast<const uint16_t *>(q);
        a.q_stride = q_stride;
        a.ctx = ctx;
        a.status = status;
        a.n = n_seq;
        a.H = n_heads;
        a.type = type;
        a.count = at<int>(workspace, w.own);
        a.part = reinterpret_cast<float *>(at<uint8_t>(workspace, w.own) + attn_kv8_count_bytes());
        a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)hd));
        if (shared_alone(n_seq, n_groups, cache->n_kv_heads, hd, cache->max_blocks)) {
            a.first = first;
            a.out = static_cast<uint16_t *>(out);
            a.lse = lse;
            a.start = group_start;
            a.prefix = prefix;
            a.groups = n_groups;
            attn_kv8_launch(cache, a, warps, s);
            return;
        }
        SharedParams p{};
        p.c = a.c;
        p.q = a.q;
        p.q_stride = q_stride;
        p.ctx = ctx;
        p.first = first;
        p.start = group_start;
        p.prefix = prefix;
        p.n = n_seq;
        p.groups = n_groups;
        p.H = n_heads;
        p.type = type;
        p.scale_log2 = a.scale_log2;
        p.status = status;
        p.plan = at<SharedPlan>(workspace, 0);
        p.group = at<SharedGroup>(workspace, w.group);
        p.row_group = at<int>(workspace, w.row_group);
        p.row_first = at<int>(workspace, w.row_first);
        p.row_prefix = at<int>(workspace, w.row_prefix);
        p.whole = at<float>(workspace, w.whole);
        p.part = at<float>(workspace, w.part);
        p.own = at<float>(workspace, w.out32);
        p.own_lse = at<float>(workspace, w.lse);
        p.out = static_cast<uint16_t *>(out);
        p.lse = lse;
        const int shares = std::min(sm_count(), kSharedMaxShares);
        p.max_shares = shares;
        shared_plan_kernel<<<1, 1024, 0, s>>>(p);
        CK(cudaGetLastError());
        by_shape(cache, [&](auto d, auto fmt) { shared_launch<d.value, fmt.value>(p, shares, s); });
        a.first = p.row_first;
        a.out32 = at<float>(workspace, w.out32);
        a.lse = at<float>(workspace, w.lse);
        attn_kv8_launch(cache, a, warps, s);
        by_shape(cache, [&](auto d, auto) { shared_join<d.value>(p, shares, s); });
    });
}

}  // extern "C"
