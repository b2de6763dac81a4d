// Entry points of log-probabilities from hidden states: sara_linear_logprobs, sara_linear_logprobs_backward.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "../../include/sara.h"
#include "host_util.h"
#include "linear_logprob.cuh"

using namespace sara;

namespace {

struct Operand {
    const void *p;
    int64_t rows, stride, d;  // rows of d elements, stride elements apart
    const uint8_t *begin() const { return static_cast<const uint8_t *>(p); }
    const uint8_t *end() const { return begin() + ((rows - 1) * stride + d) * 2; }
    bool ok() const { return p && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0 && (rows <= 1 || stride >= d); }
    bool meets(const Operand &o) const { return p && o.p && rows && o.rows && begin() < o.end() && o.begin() < end(); }
};

// Rows of 16-bit elements as a 2-D tensor map with 128-byte swizzling, boxes of 64 x `box` (elements out of range: 0)
CUtensorMap rows_map(const Operand &x, int box) {
    CUtensorMap tm;
    const cuuint64_t dims[2] = {(cuuint64_t)x.d, (cuuint64_t)x.rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(x.rows > 1 ? x.stride : lin_up(x.d, 8)) * 2};
    const cuuint32_t size[2] = {64, (cuuint32_t)box}, step[2] = {1, 1};
    const CUresult r = encode_tiled_fn()(&tm, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void *>(x.p), dims, strides, size, step,
                                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) throw SaraError(SARA_EINVAL, "cuTensorMapEncodeTiled failed (" + std::to_string((int)r) + ")");
    return tm;
}

bool sizes_ok(int type, int R, int d, int V, float scale) {
    return (type == SARA_BF16 || type == SARA_FP16) && R >= 0 && R <= (1 << 22) && d >= 8 && d <= 65536 && d % 8 == 0 && V >= 1 &&
           V <= (1 << 24) && scale > 0.f && scale <= 0x1p127f;  // (log2(e) times it is finite)
}

template <int MODE, int CTAS, int TYPE, bool STAGED, bool LONG = false>
void launch(cudaStream_t s, int sms, bool after, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &a2, const CUtensorMap &b2,
            const CUtensorMap &out, const LinParams &p) {
    const auto kern = lin_kernel<MODE, CTAS, TYPE, STAGED, LONG>;
    static SmemOnce smem;
    smem.ask(kern, lin_smem(CTAS, STAGED));
    launch_cluster(s, after, dim3((unsigned)(sms / CTAS * CTAS)), dim3(kLinThreads), lin_smem(CTAS, STAGED), CTAS, kern, a, b, a2, b2, out, p);
}

template <typename T>
T *at(void *ws, size_t off) {
    return reinterpret_cast<T *>(static_cast<uint8_t *>(ws) + off);
}

// The live rows gathered, with what the gradient's rows are raised by, and (where dW is wanted) the order of their tokens and the rows as its product has them
template <int TYPE>
void gather(cudaStream_t s, void *ws, const LinPlan &q, const Operand &h, const int32_t *tokens, const float *glp, const float *gent, bool backward,
            bool weights) {
    const int R = (int)h.rows, d = (int)h.d;
    int *kexp = backward ? at<int>(ws, q.kexp) : nullptr, *tokc = backward ? at<int>(ws, q.tokc) : nullptr;
    const LinRowParams rows{at<LinHeader>(ws, 0), R, tokens, glp, gent, at<int>(ws, q.src), at<int>(ws, q.pos), kexp, tokc, TYPE == SARA_FP16};
    const int row_ctas = q.rows_cap / 8, sort_ctas = weights ? (int)std::min<int64_t>(((int64_t)R + q.buckets + 32) / 32, 2048) : 0;
    const LinGatherParams p{at<LinHeader>(ws, 0), static_cast<const uint16_t *>(h.p), h.stride, d, kLinRows * q.ctas, at<int>(ws, q.src), kexp,
                            at<uint16_t>(ws, q.rows), weights && TYPE == SARA_FP16, row_ctas, tokc,
                            backward ? at<int2>(ws, q.sorted) : nullptr, backward ? at<int>(ws, q.start) : nullptr, q.buckets};
    const dim3 grid((unsigned)(row_ctas + sort_ctas), (unsigned)((d + kLinGatherCols - 1) / kLinGatherCols));
    if (R <= kLinFew) {
        launch_cluster(s, false, grid, dim3(256), 0, 1, lin_gather_kernel<true>, p, rows);
    } else {
        lin_rows_kernel<<<1, 1024, 0, s>>>(rows);
        CK(cudaGetLastError());
        launch_cluster(s, true, grid, dim3(256), 0, 1, lin_gather_kernel<false>, p, rows);
    }
    if (!p.raise) return;
    const LinLowParams low{p.head, d, p.tile, p.src, kexp, p.out, at<uint16_t>(ws, q.low)};
    launch_cluster(s, true, dim3((unsigned)row_ctas, grid.y), dim3(256), 0, 1, lin_low_kernel, low);
}

template <int CTAS, int TYPE>
void score(cudaStream_t s, int sms, void *ws, const LinPlan &q, const Operand &h, const Operand &w, const int32_t *tokens, float scale,
           float *logprob, float *entropy, float *stats) {
    const int R = (int)h.rows, d = (int)h.d, V = (int)w.rows;
    Operand x = h;
    if (q.gather) {
        gather<TYPE>(s, ws, q, h, tokens, nullptr, nullptr, false, false);
        x = {at<void>(ws, q.rows), q.rows_cap, d, d};
    }
    LinParams p{};
    p.head = at<LinHeader>(ws, 0);
    p.R = R;
    p.d = d;
    p.V = V;
    p.cols = V;
    p.tokens = tokens;
    p.src = q.gather ? at<int>(ws, q.src) : nullptr;
    p.scale = scale;
    p.part = at<float>(ws, q.part);
    p.ztok = at<float>(ws, q.ztok);
    p.rows_cap = q.rows_cap;
    p.token_tiles = q.tiles;
    p.a_rows = CTAS == 1 ? (int)lin_up(R, 8) : kLinRows;
    const CUtensorMap a = rows_map(x, p.a_rows), b = rows_map(w, kLinCols / CTAS);
    launch<LIN_SCORE, CTAS, TYPE, false>(s, sms, q.gather, a, b, a, b, a, p);
    const LinJoinParams j{p.head, R, V, q.tiles, q.rows_cap, tokens, q.gather ? at<int>(ws, q.pos) : nullptr, p.part, p.ztok, scale, logprob, entropy, stats};
    if (R <= 64) launch_cluster(s, true, dim3((unsigned)R), dim3(256), 0, 1, lin_join_kernel<1>, j);
    else launch_cluster(s, true, dim3((unsigned)(R + 7) / 8), dim3(256), 0, 1, lin_join_kernel<8>, j);
}

template <int CTAS, int TYPE>
void gradient(cudaStream_t s, int sms, void *ws, const LinPlan &q, const Operand &h, const Operand &w, const int32_t *tokens, const float *stats,
              const float *entropy, const float *glp, const float *gent, float scale, const Operand &dh, const Operand &dw) {
    const int R = (int)h.rows, d = (int)h.d, V = (int)w.rows;
    gather<TYPE>(s, ws, q, h, tokens, glp, gent, true, dw.p != nullptr);
    const Operand x{at<void>(ws, q.rows), q.rows_cap, d, d}, low{TYPE == SARA_FP16 ? at<void>(ws, q.low) : x.p, q.rows_cap, d, d};
    const Operand dz{at<void>(ws, q.dz), (int64_t)q.rows_cap * (q.piece / 64), 64, 64};  // blocks of 64 columns
    LinParams p{};
    p.head = at<LinHeader>(ws, 0);
    p.R = R;
    p.d = d;
    p.V = V;
    p.tokens = tokens;
    p.src = at<int>(ws, q.src);
    p.kexp = at<int>(ws, q.kexp);
    p.scale = scale;
    p.rows_cap = q.rows_cap;
    p.stats = stats;
    p.entropy = entropy;
    p.glp = glp;
    p.gent = gent;
    p.sorted = at<int2>(ws, q.sorted);
    p.start = at<int>(ws, q.start);
    p.buckets = q.buckets;
    p.delta = at<float>(ws, q.delta);
    p.low = static_cast<const uint16_t *>(low.p);
    p.acc = at<float>(ws, q.acc);
    p.splits = q.splits;
    p.dh = dh.p != nullptr;
    p.dw = dw.p != nullptr;
    p.a_rows = CTAS == 1 ? (int)lin_up(R, 8) : kLinRows;
    const CUtensorMap xk = rows_map(x, p.a_rows), wk = rows_map(w, kLinCols / CTAS), dzk = rows_map(dz, p.a_rows), dzs = rows_map(dz, kLinRows);
    const CUtensorMap dzm = rows_map(dz, kLinK), wn = rows_map(w, kLinK), xn = rows_map(low, kLinK), out = dw.p ? rows_map(dw, kLinRows) : dzs;
    // (up to 128 rows a piece is not that long)
    const bool many = CTAS == 2 && std::max(lin_up(R, kLinK), lin_up(std::min(q.piece, V), kLinK) / q.splits) > (int64_t)kLinLong * kLinK;
    for (int v = 0; v < V; v += q.piece) {
        p.v0 = v;
        p.cols = V - v < q.piece ? V - v : q.piece;
        p.first = v == 0;
        p.out = at<uint16_t>(ws, q.dz);
        p.out_stride = 64;
        p.wide = true;
        if (TYPE == SARA_BF16 && d > kLinLongPart * kLinK) launch<LIN_DZ, CTAS, TYPE, CTAS == 1, TYPE == SARA_BF16>(s, sms, true, xk, wk, xk, wk, dzs, p);
        else launch<LIN_DZ, CTAS, TYPE, CTAS == 1>(s, sms, true, xk, wk, xk, wk, dzs, p);
        p.out = static_cast<uint16_t *>(const_cast<void *>(dw.p));
        p.out_stride = dw.stride;
        p.wide = (reinterpret_cast<uintptr_t>(dw.p) & 31) == 0 && dw.stride % 16 == 0;
        if (many) launch<LIN_GRAD, 2, TYPE, false, true>(s, sms, true, dzk, wn, dzm, xn, out, p);
        else if (CTAS == 1 || R <= kLinStagedRows) launch<LIN_GRAD, CTAS, TYPE, true>(s, sms, true, dzk, wn, dzm, xn, out, p);
        else launch<LIN_GRAD, CTAS, TYPE, CTAS == 1>(s, sms, true, dzk, wn, dzm, xn, out, p);
    }
    const LinOutParams o{p.head, R, d, q.splits, q.rows_cap, at<int>(ws, q.pos), p.kexp, p.acc, p.delta, tokens, V, static_cast<const uint16_t *>(w.p), w.stride,
                         scale, static_cast<uint16_t *>(const_cast<void *>(dh.p)), dh.stride, static_cast<uint16_t *>(const_cast<void *>(dw.p)), dw.stride};
    launch_cluster(s, true, dim3((unsigned)(R + 7) / 8, (unsigned)((d + kLinOutCols - 1) / kLinOutCols)), dim3(256), 0, 1, lin_out_kernel<TYPE>, o);
}

template <typename F>
void by_type(int ctas, int type, F f) {
    auto with = [&](auto c) {
        if (type == SARA_BF16) f(c, std::integral_constant<int, SARA_BF16>());
        else f(c, std::integral_constant<int, SARA_FP16>());
    };
    if (ctas == 2) with(std::integral_constant<int, 2>());
    else with(std::integral_constant<int, 1>());
}

}  // namespace

extern "C" {

size_t sara_linear_logprobs_workspace_bytes(int32_t R, int32_t d, int32_t V, int32_t backward) {
    if (!sizes_ok(SARA_BF16, R, d, V, 1.f)) return 0;
    size_t bytes = 0;
    op_guard([&] { bytes = lin_plan(R, d, V, backward != 0).bytes; });
    return bytes;
}

int sara_linear_logprobs(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride, int32_t type, int32_t R,
                         int32_t d, int32_t V, const int32_t *tokens, float scale, float *logprob, float *entropy, float *stats,
                         void *workspace, size_t workspace_bytes, void *stream) {
    if (!sizes_ok(type, R, d, V, scale)) return SARA_EINVAL;
    if (R == 0) return SARA_OK;
    const Operand h{hidden, R, hidden_stride, d}, w{weight, V, weight_stride, d};
    if (!h.ok() || !w.ok() || (logprob && !tokens)) return SARA_EINVAL;
    const LinPlan q = lin_plan(R, d, V, false);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < q.bytes) return SARA_EINVAL;
    return op_guard([&] {
        by_type(q.ctas, type, [&](auto c, auto t) {
            score<c.value, t.value>(static_cast<cudaStream_t>(stream), sm_count(), workspace, q, h, w, tokens, scale, logprob, entropy, stats);
        });
    });
}

int sara_linear_logprobs_backward(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride, int32_t type,
                                  int32_t R, int32_t d, int32_t V, const int32_t *tokens, float scale, const float *stats,
                                  const float *entropy, const float *grad_logprob, const float *grad_entropy, void *grad_hidden,
                                  int64_t grad_hidden_stride, void *grad_weight, int64_t grad_weight_stride, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    if (!sizes_ok(type, R, d, V, scale)) return SARA_EINVAL;
    const Operand h{hidden, R, hidden_stride, d}, w{weight, V, weight_stride, d};
    const Operand dh{grad_hidden, R, grad_hidden_stride, d}, dw{grad_weight, V, grad_weight_stride, d};
    if ((dw.p && !dw.ok()) || (!dh.p && !dw.p)) return SARA_EINVAL;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (R == 0) {  // a sum over no rows
        if (!dw.p) return SARA_OK;
        return op_guard([&] { CK(cudaMemset2DAsync(grad_weight, grad_weight_stride * 2, 0, (size_t)d * 2, V, s)); });
    }
    if (!h.ok() || !w.ok() || (dh.p && !dh.ok()) || !stats || (grad_logprob && !tokens) || (grad_entropy && !entropy)) return SARA_EINVAL;
    if (dh.meets(h) || dh.meets(w) || dw.meets(h) || dw.meets(w) || dh.meets(dw)) return SARA_EINVAL;
    const LinPlan q = lin_plan(R, d, V, true);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < q.bytes) return SARA_EINVAL;
    return op_guard([&] {
        by_type(q.ctas, type, [&](auto c, auto t) {
            gradient<c.value, t.value>(s, sm_count(), workspace, q, h, w, tokens, stats, entropy, grad_logprob, grad_entropy, scale, dh, dw);
        });
    });
}

}  // extern "C"
