// Entry points of the scoring of sampled tokens: sara_logprobs, sara_logprobs_backward.
#include <cuda.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "../../include/sara.h"
#include "host_util.h"
#include "logprob.cuh"

using namespace sara;

namespace {

bool logits_ok(const void *p, int64_t stride, int type, int R, int V) {
    const uintptr_t size = type == SARA_FP32 ? 4 : 2;
    return p && (reinterpret_cast<uintptr_t>(p) & (size - 1)) == 0 && (R <= 1 || stride >= V);
}

}  // namespace

extern "C" {

int sara_logprobs(const void *logits, int64_t row_stride, int32_t type, int32_t R, int32_t V, const int32_t *tokens, int32_t top,
                  float *logprob, float *entropy, float *stats, int32_t *top_token, float *top_logprob, void *stream) {
    if (type < SARA_BF16 || type > SARA_FP32 || R < 0 || V < 1 || top < 0 || top > kScoreMaxTop) return SARA_EINVAL;
    if (R == 0) return SARA_OK;
    if ((logprob && !tokens) || (top > 0 && (!top_token || !top_logprob))) return SARA_EINVAL;
    if (!logits_ok(logits, row_stride, type, R, V)) return SARA_EINVAL;
    return op_guard([&] {
        const ScoreParams p{logits, row_stride, R, V, top, tokens, logprob, entropy, stats, top_token, top_logprob, 1, 0};
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        const int sms = sm_count();
        auto launch = [&](auto t) {
            if (top > 0) launch_score<t.value, true>(s, sms, p);
            else launch_score<t.value, false>(s, sms, p);
        };
        if (type == SARA_FP32) launch(std::integral_constant<int, SARA_FP32>());
        else if (type == SARA_BF16) launch(std::integral_constant<int, SARA_BF16>());
        else launch(std::integral_constant<int, SARA_FP16>());
    });
}

int sara_logprobs_backward(const void *logits, int64_t row_stride, int32_t type, int32_t R, int32_t V, const int32_t *tokens,
                           const float *stats, const float *entropy, const float *grad_logprob, const float *grad_entropy,
                           void *grad_logits, int64_t grad_stride, void *stream) {
    if (type < SARA_BF16 || type > SARA_FP32 || R < 0 || V < 1) return SARA_EINVAL;
    if (R == 0) return SARA_OK;
    if ((grad_logprob && !tokens) || (grad_entropy && !entropy)) return SARA_EINVAL;
    if (!logits_ok(logits, row_stride, type, R, V) || !logits_ok(grad_logits, grad_stride, type, R, V) || !stats) return SARA_EINVAL;
    if (logits == grad_logits && R > 1 && row_stride != grad_stride) return SARA_EINVAL;
    return op_guard([&] {
        const ScoreGradParams p{logits, row_stride, R, V, tokens, stats, entropy, grad_logprob, grad_entropy, grad_logits, grad_stride,
                                0, 0};
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        if (type == SARA_FP32) launch_score_grad<SARA_FP32>(s, p);
        else if (type == SARA_BF16) launch_score_grad<SARA_BF16>(s, p);
        else launch_score_grad<SARA_FP16>(s, p);
    });
}

}  // extern "C"
