// Launchers of the operators of a layer without dropped tokens and of its optimizer.  Shapes were validated by the entry points
// (sorted_api.hip); layouts and formulas as include/smile.h says.
#pragma once

#include "smile_internal.hpp"

namespace smile {

// ---- k experts for a token (topk.hip)
struct TopkIo {
    const float *logits, *bias;
    int32_t *idx;
    float *weight, *p_sum, *partial;
    int T, N, k;
    bool normalize;
};
size_t topk_workspace(int T, int N);
hipError_t launch_topk(const TopkIo &io, hipStream_t s);

struct TopkGradIo {
    const float *logits, *bias;
    const int32_t *idx;
    const float *dweight;
    const int32_t *count;
    float coef;
    float *dlogits;
    int T, N, k;
    bool normalize;
};
hipError_t launch_topk_backward(const TopkGradIo &io, hipStream_t s);

// ---- the pairs sorted by expert, and their rows (sorted_rows.hip)
struct SortIo {
    const int32_t *idx;
    int32_t *count, *start, *pos, *source, *hist;
    int pairs, N;
};
size_t sort_experts_workspace(int pairs, int N);
hipError_t launch_sort_experts(const SortIo &io, hipStream_t s);

struct SortedRowsIo {
    const void *x;             // dispatch: tokens; combine: sorted rows; combine backwards: gradients of the tokens' rows
    const void *rows;          // combine backwards: the sorted rows
    const int32_t *pos;
    const float *weight;
    const void *residual;
    void *y;                   // dispatch, combine backwards: sorted rows; combine: tokens
    float *dweight;
    int T, k, d, R;
};
hipError_t launch_sorted_dispatch(int dtype, const SortedRowsIo &io, hipStream_t s);
hipError_t launch_sorted_combine(int dtype, const SortedRowsIo &io, hipStream_t s);
hipError_t launch_sorted_combine_backward(int dtype, const SortedRowsIo &io, hipStream_t s);

// ---- products of sorted or dense rows (linear.hip)
hipError_t launch_linear(const smile_linear_args &a, const Tuning &tune, hipStream_t s);
size_t linear_backward_workspace(const smile_linear_backward_args &a);
hipError_t launch_linear_backward(const smile_linear_backward_args &a, const Tuning &tune, void *workspace, hipStream_t s);

// ---- AdamW (adamw.hip).  A plan: the step's counter, the tensors, and for each chunk of kAdamwChunk elements its tensor and its number there.
constexpr int kAdamwChunk = 2048;
struct AdamwTensor {
    void *param;
    const void *grad;
    float *master;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    long long n;
    float weight_decay;
    int32_t pad;
};
struct AdamwChunk {
    int32_t tensor, chunk;
};
constexpr size_t kAdamwTensorsAt = 256;   // bytes: the counter in front
hipError_t launch_adamw(const smile_adamw_args &a, void *plan, const float *lr, int32_t *step, const Tuning &tune, hipStream_t s);
hipError_t launch_adamw_unpack(int dtype, long long n, const uint8_t *m, const uint8_t *m_scale, const uint8_t *v, const uint8_t *v_scale, void *m_value,
                               void *v_value, hipStream_t s);

}  // namespace smile
