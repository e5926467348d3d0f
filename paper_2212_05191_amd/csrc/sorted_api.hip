// C-ABI entry points of the operators of a layer without dropped tokens and of its optimizer: argument checks, all of them on the host before anything is
// enqueued, and the plan of an optimizer step.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <memory>
#include <new>

#include "api_checks.hpp"
#include "sorted_internal.hpp"

namespace smile {

namespace {

constexpr int kWidest = 32768, kWidestRow = 16384, kMostExperts = 4096, kMostChoices = 64;
constexpr long long kMostRows = 1ll << 27, kMostPairs = 1ll << 26;
constexpr double kMostElements = 1099511627776.0;   // 2^40
constexpr double kMostGroupRows = 68719476736.0;    // 2^36: first rows that each let a group begin at row 0 still add up to less than 2^31 tiles of 64 rows

bool known(int dtype) { return dtype == SMILE_DTYPE_F32 || dtype == SMILE_DTYPE_BF16 || dtype == SMILE_DTYPE_F16; }
bool known_act(int act) { return act == SMILE_ACT_NONE || act == SMILE_ACT_RELU || act == SMILE_ACT_GELU; }
bool bad_workspace(const void *p, size_t bytes, size_t needed)
{
    return needed != 0 && ((reinterpret_cast<uintptr_t>(p) & 255u) != 0 || bytes < needed);
}

// memory of a call: NULL overlaps nothing, nor do no bytes
struct Span {
    const void *at;
    size_t bytes;
};
bool overlap(Span a, Span b)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.at), q = reinterpret_cast<uintptr_t>(b.at);
    return p && q && a.bytes && b.bytes && p < q + b.bytes && q < p + a.bytes;
}
// one of what is written overlaps another, or what is read (`in_place`: the first one written may be the first one read)
bool overlapping(std::initializer_list<Span> written, std::initializer_list<Span> read, bool in_place = false)
{
    for (auto w = written.begin(); w != written.end(); ++w) {
        for (auto o = w + 1; o != written.end(); ++o)
            if (overlap(*w, *o)) return true;
        for (const Span &r : read)
            if (overlap(*w, r) && !(in_place && w == written.begin() && &r == read.begin() && w->at == r.at)) return true;
    }
    return false;
}
Span words(const void *at, double n) { return {at, (size_t)n * 4}; }

smile_status check_choices(int T, int N, int k)
{
    if (T < 1 || N < 1 || N > kMostExperts || k < 1 || k > N || k > kMostChoices) return SMILE_BAD_SHAPE;
    if ((long long)T * k >= kMostPairs || (double)T * N >= kMostElements) return SMILE_BAD_SHAPE;
    return SMILE_OK;
}

smile_status check_rows(int T, int k, int d, int R, int dtype)
{
    if (!known(dtype)) return SMILE_UNSUPPORTED;
    if (T < 1 || k < 1 || k > kMostChoices || (long long)T * k >= kMostPairs || R < 1 || R > kMostRows) return SMILE_BAD_SHAPE;
    if (d < 8 || d % 8 || d > kWidestRow || (double)R * d >= kMostElements) return SMILE_BAD_SHAPE;
    return SMILE_OK;
}

smile_status check_linear(int N, int rows, int K, int F, int dtype, int act, const int32_t *start)
{
    if (!known(dtype) || !known_act(act)) return SMILE_UNSUPPORTED;
    if (N < 1 || N > kMostExperts || rows < 1 || rows > kMostRows) return SMILE_BAD_SHAPE;
    if (K < 8 || K % 8 || K > kWidest || F < 8 || F % 8 || F > kWidest) return SMILE_BAD_SHAPE;
    if ((double)rows * std::max(K, F) >= kMostElements || (double)N * K * F >= kMostElements) return SMILE_BAD_SHAPE;
    if ((double)rows * N >= kMostGroupRows) return SMILE_BAD_SHAPE;
    return N > 1 && !start ? SMILE_INVALID_ARG : SMILE_OK;
}

smile_status check_linear_backward(const smile_linear_backward_args *p)
{
    if (!p) return SMILE_INVALID_ARG;
    const smile_linear_backward_args &a = *p;
    if (bad(a.dy) || bad_opt(a.x) || bad_opt(a.w) || bad_opt(a.pre) || bad_opt(a.start) || bad_opt(a.dx) || bad_opt(a.dw) || bad_opt(a.dbias))
        return SMILE_INVALID_ARG;
    if ((!a.dx && !a.dw && !a.dbias) || (a.dx && !a.w) || (a.dw && !a.x)) return SMILE_INVALID_ARG;
    if (a.act != SMILE_ACT_NONE && known_act(a.act) && !a.pre) return SMILE_INVALID_ARG;
    return check_linear(a.N, a.rows, a.K, a.F, a.dtype, a.act, a.start);
}

smile_status check_adamw(const smile_adamw_args &a)
{
    if (a.tensors < 1 || a.tensors > 1 << 24) return SMILE_BAD_SHAPE;
    if (!known(a.dtype) || (a.grad_dtype != a.dtype && a.grad_dtype != SMILE_DTYPE_F32)) return SMILE_UNSUPPORTED;
    if ((a.state_bits != 32 && a.state_bits != 8) || (a.has_master && a.dtype == SMILE_DTYPE_F32)) return SMILE_UNSUPPORTED;
    if (!(a.beta1 >= 0.0 && a.beta1 < 1.0 && a.beta2 >= 0.0 && a.beta2 < 1.0)) return SMILE_BAD_SHAPE;
    // (below fp32's normal range a reciprocal is infinite, and an element without gradient and moments would be 0 times that)
    if (!(a.eps <= 1.0 && (float)a.eps >= FLT_MIN)) return SMILE_BAD_SHAPE;
    return SMILE_OK;
}

smile_status check_adamw_tensors(const smile_adamw_args &a, const smile_adamw_tensor *tensors, long long &chunks)
{
    chunks = 0;
    for (int i = 0; i < a.tensors; ++i) {
        const smile_adamw_tensor &x = tensors[i];
        if (bad(x.param) || bad(x.grad) || bad(x.m) || bad(x.v) || bad_opt(x.master) || (x.master != nullptr) != (a.has_master != 0)) return SMILE_INVALID_ARG;
        if ((x.m_scale != nullptr) != (a.state_bits == 8) || (x.v_scale != nullptr) != (a.state_bits == 8)) return SMILE_INVALID_ARG;
        if (x.n < 1 || x.n > 1ll << 32 || !std::isfinite(x.weight_decay)) return SMILE_BAD_SHAPE;
        chunks += (x.n + kAdamwChunk - 1) / kAdamwChunk;
    }
    return SMILE_OK;
}

// What a step writes, tensor by tensor: nothing of it may be there twice, and no gradient among it, or its chunks would race
smile_status check_adamw_apart(const smile_adamw_args &a, const smile_adamw_tensor *tensors)
{
    const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[(size_t)a.tensors * 6]);
    if (!spans) return SMILE_HIP_ERROR;
    Span *end = spans.get();
    for (int i = 0; i < a.tensors; ++i) {
        const smile_adamw_tensor &x = tensors[i];
        const size_t n = (size_t)x.n, blocks = (n + 127) / 128, state = a.state_bits == 8 ? blocks * 128 : n * 4;
        for (const Span &w : {Span{x.param, n * elem_size(a.dtype)}, Span{x.master, n * 4}, Span{x.m, state}, Span{x.v, state}, Span{x.m_scale, blocks}, Span{x.v_scale, blocks}})
            if (w.at) *end++ = w;
    }
    std::sort(spans.get(), end, [](const Span &p, const Span &q) { return p.at < q.at; });
    for (const Span *w = spans.get(); w + 1 < end; ++w)
        if (overlap(w[0], w[1])) return SMILE_INVALID_ARG;
    for (int i = 0; i < a.tensors; ++i) {
        // of what lies in order and apart, the last that begins in front of the gradient's end
        const Span grad{tensors[i].grad, (size_t)tensors[i].n * elem_size(a.grad_dtype)};
        const void *behind = static_cast<const char *>(grad.at) + grad.bytes;
        const Span *w = std::lower_bound(spans.get(), end, behind, [](const Span &p, const void *at) { return p.at < at; });
        if (w != spans.get() && overlap(w[-1], grad)) return SMILE_INVALID_ARG;
    }
    return SMILE_OK;
}

size_t adamw_plan_bytes(int tensors, long long chunks) { return kAdamwTensorsAt + (size_t)tensors * sizeof(AdamwTensor) + (size_t)chunks * sizeof(AdamwChunk); }

}  // namespace

}  // namespace smile

using namespace smile;

extern "C" {

smile_status smile_topk_workspace_bytes(int32_t T, int32_t N, size_t *bytes)
{
    if (!bytes) return SMILE_INVALID_ARG;
    const smile_status st = check_choices(T, N, 1);
    if (st != SMILE_OK) return st;
    *bytes = topk_workspace(T, N);
    return SMILE_OK;
}

smile_status smile_topk(int32_t T, int32_t N, int32_t k, int32_t normalize, const float *logits, const float *bias, int32_t *idx, float *weight,
                        float *p_sum, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad(logits) || bad_opt(bias) || bad(idx) || bad(weight) || bad_opt(p_sum)) return SMILE_INVALID_ARG;
    const smile_status st = check_choices(T, N, k);
    if (st != SMILE_OK) return st;
    const size_t needed = p_sum ? topk_workspace(T, N) : 0;
    if (needed && !workspace) return SMILE_INVALID_ARG;
    if (bad_workspace(workspace, workspace_bytes, needed)) return SMILE_WORKSPACE;
    const double pairs = (double)T * k;
    if (overlapping({words(idx, pairs), words(weight, pairs), words(p_sum, N), {workspace, needed}}, {words(logits, (double)T * N), words(bias, N)})) return SMILE_INVALID_ARG;
    return from_hip(launch_topk(TopkIo{logits, bias, idx, weight, p_sum, static_cast<float *>(workspace), T, N, k, normalize != 0},
                                static_cast<hipStream_t>(stream)));
}

smile_status smile_topk_backward(int32_t T, int32_t N, int32_t k, int32_t normalize, const float *logits, const float *bias, const int32_t *idx,
                                 const float *dweight, const int32_t *count, float coef, float *dlogits, void *stream)
{
    if (bad(logits) || bad_opt(bias) || bad(idx) || bad(dweight) || bad_opt(count) || bad(dlogits)) return SMILE_INVALID_ARG;
    const smile_status st = check_choices(T, N, k);
    if (st != SMILE_OK) return st;
    const double all = (double)T * N, pairs = (double)T * k;
    if (overlapping({words(dlogits, all)}, {words(logits, all), words(bias, N), words(idx, pairs), words(dweight, pairs), words(count, N)}, true)) return SMILE_INVALID_ARG;
    return from_hip(launch_topk_backward(TopkGradIo{logits, bias, idx, dweight, count, coef, dlogits, T, N, k, normalize != 0},
                                         static_cast<hipStream_t>(stream)));
}

smile_status smile_sort_experts_workspace_bytes(int32_t T, int32_t k, int32_t N, size_t *bytes)
{
    if (!bytes) return SMILE_INVALID_ARG;
    if (T < 1 || k < 1 || k > kMostChoices || (long long)T * k >= kMostPairs || N < 1 || N > kMostExperts) return SMILE_BAD_SHAPE;
    *bytes = sort_experts_workspace(T * k, N);
    return SMILE_OK;
}

smile_status smile_sort_experts(int32_t T, int32_t k, int32_t N, const int32_t *idx, int32_t *count, int32_t *start, int32_t *pos, int32_t *source,
                                void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad(idx) || bad(count) || bad(start) || bad(pos) || bad(source)) return SMILE_INVALID_ARG;
    size_t needed = 0;
    const smile_status st = smile_sort_experts_workspace_bytes(T, k, N, &needed);
    if (st != SMILE_OK) return st;
    if (needed && !workspace) return SMILE_INVALID_ARG;
    if (bad_workspace(workspace, workspace_bytes, needed)) return SMILE_WORKSPACE;
    const double pairs = (double)T * k;
    if (overlapping({words(count, N), words(start, N + 1.0), words(pos, pairs), words(source, pairs), {workspace, needed}}, {words(idx, pairs)})) return SMILE_INVALID_ARG;
    return from_hip(launch_sort_experts(SortIo{idx, count, start, pos, source, static_cast<int32_t *>(workspace), T * k, N}, static_cast<hipStream_t>(stream)));
}

smile_status smile_sorted_dispatch(int32_t T, int32_t k, int32_t d, int32_t R, int32_t dtype, const void *x, const int32_t *pos, void *xs, void *stream)
{
    if (bad(x) || bad(pos) || bad(xs)) return SMILE_INVALID_ARG;
    const smile_status st = check_rows(T, k, d, R, dtype);
    if (st != SMILE_OK) return st;
    const size_t row = (size_t)d * elem_size(dtype), pairs = (size_t)T * k;
    if (overlapping({{xs, R * row}}, {{x, T * row}, words(pos, pairs)})) return SMILE_INVALID_ARG;
    return from_hip(launch_sorted_dispatch(dtype, SortedRowsIo{x, nullptr, pos, nullptr, nullptr, xs, nullptr, T, k, d, R}, static_cast<hipStream_t>(stream)));
}

smile_status smile_sorted_combine(int32_t T, int32_t k, int32_t d, int32_t R, int32_t dtype, const void *ys, const int32_t *pos, const float *weight,
                                  const void *residual, void *y, void *stream)
{
    if (bad(ys) || bad(pos) || bad_opt(weight) || bad_opt(residual) || bad(y)) return SMILE_INVALID_ARG;
    const smile_status st = check_rows(T, k, d, R, dtype);
    if (st != SMILE_OK) return st;
    const size_t row = (size_t)d * elem_size(dtype), pairs = (size_t)T * k;
    if (overlapping({{y, T * row}}, {{residual, T * row}, {ys, R * row}, words(pos, pairs), words(weight, pairs)}, true)) return SMILE_INVALID_ARG;
    return from_hip(launch_sorted_combine(dtype, SortedRowsIo{ys, nullptr, pos, weight, residual, y, nullptr, T, k, d, R}, static_cast<hipStream_t>(stream)));
}

smile_status smile_sorted_combine_backward(int32_t T, int32_t k, int32_t d, int32_t R, int32_t dtype, const void *dy, const void *ys, const int32_t *pos,
                                           const float *weight, void *dys, float *dweight, void *stream)
{
    if (bad(dy) || bad_opt(ys) || bad(pos) || bad(weight) || bad(dys) || bad_opt(dweight) || (ys == nullptr) != (dweight == nullptr)) return SMILE_INVALID_ARG;
    const smile_status st = check_rows(T, k, d, R, dtype);
    if (st != SMILE_OK) return st;
    const size_t row = (size_t)d * elem_size(dtype), pairs = (size_t)T * k;
    if (overlapping({{dys, R * row}, words(dweight, pairs)}, {{dy, T * row}, {ys, R * row}, words(pos, pairs), words(weight, pairs)})) return SMILE_INVALID_ARG;
    return from_hip(launch_sorted_combine_backward(dtype, SortedRowsIo{dy, ys, pos, weight, nullptr, dys, dweight, T, k, d, R}, static_cast<hipStream_t>(stream)));
}

smile_status smile_linear(const smile_linear_args *p, void *stream)
{
    if (!p) return SMILE_INVALID_ARG;
    const smile_linear_args &a = *p;
    if (bad(a.x) || bad(a.w) || bad_opt(a.bias) || bad_opt(a.residual) || bad_opt(a.start) || bad(a.y) || bad_opt(a.pre)) return SMILE_INVALID_ARG;
    const smile_status st = check_linear(a.N, a.rows, a.K, a.F, a.dtype, a.act, a.start);
    if (st != SMILE_OK) return st;
    const size_t es = elem_size(a.dtype), out = (size_t)a.rows * a.F * es, bias = (size_t)a.N * a.F * es;
    if (overlapping({{a.y, out}, {a.pre, out}}, {{a.residual, out}, {a.x, (size_t)a.rows * a.K * es}, {a.w, bias * a.K}, {a.bias, bias}, words(a.start, a.N + 1.0)}, true))
        return SMILE_INVALID_ARG;
    return from_hip(launch_linear(a, device_tuning(), static_cast<hipStream_t>(stream)));
}

smile_status smile_linear_backward_workspace_bytes(const smile_linear_backward_args *args, size_t *bytes)
{
    if (!bytes) return SMILE_INVALID_ARG;
    const smile_status st = check_linear_backward(args);
    if (st != SMILE_OK) return st;
    *bytes = linear_backward_workspace(*args);
    return SMILE_OK;
}

smile_status smile_linear_backward(const smile_linear_backward_args *args, void *workspace, size_t workspace_bytes, void *stream)
{
    const smile_status st = check_linear_backward(args);
    if (st != SMILE_OK) return st;
    const size_t needed = linear_backward_workspace(*args);
    if (needed && !workspace) return SMILE_INVALID_ARG;
    if (bad_workspace(workspace, workspace_bytes, needed)) return SMILE_WORKSPACE;
    const smile_linear_backward_args &a = *args;
    const size_t es = elem_size(a.dtype), in = (size_t)a.rows * a.K * es, out = (size_t)a.rows * a.F * es, bias = (size_t)a.N * a.F * es;
    if (overlapping({{a.dx, in}, {a.dw, bias * a.K}, {a.dbias, bias}, {workspace, needed}},
                    {{a.dy, out}, {a.dw ? a.x : nullptr, in}, {a.dx ? a.w : nullptr, bias * a.K}, {a.act != SMILE_ACT_NONE ? a.pre : nullptr, out}, words(a.start, a.N + 1.0)}))
        return SMILE_INVALID_ARG;
    return from_hip(launch_linear_backward(*args, device_tuning(), workspace, static_cast<hipStream_t>(stream)));
}

smile_status smile_adamw_plan_bytes(const smile_adamw_args *args, const smile_adamw_tensor *tensors, size_t *bytes)
{
    if (!args || !tensors || !bytes) return SMILE_INVALID_ARG;
    long long chunks = 0;
    smile_status st = check_adamw(*args);
    if (st == SMILE_OK) st = check_adamw_tensors(*args, tensors, chunks);
    if (st == SMILE_OK) *bytes = adamw_plan_bytes(args->tensors, chunks);
    return st;
}

smile_status smile_adamw_plan(smile_adamw_args *args, const smile_adamw_tensor *tensors, void *plan, size_t plan_bytes)
{
    if (!args || !tensors || bad(plan)) return SMILE_INVALID_ARG;
    long long chunks = 0;
    smile_status st = check_adamw(*args);
    if (st == SMILE_OK) st = check_adamw_tensors(*args, tensors, chunks);
    if (st == SMILE_OK) st = check_adamw_apart(*args, tensors);
    if (st != SMILE_OK) return st;
    if (plan_bytes < adamw_plan_bytes(args->tensors, chunks)) return SMILE_WORKSPACE;
    char *base = static_cast<char *>(plan);
    memset(base, 0, kAdamwTensorsAt);
    AdamwTensor *to = reinterpret_cast<AdamwTensor *>(base + kAdamwTensorsAt);
    AdamwChunk *list = reinterpret_cast<AdamwChunk *>(to + args->tensors);
    for (int i = 0; i < args->tensors; ++i) {
        const smile_adamw_tensor &x = tensors[i];
        to[i] = AdamwTensor{x.param, x.grad, x.master, x.m, x.v, static_cast<uint8_t *>(x.m_scale), static_cast<uint8_t *>(x.v_scale), x.n, x.weight_decay, 0};
        for (long long c = 0; c < (x.n + kAdamwChunk - 1) / kAdamwChunk; ++c) *list++ = AdamwChunk{i, (int32_t)c};
    }
    args->chunks = chunks;
    return SMILE_OK;
}

smile_status smile_adamw(const smile_adamw_args *args, void *device_plan, size_t plan_bytes, const float *lr, int32_t *step, void *stream)
{
    if (!args || !device_plan || !lr || !step) return SMILE_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(lr) & 3u) || (reinterpret_cast<uintptr_t>(step) & 3u)) return SMILE_INVALID_ARG;
    const smile_status st = check_adamw(*args);
    if (st != SMILE_OK) return st;
    if (args->chunks < args->tensors || args->chunks > 1ll << 40) return SMILE_BAD_SHAPE;
    const size_t needed = adamw_plan_bytes(args->tensors, args->chunks);
    if (bad_workspace(device_plan, plan_bytes, needed)) return SMILE_WORKSPACE;
    if (overlapping({words(step, 1), {device_plan, needed}}, {words(lr, 1)})) return SMILE_INVALID_ARG;
    return from_hip(launch_adamw(*args, device_plan, lr, step, device_tuning(), static_cast<hipStream_t>(stream)));
}

smile_status smile_adamw_unpack_states(int64_t n, int32_t dtype, const void *m, const void *m_scale, const void *v, const void *v_scale, void *m_value,
                                       void *v_value, void *stream)
{
    if (bad(m) || !m_scale || bad(v) || !v_scale || bad(m_value) || bad(v_value)) return SMILE_INVALID_ARG;
    if (dtype != SMILE_DTYPE_F32 && dtype != SMILE_DTYPE_BF16) return SMILE_UNSUPPORTED;
    if (n < 128 || n % 128 || (double)n >= kMostElements) return SMILE_BAD_SHAPE;
    const size_t codes = (size_t)n, values = codes * elem_size(dtype);
    if (overlapping({{m_value, values}, {v_value, values}}, {{m, codes}, {m_scale, codes / 128}, {v, codes}, {v_scale, codes / 128}})) return SMILE_INVALID_ARG;
    return from_hip(launch_adamw_unpack(dtype, n, static_cast<const uint8_t *>(m), static_cast<const uint8_t *>(m_scale), static_cast<const uint8_t *>(v),
                                        static_cast<const uint8_t *>(v_scale), m_value, v_value, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
