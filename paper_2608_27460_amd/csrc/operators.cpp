// C ABI of the operators around the head's logits (include/vie.h): the int8
// head, sampling and distillation.  Arguments are checked here, before
// anything is enqueued.
#include <hip/hip_runtime.h>

#include <initializer_list>

#include "operators.hpp"

using namespace vie;

namespace {

vie_status check_type(int32_t dtype, const char *what)
{
    if (dtype != VIE_F32 && dtype != VIE_BF16) return fail(VIE_EINVAL, "unknown dtype %d of %s", dtype, what);
    return VIE_OK;
}

vie_status check_rows(int32_t B, int64_t V)
{
    if (B < 1 || B > 65535) return fail(VIE_EINVAL, "%d rows out of range [1, 65535]", B);
    if (V < 1 || V >= (int64_t(1) << 31)) return fail(VIE_EINVAL, "V = %lld out of range", (long long)V);
    return VIE_OK;
}

// Rows of V values, ld values apart, aligned to their type.
vie_status check_matrix(const void *p, int32_t dtype, int64_t V, int64_t ld, const char *what)
{
    if (vie_status s = check_type(dtype, what)) return s;
    if (ld < V || ld >= (int64_t(1) << 40))
        return fail(VIE_EINVAL, "row stride %lld of %s outside [V, 2^40)", (long long)ld, what);
    if ((uintptr_t)p % elem_bytes(dtype)) return fail(VIE_EINVAL, "%s is not aligned to its type", what);
    return VIE_OK;
}

// Arrays of 4-byte values.
vie_status check_words(std::initializer_list<const void *> arrays)
{
    for (const void *p : arrays)
        if ((uintptr_t)p % 4) return fail(VIE_EINVAL, "an array of 4-byte values is not aligned to its type");
    return VIE_OK;
}

vie_status check_list(int32_t k)
{
    if (k < 1 || k > kMaxList) return fail(VIE_EINVAL, "k = %d out of range [1, %d]", k, kMaxList);
    return VIE_OK;
}

vie_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return VIE_OK;
    if (!ws) return fail(VIE_EINVAL, "NULL workspace (%zu bytes needed)", need);
    if ((uintptr_t)ws % 256) return fail(VIE_EINVAL, "workspace is not 256-byte aligned");
    if (have < need) return fail(VIE_EINVAL, "workspace holds %zu bytes, needs %zu", have, need);
    return VIE_OK;
}

vie_status check_distill(const void *logits, int32_t dtype, int32_t N, int64_t V, int64_t ld, const int32_t *ids,
                         const float *teacher, int32_t k, float tau)
{
    if (!logits || !ids || !teacher) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_rows(N, V)) return s;
    if (vie_status s = check_matrix(logits, dtype, V, ld, "logits")) return s;
    if (vie_status s = check_list(k)) return s;
    if (!(tau >= 1e-4f && tau <= 1e4f)) return fail(VIE_EINVAL, "tau = %g outside [1e-4, 1e4]", (double)tau);
    return VIE_OK;
}

// Bytes that an argument takes: `bytes` of them, or rows of `width` that begin
// `stride` apart and take `bytes` from the first to the last.
struct Range {
    const void *p;
    size_t bytes, width = 0, stride = 0;
};
Range matrix(const void *p, int32_t rows, int64_t V, int64_t ld, int32_t dtype)
{
    const size_t e = elem_bytes(dtype), span = ((size_t)(rows - 1) * ld + V) * e;
    if (rows == 1) return {p, span};
    return {p, span, (size_t)V * e, (size_t)ld * e};
}
// What lies between the rows of a matrix is not the matrix: another argument
// may be there (two matrices of one stride only, as in the halves of wider
// rows).
bool overlap(const Range &a, const Range &b)
{
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    if (pa >= pb + b.bytes || pb >= pa + a.bytes) return false;
    if (!a.stride) return b.stride ? overlap(b, a) : true;
    if (b.stride && b.stride != a.stride) return true;
    const size_t by = pb >= pa ? (pb - pa) % a.stride : (a.stride - (pa - pb) % a.stride) % a.stride;
    return by < a.width || by + (b.stride ? b.width : b.bytes) > a.stride;
}
// What is written (the first n_out ranges) apart from each other and from the
// inputs; a NULL range is none.
template <int N> vie_status check_ranges(const Range (&r)[N], int n_out)
{
    for (int i = 0; i < n_out; ++i)
        for (int j = i + 1; j < N; ++j)
            if (r[i].p && r[j].p && overlap(r[i], r[j]))
                return fail(VIE_EINVAL, "an output or the workspace overlaps another argument");
    return VIE_OK;
}
vie_status check_sample(const SampleLaunch &a, size_t ws_bytes)
{
    if (vie_status s = check_words({a.token, a.prob, a.kept, a.u, a.ids, a.prm.temperature_dev, a.prm.top_k_dev,
                                    a.prm.top_p_dev, a.prm.min_p_dev}))
        return s;
    const size_t n = (size_t)a.B * 4;
    const Range r[] = {{a.token, n}, {a.prob, n}, {a.kept, n}, {a.ws, ws_bytes}, {a.u, n}, matrix(a.logits, a.B, a.n, a.ld, a.dtype),
                       {a.ids, n * (size_t)a.n}, {a.prm.temperature_dev, n}, {a.prm.top_k_dev, n},
                       {a.prm.top_p_dev, n}, {a.prm.min_p_dev, n}};
    return check_ranges(r, 4);
}

// The gradient's rows are the logits' own or apart from them.
vie_status check_apart(const DistillLaunch &a)
{
    if (a.grad == a.logits) {
        if (a.grad_ld != a.ld && a.N > 1)
            return fail(VIE_EINVAL, "a gradient in place of the logits needs their row stride");
        return VIE_OK;
    }
    if (overlap(matrix(a.logits, a.N, a.V, a.ld, a.dtype), matrix(a.grad, a.N, a.V, a.grad_ld, a.dtype)))
        return fail(VIE_EINVAL, "the gradient overlaps the logits without being in their place");
    return VIE_OK;
}
// Every array aligned, and what is written of a distillation apart from the rest (but for a gradient
// in place of the logits).
vie_status check_distilled(const DistillLaunch &a, bool stats_out)
{
    if (vie_status s = check_words({a.ids, a.teacher, a.loss, a.stats, a.gloss})) return s;
    const size_t n = (size_t)a.N * 4, list = n * (size_t)a.k;
    const Range none{nullptr, 0};
    const Range g = a.grad ? matrix(a.grad, a.N, a.V, a.grad_ld, a.dtype) : none;
    const Range logits = a.grad == a.logits ? none : matrix(a.logits, a.N, a.V, a.ld, a.dtype);
    const Range stats{a.stats, 2 * n};
    const Range r[] = {g, {a.loss, n}, stats_out ? stats : none, {a.ws, distill_workspace_bytes(a.V, a.N)}, logits, stats_out ? none : stats, {a.ids, list},
                       {a.teacher, list}, {a.gloss, n}};
    return check_ranges(r, 4);
}

}  // namespace

extern "C" {

vie_status vie_int8_logits_workspace(int64_t V, int32_t d, int32_t B, size_t *bytes)
{
    set_error("%s", "");
    if (!bytes) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_rows(B, V)) return s;
    if (d < 1 || d > kMaxD) return fail(VIE_EINVAL, "d = %d out of range [1, %d]", d, kMaxD);
    *bytes = int8_workspace_bytes(V, d, B);
    return VIE_OK;
}

vie_status vie_int8_logits(const int8_t *q_dev, const float *scale_dev, int64_t V, int32_t d, const void *h_dev,
                           vie_dtype h_dtype, int32_t B, void *out_dev, vie_dtype out_dtype, int64_t out_ld,
                           void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    set_error("%s", "");
    if (!q_dev || !scale_dev || !h_dev || !out_dev) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_rows(B, V)) return s;
    if (d < 1 || d > kMaxD) return fail(VIE_EINVAL, "d = %d out of range [1, %d]", d, kMaxD);
    if (vie_status s = check_matrix(h_dev, h_dtype, d, d, "h")) return s;
    if (vie_status s = check_matrix(out_dev, out_dtype, V, out_ld, "the logits")) return s;
    if (vie_status s = check_words({scale_dev})) return s;
    const size_t need = int8_workspace_bytes(V, d, B);
    if (vie_status s = check_workspace(workspace_dev, workspace_bytes, need)) return s;
    const Range r[] = {matrix(out_dev, B, V, out_ld, out_dtype), {need ? workspace_dev : nullptr, need},
                       {q_dev, (size_t)V * d}, {scale_dev, (size_t)V * 4}, {h_dev, (size_t)B * d * elem_bytes(h_dtype)}};
    if (vie_status s = check_ranges(r, 2)) return s;
    const Int8Launch a{q_dev, scale_dev, V, d, h_dev, h_dtype, B, out_dev, out_dtype, out_ld, workspace_dev};
    return launch_int8_logits(a, static_cast<hipStream_t>(hip_stream));
}

vie_status vie_sample(const int32_t *ids_dev, const float *logits_dev, int32_t B, int32_t k,
                      const vie_sample_params *params, const float *u_dev, int32_t *token_dev, float *prob_dev,
                      int32_t *kept_dev, void *hip_stream)
{
    set_error("%s", "");
    if (!ids_dev || !logits_dev || !params || !u_dev || !token_dev) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_rows(B, 1)) return s;
    if (vie_status s = check_list(k)) return s;
    if (vie_status s = check_words({logits_dev})) return s;
    const SampleLaunch a{ids_dev, logits_dev, VIE_F32, k, k, B, *params, u_dev, token_dev, prob_dev, kept_dev, nullptr};
    if (vie_status s = check_sample(a, 0)) return s;
    return launch_sample_lists(a, static_cast<hipStream_t>(hip_stream));
}

vie_status vie_sample_rows_workspace(int64_t V, int32_t B, size_t *bytes)
{
    set_error("%s", "");
    if (!bytes) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_rows(B, V)) return s;
    *bytes = sample_rows_workspace_bytes(V, B);
    return VIE_OK;
}

vie_status vie_sample_rows(const void *logits_dev, vie_dtype dtype, int64_t V, int64_t ld, int32_t B,
                           const vie_sample_params *params, const float *u_dev, int32_t *token_dev, float *prob_dev,
                           int32_t *kept_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    set_error("%s", "");
    if (!logits_dev || !params || !u_dev || !token_dev) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_rows(B, V)) return s;
    if (vie_status s = check_matrix(logits_dev, dtype, V, ld, "logits")) return s;
    const size_t need = sample_rows_workspace_bytes(V, B);
    if (vie_status s = check_workspace(workspace_dev, workspace_bytes, need)) return s;
    const SampleLaunch a{nullptr, logits_dev, dtype, V, ld, B, *params, u_dev, token_dev, prob_dev, kept_dev,
                         workspace_dev};
    if (vie_status s = check_sample(a, need)) return s;
    return launch_sample_rows(a, static_cast<hipStream_t>(hip_stream));
}

vie_status vie_distill_workspace(int64_t V, int32_t N, size_t *bytes)
{
    set_error("%s", "");
    if (!bytes) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_rows(N, V)) return s;
    *bytes = distill_workspace_bytes(V, N);
    return VIE_OK;
}

vie_status vie_distill(const void *logits_dev, vie_dtype dtype, int32_t N, int64_t V, int64_t ld,
                       const int32_t *ids_dev, const float *teacher_dev, int32_t k, float tau, float *loss_dev,
                       float *stats_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    set_error("%s", "");
    if (vie_status s = check_distill(logits_dev, dtype, N, V, ld, ids_dev, teacher_dev, k, tau)) return s;
    if (!loss_dev || !stats_dev) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_workspace(workspace_dev, workspace_bytes, distill_workspace_bytes(V, N))) return s;
    const DistillLaunch a{logits_dev, dtype, N, V, ld, ids_dev, teacher_dev, k, tau, loss_dev, stats_dev,
                          nullptr, 1.0f, nullptr, 0, workspace_dev};
    if (vie_status s = check_distilled(a, true)) return s;
    return launch_distill(a, static_cast<hipStream_t>(hip_stream));
}

vie_status vie_distill_grad(const void *logits_dev, vie_dtype dtype, int32_t N, int64_t V, int64_t ld,
                            const int32_t *ids_dev, const float *teacher_dev, int32_t k, float tau,
                            const float *stats_dev, const float *gloss_dev, float weight, void *grad_dev,
                            int64_t grad_ld, void *hip_stream)
{
    set_error("%s", "");
    if (vie_status s = check_distill(logits_dev, dtype, N, V, ld, ids_dev, teacher_dev, k, tau)) return s;
    if (!stats_dev || !grad_dev) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_matrix(grad_dev, dtype, V, grad_ld, "the gradient")) return s;
    const DistillLaunch a{logits_dev, dtype, N, V, ld, ids_dev, teacher_dev, k, tau, nullptr,
                          const_cast<float *>(stats_dev), gloss_dev, weight, grad_dev, grad_ld, nullptr};
    if (vie_status s = check_apart(a)) return s;
    if (vie_status s = check_distilled(a, false)) return s;
    return launch_distill_grad(a, static_cast<hipStream_t>(hip_stream));
}

vie_status vie_distill_step(const void *logits_dev, vie_dtype dtype, int32_t N, int64_t V, int64_t ld,
                            const int32_t *ids_dev, const float *teacher_dev, int32_t k, float tau,
                            const float *gloss_dev, float weight, float *loss_dev, void *grad_dev, int64_t grad_ld,
                            void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    set_error("%s", "");
    if (vie_status s = check_distill(logits_dev, dtype, N, V, ld, ids_dev, teacher_dev, k, tau)) return s;
    if (!loss_dev || !grad_dev) return fail(VIE_EINVAL, "NULL argument");
    if (vie_status s = check_matrix(grad_dev, dtype, V, grad_ld, "the gradient")) return s;
    if (vie_status s = check_workspace(workspace_dev, workspace_bytes, distill_workspace_bytes(V, N))) return s;
    const DistillLaunch a{logits_dev, dtype, N, V, ld, ids_dev, teacher_dev, k, tau, loss_dev, nullptr,
                          gloss_dev, weight, grad_dev, grad_ld, workspace_dev};
    if (vie_status s = check_apart(a)) return s;
    if (vie_status s = check_distilled(a, false)) return s;
    return launch_distill_step(a, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
