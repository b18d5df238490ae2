// Distillation from a teacher's top logits (gfx950).
//
// For a token with the student's logits s over V ids and the teacher's list
// (id_j, t_j), at temperature tau:
//
//   p = softmax(t / tau) over the list,  q = softmax(s / tau) over the V ids
//   loss = tau^2 sum_j p_j (log p_j - log q[id_j])
//   d loss / d s_v = tau (q_v - p_v),   p_v = sum of the p_j with id_j = v
//
// q needs the row's maximum m and the sum Z of exp((s - m) / tau), which one
// pass over the row gives: a thread keeps the maximum of what it has seen
// and the sum relative to it, and rescales the sum when the maximum grows.
// The pair (m, Z) is what the backward pass needs of the forward pass; it
// is kept as two fp32 numbers rather than as log Z + m / tau, whose rounding
// would be relative to m.  Sums are fp32 per thread (at most a few hundred
// terms) and merged pairwise; the list's sums are fp64.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "block.hpp"
#include "operators.hpp"

namespace vie {

namespace {

constexpr int kRowThreads = 512;
constexpr int kRowWaves = kRowThreads / kLanes;
constexpr int kListPer = kMaxList / kRowThreads;  // list entries of a thread
static_assert(kListPer * kRowThreads == kMaxList, "every list entry has a thread");

// Maximum and sum of exp2((s - m) c) of a set of logits.  The empty set has
// the lowest finite maximum, so that rows of -inf or of the lowest value make
// no NaN on the way: s - m is then 0 or -inf.
struct Part {
    float m, z;
};
__device__ __forceinline__ Part merge(Part a, Part b, float c)
{
    const float m = fmaxf(a.m, b.m);
    return {m, a.z * exp2f((a.m - m) * c) + b.z * exp2f((b.m - m) * c)};
}
template <int N> __device__ __forceinline__ void add(Part &p, const float *f, float c)
{
    float m = f[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, f[i]);
    m = fmaxf(m, p.m);
    float z = p.z * exp2f((p.m - m) * c);
#pragma unroll
    for (int i = 0; i < N; ++i) z += exp2f((f[i] - m) * c);
    p = {m, z};
}

// The part of n logits from s on, in every thread.
template <bool BF16> __device__ Part row_part(const typename Elem<BF16>::T *s, int64_t n, float c, Part *tmp)
{
    typedef Elem<BF16> E;
    const Span<typename E::T> sp(s, n);
    Part p{-FLT_MAX, 0.0f};
    const word4 *v = reinterpret_cast<const word4 *>(s + sp.head);
    for (int64_t i = threadIdx.x; i < sp.vecs; i += kRowThreads) {
        float f[E::kVec];
        E::unpack(v[i], f);
        add<E::kVec>(p, f, c);
    }
    for (int64_t i = threadIdx.x; i < sp.head + n - sp.tail0; i += kRowThreads) {
        const float f = E::get(s[i < sp.head ? i : sp.tail0 + i - sp.head]);
        add<1>(p, &f, c);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) p = merge(p, Part{__shfl_xor(p.m, o, kLanes), __shfl_xor(p.z, o, kLanes)}, c);
    __syncthreads();
    if ((threadIdx.x & (kLanes - 1)) == 0) tmp[threadIdx.x / kLanes] = p;
    __syncthreads();
    p = tmp[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) p = merge(p, tmp[w], c);
    return p;
}

// The teacher's list of a row: this thread's entries, and the list's maximum
// and sum.  An entry counts if its id lies in [0, V) and its logit is not
// -inf; the others have id -1.
struct List {
    int32_t id[kListPer];
    float t[kListPer];
    float top;
    double total;  // 0: nothing listed
    double inv_tau;
    __device__ __forceinline__ double x(int i) const { return ((double)t[i] - (double)top) * inv_tau; }
    __device__ __forceinline__ double p(int i) const { return exp(x(i)) / total; }
};

__device__ __forceinline__ void read_list(List &l, const int32_t *ids, const float *t, int k, int64_t V, float tau,
                                          double *tmp)
{
    l.inv_tau = 1.0 / (double)tau;
    float top = -FLT_MAX;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kListPer; ++i) {
        const int j = i * kRowThreads + threadIdx.x;
        l.id[i] = -1;
        l.t[i] = 0.0f;
        if (j >= k) continue;
        const int32_t id = ids[j];
        const float v = t[j];
        if (id < 0 || id >= V || v == -__builtin_inff()) continue;
        l.id[i] = id;
        l.t[i] = v;
        nan |= v != v;
        top = fmaxf(top, v);
    }
    top = nan ? __builtin_nanf("") : top;
    l.top = block_reduce<kRowThreads>(top, reinterpret_cast<float *>(tmp),
                                      [](float a, float b) { return a != a || b != b ? a + b : fmaxf(a, b); });
    double total = 0.0;
#pragma unroll
    for (int i = 0; i < kListPer; ++i)
        if (l.id[i] >= 0) total += exp(l.x(i));
    __syncthreads();
    l.total = block_reduce<kRowThreads>(total, tmp, [](double a, double b) { return a + b; });
}

// The loss of a row from its part and its list (in every thread).
template <bool BF16>
__device__ __forceinline__ float row_loss(const List &l, const typename Elem<BF16>::T *s, Part r, float tau, double *tmp)
{
    double sum = 0.0;
    const double log_total = log(l.total), log_z = log((double)r.z);
#pragma unroll
    for (int i = 0; i < kListPer; ++i) {
        if (l.id[i] < 0) continue;
        const double p = l.p(i);
        if (p == 0.0) continue;
        const double logq = ((double)Elem<BF16>::get(s[l.id[i]]) - (double)r.m) * l.inv_tau - log_z;
        sum += p * (l.x(i) - log_total - logq);
    }
    __syncthreads();
    sum = block_reduce<kRowThreads>(sum, tmp, [](double a, double b) { return a + b; });
    return l.total == 0.0 ? 0.0f : (float)((double)tau * (double)tau * sum);
}

// The gradient of n logits from v0 on: f = g tau, the row's part r.  `grad`
// may be `s`: what the listed ids need of s is read before anything is
// written.
template <bool BF16>
__device__ void row_grad(const List &l, const typename Elem<BF16>::T *s, typename Elem<BF16>::T *grad, int64_t v0,
                         int64_t n, Part r, float c, float f, int32_t *s_id, float *s_p)
{
    typedef Elem<BF16> E;
    const int tid = threadIdx.x;
    const float inv = 1.0f / r.z;
    const bool none = l.total == 0.0;
    if (none) f = 0.0f;
    // listed ids: q - p, p summed over the entries of an id; its first entry writes it
#pragma unroll
    for (int i = 0; i < kListPer; ++i) {
        const int j = i * kRowThreads + tid;
        s_id[j] = l.id[i];
        s_p[j] = l.id[i] >= 0 ? (float)l.p(i) : 0.0f;
    }
    __syncthreads();
    float val[kListPer];
    bool mine[kListPer];
#pragma unroll
    for (int i = 0; i < kListPer; ++i) {
        const int j = i * kRowThreads + tid;
        const int32_t id = l.id[i];
        mine[i] = id >= v0 && id < v0 + n;
        val[i] = 0.0f;
        if (!mine[i]) continue;
        double p = 0.0;  // (2048 fp32 additions would lose four digits)
        for (int e = 0; e < kMaxList; ++e) {
            if (s_id[e] != id) continue;
            if (e < j) mine[i] = false;
            p += (double)s_p[e];
        }
        val[i] = f * (exp2f((E::get(s[id]) - r.m) * c) * inv - (float)p);
    }
    __syncthreads();
    auto one = [&](float x) { return none ? 0.0f : f * (exp2f((x - r.m) * c) * inv); };
    const typename E::T *src = s + v0;
    typename E::T *dst = grad + v0;
    const Span<typename E::T> sp(src, n);
    const word4 *v = reinterpret_cast<const word4 *>(src + sp.head);
    const bool alike = (((uintptr_t)src ^ (uintptr_t)dst) & 15) == 0;
    for (int64_t i = tid; i < sp.vecs; i += kRowThreads) {
        float x[E::kVec];
        E::unpack(v[i], x);
#pragma unroll
        for (int e = 0; e < E::kVec; ++e) x[e] = one(x[e]);
        if (alike) {
            reinterpret_cast<word4 *>(dst + sp.head)[i] = E::pack(x);
        } else {
#pragma unroll
            for (int e = 0; e < E::kVec; ++e) dst[sp.head + i * E::kVec + e] = E::put(x[e]);
        }
    }
    for (int64_t i = tid; i < sp.head + n - sp.tail0; i += kRowThreads) {
        const int64_t at = i < sp.head ? i : sp.tail0 + i - sp.head;
        dst[at] = E::put(one(E::get(src[at])));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kListPer; ++i)
        if (mine[i]) grad[l.id[i]] = E::put(val[i]);
}

// One workgroup per row: the loss and the row's part, and where GRAD the
// gradient too, whose pass over the row follows at once.
template <bool BF16, bool GRAD> __global__ __launch_bounds__(kRowThreads) void distill_row_kernel(DistillLaunch a)
{
    typedef typename Elem<BF16>::T T;
    __shared__ double s_tmp[kRowWaves];
    __shared__ Part s_part[kRowWaves];
    __shared__ int32_t s_id[GRAD ? kMaxList : 1];
    __shared__ float s_p[GRAD ? kMaxList : 1];
    const int64_t row = blockIdx.x;
    const T *s = static_cast<const T *>(a.logits) + row * a.ld;
    const float c = (float)(1.4426950408889634 / (double)a.tau);
    List l;
    read_list(l, a.ids + row * a.k, a.teacher + row * a.k, a.k, a.V, a.tau, s_tmp);
    const Part r = row_part<BF16>(s, a.V, c, s_part);
    const float loss = row_loss<BF16>(l, s, r, a.tau, s_tmp);
    if (threadIdx.x == 0) {
        a.loss[row] = loss;
        if (a.stats) a.stats[2 * row] = r.m, a.stats[2 * row + 1] = r.z;
    }
    if constexpr (GRAD) {
        const float g = a.weight * (a.gloss ? a.gloss[row] : 1.0f);
        row_grad<BF16>(l, s, static_cast<T *>(a.grad) + row * a.grad_ld, 0, a.V, r, c, g * a.tau, s_id, s_p);
    }
}

// The gradient from the part that the forward pass kept.
template <bool BF16> __global__ __launch_bounds__(kRowThreads) void distill_grad_kernel(DistillLaunch a)
{
    typedef typename Elem<BF16>::T T;
    __shared__ double s_tmp[kRowWaves];
    __shared__ int32_t s_id[kMaxList];
    __shared__ float s_p[kMaxList];
    const int64_t row = blockIdx.x;
    const float c = (float)(1.4426950408889634 / (double)a.tau);
    List l;
    read_list(l, a.ids + row * a.k, a.teacher + row * a.k, a.k, a.V, a.tau, s_tmp);
    const Part r{a.stats[2 * row], a.stats[2 * row + 1]};
    const float g = a.weight * (a.gloss ? a.gloss[row] : 1.0f);
    row_grad<BF16>(l, static_cast<const T *>(a.logits) + row * a.ld, static_cast<T *>(a.grad) + row * a.grad_ld, 0, a.V,
                   r, c, g * a.tau, s_id, s_p);
}

vie_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

size_t distill_workspace_bytes(int64_t, int) { return 0; }

vie_status launch_distill(const DistillLaunch &a, hipStream_t s)
{
    if (a.dtype == VIE_BF16) distill_row_kernel<true, false><<<a.N, kRowThreads, 0, s>>>(a);
    else distill_row_kernel<false, false><<<a.N, kRowThreads, 0, s>>>(a);
    return launched("distillation launch");
}

vie_status launch_distill_grad(const DistillLaunch &a, hipStream_t s)
{
    if (a.dtype == VIE_BF16) distill_grad_kernel<true><<<a.N, kRowThreads, 0, s>>>(a);
    else distill_grad_kernel<false><<<a.N, kRowThreads, 0, s>>>(a);
    return launched("distillation gradient launch");
}

vie_status launch_distill_step(const DistillLaunch &a, hipStream_t s)
{
    if (a.dtype == VIE_BF16) distill_row_kernel<true, true><<<a.N, kRowThreads, 0, s>>>(a);
    else distill_row_kernel<false, true><<<a.N, kRowThreads, 0, s>>>(a);
    return launched("distillation step launch");
}

}  // namespace vie
