// A token drawn from a head's candidates (gfx950): temperature, top-k, top-p
// and min-p, from a given uniform number.
//
// The candidates of a row (logit above -inf, not NaN; in a list also id >= 0)
// are ordered by logit descending, then id ascending.  With l_1 the best
// logit and t the temperature, candidate j weighs w_j = exp((l_j - l_1) / t)
// (1 where l_j = l_1, else 0 where l_1 is +inf), and C_j = w_1 + .. + w_j.  The three limits keep a
// prefix of the order:
//   top-k  the first K = min(top_k, candidates),
//   top-p  the first n with C_n >= top_p C_K,
//   min-p  those with w_j >= min_p,
// and the token is the first j with C_j > u C_kept.
//
// Which token that is goes by comparing sums, so weights are fp64 and sums
// are integers: w 2^sh rounded to a 64-bit integer, with sh as large as n
// weights allow (62 - ceil(log2 n): 2^-45 of the best weight per candidate at
// 262144 candidates).  Integer sums do not depend on their order, so that
// the result is the same from run to run however the additions fall.
#include <hip/hip_runtime.h>

#include "block.hpp"
#include "keys.hpp"
#include "operators.hpp"

namespace vie {

namespace {

struct Settings {
    float t, p, m;
    int k;
};
__device__ __forceinline__ Settings settings(const vie_sample_params &a, int b)
{
    return {a.temperature_dev ? a.temperature_dev[b] : a.temperature, a.top_p_dev ? a.top_p_dev[b] : a.top_p,
            a.min_p_dev ? a.min_p_dev[b] : a.min_p, a.top_k_dev ? a.top_k_dev[b] : a.top_k};
}

__host__ __device__ inline int fixed_shift(int64_t n)
{
    int lg = 0;
    while ((int64_t(1) << lg) < n) ++lg;
    return 62 - lg;
}

__device__ __forceinline__ double weight(float l, float best, double inv_t)
{
    const double x = ((double)l - (double)best) * inv_t;
    return l == best ? 1.0 : x == x ? exp(x) : 0.0;  // (no number: the best is +inf and so is t)
}
__device__ __forceinline__ uint64_t fixed(double w, double one) { return (uint64_t)(w * one + 0.5); }

// Borders as integers: C >= p T iff C >= reach(p, T), C > u T iff C > below(u, T).
__device__ __forceinline__ uint64_t reach(float p, uint64_t total) { return p > 0.0f ? (uint64_t)ceil((double)p * (double)total) : 0ull; }
__device__ __forceinline__ uint64_t below(float u, uint64_t total)
{
    return u > 0.0f ? (uint64_t)fmin((double)u * (double)total, 9.2e18) : 0ull;
}

struct Result {
    int32_t token;
    float prob;
    int32_t kept;
};
__device__ __forceinline__ void put(const SampleLaunch &a, int b, Result r)
{
    a.token[b] = r.token;
    if (a.prob) a.prob[b] = r.prob;
    if (a.kept) a.kept[b] = r.kept;
}

__device__ __forceinline__ bool candidate(float l) { return l > -__builtin_inff(); }  // false for NaN

// ---------------------------------------------------------------------------
// lists
// ---------------------------------------------------------------------------

// Ascending position of the first of n inclusive sums that is at least
// (STRICT: above) x; n if there is none.
template <bool STRICT> __device__ __forceinline__ int first_at(const uint64_t *sums, int n, uint64_t x)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (STRICT ? sums[mid] > x : sums[mid] >= x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// P keys (a power of two) in descending order, by NT threads.
template <int NT> __device__ void sort_keys(uint64_t *key, int P)
{
    for (int k = 2; k <= P; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < P / 2; i += NT) {
                const int x = ((i & ~(j - 1)) << 1) | (i & (j - 1)), y = x | j;
                const uint64_t u = key[x], v = key[y];
                if ((x & k) == 0 ? u < v : u > v) key[x] = v, key[y] = u;
            }
        }
    __syncthreads();
}

// One workgroup per list.  The keys are put in order if they are not (a
// head's lists are), weighed and summed in LDS.
template <int NT> __global__ __launch_bounds__(NT) void sample_list_kernel(SampleLaunch a)
{
    constexpr int W = NT / kLanes;
    extern __shared__ uint64_t s_key[];
    __shared__ uint64_t s_wave[W];
    __shared__ int s_min;
    const int b = blockIdx.x, n = (int)a.n, tid = threadIdx.x;
    int P = 64;
    while (P < n) P <<= 1;
    uint64_t *s_sum = s_key + P;
    const int32_t *ids = a.ids + (int64_t)b * a.ld;
    const float *l = static_cast<const float *>(a.logits) + (int64_t)b * a.ld;
    const Settings st = settings(a.prm, b);
    const float u = a.u[b];
    for (int j = tid; j < P; j += NT) {
        uint64_t key = 0;
        if (j < n && ids[j] >= 0 && candidate(l[j])) key = make_key(l[j], ids[j]);
        s_key[j] = key;
    }
    if (tid == 0) s_min = 0;
    __syncthreads();
    bool off = false;
    int live = 0;
    for (int j = tid; j < P; j += NT) {
        off |= j + 1 < P && s_key[j] < s_key[j + 1];
        live += s_key[j] != 0;
    }
    if (__syncthreads_or(off)) sort_keys<NT>(s_key, P);
    __shared__ int s_live[W];
    live = block_reduce<NT>(live, s_live, [](int x, int y) { return x + y; });
    if (live == 0) {
        if (tid == 0) put(a, b, {-1, 0.0f, 0});
        return;
    }
    if (!(st.t > 0.0f)) {
        if (tid == 0) put(a, b, {key_id(s_key[0]), 1.0f, 1});
        return;
    }
    const float best = key_logit(s_key[0]);
    const double inv_t = 1.0 / (double)st.t, one = ldexp(1.0, fixed_shift(kMaxList));
    const int K = st.k > 0 && st.k < live ? st.k : live;
    // sums in order, NT candidates at a time; the prefix that passes min-p
    uint64_t base = 0;
    for (int j0 = 0; j0 < K; j0 += NT) {
        const int j = j0 + tid;
        double w = 0.0;
        if (j < K) w = weight(key_logit(s_key[j]), best, inv_t);
        const bool ok = j < K && w >= (double)st.m;
        uint64_t x = wave_scan(j < K ? fixed(w, one) : 0ull);
        const unsigned long long pass = __ballot(ok);
        if (W > 1) {
            if ((tid & (kLanes - 1)) == kLanes - 1) s_wave[tid / kLanes] = x;
            __syncthreads();
            for (int i = 0; i < tid / kLanes; ++i) x += s_wave[i];
        }
        if ((tid & (kLanes - 1)) == 0) atomicAdd(&s_min, __popcll(pass));
        x += base;
        if (j < K) s_sum[j] = x;
        __syncthreads();
        base = s_sum[min(j0 + NT, K) - 1];
        if (W > 1) __syncthreads();
    }
    __syncthreads();
    if (tid != 0) return;
    int kept = K;
    if (st.p < 1.0f) kept = min(kept, first_at<false>(s_sum, K, reach(st.p, s_sum[K - 1])) + 1);
    if (st.m > 0.0f) kept = min(kept, s_min);
    kept = max(kept, 1);
    const uint64_t total = s_sum[kept - 1];
    const int j = min(first_at<true>(s_sum, kept, below(u, total)), kept - 1);
    put(a, b, {key_id(s_key[j]), (float)(weight(key_logit(s_key[j]), best, inv_t) * one / (double)total), kept});
}

// ---------------------------------------------------------------------------
// full rows
// ---------------------------------------------------------------------------

constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / kLanes;
constexpr int kDigit = 11;                 // key bits settled by a pass
constexpr int kBins = 1 << kDigit;

// A candidate's place in the order: how many and how much weight come up to
// it (itself included), and its key.
struct Place {
    uint64_t key, sum;
    int64_t rank;
};

struct RowLds {
    uint64_t sum[kBins];
    uint32_t count[kBins];
    uint64_t wave_sum[kRowWaves];
    uint32_t wave_count[kRowWaves];
    uint64_t key[kRowWaves];
    Place at;
    int bin;
};

template <bool BF16> struct Row {
    typedef Elem<BF16> E;
    const typename E::T *l;
    int64_t n;
    float best;
    double inv_t, one;

    // f(logit, id) for every candidate, by the whole workgroup
    template <typename F> __device__ __forceinline__ void each(F f) const
    {
        const Span<typename E::T> sp(l, n);
        const word4 *v = reinterpret_cast<const word4 *>(l + sp.head);
        for (int64_t i = threadIdx.x; i < sp.vecs; i += kRowThreads) {
            float x[E::kVec];
            E::unpack(v[i], x);
#pragma unroll
            for (int e = 0; e < E::kVec; ++e)
                if (candidate(x[e])) f(x[e], (int32_t)(sp.head + i * E::kVec + e));
        }
        for (int64_t i = threadIdx.x; i < sp.head + n - sp.tail0; i += kRowThreads) {
            const int64_t at = i < sp.head ? i : sp.tail0 + i - sp.head;
            const float x = E::get(l[at]);
            if (candidate(x)) f(x, (int32_t)at);
        }
    }
};

// The first candidate in the order whose rank is at least `rank` (BY_RANK),
// or else whose sum is at least `sum`: digits of the keys from the top, each
// by a histogram of the candidates that share the digits before.  If there is
// none (`sum` above the total), the last candidate.
template <bool BF16, bool BY_RANK>
__device__ Place find(const Row<BF16> &row, int64_t rank, uint64_t sum, RowLds &s)
{
    const int tid = threadIdx.x;
    uint64_t prefix = 0, before_sum = 0;
    int64_t before = 0;
    for (int shift = 64; shift > 0;) {
        const int bits = shift < kDigit ? shift : kDigit;
        shift -= bits;
        __syncthreads();
        for (int i = tid; i < kBins; i += kRowThreads) s.sum[i] = 0, s.count[i] = 0;
        __syncthreads();
        row.each([&](float l, int32_t id) {
            const uint64_t key = make_key(l, id);
            if (shift + bits < 64 && (key >> (shift + bits)) != prefix) return;
            const int bin = (int)((key >> shift) & ((1u << bits) - 1));
            atomicAdd(&s.count[bin], 1u);
            atomicAdd((unsigned long long *)&s.sum[bin], (unsigned long long)fixed(weight(l, row.best, row.inv_t), row.one));
        });
        __syncthreads();
        // bins from the top, two a thread
        const int top = kBins - 1 - 2 * tid;
        const uint64_t s0 = s.sum[top], s1 = s.sum[top - 1];
        const uint32_t c0 = s.count[top], c1 = s.count[top - 1];
        uint64_t cs = wave_scan(s0 + s1);
        uint32_t cc = wave_scan(c0 + c1);
        if ((tid & (kLanes - 1)) == kLanes - 1) s.wave_sum[tid / kLanes] = cs, s.wave_count[tid / kLanes] = cc;
        if (tid == 0) s.bin = -1;
        __syncthreads();
        cs += before_sum;
        int64_t rc = before + cc;
        for (int w = 0; w < tid / kLanes; ++w) cs += s.wave_sum[w], rc += s.wave_count[w];
        // (the places after bins `top` and `top - 1`)
        const uint64_t e1 = cs, e0 = cs - s1, b0 = e0 - s0;
        const int64_t r1 = rc, r0 = rc - c1, q0 = r0 - c0;
        auto take = [&](int bin, uint64_t sum0, int64_t rank0) { s.bin = bin, s.at.sum = sum0, s.at.rank = rank0; };
        auto hit = [&](int64_t r, uint64_t c) { return BY_RANK ? r >= rank : c >= sum; };
        if (c0 && hit(r0, e0) && !(q0 > before && hit(q0, b0))) take(top, b0, q0);
        if (c1 && hit(r1, e1) && !(r0 > before && hit(r0, e0))) take(top - 1, e0, r0);
        __syncthreads();
        if (s.bin < 0) {  // beyond the last candidate: its bin
            int last = -1;
            if (c0) last = top;
            if (c1) last = top - 1;
            int low = last < 0 ? kBins : last;
            low = block_reduce<kRowThreads>(low, reinterpret_cast<int *>(s.key), [](int x, int y) { return x < y ? x : y; });
            if (low == top) take(top, b0, q0);
            if (low == top - 1) take(top - 1, e0, r0);
            __syncthreads();
        }
        prefix = (prefix << bits) | (uint64_t)s.bin;
        before_sum = s.at.sum;
        before = s.at.rank;
    }
    const uint64_t w = fixed(weight(key_logit(prefix), row.best, row.inv_t), row.one);
    return {prefix, before_sum + w, before + 1};
}

// One workgroup per row.
template <bool BF16> __global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleLaunch a)
{
    typedef typename Elem<BF16>::T T;
    __shared__ RowLds s;
    const int b = blockIdx.x, tid = threadIdx.x;
    const Settings st = settings(a.prm, b);
    Row<BF16> row{static_cast<const T *>(a.logits) + (int64_t)b * a.ld, a.n, 0.0f, 0.0, 0.0};
    uint64_t top = 0;
    row.each([&](float l, int32_t id) { top = max(top, make_key(l, id)); });
    top = block_reduce<kRowThreads>(top, s.key, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
    if (top == 0 || !(st.t > 0.0f)) {
        if (tid == 0) put(a, b, top == 0 ? Result{-1, 0.0f, 0} : Result{key_id(top), 1.0f, 1});
        return;
    }
    row.best = key_logit(top);
    row.inv_t = 1.0 / (double)st.t;
    row.one = ldexp(1.0, fixed_shift(a.n));
    // how many candidates there are, how many pass min-p, and the total
    uint64_t total = 0;
    uint32_t live = 0, pass = 0;
    row.each([&](float l, int32_t) {
        const double w = weight(l, row.best, row.inv_t);
        total += fixed(w, row.one);
        ++live;
        pass += w >= (double)st.m;
    });
    auto plus = [](auto x, auto y) { return x + y; };
    total = block_reduce<kRowThreads>(total, s.wave_sum, plus);
    live = block_reduce<kRowThreads>(live, s.wave_count, plus);
    __syncthreads();
    pass = block_reduce<kRowThreads>(pass, s.wave_count, plus);
    Place end{0, total, (int64_t)live};  // the last candidate kept
    if (st.k > 0 && st.k < live) end = find<BF16, true>(row, st.k, 0, s);
    if (st.p < 1.0f) end = find<BF16, false>(row, 0, reach(st.p, end.sum), s);
    if (st.m > 0.0f && (int64_t)pass < end.rank) end = find<BF16, true>(row, max(pass, 1u), 0, s);
    // (never beyond the kept ones, also for u of 1 and above)
    const uint64_t past = below(a.u[b], end.sum) + 1;
    const Place at = find<BF16, false>(row, 0, past < end.sum ? past : end.sum, s);
    if (tid == 0) {
        const double w = weight(key_logit(at.key), row.best, row.inv_t);
        put(a, b, {key_id(at.key), (float)(w * row.one / (double)end.sum), (int32_t)end.rank});
    }
}

vie_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

size_t sample_rows_workspace_bytes(int64_t, int) { return 0; }

vie_status launch_sample_lists(const SampleLaunch &a, hipStream_t s)
{
    int P = 64;
    while (P < a.n) P <<= 1;
    const size_t lds = (size_t)P * 16;
    if (a.n <= 64) sample_list_kernel<64><<<a.B, 64, lds, s>>>(a);
    else sample_list_kernel<256><<<a.B, 256, lds, s>>>(a);
    return launched("list sampling launch");
}

vie_status launch_sample_rows(const SampleLaunch &a, hipStream_t s)
{
    if (a.dtype == VIE_BF16) sample_row_kernel<true><<<a.B, kRowThreads, 0, s>>>(a);
    else sample_row_kernel<false><<<a.B, kRowThreads, 0, s>>>(a);
    return launched("row sampling launch");
}

}  // namespace vie
