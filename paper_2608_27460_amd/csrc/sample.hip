// A token drawn from a head's candidates (gfx950): temperature, top-k, top-p
// and min-p, from a given uniform number.
//
// The candidates of a row (logit above -inf, not NaN; in a list also id >= 0)
// are ordered by logit descending, then id ascending.  With l_1 the best
// logit and t the temperature, candidate j weighs w_j = exp((l_j - l_1) / t)
// (1 where l_j = l_1, else 0 where l_1 is +inf), and C_j = w_1 + .. + w_j.
// The three limits keep a prefix of the order:
//   top-k  the first K = min(top_k, candidates),
//   top-p  the first n with C_n >= top_p C_K,
//   min-p  those with w_j >= min_p,
// and the token is the first j with C_j > u C_kept.
//
// Which token that is goes by comparing sums, so weights are fp64 and sums
// are integers: w 2^sh rounded to a 64-bit integer, with sh as large as n
// weights and the rounding in fp64 allow (62 - ceil(log2 n), at most 51: an
// error of at most 2^-45 of the best weight a candidate at 262144 of them).
// Integer sums do not depend on their order, so that the result is the same
// from run to run however the additions fall.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "block.hpp"
#include "keys.hpp"
#include "operators.hpp"

namespace vie {

namespace {

struct Settings {
    double t, p, m;
    int k;
};
__device__ __forceinline__ Settings settings(const vie_sample_params &a, int b)
{
    return {a.temperature_dev ? (double)a.temperature_dev[b] : a.temperature,
            a.top_p_dev ? (double)a.top_p_dev[b] : a.top_p, a.min_p_dev ? (double)a.min_p_dev[b] : a.min_p,
            a.top_k_dev ? a.top_k_dev[b] : a.top_k};
}

__host__ __device__ inline int fixed_shift(int64_t n)
{
    int lg = 11;  // (at most 2^51 a weight, which fp64 holds with its rounding)
    while ((int64_t(1) << lg) < n) ++lg;
    return 62 - lg;
}

// 2^(i / 64) by its series
struct Exp2Table {
    double v[64];
};
constexpr double exp2_64(int i)
{
    const double x = i * 0.69314718055994530942 / 64;
    double t = 1.0, s = 1.0;
    for (int n = 1; n < 26; ++n) t *= x / n, s += t;
    return s;
}
constexpr Exp2Table make_table()
{
    Exp2Table t{};
    for (int i = 0; i < 64; ++i) t.v[i] = exp2_64(i);
    return t;
}
__device__ constexpr Exp2Table kExp2 = make_table();

// Weights in units of 2^-shift of the best one, without branches, so that the
// latencies of several overlap: exp((l - best) / t) = 2^(y / 64), y the
// difference times 64 log2(e) / t; a table gives the whole part of y, the
// Taylor sum to the fifth power the rest (at most 1/2: the sixth power is
// below 2^-55 of the sum).  The error is that of y, 2^-47 relative for the
// smallest weights.  Exactly 1 at the best logit.  An infinite best logit is
// 1e300 here, as are all infinite ones, so that no difference is NaN, and the
// factor is kept where such a difference is still -inf or large.
struct Weights {
    double best, scale;
    int shift;
    const double *table;  // kExp2's values, or a copy of them in LDS
    __device__ __forceinline__ Weights(float best, double t, int shift, const double *table = kExp2.v)
        : best(fmin((double)best, 1e300)), scale(fmin(fmax(64 * 1.4426950408889634074 / t, 1e-290), 1e300)), shift(shift),
          table(table)
    {
    }
    __device__ __forceinline__ double real(float l) const  // times 2^shift
    {
        const double y = fmax((fmin((double)l, 1e300) - best) * scale, -64.0 * 1100.0);  // (2^-1100 is 0 in any units)
        const double k = rint(y), f = y - k;
        constexpr double c = 0.69314718055994530942 / 64;
        double p = fma(f, c * c * c * c * c / 120, c * c * c * c / 24);
        p = fma(p, f, c * c * c / 6);
        p = fma(p, f, c * c / 2);
        p = fma(p, f, c);
        p = fma(p, f, 1.0);
        const int n = (int)k;
        return ldexp(table[n & 63] * p, (n >> 6) + shift);
    }
    static __device__ __forceinline__ uint64_t round(double w)  // to the nearest integer, from the bits of 2^52 + w
    {
        return __builtin_bit_cast(uint64_t, w + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
    }
    __device__ __forceinline__ uint64_t units(float l) const { return round(real(l)); }
    __device__ __forceinline__ double least(double min_p) const { return ldexp(min_p, shift); }
};

// Borders as integers: C >= p T iff C >= reach(p, T), C > u T iff C > below(u, T).
// (p T, rounded to fp64, may pass T for p within 2^-52 of 1: T is reached.)
__device__ __forceinline__ uint64_t reach(double p, uint64_t total)
{
    return p > 0.0 ? min((uint64_t)ceil(p * (double)total), total) : 0ull;
}
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
// head's lists are), weighed and summed in LDS.  Latency bounds it, of the
// loads, the weights and the searches one after the other: 3.4 us for a list
// of 50 and 5.3 for 256 lists of 114 with settings of their own (9 where they
// come from memory), of which a launch is 3.5.
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
    if (!(st.t > 0.0)) {
        if (tid == 0) put(a, b, {key_id(s_key[0]), 1.0f, 1});
        return;
    }
    const Weights weights(key_logit(s_key[0]), st.t, fixed_shift(kMaxList));
    const double least = weights.least(st.m);
    const int K = st.k > 0 && st.k < live ? st.k : live;
    // sums in order, NT candidates at a time; the prefix that passes min-p
    uint64_t base = 0;
    for (int j0 = 0; j0 < K; j0 += NT) {
        const int j = j0 + tid;
        double w = 0.0;
        if (j < K) w = weights.real(key_logit(s_key[j]));
        const bool ok = j < K && w >= least;
        uint64_t x = wave_scan<uint64_t>(j < K ? Weights::round(w) : 0ull);
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
    if (st.p < 1.0) kept = min(kept, first_at<false>(s_sum, K, reach(st.p, s_sum[K - 1])) + 1);
    if (st.m > 0.0) kept = min(kept, s_min);
    kept = max(kept, 1);
    const uint64_t total = s_sum[kept - 1];
    const int j = min(first_at<true>(s_sum, kept, below(u, total)), kept - 1);
    put(a, b, {key_id(s_key[j]), (float)(weights.real(key_logit(s_key[j])) / (double)total), kept});
}

// ---------------------------------------------------------------------------
// full rows
// ---------------------------------------------------------------------------
//
// A row of V logits would have to be sorted for its limits and its token to
// be read off; but all of them are borders in one order, and only the
// candidates around a border matter one by one.  So the candidates are
// counted and weighed in bins that keep the order, by their distance from the
// best logit, and only those of a bin that a border may fall into are put in
// order themselves:
//
//   rows_best_kernel   the best key of each part of a row,
//   rows_bins_kernel   how many candidates and how much weight each bin holds
//                      (in LDS, then added up in memory), and how many
//                      candidates pass min-p,
//   rows_draw_kernel   sums over the bins; the bins that each border can fall
//                      into, given those before it (top-k, then top-p, then
//                      the token); their candidates, collected.  The last
//                      workgroup of a row to finish orders them, and their
//                      sums, from those of the bins before, give the exact
//                      borders.
//
// A bin of an fp32 row is the leading bits of the distance: 1024 to the
// octave from 1/8 to 32, so that the bins are finest where the candidates are
// few and weigh most.  A bf16 row has few enough values for a bin each; its
// candidates are counted only, and weighed by the bin.  A border in the bulk
// of 262144 normal logits meets some 400 candidates of its bin.
//
// Latency bounds it: each kernel is a chain of loads, sums and searches that
// wait for one another, from 1 to 3 us each.  One row of 262144 fp32: 3.8, 7.1
// and 15.0 us; 64 rows of 151936 bf16: 7.8, 14.6 and 21.8, where reading them
// takes 4.
//
// Short rows, or many, take a workgroup each, which does all of this in one
// kernel (rows_one_kernel).
//
// Rows whose border bins hold more than kCollect candidates take one of two
// other ways.  Where each of these bins holds one value (logits that were
// rounded to bf16 somewhere, constant rows), its candidates weigh the same,
// and borders and the token's place among them follow from their number.
// Otherwise the borders are found one after the other from histograms of the
// keys' digits: exact too, in up to 24 passes of one workgroup.  That is slow,
// and happens to fp32 rows whose border falls where the bins are coarse: within
// 1/8 of the best logit, or more than 32 below it.  Normal logits with top_p
// 0.95, in us: one row of 262144 30 down to a standard deviation of 0.05 and 645
// at 0.02 and less; 64 rows of 151936 57 down to 0.1 and 425 to 510 from 0.05 on;
// deviations of 20 and more at a temperature as large 640 and 540.

constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / kLanes;
constexpr int kDigit = 11;                 // key bits settled by a pass
constexpr int kDigits = 1 << kDigit;
constexpr int kBins = 8192;
constexpr int kBinsPer = kBins / kRowThreads;
constexpr int kCollect = 2048;             // candidates put in order one by one
constexpr int kMaxParts = 128;
constexpr int kMaxSlots = 256;             // bins that borders can fall into
constexpr int kTies = 8;                   // border bins that may be too full to be collected

// Bins of a row of this best key: `of` is monotone in the logit and 0 at the
// best one.
template <bool BF16> struct Bins;

// fp32: the distance's leading bits.  Infinite logits count as the largest
// finite one, so that none is NaN; a NaN falls into the last bin.
template <> struct Bins<false> {
    float top;
    __device__ __forceinline__ explicit Bins(uint64_t best) : top(fminf(key_logit(best), __FLT_MAX__)) {}
    __device__ __forceinline__ int of(float l) const
    {
        constexpr int kFirst = 124 << 10;  // 2^-3: exponent 124, ten mantissa bits
        const int x = (int)(__float_as_uint(top - fminf(l, __FLT_MAX__)) >> 13) - kFirst + 1;
        return x < 0 ? 0 : x > kBins - 1 ? kBins - 1 : x;
    }
};

// bf16: a bin for each value of 2^-12 and more in size, one for those between,
// the last one for all from 8191 values below the best.
template <> struct Bins<true> {
    static constexpr int kSmall = 115 << 7;  // the bits of 2^-12
    int top;
    __device__ __forceinline__ explicit Bins(uint64_t best) : top(place(key_logit(best))) {}
    static __device__ __forceinline__ int place(float l)
    {
        const int m = max((int)(__float_as_uint(l) >> 16 & 0x7FFF) - kSmall + 1, 0);
        return __float_as_int(l) < 0 ? -m : m;
    }
    __device__ __forceinline__ int of(float l) const { return min(max(top - place(l), 0), kBins - 1); }
    // whether a bin holds one value, and that value
    __device__ __forceinline__ bool one(int bin) const { return bin != top && bin != kBins - 1; }
    __device__ __forceinline__ float value(int bin) const
    {
        const int at = top - bin;
        return from_bf16((uint32_t)(at < 0 ? 0x8000 - at - 1 + kSmall : at - 1 + kSmall));
    }
};

// A row's part of the workspace.
struct RowSpace {
    uint64_t best[kMaxParts];
    uint64_t sum[kBins];
    uint64_t key[kCollect];
    uint32_t count[kBins];
    uint32_t pass, collected, done, unused;
};
static_assert(kMaxParts * kTies * 2 <= kCollect, "the parts' counts take the place of the collected keys");
// The same where one workgroup takes the row, whose bins and keys stay in LDS.
struct OneSpace {
    uint64_t key[kTies * 2];
    uint32_t collected, done;
};
// What the draw uses of either.
struct Exchange {
    uint64_t *key;
    uint32_t *collected, *done;
};

// A candidate's place in the order: how many and how much weight come up to
// it (itself included), and its key.
struct Place {
    uint64_t key, sum;
    int64_t rank;
};

struct DigitLds {
    uint64_t sum[kDigits];
    uint32_t count[kDigits];
    uint64_t wave_sum[kRowWaves];
    uint32_t wave_count[kRowWaves];
    int wave_bin[kRowWaves];
    Place at;
    int bin;
};

template <bool BF16> struct Row {
    typedef Elem<BF16> E;
    const typename E::T *l;
    int64_t n;

    // f(logit, id) for every candidate of the n logits from i0 on, by the whole workgroup
    template <typename F> __device__ __forceinline__ void each(int64_t i0, int64_t n, F f) const
    {
        groups(i0, n, [&](const float *x, int32_t id, auto count) {
#pragma unroll
            for (int e = 0; e < decltype(count)::value; ++e)
                if (candidate(x[e])) f(x[e], id + e);
        });
    }
    // f(logits, first id, how many) for groups of them: 16 bytes, or one at the ends
    template <typename F> __device__ __forceinline__ void groups(int64_t i0, int64_t n, F f) const
    {
        const typename E::T *p = l + i0;
        const Span<typename E::T> sp(p, n);
        const word4 *v = reinterpret_cast<const word4 *>(p + sp.head);
        // (the next 16 bytes are on their way while these are worked on)
        word4 next = {0, 0, 0, 0};
        if (threadIdx.x < sp.vecs) next = v[threadIdx.x];
        for (int64_t i = threadIdx.x; i < sp.vecs; i += kRowThreads) {
            const word4 w = next;
            if (i + kRowThreads < sp.vecs) next = v[i + kRowThreads];
            float x[E::kVec];
            E::unpack(w, x);
            f(x, (int32_t)(i0 + sp.head + i * E::kVec), std::integral_constant<int, E::kVec>());
        }
        for (int64_t i = threadIdx.x; i < sp.head + n - sp.tail0; i += kRowThreads) {
            const int64_t at = i < sp.head ? i : sp.tail0 + i - sp.head;
            const float x = E::get(p[at]);
            f(&x, (int32_t)(i0 + at), std::integral_constant<int, 1>());
        }
    }
};

// Inclusive sums over the workgroup's threads of a count and a sum, and the
// totals.
__device__ __forceinline__ void block_scan(uint32_t &c, uint64_t &s, uint32_t &c_total, uint64_t &s_total,
                                           uint32_t *wave_count, uint64_t *wave_sum)
{
    c = wave_scan(c);
    s = wave_scan(s);
    wave_total(c, wave_count);
    wave_total(s, wave_sum);
    __syncthreads();
    const auto cs = after_waves(c, wave_count, kRowWaves);
    const auto ss = after_waves(s, wave_sum, kRowWaves);
    c = cs.upto, c_total = cs.total, s = ss.upto, s_total = ss.total;
}

// The first candidate in the order whose rank is at least `rank` (by_rank),
// or else whose sum is at least `sum`: digits of the keys from the top, each
// by a histogram of the candidates that share the digits before.  If there is
// none (`sum` above the total), the last candidate.
template <bool BF16>
__device__ __forceinline__ Place find(const Row<BF16> &row, const Weights &weights, bool by_rank, int64_t rank, uint64_t sum, DigitLds &s)
{
    const int tid = threadIdx.x;
    uint64_t prefix = 0, before_sum = 0;
    int64_t before = 0;
    for (int shift = 64; shift > 0;) {
        const int bits = shift < kDigit ? shift : kDigit;
        shift -= bits;
        __syncthreads();
        for (int i = tid; i < kDigits; i += kRowThreads) s.sum[i] = 0, s.count[i] = 0;
        __syncthreads();
        row.each(0, row.n, [&](float l, int32_t id) {
            const uint64_t key = make_key(l, id);
            if (shift + bits < 64 && (key >> (shift + bits)) != prefix) return;
            const int bin = (int)((key >> shift) & ((1u << bits) - 1));
            const uint64_t units = weights.units(l);
            // (where a wave's candidates share a digit and a weight, as equal
            // logits do, one of them adds for all)
            const unsigned long long active = __ballot(1);
            if (__all(bin == __builtin_amdgcn_readfirstlane(bin)) && __all(l == __shfl(l, __ffsll(active) - 1, kLanes))) {
                if ((threadIdx.x & (kLanes - 1)) == __ffsll(active) - 1) {
                    atomicAdd(&s.count[bin], (uint32_t)__popcll(active));
                    atomicAdd((unsigned long long *)&s.sum[bin], (unsigned long long)(units * __popcll(active)));
                }
            } else {
                atomicAdd(&s.count[bin], 1u);
                atomicAdd((unsigned long long *)&s.sum[bin], (unsigned long long)units);
            }
        });
        __syncthreads();
        // bins from the top, two a thread
        const int top = kDigits - 1 - 2 * tid;
        const uint64_t s0 = s.sum[top], s1 = s.sum[top - 1];
        const uint32_t c0 = s.count[top], c1 = s.count[top - 1];
        uint64_t cs = s0 + s1;
        uint32_t cc = c0 + c1;
        if (tid == 0) s.bin = -1;
        uint32_t all_count;
        uint64_t all_sum;
        block_scan(cc, cs, all_count, all_sum, s.wave_count, s.wave_sum);
        cs += before_sum;
        const int64_t rc = before + cc;
        // (the places after bins `top` and `top - 1`)
        const uint64_t e1 = cs, e0 = cs - s1, b0 = e0 - s0;
        const int64_t r1 = rc, r0 = rc - c1, q0 = r0 - c0;
        auto take = [&](int bin, uint64_t sum0, int64_t rank0) { s.bin = bin, s.at.sum = sum0, s.at.rank = rank0; };
        auto hit = [&](int64_t r, uint64_t c) { return by_rank ? r >= rank : c >= sum; };
        if (c0 && hit(r0, e0) && !(q0 > before && hit(q0, b0))) take(top, b0, q0);
        if (c1 && hit(r1, e1) && !(r0 > before && hit(r0, e0))) take(top - 1, e0, r0);
        __syncthreads();
        if (s.bin < 0) {  // beyond the last candidate: its bin
            int low = c1 ? top - 1 : c0 ? top : kDigits;
            low = block_reduce<kRowThreads>(low, s.wave_bin, [](int x, int y) { return x < y ? x : y; });
            if (low == top) take(top, b0, q0);
            if (low == top - 1) take(top - 1, e0, r0);
            __syncthreads();
        }
        prefix = (prefix << bits) | (uint64_t)s.bin;
        before_sum = s.at.sum;
        before = s.at.rank;
    }
    return {prefix, before_sum + weights.units(key_logit(prefix)), before + 1};
}

// The drawn candidate as a result; `end` units of weight are kept.
__device__ __forceinline__ Result drawn(const Weights &weights, uint64_t key, uint64_t end, int64_t kept)
{
    return {key_id(key), (float)(weights.real(key_logit(key)) / (double)end), (int32_t)kept};
}

// The borders one after the other, over the whole row: `live` candidates,
// `total` units of weight, `pass` candidates within min-p.
template <bool BF16>
__device__ __forceinline__ Result draw_by_digits(const Row<BF16> &row, const Weights &weights, Settings st, float u, uint32_t live, uint64_t total, uint32_t pass,
                                 DigitLds &s)
{
    Place end{0, total, (int64_t)live};  // the last candidate kept
    if (st.k > 0 && st.k < live) end = find<BF16>(row, weights, true, st.k, 0, s);
    if (st.p < 1.0) end = find<BF16>(row, weights, false, 0, reach(st.p, end.sum), s);
    if (st.m > 0.0 && (int64_t)pass < end.rank) end = find<BF16>(row, weights, true, max(pass, 1u), 0, s);
    // (never beyond the kept ones, also for u of 1 and above)
    const uint64_t past = below(u, end.sum) + 1;
    const Place at = find<BF16>(row, weights, false, 0, past < end.sum ? past : end.sum, s);
    return drawn(weights, at.key, end.sum, end.rank);
}

// Workgroup (c, b) takes part c of row b in each of the three kernels.
struct Parts {
    int64_t len;  // candidates of a part
    RowSpace *ws;
};
template <bool BF16> __device__ __forceinline__ Row<BF16> row_of(const SampleLaunch &a, int b)
{
    return {static_cast<const typename Elem<BF16>::T *>(a.logits) + (int64_t)b * a.ld, a.n};
}

// The best key among n logits from i0 on, in every thread (0: no candidate).
template <bool BF16> __device__ __forceinline__ uint64_t best_of(const Row<BF16> &row, int64_t i0, int64_t n, uint64_t *tmp)
{
    uint64_t best = 0;
    row.each(i0, n, [&](float l, int32_t id) {
        const uint64_t key = make_key(l, id);
        best = key > best ? key : best;
    });
    return block_reduce<kRowThreads>(best, tmp, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
}

template <bool BF16> __global__ __launch_bounds__(kRowThreads) void rows_best_kernel(SampleLaunch a, Parts parts)
{
    __shared__ uint64_t tmp[kRowWaves];
    const int b = blockIdx.y, c = blockIdx.x, S = gridDim.x;
    RowSpace &ws = parts.ws[b];
    for (int i = c * kRowThreads + threadIdx.x; i < kBins; i += S * kRowThreads) ws.sum[i] = 0, ws.count[i] = 0;
    if (c == 0 && threadIdx.x == 0) ws.pass = ws.collected = ws.done = 0;
    const Row<BF16> row = row_of<BF16>(a, b);
    const int64_t i0 = c * parts.len;
    const uint64_t best = best_of(row, i0, min(parts.len, a.n - i0), tmp);
    if (threadIdx.x == 0) ws.best[c] = best;
}

__device__ __forceinline__ uint64_t best_key(const RowSpace &ws, int S)
{
    uint64_t k = 0;
    for (int i = threadIdx.x & (kLanes - 1); i < S; i += kLanes) k = ws.best[i] > k ? ws.best[i] : k;
    return wave_max(k);
}

// Whether a row has more to draw than its best candidate, or none, and the
// result where not.
__device__ __forceinline__ bool open(uint64_t best, Settings st) { return best != 0 && st.t > 0.0; }
__device__ __forceinline__ Result closed(uint64_t best)
{
    return best == 0 ? Result{-1, 0.0f, 0} : Result{key_id(best), 1.0f, 1};
}

// A row's bins in LDS: counts, and sums (bf16: of the bins of more than one
// value, the others' follow from their counts).
template <bool BF16> struct BinLds {
    static constexpr int kSums = BF16 ? 2 : kBins;
    uint64_t sum[kSums];
    uint32_t count[kBins];
    double exp[64];
    uint32_t pass;
    uint64_t tmp[kRowWaves];

    __device__ __forceinline__ void clear()
    {
        const int tid = threadIdx.x;
        for (int i = tid; i < kSums / 2; i += kRowThreads) reinterpret_cast<ulonglong2 *>(sum)[i] = {0, 0};
        for (int i = tid; i < kBins / 4; i += kRowThreads) reinterpret_cast<uint4 *>(count)[i] = {0, 0, 0, 0};
        if (tid < 64) exp[tid] = kExp2.v[tid];
        if (tid == 0) pass = 0;
    }
    // n logits from i0 on; returns how many of this thread's pass min-p
    // (bf16: of those in bins of more than one value)
    __device__ __forceinline__ uint32_t add(const Row<BF16> &row, int64_t i0, int64_t n, const Weights &weights,
                                            const Bins<BF16> &bin_map, double least)
    {
        uint32_t passed = 0;
        row.groups(i0, n, [&](const float *l, int32_t, auto number) {
            constexpr int N = decltype(number)::value;
            int bin[N];
            uint64_t units[N];
            if constexpr (BF16) {
#pragma unroll
                for (int e = 0; e < N; ++e) bin[e] = bin_map.of(l[e]);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (!candidate(l[e])) continue;
                    atomicAdd(&count[bin[e]], 1u);
                    if (!bin_map.one(bin[e])) {
                        const double w = weights.real(l[e]);
                        passed += w >= least;
                        atomicAdd((unsigned long long *)&sum[bin[e] != bin_map.top], (unsigned long long)Weights::round(w));
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {  // (without branches, so that their latencies overlap)
                    bin[e] = bin_map.of(l[e]);
                    const double w = weights.real(l[e]);
                    passed += candidate(l[e]) & (w >= least);
                    units[e] = Weights::round(w);
                }
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (candidate(l[e])) {
                        atomicAdd(&count[bin[e]], 1u);
                        atomicAdd((unsigned long long *)&sum[bin[e]], (unsigned long long)units[e]);
                    }
            }
        });
        return passed;
    }
    // the weight of the n > 0 candidates of bin i, and those of them that
    // pass min-p and were not counted yet
    __device__ __forceinline__ uint64_t weight(int i, uint32_t n, const Weights &weights, const Bins<BF16> &bin_map, double least,
                                               uint32_t &passed) const
    {
        if constexpr (BF16) {
            if (!bin_map.one(i)) return sum[i != bin_map.top];
            const double w = weights.real(bin_map.value(i));
            if (w >= least) passed += n;
            return Weights::round(w) * n;
        } else {
            return sum[i];
        }
    }
    // all threads' numbers into `pass` (complete after the next barrier)
    __device__ __forceinline__ void add_pass(uint32_t passed)
    {
        passed = wave_sum(passed);
        if ((threadIdx.x & (kLanes - 1)) == 0 && passed) atomicAdd(&pass, passed);
    }
};

template <bool BF16> __global__ __launch_bounds__(kRowThreads) void rows_bins_kernel(SampleLaunch a, Parts parts)
{
    extern __shared__ __align__(16) char smem[];
    BinLds<BF16> &s = *reinterpret_cast<BinLds<BF16> *>(smem);
    const int b = blockIdx.y, tid = threadIdx.x;
    RowSpace &ws = parts.ws[b];
    const Settings st = settings(a.prm, b);
    const Row<BF16> row = row_of<BF16>(a, b);
    s.clear();
    const uint64_t best = best_key(ws, gridDim.x);
    if (!open(best, st)) return;
    const Weights weights(key_logit(best), st.t, fixed_shift(a.n), s.exp);
    const double least = weights.least(st.m);
    const Bins<BF16> bin_map(best);
    __syncthreads();
    const int64_t i0 = blockIdx.x * parts.len;
    uint32_t passed = s.add(row, i0, min(parts.len, a.n - i0), weights, bin_map, least);
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < kBins; i += kRowThreads) {
        const uint32_t n = s.count[i];
        if (n == 0) continue;
        const uint64_t sum = s.weight(i, n, weights, bin_map, least, passed);
        atomicAdd(&ws.count[i], n);
        atomicAdd((unsigned long long *)&ws.sum[i], (unsigned long long)sum);
    }
    s.add_pass(passed);
    __syncthreads();
    if (tid == 0) atomicAdd(&ws.pass, s.pass);
}

// The bin that a border falls into, with what lies before it and up to its end.
struct Bin {
    int bin;
    uint32_t count0, count1;
    uint64_t sum0, sum1;
};

// A bin whose candidates are collected: what lies before it, and how many
// collected candidates.
struct Slot {
    uint64_t base;
    uint32_t rank, first;
    int bin;
};

struct DrawLds {
    union {
        struct {
            uint64_t key[kCollect], sum[kCollect];  // the collected candidates in order, their sums
            Slot slot[kMaxSlots];
            uint32_t flag[kBins / 32];              // the bins collected
        } d;
        DigitLds digits;
    };
    uint64_t wave_sum[kRowWaves];
    uint32_t wave_count[kRowWaves];
    Bin at[2];
    uint64_t found_sum, found_key;
    int64_t found_rank;
    uint32_t base, last;
};

// P keys (a power of two, at most 2 kRowThreads) in descending order: thread
// t holds keys t and t + kRowThreads; pairs less than a wave apart meet by
// lane exchanges, the others in LDS.
__device__ void sort_row(uint64_t *key, int P)
{
    constexpr int E = 2;
    const int tid = threadIdx.x;
    uint64_t v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e * kRowThreads + tid < P ? key[e * kRowThreads + tid] : 0ull;
    auto keep = [&](int e, uint64_t o, int k, int j) {  // the larger one goes first in a descending run
        const int i = e * kRowThreads + tid;
        const bool larger = ((i & k) == 0) == ((i & j) == 0);
        v[e] = (v[e] > o) == larger ? v[e] : o;
    };
    for (int k = 2; k <= P; k <<= 1) {
        for (int j = k >> 1; j >= kLanes; j >>= 1) {
            if (j >= kRowThreads) {
                const uint64_t a = v[0], b = v[1];
                keep(0, b, k, j);
                keep(1, a, k, j);
                continue;
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e * kRowThreads + tid < P) key[e * kRowThreads + tid] = v[e];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e * kRowThreads + tid < P) keep(e, key[(e * kRowThreads + tid) ^ j], k, j);
        }
#define VIE_LANE_STEP(J)                                                                  \
    if (k > J)                                                                            \
        for (int e = 0; e < E; ++e) keep(e, lane_xor(v[e], J), k, J);
        VIE_LANE_STEP(32)
        VIE_LANE_STEP(16)
        VIE_LANE_STEP(8)
        VIE_LANE_STEP(4)
        VIE_LANE_STEP(2)
        VIE_LANE_STEP(1)
#undef VIE_LANE_STEP
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e * kRowThreads + tid < P) key[e * kRowThreads + tid] = v[e];
    __syncthreads();
}

// The same for P keys of at most kRowThreads, different but for zeros, by P
// threads: each wave puts its 64 in order, and a key's place is the number of
// larger ones in all the waves' runs, by binary searches whose latencies
// overlap, four runs at a time (439 keys: 2 us less than in sort_row's way).
// Zeros, which come last, are not put back.
__device__ __forceinline__ void sort_distinct(uint64_t *key, int P)
{
    const int tid = threadIdx.x, lane = tid & (kLanes - 1);
    uint64_t v = key[tid];
#pragma unroll
    for (int k = 2; k <= kLanes; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            const uint64_t o = lane_xor(v, j);
            const bool larger = ((lane & k) == 0) == ((lane & j) == 0);
            v = (v > o) == larger ? v : o;
        }
    if (P > kLanes) {
        key[tid] = v;
        __syncthreads();
        int place = 0;
        for (int run = 0; run < P; run += 4 * kLanes) {
            int n[4] = {0, 0, 0, 0};
#pragma unroll
            for (int step = kLanes / 2; step >= 1; step >>= 1)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key[(run + i * kLanes) % P + n[i] + step - 1] > v) n[i] += step;
#pragma unroll
            for (int i = 0; i < 4; ++i)  // (and the 64th; runs past P count nothing)
                place += run + i * kLanes < P ? n[i] + (key[(run + i * kLanes) % P + n[i]] > v) : 0;
        }
        __syncthreads();
        if (v != 0) key[place] = v;
    } else {
        key[tid] = v;
    }
    __syncthreads();
}

// What the draw knows of a row's borders: the limits, and the weight of the
// first K candidates and of the kept ones where the bins gave it exactly.
struct Borders {
    uint32_t K, most;
    bool exact_k, exact_end;
    uint64_t sum_k, sum_end;
};

// The draw where the border bins (at most kTies of them) are too full to be
// collected: every part of the row calls it.  The part's candidates of each
// bin are counted, and the lowest and the highest of them kept; the last part
// to finish has those of all.  Returns 0 in the others, 1 with the result,
// and 2, in the last part, if a bin holds more than one value.
template <bool BF16>
__device__ __forceinline__ int draw_ties(const Row<BF16> &row, const Weights &weights, const Bins<BF16> &bin_map,
                                      const Settings &st, float u, const Borders &known, int nslot, int64_t len,
                                      const Exchange &ws, DrawLds &s, Result &out)
{
    typedef Elem<BF16> E;
    const int tid = threadIdx.x, S = gridDim.x, part = blockIdx.x;
    for (int j = 0; j < nslot; ++j) {
        const int bin = s.d.slot[j].bin;
        uint32_t low = ~0u, high = 0, n = 0;
        const int64_t i0 = part * len;
        row.each(i0, min(len, row.n - i0), [&](float l, int32_t) {
            if (bin_map.of(l) != bin) return;
            const uint32_t o = f2ord(l);
            low = min(low, o);
            high = max(high, o);
            ++n;
        });
        low = block_reduce<kRowThreads>(low, s.wave_count, [](uint32_t a, uint32_t b) { return min(a, b); });
        high = block_reduce<kRowThreads>(high, s.wave_count, [](uint32_t a, uint32_t b) { return max(a, b); });
        n = block_reduce<kRowThreads>(n, s.wave_count, [](uint32_t a, uint32_t b) { return a + b; });
        if (tid == 0) {
            uint64_t *to = &ws.key[(part * kTies + j) * 2];
            __hip_atomic_store(to, (uint64_t)high << 32 | low, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(to + 1, (uint64_t)n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s.last = __hip_atomic_fetch_add(ws.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s.last != (uint32_t)S - 1) return 0;
    // all parts' counts, and a bin's value and number
    uint64_t *all = s.d.key;
    for (int i = tid; i < S * kTies * 2; i += kRowThreads)
        all[i] = i / 2 % kTies < nslot ? __hip_atomic_load(&ws.key[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0ull;
    __syncthreads();
    bool one = true;
    for (int j = 0; j < nslot; ++j) {
        uint32_t low = ~0u, high = 0, n = 0;
        for (int c = 0; c < S; ++c) {
            const uint64_t v = all[(c * kTies + j) * 2], m = all[(c * kTies + j) * 2 + 1];
            if (m == 0) continue;
            low = min(low, (uint32_t)v);
            high = max(high, (uint32_t)(v >> 32));
            n += (uint32_t)m;
        }
        one &= low == high;
        s.d.sum[2 * j] = high;  // (every thread writes the same)
        s.d.sum[2 * j + 1] = n;
    }
    __syncthreads();
    if (!one) return 2;
    // the place of a rank or a sum: its bin, and how many of it up to there
    struct At {
        int slot;
        uint64_t count, sum;
        int64_t rank;
    };
    auto at = [&](bool by_rank, uint64_t v) {
        int j = 0;
        for (;; ++j) {
            const uint64_t n = s.d.sum[2 * j + 1], unit = weights.units(ord2f((uint32_t)s.d.sum[2 * j]));
            const Slot sl = s.d.slot[j];
            const uint64_t end = by_rank ? sl.rank + n : sl.base + n * unit;
            if (end < v && j + 1 < nslot) continue;
            uint64_t k = by_rank ? v - sl.rank : v > sl.base && unit ? (v - sl.base + unit - 1) / unit : 1;
            k = k < 1 ? 1 : k > n ? n : k;
            return At{j, k, sl.base + k * unit, (int64_t)(sl.rank + k)};
        }
    };
    const uint64_t ck = known.exact_k ? known.sum_k : at(true, known.K).sum;
    int64_t kept = known.most;
    if (st.p < 1.0) kept = min(kept, at(false, reach(st.p, ck)).rank);
    const uint64_t end = known.exact_end ? known.sum_end : at(true, kept).sum;
    const At t = at(false, min(below(u, end) + 1, end));
    // the token: number t.count of its bin, by id; first its part
    uint64_t left = t.count;
    int c = 0;
    for (; c < S - 1 && left > all[(c * kTies + t.slot) * 2 + 1]; ++c) left -= all[(c * kTies + t.slot) * 2 + 1];
    const int64_t i0 = c * len, n = min(len, row.n - i0);
    const int bin = s.d.slot[t.slot].bin;
    const float l = ord2f((uint32_t)s.d.sum[2 * t.slot]);
    if (tid == 0) s.found_rank = 0;
    uint64_t before = 0;
    for (int64_t i = 0; i < n; i += kRowThreads * E::kVec) {
        const int64_t mine = i + tid * E::kVec;
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < E::kVec; ++e) {
            const float x = mine + e < n ? E::get(row.l[i0 + mine + e]) : -__builtin_inff();
            hits |= (uint32_t)(candidate(x) && bin_map.of(x) == bin) << e;
        }
        uint32_t upto = __popc(hits);
        uint64_t none = 0;
        __syncthreads();
        uint32_t sum;
        uint64_t no_sum;
        block_scan(upto, none, sum, no_sum, s.wave_count, s.wave_sum);
        const uint64_t from = before + upto - __popc(hits);
        if (from < left && left <= before + upto) {
            uint32_t h = hits;
            for (uint64_t k = from + 1; k < left; ++k) h &= h - 1;
            s.found_rank = i0 + mine + __ffs(h) - 1;
        }
        before += sum;
        if (before >= left) break;
    }
    __syncthreads();
    out = {(int32_t)s.found_rank, (float)(weights.real(l) / (double)end), (int32_t)kept};
    return 1;
}

// The draw by the row's workgroups, from the bins, kBinsPer a thread, and
// the number of candidates that pass min-p.  (The rare paths are inlined: as
// functions they would take a stack, which costs the kernel 1 us when they
// are not called.)
template <bool BF16>
__device__ __forceinline__ void draw_row(const SampleLaunch &a, int b, const Row<BF16> &row, const Settings &st, float u,
                                         const Weights &weights, const Bins<BF16> &bin_map, const uint32_t (&cnt)[kBinsPer],
                                         const uint64_t (&sum)[kBinsPer], uint32_t pass, int64_t len, const Exchange &ws, DrawLds &s);

template <bool BF16> __global__ __launch_bounds__(kRowThreads) void rows_draw_kernel(SampleLaunch a, Parts parts)
{
    extern __shared__ __align__(16) char smem[];
    const int b = blockIdx.y, tid = threadIdx.x;
    RowSpace &ws = parts.ws[b];
    // the bins (read while the row's settings are)
    uint32_t cnt[kBinsPer];
    uint64_t sum[kBinsPer];
    static_assert(kBinsPer % 4 == 0, "read 16 bytes at a time");
#pragma unroll
    for (int i = 0; i < kBinsPer; i += 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(&ws.count[tid * kBinsPer + i]);
        cnt[i] = v.x, cnt[i + 1] = v.y, cnt[i + 2] = v.z, cnt[i + 3] = v.w;
    }
#pragma unroll
    for (int i = 0; i < kBinsPer; i += 2) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(&ws.sum[tid * kBinsPer + i]);
        sum[i] = v.x, sum[i + 1] = v.y;
    }
    const uint32_t pass = ws.pass;
    const Settings st = settings(a.prm, b);
    const float u = a.u[b];
    const Row<BF16> row = row_of<BF16>(a, b);
    const uint64_t best = best_key(ws, gridDim.x);
    if (!open(best, st)) {
        if (blockIdx.x == 0 && tid == 0) put(a, b, closed(best));
        return;
    }
    draw_row<BF16>(a, b, row, st, u, Weights(key_logit(best), st.t, fixed_shift(a.n)), Bins<BF16>(best), cnt, sum, pass,
                   parts.len, Exchange{ws.key, &ws.collected, &ws.done}, *reinterpret_cast<DrawLds *>(smem));
}

// The three kernels in one, for rows of one part: a workgroup's row, whose
// bins stay in LDS.
template <bool BF16> __global__ __launch_bounds__(kRowThreads) void rows_one_kernel(SampleLaunch a)
{
    extern __shared__ __align__(16) char smem[];
    BinLds<BF16> &s = *reinterpret_cast<BinLds<BF16> *>(smem + sizeof(DrawLds));
    const int b = blockIdx.y, tid = threadIdx.x;
    OneSpace &ws = static_cast<OneSpace *>(a.ws)[b];
    const Settings st = settings(a.prm, b);
    const float u = a.u[b];
    const Row<BF16> row = row_of<BF16>(a, b);
    s.clear();
    if (tid == 0) ws.done = 0;
    const uint64_t best = best_of(row, 0, a.n, s.tmp);  // (the workgroup waits in here)
    if (!open(best, st)) {
        if (tid == 0) put(a, b, closed(best));
        return;
    }
    const Weights weights(key_logit(best), st.t, fixed_shift(a.n), s.exp);
    const double least = weights.least(st.m);
    const Bins<BF16> bin_map(best);
    uint32_t passed = s.add(row, 0, a.n, weights, bin_map, least);
    __syncthreads();
    uint32_t cnt[kBinsPer];
    uint64_t sum[kBinsPer];
#pragma unroll
    for (int i = 0; i < kBinsPer; ++i) {
        cnt[i] = s.count[tid * kBinsPer + i];
        sum[i] = cnt[i] ? s.weight(tid * kBinsPer + i, cnt[i], weights, bin_map, least, passed) : 0ull;
    }
    s.add_pass(passed);
    __syncthreads();
    draw_row<BF16>(a, b, row, st, u, weights, bin_map, cnt, sum, s.pass, a.n, Exchange{ws.key, &ws.collected, &ws.done},
                   *reinterpret_cast<DrawLds *>(smem));
}

template <bool BF16>
__device__ __forceinline__ void draw_row(const SampleLaunch &a, int b, const Row<BF16> &row, const Settings &st, float u,
                                         const Weights &weights, const Bins<BF16> &bin_map, const uint32_t (&cnt)[kBinsPer],
                                         const uint64_t (&sum)[kBinsPer], uint32_t pass, int64_t len, const Exchange &ws, DrawLds &s)
{
    const int tid = threadIdx.x, S = gridDim.x;
    uint32_t c = 0;
    uint64_t x = 0;
#pragma unroll
    for (int i = 0; i < kBinsPer; ++i) {
        c += cnt[i];
        x += sum[i];
    }
    const uint32_t call = c;
    const uint64_t xall = x;
    uint32_t live;
    uint64_t total;
    block_scan(c, x, live, total, s.wave_count, s.wave_sum);
    // before this thread's bins
    c -= call;
    x -= xall;
    for (int i = tid; i < kBins / 32; i += kRowThreads) s.d.flag[i] = 0;
    // the bins of two borders, lo <= hi: each the first bin, not empty, up to
    // whose end the rank (or the sum) is reached; one thread holds it
    const uint32_t cend = c + call;
    const uint64_t xend = x + xall;
    auto bin_at = [&](bool by_rank, uint64_t v, Bin &out) {
        const uint64_t before = by_rank ? c : x, after = by_rank ? cend : xend;
        if (call == 0 || after < v || (c != 0 && before >= v)) return;
        uint32_t ci = c;
        uint64_t xi = x;
#pragma unroll
        for (int i = 0; i < kBinsPer; ++i) {
            const uint64_t v0 = by_rank ? ci : xi, v1 = by_rank ? ci + cnt[i] : xi + sum[i];
            if (cnt[i] && v1 >= v && (ci == 0 || v0 < v)) out = {tid * kBinsPer + i, ci, ci + cnt[i], xi, xi + sum[i]};
            ci += cnt[i];
            xi += sum[i];
        }
    };
    auto bins = [&](bool by_rank, uint64_t lo, uint64_t hi) {
        __syncthreads();
        bin_at(by_rank, lo, s.at[0]);
        if (hi != lo) bin_at(by_rank, hi, s.at[1]);
        __syncthreads();
        return hi != lo ? 1 : 0;  // where the second one is
    };
    // this thread's bins from `first` to `last` are collected (a thread's
    // bits lie in one word that it shares with three others)
    auto collect = [&](int first, int last) {
        if (first >= (tid + 1) * kBinsPer || last < tid * kBinsPer) return;
        const int f = max(first - tid * kBinsPer, 0), l = min(last - tid * kBinsPer, kBinsPer - 1);
        atomicOr(&s.d.flag[tid * kBinsPer / 32], ((2u << l) - (1u << f)) << (tid * kBinsPer % 32));
    };
    // Each quantity as the range that the bins leave it: C_K, ...
    const uint32_t K = st.k > 0 && st.k < live ? st.k : live;
    uint64_t lo = total, hi = total;
    if (K < live) {
        bins(true, K, K);
        const Bin at = s.at[0];
        hi = at.sum1;
        lo = at.count1 == K ? hi : at.sum0;
        if (lo != hi) collect(at.bin, at.bin);
    }
    const bool exact_k = lo == hi;
    const uint64_t sum_k = hi;
    // ... the number kept ...
    const uint32_t most = st.m > 0.0 ? max(min(K, pass), 1u) : K;
    uint32_t kmin = most, kmax = most;
    int at_end = 0;
    if (st.p < 1.0) {
        at_end = bins(false, reach(st.p, lo), reach(st.p, hi));
        kmin = min(most, s.at[0].count0 + 1);
        kmax = min(most, s.at[at_end].count1);
        collect(s.at[0].bin, s.at[at_end].bin);
    }
    // ... their weight (the bins just found, unless another limit cuts in) ...
    bool exact_end = true;
    if (kmin == live) {
        lo = hi = total;
    } else {
        if (kmax == most) at_end = bins(true, kmin, kmax);
        hi = s.at[at_end].sum1;
        exact_end = kmin == kmax && s.at[0].count1 == kmin;
        lo = exact_end ? hi : s.at[0].sum0;
        if (!exact_end) collect(s.at[0].bin, s.at[at_end].bin);
    }
    const uint64_t sum_end = hi;
    // ... and the token.
    auto past = [&](uint64_t end) { return min(below(u, end) + 1, end); };
    const int e = bins(false, past(lo), past(hi));
    collect(s.at[0].bin, s.at[e].bin);
    __syncthreads();

    // how many bins and candidates that makes
    const uint32_t flags = s.d.flag[tid * kBinsPer / 32] >> (tid * kBinsPer % 32);
    uint32_t f = 0, n = 0;
    if (flags & ((1u << kBinsPer) - 1)) {
#pragma unroll
        for (int i = 0; i < kBinsPer; ++i)
            if (flags >> i & 1 && cnt[i]) f += cnt[i], ++n;
    }
    uint64_t slots = n;
    uint32_t fi = f;
    uint32_t M;
    uint64_t nslot;
    block_scan(fi, slots, M, nslot, s.wave_count, s.wave_sum);
    fi -= f;
    slots -= n;
    if (n) {
        uint32_t ci = c;
        uint64_t xi = x;
#pragma unroll
        for (int i = 0; i < kBinsPer; ++i) {
            if (flags >> i & 1 && cnt[i]) {
                if (slots < kMaxSlots) s.d.slot[slots] = Slot{xi, ci, fi, tid * kBinsPer + i};
                fi += cnt[i];
                ++slots;
            }
            ci += cnt[i];
            xi += sum[i];
        }
    }
    if (tid == 0) s.base = 0;
    __syncthreads();
    if (M > kCollect || nslot > kMaxSlots) {  // (the same in every workgroup of the row)
        Result r;
        int how = 2;
        if (nslot <= kTies)
            how = draw_ties(row, weights, bin_map, st, u, Borders{K, most, exact_k, exact_end, sum_k, sum_end}, (int)nslot,
                            len, ws, s, r);
        else if (blockIdx.x != 0)
            return;
        if (how == 0) return;
        if (how == 2) r = draw_by_digits(row, weights, st, u, live, total, pass, s.digits);
        if (tid == 0) put(a, b, r);
        return;
    }

    // collect: this part's in LDS, then all parts' in the workspace
    const int64_t i0 = blockIdx.x * len;
    row.groups(i0, min(len, a.n - i0), [&](const float *l, int32_t id, auto count) {
        constexpr int N = decltype(count)::value;
        uint32_t hit = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int bin = bin_map.of(l[e]);
            hit |= (s.d.flag[bin / 32] >> (bin % 32) & (uint32_t)candidate(l[e])) << e;
        }
        if (hit)
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (hit >> e & 1) s.d.key[atomicAdd(&s.base, 1u)] = make_key(l[e], id + e);
    });
    __syncthreads();
    if (S > 1) {
        const uint32_t mine = s.base;
        if (tid == 0) s.last = atomicAdd(ws.collected, mine);
        __syncthreads();
        // Stores and loads at the device's point of coherence: no cache is
        // written back for them (with fences, which do that, the kernel took
        // 46 us for a row of 262144).  A store is there once it is counted
        // down, so that the workgroup that counts last sees all of them.
        for (uint32_t i = tid; i < mine; i += kRowThreads)
            __hip_atomic_store(&ws.key[s.last + i], s.d.key[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) s.last = __hip_atomic_fetch_add(ws.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (s.last != (uint32_t)S - 1) return;
        for (uint32_t i = tid; i < M; i += kRowThreads)
            s.d.key[i] = __hip_atomic_load(&ws.key[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
    }

    // their order, and their sums: a candidate's is that of the bins before
    // its own and of those before it in its own
    int P = 64;
    while (P < (int)M) P <<= 1;
    for (int i = (int)M + tid; i < P; i += kRowThreads) s.d.key[i] = 0;
    __syncthreads();
    // Waves without a candidate end here: a barrier waits for the others only,
    // and the sooner the fewer they are.
    const int waves = min(P / kLanes, kRowWaves);
    if (tid >= waves * kLanes) return;
    if (P <= kRowThreads) sort_distinct(s.d.key, P);
    else sort_row(s.d.key, P);
    uint64_t own[kCollect / kRowThreads];
    int64_t rank[kCollect / kRowThreads];
    uint64_t base = 0;
#pragma unroll
    for (int h = 0; h < kCollect / kRowThreads; ++h) {
        const int i = h * kRowThreads + tid;
        if (h * kRowThreads >= P) break;
        const uint64_t w = wave_scan<uint64_t>(i < (int)M ? weights.units(key_logit(s.d.key[i])) : 0ull);
        wave_total(w, s.wave_sum);
        __syncthreads();
        const auto sums = after_waves(w, s.wave_sum, waves);
        s.d.sum[i] = base + sums.upto;
        base += sums.total;
        __syncthreads();
    }
#pragma unroll
    for (int h = 0; h < kCollect / kRowThreads; ++h) {
        const int i = h * kRowThreads + tid;
        own[h] = ~0ull;
        rank[h] = INT64_MAX;
        if (i >= (int)M) continue;
        int lo = 0, hi = (int)nslot - 1;  // its bin: the last slot that begins at or before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (s.d.slot[mid].first <= (uint32_t)i) lo = mid;
            else hi = mid - 1;
        }
        const Slot at = s.d.slot[lo];
        own[h] = at.base + s.d.sum[i] - (at.first ? s.d.sum[at.first - 1] : 0ull);
        rank[h] = (int64_t)at.rank + i - at.first + 1;
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < kCollect / kRowThreads; ++h) s.d.sum[h * kRowThreads + tid] = own[h];
    // the first of the collected candidates with that rank, or sum
    auto first = [&](bool by_rank, uint64_t v) {
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kCollect / kRowThreads; ++h) {
            const int i = h * kRowThreads + tid;
            if (i >= (int)M) continue;
            const bool hit = by_rank ? rank[h] == (int64_t)v : own[h] >= v && (i == 0 || s.d.sum[i - 1] < v);
            if (hit) s.found_key = s.d.key[i], s.found_sum = own[h], s.found_rank = rank[h];
        }
        __syncthreads();
    };
    uint64_t ck = sum_k;
    if (!exact_k) {
        first(true, K);
        ck = s.found_sum;
    }
    int64_t kept = most;
    if (st.p < 1.0) {
        first(false, reach(st.p, ck));
        kept = min(kept, s.found_rank);
    }
    uint64_t end = sum_end;
    if (!exact_end) {
        first(true, kept);
        end = s.found_sum;
    }
    first(false, past(end));
    if (tid == 0) put(a, b, drawn(weights, s.found_key, end, kept));
}

vie_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

// Parts of a row: one workgroup a CU (64 rows of 151936 bf16: 46 us so, 69
// with two, 57 with half of one), of 4096 candidates at least (one row of
// 262144 fp32 in parts of 2048: 30.5 us, of 4096: 27.1, of 8192: 27.7, of
// 16384: 31.2; of 50000: 22.6, 23.4, 24.5 and 28.1).
static int parts_of(int64_t V, int B)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>({(V + 4095) / 4096, 256 / B, kMaxParts}));
}
// A workgroup a row in one kernel, or three kernels.  In us, one and three:
//                  fp32                                bf16
//     1 row    of  8192 16.0 19.9, of 16384 19.5 19.7    16384 18.3 20.7
//              of 24000 24.4 20.7, of 50257 37.8 21.3    24000 21.8 20.7
//     8 rows   of 20000 22.9 21.8, of 32000 28.8 22.5    20000 20.1 22.1, 32000 25.5 23.0
//    64 rows   of 32000 30.1 35.0, of 50257 40.5 36.2    50257 33.5 37.4, 80000 46.3 40.5
//   128 rows   of 60000 45.7 46.0, of 80000 57.0 53.3    80000 46.2 47.0, 128256 66.6 59.8
static bool one_kernel(int64_t V, int B, bool bf16)
{
    return parts_of(V, B) == 1 || V <= (bf16 ? 20480 + 512 * (int64_t)B : 16384 + 352 * (int64_t)B);
}

// Enough for either type, and for fewer rows, too: the most of them (of up to
// 128, which have parts) that take three kernels, of fp32.
size_t sample_rows_workspace_bytes(int64_t V, int B)
{
    const int64_t three = V > 16384 ? std::min<int64_t>({B, 128, (V - 1 - 16384) / 352}) : 0;
    return std::max((size_t)three * sizeof(RowSpace), B * sizeof(OneSpace));
}

vie_status launch_sample_lists(const SampleLaunch &a, hipStream_t s)
{
    int P = 64;
    while (P < a.n) P <<= 1;
    const size_t lds = (size_t)P * 16;
    // A wave needs no barrier (64 entries: 3.8 us with one wave, 4.0 with four;
    // 65: 4.4 and 4.1; 256: 5.9 and 4.4).
    if (a.n <= 64) sample_list_kernel<64><<<a.B, 64, lds, s>>>(a);
    else sample_list_kernel<256><<<a.B, 256, lds, s>>>(a);
    return launched("list sampling launch");
}

namespace {
template <bool BF16> vie_status rows_launch(const SampleLaunch &a, hipStream_t s)
{
    constexpr int kBinsLds = sizeof(BinLds<BF16>), kOneLds = sizeof(DrawLds) + sizeof(BinLds<BF16>);
    hipError_t e = hipFuncSetAttribute((const void *)rows_draw_kernel<BF16>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)sizeof(DrawLds));
    if (e == hipSuccess)
        e = hipFuncSetAttribute((const void *)rows_bins_kernel<BF16>, hipFuncAttributeMaxDynamicSharedMemorySize, kBinsLds);
    if (e == hipSuccess)
        e = hipFuncSetAttribute((const void *)rows_one_kernel<BF16>, hipFuncAttributeMaxDynamicSharedMemorySize, kOneLds);
    if (e != hipSuccess) return fail(VIE_EHIP, "row sampling: %s", hipGetErrorString(e));
    if (one_kernel(a.n, a.B, BF16)) {
        rows_one_kernel<BF16><<<dim3(1, a.B), kRowThreads, kOneLds, s>>>(a);
    } else {
        const int S = parts_of(a.n, a.B);
        const Parts parts{((a.n + S - 1) / S + 63) / 64 * 64, static_cast<RowSpace *>(a.ws)};
        const dim3 grid((unsigned)((a.n + parts.len - 1) / parts.len), (unsigned)a.B);
        rows_best_kernel<BF16><<<grid, kRowThreads, 0, s>>>(a, parts);
        rows_bins_kernel<BF16><<<grid, kRowThreads, kBinsLds, s>>>(a, parts);
        rows_draw_kernel<BF16><<<grid, kRowThreads, sizeof(DrawLds), s>>>(a, parts);
    }
    return launched("row sampling launch");
}
}  // namespace

vie_status launch_sample_rows(const SampleLaunch &a, hipStream_t s)
{
    return a.dtype == VIE_BF16 ? rows_launch<true>(a, s) : rows_launch<false>(a, s);
}

}  // namespace vie
