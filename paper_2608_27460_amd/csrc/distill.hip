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

#include <algorithm>
#include <cfloat>

#include "block.hpp"
#include "operators.hpp"

namespace vie {

namespace {

// Maximum and sum of exp2((s - m) c) of a set of logits.  The empty set has
// the lowest finite maximum, so that rows of -inf or of the lowest value make
// no NaN on the way: s - m is then 0 or -inf.
struct Part {
    float m, z;
};
__device__ __forceinline__ float term(float s, float m, float c) { return __builtin_amdgcn_exp2f((s - m) * c); }
__device__ __forceinline__ Part merge(Part a, Part b, float c)
{
    const float m = fmaxf(a.m, b.m);
    return {m, a.z * term(a.m, m, c) + b.z * term(b.m, m, c)};
}
template <int N> __device__ __forceinline__ void add(Part &p, const float *f, float c)
{
    float m = p.m;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, f[i]);
    float z = p.z * term(p.m, m, c);
#pragma unroll
    for (int i = 0; i < N; ++i) z += term(f[i], m, c);
    p = {m, z};
}
// The part of W lanes, in each of them.
template <int W> __device__ __forceinline__ Part wave_merge(Part p, float c)
{
    if constexpr (W > 1) {
        p = merge(p, Part{lane_xor_as(p.m, W / 2), lane_xor_as(p.z, W / 2)}, c);
        return wave_merge<W / 2>(p, c);
    }
    return p;
}
// The whole workgroup's part, in every thread; `tmp`: NT / 64 parts.
template <int NT> __device__ __forceinline__ Part block_merge(Part p, float c, Part *tmp)
{
    p = wave_merge<kLanes>(p, c);
    __syncthreads();
    if ((threadIdx.x & (kLanes - 1)) == 0) tmp[threadIdx.x / kLanes] = p;
    __syncthreads();
    // (lanes past the waves repeat them: the exchanges stay among NT / 64)
    return wave_merge<NT / kLanes>(tmp[threadIdx.x & (NT / kLanes - 1)], c);
}

// 16 bytes at any alignment of the elements
template <typename T> __device__ __forceinline__ word4 load_vec(const T *p)
{
    word4 w;
    __builtin_memcpy(&w, p, 16);
    return w;
}
typedef word4 any_word4 __attribute__((aligned(2)));
// The same past the caches' keeping: what is read for the last time, and
// gradients, which would push out rows still to be read again (a step of 2048
// rows of 128256 bf16: 294 us without, 267 with).
template <typename T> __device__ __forceinline__ word4 load_last(const T *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const any_word4 *>(p));
}
template <typename T> __device__ __forceinline__ void store_vec(T *p, word4 w)
{
    __builtin_nontemporal_store(w, reinterpret_cast<any_word4 *>(p));
}

// The teacher's list of a row, in LDS: 16 bytes an entry.  An entry counts if
// its id lies in [0, V) and its logit is not -inf; the others have id -1.
// Entry j belongs to thread j % NT in every step, so the steps need no
// barrier; its fp64 work is one entry at a time, whose registers the rows'
// kernels could not spare for more.
struct Entry {
    int32_t id;
    float t, at;  // the teacher's logit, the student's at that id
    float e;      // exp((t - top) / tau)
};
template <int NT> struct List {
    Entry *entry;
    int k;
    float top;
    double total;  // 0: nothing listed
    double inv_tau;

    static __device__ __forceinline__ Entry get(const int32_t *ids, const float *teacher, int j, int k, int64_t V)
    {
        Entry x{-1, 0.0f, 0.0f, 0.0f};
        if (j < k) {
            x.id = ids[j];
            x.t = teacher[j];
            if (x.id >= V || x.t == -__builtin_inff()) x.id = -1;
        }
        return x;
    }
    // `s` (of BF16 elements) nullptr: without the student's logits
    template <bool BF16>
    __device__ __forceinline__ void read(const int32_t *ids, const float *teacher, int64_t V, const typename Elem<BF16>::T *s)
    {
        for (int j = threadIdx.x; j < k; j += NT) {
            Entry x = get(ids, teacher, j, k, V);
            if (s && x.id >= 0) x.at = Elem<BF16>::get(s[x.id]);
            entry[j] = x;
        }
    }
    // the list's maximum and sum (the workgroup waits in here)
    __device__ __forceinline__ void sum(float tau, double *tmp)
    {
        inv_tau = 1.0 / (double)tau;
        float m = -FLT_MAX;
        for (int j = threadIdx.x; j < k; j += NT) {
            const float t = entry[j].t;
            if (entry[j].id >= 0) m = m != m || t != t ? m + t : fmaxf(m, t);
        }
        top = block_reduce<NT>(m, reinterpret_cast<float *>(tmp),
                               [](float a, float b) { return a != a || b != b ? a + b : fmaxf(a, b); });
        double z = 0.0;
#pragma unroll 1
        for (int j = threadIdx.x; j < k; j += NT) {
            const double e = entry[j].id >= 0 ? exp(x(j)) : 0.0;
            entry[j].e = (float)e;
            z += e;
        }
        total = block_reduce<NT>(z, tmp + NT / kLanes, [](double a, double b) { return a + b; });
    }
    __device__ __forceinline__ double x(int j) const { return ((double)entry[j].t - (double)top) * inv_tau; }
    __device__ __forceinline__ double p(int j) const { return (double)entry[j].e / total; }

    // The row's loss from its part and the student's logits, in every thread.
    __device__ __forceinline__ float loss(Part r, float tau, double *tmp) const
    {
        double sum = 0.0;
        if ((int)threadIdx.x < k) {
            // log p - log q: the logarithms of the two sums together
            const double log_ratio = log((double)r.z / total);
#pragma unroll 1
            for (int j = threadIdx.x; j < k; j += NT) {
                if (entry[j].id < 0 || entry[j].e == 0.0f) continue;
                sum += p(j) * (x(j) - ((double)entry[j].at - (double)r.m) * inv_tau + log_ratio);
            }
        }
        sum = block_reduce<NT>(sum, tmp, [](double a, double b) { return a + b; });
        return total == 0.0 ? 0.0f : (float)((double)tau * (double)tau * sum);
    }
};

// The list's probabilities by id, for the ids of [v0, v0 + n): a hash table
// of 2^bits places, at least twice the entries, and a bit for every 16 bytes
// of logits that hold a listed id.
constexpr int kMapWords = 1024;  // for up to 32768 groups of 16 bytes
struct Table {
    uint32_t *map;
    int32_t *id;
    float *prob;
    int bits;
    __device__ __forceinline__ Table(char *lds, int bits)
        : map(reinterpret_cast<uint32_t *>(lds)), id(reinterpret_cast<int32_t *>(lds + kMapWords * 4)),
          prob(reinterpret_cast<float *>(lds + kMapWords * 4 + (4 << bits))), bits(bits)
    {
    }
    __device__ __forceinline__ uint32_t place(int32_t v) const { return (uint32_t)v * 2654435761u >> (32 - bits); }
    template <int NT> __device__ __forceinline__ void clear()
    {
        for (int i = threadIdx.x; i < kMapWords; i += NT) map[i] = 0;
        for (int i = threadIdx.x; i < 1 << bits; i += NT) id[i] = -1;
    }
    // (between clear and fill the workgroup waits; in fill it does so itself)
    template <int NT> __device__ __forceinline__ void fill(const List<NT> &l, int64_t v0, int64_t n, int vec)
    {
        bool twice = false;
#pragma unroll 1
        for (int j = threadIdx.x; j < l.k; j += NT) {
            const int32_t v = l.entry[j].id;
            const int64_t off = (int64_t)v - v0;
            if (v < 0 || off < 0 || off >= n) continue;
            uint32_t h = place(v);
            int32_t was;
            while ((was = atomicCAS(&id[h], -1, v)) != -1 && was != v) h = (h + 1) & ((1u << bits) - 1);
            twice |= was == v;
            prob[h] = (float)l.p(j);
            const uint32_t g = (uint32_t)off / vec;
            atomicOr(&map[g / 32], 1u << (g % 32));
        }
        if (!__syncthreads_or(twice)) return;
        // Ids listed more than once (no list of a head's): their first entry
        // adds up all of them, in the list's order.
#pragma unroll 1
        for (int j = threadIdx.x; j < l.k; j += NT) {
            const int32_t v = l.entry[j].id;
            const int64_t off = (int64_t)v - v0;
            if (v < 0 || off < 0 || off >= n) continue;
            bool first = true;
            double p = 0.0;
            for (int e = 0; e < l.k; ++e) {
                if (l.entry[e].id != v) continue;
                first &= e >= j;
                p += l.p(e);
            }
            if (!first) continue;
            uint32_t h = place(v);
            while (id[h] != v) h = (h + 1) & ((1u << bits) - 1);
            prob[h] = (float)p;
        }
        __syncthreads();
    }
    __device__ __forceinline__ bool any(uint32_t group) const { return map[group / 32] >> (group % 32) & 1; }
    __device__ __forceinline__ float p(int32_t v) const
    {
        for (uint32_t h = place(v);; h = (h + 1) & ((1u << bits) - 1)) {
            if (id[h] == v) return prob[h];
            if (id[h] == -1) return 0.0f;
        }
    }
};
__host__ __device__ inline int table_bits(int k)
{
    int b = 6;
    while ((1 << b) < 2 * k) ++b;
    return b;
}
__host__ __device__ inline size_t list_lds(int k) { return (size_t)k * sizeof(Entry); }
inline size_t table_lds(int k) { return kMapWords * 4 + ((size_t)8 << table_bits(k)) + list_lds(k); }  // and the list

// The gradient of a row, value by value: f (q - p) with q = term / Z; of a row that lists
// nothing 0, whatever its logits.
struct Slope {
    Part r;
    float c, f, f_z;  // f / Z
    bool none;
    __device__ __forceinline__ Slope(Part r, float c, float f, bool none) : r(r), c(c), f(f), f_z(f / r.z), none(none) {}
    __device__ __forceinline__ float at(float s) const { return term(s, r.m, c) * f_z; }
    __device__ __forceinline__ float at(float s, float p) const { return fmaf(-f, p, at(s)); }
};
// Element e of 16 bytes.
template <bool BF16> __device__ __forceinline__ float element(word4 w, int e)
{
    const int k = BF16 ? e >> 1 : e;
    const uint32_t word = k == 0 ? w.x : k == 1 ? w.y : k == 2 ? w.z : w.w;
    return BF16 ? __uint_as_float(e & 1 ? word & 0xFFFF0000u : word << 16) : __uint_as_float(word);
}
// The gradient of a group of 16 bytes, from v on; the listed ids' values are
// written over by the same thread.
template <bool BF16>
__device__ __forceinline__ void put_group(const Slope &g, const Table &t, uint32_t group, int32_t v, word4 w,
                                          typename Elem<BF16>::T *dst)
{
    typedef Elem<BF16> E;
    if (g.none) {
        store_vec(dst, word4{0, 0, 0, 0});
        return;
    }
    float x[E::kVec];
    E::unpack(w, x);
#pragma unroll
    for (int e = 0; e < E::kVec; ++e) x[e] = g.at(x[e]);
    store_vec(dst, E::pack(x));
    if (t.any(group)) {
#pragma unroll 1
        for (int e = 0; e < E::kVec; ++e) {
            const float p = t.p(v + e);
            if (p != 0.0f) dst[e] = E::put(g.at(element<BF16>(w, e), p));
        }
    }
}
template <bool BF16>
__device__ __forceinline__ void put_one(const Slope &g, const Table &t, uint32_t group, int32_t v, float x,
                                        typename Elem<BF16>::T *dst)
{
    *dst = Elem<BF16>::put(g.none ? 0.0f : g.at(x, t.any(group) ? t.p(v) : 0.0f));
}

__device__ __forceinline__ float exponent_scale(float tau) { return (float)(1.4426950408889634 / (double)tau); }

// ---------------------------------------------------------------------------
// forward and backward apart: rows in parts, streamed
// ---------------------------------------------------------------------------

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kLanes;
constexpr int kFlight = 4;                       // 16-byte loads of a thread in flight
constexpr int kMaxParts = 64;                    // of a row
constexpr int kMapGroups = 32 * kMapWords;       // 16-byte groups that a map has bits for

template <bool BF16> __global__ __launch_bounds__(kThreads) void distill_forward_kernel(DistillLaunch a, int64_t len)
{
    typedef Elem<BF16> E;
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * kWaves];
    __shared__ Part s_part[kWaves];
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= a.N) return;
    const int tid = threadIdx.x;
    const typename E::T *s = static_cast<const typename E::T *>(a.logits) + row * a.ld;
    const float c = exponent_scale(a.tau);
    const int64_t v0 = blockIdx.x * len, n = min(len, a.V - v0), groups = n / E::kVec;
    Part p{-FLT_MAX, 0.0f};
    const typename E::T *src = s + v0;
    int64_t i = tid;
    for (; i + (kFlight - 1) * kThreads < groups; i += kFlight * kThreads) {
        word4 w[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_vec(src + (i + u * kThreads) * E::kVec);
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            float f[E::kVec];
            E::unpack(w[u], f);
            add<E::kVec>(p, f, c);
        }
    }
    for (; i < groups; i += kThreads) {
        float f[E::kVec];
        E::unpack(load_vec(src + i * E::kVec), f);
        add<E::kVec>(p, f, c);
    }
    if (groups * E::kVec + tid < n) {
        const float f = E::get(src[groups * E::kVec + tid]);
        add<1>(p, &f, c);
    }
    p = block_merge<kThreads>(p, c, s_part);
    if (gridDim.x > 1) {
        if (tid == 0) static_cast<Part *>(a.ws)[row * kMaxParts + blockIdx.x] = p;
        return;
    }
    List<kThreads> l{reinterpret_cast<Entry *>(smem), a.k};
    l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V, s);
    l.sum(a.tau, s_tmp);
    const float loss = l.loss(p, a.tau, s_tmp);
    if (tid == 0) {
        a.loss[row] = loss;
        a.stats[2 * row] = p.m;
        a.stats[2 * row + 1] = p.z;
    }
}

// The losses of rows that were taken in parts.
template <bool BF16> __global__ __launch_bounds__(kThreads) void distill_join_kernel(DistillLaunch a, int parts)
{
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * kWaves];
    const int64_t row = blockIdx.x;
    const float c = exponent_scale(a.tau);
    List<kThreads> l{reinterpret_cast<Entry *>(smem), a.k};
    l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V,
                          static_cast<const typename Elem<BF16>::T *>(a.logits) + row * a.ld);
    const int lane = threadIdx.x & (kLanes - 1);
    Part p{-FLT_MAX, 0.0f};
    if (lane < parts) p = static_cast<const Part *>(a.ws)[row * kMaxParts + lane];
    p = wave_merge<kLanes>(p, c);
    l.sum(a.tau, s_tmp);
    const float loss = l.loss(p, a.tau, s_tmp);
    if (threadIdx.x == 0) {
        a.loss[row] = loss;
        a.stats[2 * row] = p.m;
        a.stats[2 * row + 1] = p.z;
    }
}

template <bool BF16> __global__ __launch_bounds__(kThreads) void distill_backward_kernel(DistillLaunch a, int64_t len)
{
    typedef Elem<BF16> E;
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * kWaves];
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= a.N) return;
    const int tid = threadIdx.x;
    const int64_t v0 = blockIdx.x * len, n = min(len, a.V - v0), groups = n / E::kVec;
    const typename E::T *src = static_cast<const typename E::T *>(a.logits) + row * a.ld + v0;
    typename E::T *dst = static_cast<typename E::T *>(a.grad) + row * a.grad_ld + v0;
    List<kThreads> l{reinterpret_cast<Entry *>(smem), a.k};
    Table t(smem + list_lds(a.k), table_bits(a.k));
    t.clear<kThreads>();
    l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V, nullptr);
    l.sum(a.tau, s_tmp);  // (the workgroup waits in here)
    t.fill(l, v0, n, E::kVec);
    const float g = a.weight * (a.gloss ? a.gloss[row] : 1.0f);
    const Slope sl({a.stats[2 * row], a.stats[2 * row + 1]}, exponent_scale(a.tau), g * a.tau, l.total == 0.0);
    __syncthreads();
    int64_t i = tid;
    for (; i + (kFlight - 1) * kThreads < groups; i += kFlight * kThreads) {
        word4 w[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_last(src + (i + u * kThreads) * E::kVec);
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const int64_t at = i + u * kThreads;
            put_group<BF16>(sl, t, (uint32_t)at, (int32_t)(v0 + at * E::kVec), w[u], dst + at * E::kVec);
        }
    }
    for (; i < groups; i += kThreads) {
        put_group<BF16>(sl, t, (uint32_t)i, (int32_t)(v0 + i * E::kVec), load_vec(src + i * E::kVec), dst + i * E::kVec);
    }
    if (groups * E::kVec + tid < n) {
        const int64_t at = groups * E::kVec + tid;
        put_one<BF16>(sl, t, (uint32_t)groups, (int32_t)(v0 + at), E::get(src[at]), dst + at);
    }
}

// ---------------------------------------------------------------------------
// both at once
// ---------------------------------------------------------------------------
//
// A workgroup of 1024 threads, two of them a CU, takes a row: its part first,
// then its gradient, from the row's end to its beginning, so that the second
// reading finds what the caches hold of the first.

constexpr int kBothThreads = 1024;
constexpr int kBothWaves = kBothThreads / kLanes;

template <bool BF16>
__global__ __launch_bounds__(kBothThreads) __attribute__((amdgpu_waves_per_eu(8, 8))) void distill_both_kernel(DistillLaunch a)
{
    typedef Elem<BF16> E;
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * kBothWaves];
    __shared__ Part s_part[kBothWaves];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const float c = exponent_scale(a.tau);
    const typename E::T *src = static_cast<const typename E::T *>(a.logits) + row * a.ld;
    typename E::T *dst = static_cast<typename E::T *>(a.grad) + row * a.grad_ld;
    const int groups = (int)(a.V / E::kVec), rest = (int)(a.V - (int64_t)groups * E::kVec);
    List<kBothThreads> l{reinterpret_cast<Entry *>(smem), a.k};
    Table t(smem + list_lds(a.k), table_bits(a.k));
    // (the first loads of either pass are on their way while the list is
    // worked on)
    const int step = kFlight * kBothThreads;
    word4 w[kFlight];
    auto load_up = [&](int i) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_vec(src + (int64_t)min(i + u * kBothThreads, groups - 1) * E::kVec);
    };
    auto load_down = [&](int i) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_last(src + (int64_t)max(i - u * kBothThreads, 0) * E::kVec);
    };
    if (groups) load_up(tid);
    t.clear<kBothThreads>();
    l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V, src);
    Part p{-FLT_MAX, 0.0f};
    for (int i = tid; i < groups; i += step) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            float f[E::kVec];
            E::unpack(w[u], f);
            if (i + u * kBothThreads < groups) add<E::kVec>(p, f, c);
        }
        if (i + step < groups) load_up(i + step);
    }
    const int down = groups - 1 - tid;
    if (groups) load_down(down);
    const int64_t last = (int64_t)groups * E::kVec + tid;
    float tail = 0.0f;
    if (tid < rest) {
        tail = E::get(src[last]);
        add<1>(p, &tail, c);
    }
    l.sum(a.tau, s_tmp);  // (the workgroup waits in here)
    t.fill(l, 0, a.V, E::kVec);
    p = block_merge<kBothThreads>(p, c, s_part);
    const float loss = l.loss(p, a.tau, s_tmp);
    if (tid == 0) a.loss[row] = loss;
    const float g = a.weight * (a.gloss ? a.gloss[row] : 1.0f);
    const Slope sl(p, c, g * a.tau, l.total == 0.0);
    if (tid < rest) put_one<BF16>(sl, t, (uint32_t)groups, (int32_t)last, tail, dst + last);
    for (int i = down; i >= 0; i -= step) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const int at = i - u * kBothThreads;
            if (at >= 0) put_group<BF16>(sl, t, (uint32_t)at, at * E::kVec, w[u], dst + (int64_t)at * E::kVec);
        }
        if (i - step >= 0) load_down(i - step);
    }
}

vie_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// LDS above 64 KB has to be asked for.
vie_status allow_lds(const void *kernel, size_t lds)
{
    if (lds <= 64 * 1024) return VIE_OK;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "distillation: %s", hipGetErrorString(e));
}

// Rows in parts: as many as give the device two workgroups a CU, of `least`
// logits at least, and as many as a part's map of groups asks for.
struct Split {
    int parts;
    int64_t len;
    dim3 grid;
};
Split split_rows(const DistillLaunch &a, int64_t least, int most_groups)
{
    const int vec = a.dtype == VIE_BF16 ? 8 : 4;
    int64_t parts = std::min<int64_t>((a.V + least - 1) / least, 512 / a.N);
    parts = std::max<int64_t>(parts, (a.V / vec + most_groups - 1) / most_groups);
    parts = std::max<int64_t>(parts, 1);
    Split s;
    s.len = ((a.V + parts - 1) / parts + 63) / 64 * 64;
    s.parts = (int)((a.V + s.len - 1) / s.len);
    s.grid = dim3((unsigned)s.parts, (unsigned)std::min(a.N, 32768), (unsigned)((a.N + 32767) / 32768));
    return s;
}

// The rows' parts (more than 256 rows have none: split_rows) and, in a step
// that keeps none for the caller, their stats.
size_t parts_bytes(int N) { return N > 256 ? 0 : (size_t)N * kMaxParts * sizeof(Part); }

template <bool BF16> vie_status forward(const DistillLaunch &a, hipStream_t s)
{
    // Joining parts is a launch more, in which a workgroup reads some 200 KB
    // of a row (one row of 65536 bf16: 12 us whole, 14 in parts; of 262144:
    // 18 and 15).
    const bool whole = a.V * elem_bytes(a.dtype) <= 192 * 1024;
    Split sp = split_rows(a, whole ? a.V : 32768, INT32_MAX);
    if (sp.parts > kMaxParts) {
        sp.len = ((a.V + kMaxParts - 1) / kMaxParts + 63) / 64 * 64;
        sp.parts = (int)((a.V + sp.len - 1) / sp.len);
        sp.grid.x = (unsigned)sp.parts;
    }
    distill_forward_kernel<BF16><<<sp.grid, kThreads, list_lds(a.k), s>>>(a, sp.len);
    if (sp.parts > 1) distill_join_kernel<BF16><<<a.N, kThreads, list_lds(a.k), s>>>(a, sp.parts);
    return launched("distillation launch");
}

template <bool BF16> vie_status backward(const DistillLaunch &a, hipStream_t s)
{
    // (parts of 64 KB: more workgroups than fit at once, whose ends and lists
    // others stream over; 2048 rows of 128256 bf16: 237 us as whole rows, 209)
    const Split sp = split_rows(a, 8192, 4096);
    if (vie_status e = allow_lds((const void *)distill_backward_kernel<BF16>, table_lds(a.k))) return e;
    distill_backward_kernel<BF16><<<sp.grid, kThreads, table_lds(a.k), s>>>(a, sp.len);
    return launched("distillation gradient launch");
}

template <bool BF16> vie_status step(const DistillLaunch &a, hipStream_t s)
{
    // One kernel where its workgroups fill half of the CUs, or where the row
    // is read in less time than another launch takes (8 rows of 8000 bf16: 15
    // us so, 22 as two kernels; of 32000: 21 and 16).
    const bool one = a.N >= 128 || a.V * elem_bytes(a.dtype) <= 32 * 1024;
    if (one && a.V / Elem<BF16>::kVec < kMapGroups) {
        if (vie_status e = allow_lds((const void *)distill_both_kernel<BF16>, table_lds(a.k))) return e;
        distill_both_kernel<BF16><<<a.N, kBothThreads, table_lds(a.k), s>>>(a);
        return launched("distillation step launch");
    }
    DistillLaunch b = a;
    b.stats = reinterpret_cast<float *>(static_cast<char *>(a.ws) + parts_bytes(a.N));
    if (vie_status e = forward<BF16>(b, s)) return e;
    return backward<BF16>(b, s);
}

}  // namespace

size_t distill_workspace_bytes(int64_t, int N) { return parts_bytes(N) + (size_t)N * 8; }

vie_status launch_distill(const DistillLaunch &a, hipStream_t s)
{
    return a.dtype == VIE_BF16 ? forward<true>(a, s) : forward<false>(a, s);
}

vie_status launch_distill_grad(const DistillLaunch &a, hipStream_t s)
{
    return a.dtype == VIE_BF16 ? backward<true>(a, s) : backward<false>(a, s);
}

vie_status launch_distill_step(const DistillLaunch &a, hipStream_t s)
{
    return a.dtype == VIE_BF16 ? step<true>(a, s) : step<false>(a, s);
}

}  // namespace vie
