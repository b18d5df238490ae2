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
// would be relative to m.  Sums are fp32 over at most 512 terms of a thread,
// fp64 over those, and merged pairwise among the threads; the list's sums are
// fp64.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <type_traits>

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
// (Contracted to one product and a multiply-add, it would round differently
// in the two lanes that exchange their parts, and the threads of a row would
// end with different sums.)
__device__ __forceinline__ Part merge(Part a, Part b, float c)
{
#pragma clang fp contract(off)
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
// A long row's sum, in 64 bits: what a thread (or a wave) has folded into it
// after every kFold terms.
constexpr int kFold = 512;
struct Folded {
    float m;
    double z;
};
__device__ __forceinline__ void fold(Folded &all, Part &p, float c)
{
    const float m = fmaxf(all.m, p.m);
    all = {m, all.z * (double)term(all.m, m, c) + (double)(p.z * term(p.m, m, c))};
    p = {m, 0.0f};
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
// kernels could not spare for more.  NT = 64: the workgroup's first wave
// works on the list, while the others stream the row (4096 rows of 8000 bf16
// with 50 entries, forward: 22.5 us, 30 where all waves met in the list's
// reductions).
struct Entry {
    int32_t id;
    float t, at;  // the teacher's logit, the student's at that id
    float e;      // exp((t - top) / tau)
};
template <int NT> __device__ __forceinline__ void list_barrier()
{
    if constexpr (NT > kLanes) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}
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
    // with the student's logits s (of BF16 elements) of the ids in [v0, v0 + n)
    template <bool BF16>
    __device__ __forceinline__ void read(const int32_t *ids, const float *teacher, int64_t V, const typename Elem<BF16>::T *s,
                                         int64_t v0, int64_t n)
    {
        for (int j = threadIdx.x; j < k; j += NT) {
            Entry x = get(ids, teacher, j, k, V);
            if (in(x.id, v0, n)) x.at = Elem<BF16>::get(s[x.id]);
            entry[j] = x;
        }
    }
    static __device__ __forceinline__ bool in(int32_t id, int64_t v0, int64_t n) { return id >= 0 && id >= v0 && id - v0 < n; }
    // the list's maximum and sum
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
        list_barrier<NT>();
    }
    __device__ __forceinline__ double x(int j) const { return ((double)entry[j].t - (double)top) * inv_tau; }
    __device__ __forceinline__ double p(int j) const { return (double)entry[j].e / total; }

    // The row's loss from its part and the student's logits.
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

    // Whether an id of [v0, v0 + n) is listed more than once (the list of a
    // head has no such id).  `place`: 2^bits words of LDS, at least twice the
    // entries, a hash table.
    __device__ __forceinline__ void clear(int32_t *place, int bits) const
    {
        for (int i = threadIdx.x; i < 1 << bits; i += NT) place[i] = -1;
    }
    __device__ __forceinline__ bool twice(int32_t *place, int bits, int64_t v0, int64_t n) const
    {
        bool found = false;
#pragma unroll 1
        for (int j = threadIdx.x; j < k; j += NT) {
            if (!in(entry[j].id, v0, n)) continue;
            const int32_t v = entry[j].id;
            uint32_t h = (uint32_t)v * 2654435761u >> (32 - bits);
            int32_t was;
            while ((was = atomicCAS(&place[h], -1, v)) != -1 && was != v) h = (h + 1) & ((1u << bits) - 1);
            found |= was == v;
        }
        if constexpr (NT > kLanes) return __syncthreads_or(found);
        else return __any(found);
    }
    // The gradient at the listed ids of [v0, v0 + n), in grad[id - v0]; of an
    // id listed more than once its first entry takes the sum, in the list's
    // order.
    template <bool BF16, typename G>
    __device__ __forceinline__ void put(const G &g, int64_t v0, int64_t n, bool twice, typename Elem<BF16>::T *grad) const
    {
#pragma unroll 1
        for (int j = threadIdx.x; j < k; j += NT) {
            if (!in(entry[j].id, v0, n)) continue;
            const int32_t v = entry[j].id;
            double sum = p(j);
            bool first = true;
            if (twice) {
                sum = 0.0;
                for (int e = 0; e < k; ++e) {
                    if (entry[e].id != v) continue;
                    first &= e >= j;
                    sum += p(e);
                }
            }
            if (first && (float)sum != 0.0f) grad[v - v0] = Elem<BF16>::put(g.at(entry[j].at, (float)sum));
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
inline size_t table_lds(int k) { return list_lds(k) + ((size_t)4 << table_bits(k)); }  // and the list


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
// The gradient of a group of 16 bytes as if nothing in it were listed.
template <bool BF16> __device__ __forceinline__ void put_group(const Slope &g, word4 w, typename Elem<BF16>::T *dst)
{
    typedef Elem<BF16> E;
    float x[E::kVec];
    E::unpack(w, x);
#pragma unroll
    for (int e = 0; e < E::kVec; ++e) x[e] = g.at(x[e]);
    store_vec(dst, g.none ? word4{0, 0, 0, 0} : E::pack(x));
}
template <bool BF16> __device__ __forceinline__ void put_one(const Slope &g, float x, typename Elem<BF16>::T *dst)
{
    *dst = Elem<BF16>::put(g.none ? 0.0f : g.at(x));
}
// Until the workgroup's stores are done: those after it, from any of its
// threads, come after them.  The listed ids' gradients are stored so, over
// the others; looking each value up while it is stored (in a table of the
// listed ids, behind a bit for every 16 bytes that hold one) took 73 us
// instead of 30 for the gradients of 4096 rows of 8000 bf16 with 50 entries,
// because nearly every wave has one to look up.
__device__ __forceinline__ void after_stores()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

__device__ __forceinline__ float exponent_scale(float tau) { return (float)(1.4426950408889634 / (double)tau); }

// ---------------------------------------------------------------------------
// forward and backward apart: rows in parts, streamed
// ---------------------------------------------------------------------------
//
// Both are bound by memory where there are rows enough: 2048 rows of 128256
// bf16 forward in 98 us (5.4 TB/s read), backward in 177 (5.9 TB/s read and
// written).  Few rows are bound by one workgroup's way through a row: 48 rows
// of 32768 fp32 forward in 6 us, of which a launch is 3.5.

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kLanes;
constexpr int kFlight = 4;                       // 16-byte loads of a thread in flight
constexpr int kMaxParts = 64;                    // of a row
constexpr int kBackGroups = 4096;                // 16-byte groups of a part of the backward pass

// LONG: parts of more than kFold terms a thread (folding in every kernel took
// 0.2 us of 48 rows of 32768 fp32, and 0.8 of 600 rows of 128256 bf16).
template <bool BF16, int LT, bool LONG>
__global__ __launch_bounds__(kThreads) void distill_forward_kernel(DistillLaunch a, int64_t len)
{
    typedef Elem<BF16> E;
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * kWaves];
    __shared__ Part s_part[kWaves];
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= a.N) return;
    const int tid = threadIdx.x;
    const bool lists = gridDim.x == 1 && tid < LT;
    const typename E::T *s = static_cast<const typename E::T *>(a.logits) + row * a.ld;
    const float c = exponent_scale(a.tau);
    const int64_t v0 = blockIdx.x * len, n = min(len, a.V - v0), groups = n / E::kVec;
    List<LT> l{reinterpret_cast<Entry *>(smem), a.k};
    Part p{-FLT_MAX, 0.0f};
    const typename E::T *src = s + v0;
    const int64_t first = tid;
    word4 w[kFlight];
    auto load = [&](int64_t i) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_vec(src + (i + u * kThreads) * E::kVec);
    };
    // whether a thread has kFlight groups from i on
    auto full = [&](int64_t i) { return i + (kFlight - 1) * kThreads < groups; };
    if (full(first)) load(first);
    if (lists) l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V, s, 0, a.V);
    int64_t i = first;
    [[maybe_unused]] Folded all{-FLT_MAX, 0.0};
    for (int turn = 1; full(i); ++turn) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            float f[E::kVec];
            E::unpack(w[u], f);
            add<E::kVec>(p, f, c);
        }
        i += kFlight * kThreads;
        if (full(i)) load(i);
        if constexpr (LONG)
            if (turn % (kFold / (kFlight * E::kVec)) == 0) fold(all, p, c);
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
    if constexpr (LONG) {
        fold(all, p, c);
        p.z = (float)all.z;
    }
    if (lists) l.sum(a.tau, s_tmp);
    p = block_merge<kThreads>(p, c, s_part);
    if (gridDim.x > 1) {
        if (tid == 0) static_cast<Part *>(a.ws)[row * kMaxParts + blockIdx.x] = p;
        return;
    }
    if (!lists) return;
    const float loss = l.loss(p, a.tau, s_tmp);
    if (tid == 0) {
        a.loss[row] = loss;
        a.stats[2 * row] = p.m;
        a.stats[2 * row + 1] = p.z;
    }
}

// The losses of rows that were taken in parts.
template <bool BF16, int LT> __global__ __launch_bounds__(LT) void distill_join_kernel(DistillLaunch a, int parts)
{
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * LT / kLanes];
    const int64_t row = blockIdx.x;
    const float c = exponent_scale(a.tau);
    List<LT> l{reinterpret_cast<Entry *>(smem), a.k};
    l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V,
                          static_cast<const typename Elem<BF16>::T *>(a.logits) + row * a.ld, 0, a.V);
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

template <bool BF16, int LT>
__global__ __launch_bounds__(kThreads) void distill_backward_kernel(DistillLaunch a, int64_t len)
{
    typedef Elem<BF16> E;
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * kWaves];
    __shared__ bool s_none;
    const int64_t row = blockIdx.y + (int64_t)blockIdx.z * 32768;
    if (row >= a.N) return;
    const int tid = threadIdx.x;
    const int64_t v0 = blockIdx.x * len, n = min(len, a.V - v0), groups = n / E::kVec;
    const typename E::T *src = static_cast<const typename E::T *>(a.logits) + row * a.ld + v0;
    typename E::T *dst = static_cast<typename E::T *>(a.grad) + row * a.grad_ld + v0;
    int32_t *place = reinterpret_cast<int32_t *>(smem + list_lds(a.k));
    const int bits = table_bits(a.k);
    List<LT> l{reinterpret_cast<Entry *>(smem), a.k};
    bool twice = false;
    word4 w[kFlight];
    auto load = [&](int64_t i) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_last(src + (i + u * kThreads) * E::kVec);
    };
    auto full = [&](int64_t i) { return i + (kFlight - 1) * kThreads < groups; };
    int64_t i = tid;
    if (full(i)) load(i);
    if (tid < LT) {
        l.clear(place, bits);
        l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V, src - v0, v0, n);
        l.sum(a.tau, s_tmp);
        twice = l.twice(place, bits, v0, n);
        if (tid == 0) s_none = l.total == 0.0;
    }
    const float g = a.weight * (a.gloss ? a.gloss[row] : 1.0f);
    const Part r{a.stats[2 * row], a.stats[2 * row + 1]};
    __syncthreads();
    const Slope sl(r, exponent_scale(a.tau), g * a.tau, s_none);
    while (full(i)) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const int64_t at = i + u * kThreads;
            put_group<BF16>(sl, w[u], dst + at * E::kVec);
        }
        i += kFlight * kThreads;
        if (full(i)) load(i);
    }
    for (; i < groups; i += kThreads) put_group<BF16>(sl, load_vec(src + i * E::kVec), dst + i * E::kVec);
    if (groups * E::kVec + tid < n) {
        const int64_t at = groups * E::kVec + tid;
        put_one<BF16>(sl, E::get(src[at]), dst + at);
    }
    after_stores();
    if (tid < LT) l.template put<BF16>(sl, v0, n, twice, dst);
}

// ---------------------------------------------------------------------------
// both at once
// ---------------------------------------------------------------------------
//
// A workgroup of NT threads, 2048 / NT of them a CU, takes a row: its part
// first, then its gradient, from the row's end to its beginning, so that the
// second reading finds what the caches hold of the first.  What it took last
// stays in the registers, and what it took before that in LDS if all the
// workgroups of a CU have room for it: a row of two steps is read once.
// 2048 rows of 128256 bf16, 1.05 GB read and written: 200 to 208 us, what a
// copy of the same bytes takes (197 to 212).  Lists that all threads take
// (LT = NT) cost 2 to 4 vector registers, in scratch memory: 4096 rows of 32000
// with lists of 300 in 188 us.

// Groups of 16 bytes that a workgroup of NT threads takes at a time.
template <int NT> constexpr int kStep = kFlight * NT;

// LT: the list's threads
template <bool BF16, int NT, int LT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(8, 8))) void distill_both_kernel(DistillLaunch a, int keep)
{
    typedef Elem<BF16> E;
    extern __shared__ __align__(16) char smem[];
    __shared__ double s_tmp[2 * NT / kLanes];
    __shared__ bool s_none;
    __shared__ Part s_part[NT / kLanes];
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const float c = exponent_scale(a.tau);
    const typename E::T *src = static_cast<const typename E::T *>(a.logits) + row * a.ld;
    typename E::T *dst = static_cast<typename E::T *>(a.grad) + row * a.grad_ld;
    const int groups = (int)(a.V / E::kVec), rest = (int)(a.V - (int64_t)groups * E::kVec);
    const int steps = (groups + kStep<NT> - 1) / kStep<NT>;
    word4 *kept = reinterpret_cast<word4 *>(smem);  // a thread's own values at tid + u * NT
    char *list = smem + (keep ? kStep<NT> * 16 : 0);
    List<LT> l{reinterpret_cast<Entry *>(list), a.k};
    int32_t *place = reinterpret_cast<int32_t *>(list + list_lds(a.k));
    const int bits = table_bits(a.k);
    bool twice = false;
    word4 w[kFlight];
    auto at = [&](int j, int u) { return j * kStep<NT> + u * NT + tid; };
    auto load_up = [&](int j) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_vec(src + (int64_t)min(at(j, u), groups - 1) * E::kVec);
    };
    auto load_down = [&](int j) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) w[u] = load_last(src + (int64_t)at(j, u) * E::kVec);
    };
    if (steps) load_up(0);
    if (tid < LT) {
        l.clear(place, bits);
        l.template read<BF16>(a.ids + row * a.k, a.teacher + row * a.k, a.V, src, 0, a.V);
    }
    Part p{-FLT_MAX, 0.0f};
    // (a wave's sum lies in LDS: the registers are taken.  Only the widest
    // workgroups take rows of more than two steps.)
    __shared__ Folded s_all[NT / kLanes];
    constexpr int kTurns = kFold / (kFlight * E::kVec);
    const bool folds = NT == 1024 && steps > kTurns;
    Folded &all = s_all[tid / kLanes];
    auto fold_wave = [&] {
        p = wave_merge<kLanes>(p, c);
        if ((tid & (kLanes - 1)) == 0) {
            Folded x = all;
            fold(x, p, c);
            all = x;
        }
        p.z = 0.0f;
    };
    if (folds && (tid & (kLanes - 1)) == 0) all = {-FLT_MAX, 0.0};
    for (int j = 0; j < steps; ++j) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            float f[E::kVec];
            E::unpack(w[u], f);
            if (at(j, u) < groups) add<E::kVec>(p, f, c);
        }
        if (folds && (j + 1) % kTurns == 0) fold_wave();
        if (keep && j == steps - 2) {
#pragma unroll
            for (int u = 0; u < kFlight; ++u) kept[u * NT + tid] = w[u];
        }
        if (j + 1 < steps) load_up(j + 1);
    }
    const int64_t last = (int64_t)groups * E::kVec + tid;
    float tail = 0.0f;
    if (tid < rest) {
        tail = E::get(src[last]);
        add<1>(p, &tail, c);
    }
    if (folds) {
        fold_wave();
        if ((tid & (kLanes - 1)) == 0) p = {all.m, (float)all.z};
    }
    const float g = a.weight * (a.gloss ? a.gloss[row] : 1.0f);
    if (tid < LT) {
        l.sum(a.tau, s_tmp);
        twice = l.twice(place, bits, 0, a.V);
        if (tid == 0) s_none = l.total == 0.0;
    }
    p = block_merge<NT>(p, c, s_part);  // (the workgroup waits in here)
    if (tid < LT) {
        const float loss = l.loss(p, a.tau, s_tmp);
        if (tid == 0) a.loss[row] = loss;
    }
    const Slope sl(p, c, g * a.tau, s_none);
    if (tid < rest) put_one<BF16>(sl, tail, dst + last);
    auto put = [&](int i, word4 x) {
        if (i < groups) put_group<BF16>(sl, x, dst + (int64_t)i * E::kVec);
    };
    int j = steps - 1;
    if (j >= 0) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) put(at(j, u), w[u]);
        --j;
    }
    if (keep && j >= 0) {
        if (j > 0) load_down(j - 1);
#pragma unroll
        for (int u = 0; u < kFlight; ++u) put(at(j, u), kept[u * NT + tid]);
        --j;
    } else if (j >= 0) {
        load_down(j);
    }
    for (; j >= 0; --j) {
#pragma unroll
        for (int u = 0; u < kFlight; ++u) put(at(j, u), w[u]);
        if (j > 0) load_down(j - 1);
    }
    after_stores();
    if (tid < LT) l.template put<BF16>(sl, 0, a.V, twice, dst);
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

// Calls f with the number of threads that take the list (List): a wave while
// it is no longer at it than the others at the row.  Forward, gradient and
// both in us with a wave and with all, for 1024 rows of 32000 bf16: lists of
// 128 17/30/28 and 19/29/28, of 256 17/36/34 and 20/31/31, of 512 22/48/45
// and 23/37/38; for 48 rows: of 128 6.1/6.0/9.9 and 6.9/5.9/10.5, of 256
// 7.5/8.2/13.6 and 7.1/6.0/11.2.
constexpr int kListWave = 128;
template <int NT, typename F> void by_list(int k, F f)
{
    if (k <= kListWave) f(std::integral_constant<int, kLanes>());
    else f(std::integral_constant<int, NT>());
}

template <bool BF16> vie_status forward(const DistillLaunch &a, hipStream_t s)
{
    // Joining parts is a launch more, in which a workgroup reads 150 KB of a
    // row (one row of 65536 bf16: 6.7 us whole, 7.6 in parts; of 98304: 8.4
    // and 7.6; 48 rows of 65536: 7.1 and 8.1, of 98304: 8.8 and 8.1).
    const bool whole = a.V * elem_bytes(a.dtype) <= 150 * 1024;
    Split sp = split_rows(a, whole ? a.V : 32768, INT32_MAX);
    if (sp.parts > kMaxParts) {
        sp.len = ((a.V + kMaxParts - 1) / kMaxParts + 63) / 64 * 64;
        sp.parts = (int)((a.V + sp.len - 1) / sp.len);
        sp.grid.x = (unsigned)sp.parts;
    }
    by_list<kThreads>(a.k, [&](auto lt) {
        constexpr int LT = decltype(lt)::value;
        if (sp.len > kFold * kThreads) distill_forward_kernel<BF16, LT, true><<<sp.grid, kThreads, list_lds(a.k), s>>>(a, sp.len);
        else distill_forward_kernel<BF16, LT, false><<<sp.grid, kThreads, list_lds(a.k), s>>>(a, sp.len);
        if (sp.parts > 1) distill_join_kernel<BF16, LT><<<a.N, LT, list_lds(a.k), s>>>(a, sp.parts);
    });
    return launched("distillation launch");
}

template <bool BF16> vie_status backward(const DistillLaunch &a, hipStream_t s)
{
    // (parts of 64 KB: more workgroups than fit at once, whose ends and lists
    // others stream over; 2048 rows of 128256 bf16: 200 us as whole rows, 187
    // in parts of 128 KB, 177 so and in parts of 32)
    const Split sp = split_rows(a, 8192, kBackGroups);
    const size_t lds = table_lds(a.k);
    vie_status e = VIE_OK;
    by_list<kThreads>(a.k, [&](auto lt) {
        constexpr int LT = decltype(lt)::value;
        e = allow_lds((const void *)distill_backward_kernel<BF16, LT>, lds);
        if (e == VIE_OK) distill_backward_kernel<BF16, LT><<<sp.grid, kThreads, lds, s>>>(a, sp.len);
    });
    return e == VIE_OK ? launched("distillation gradient launch") : e;
}

template <bool BF16, int NT> vie_status both(const DistillLaunch &a, hipStream_t s)
{
    constexpr int64_t kGroups = kStep<NT>;
    size_t lds = table_lds(a.k);
    // of a CU's 160 KB, with 2 KB for the static arrays
    const bool keep = a.V / Elem<BF16>::kVec > kGroups && lds + kGroups * 16 + 1024 * NT / 1024 <= 80 * NT;
    if (keep) lds += kGroups * 16;
    vie_status e = VIE_OK;
    by_list<NT>(a.k, [&](auto lt) {
        constexpr int LT = decltype(lt)::value;
        e = allow_lds((const void *)distill_both_kernel<BF16, NT, LT>, lds);
        if (e == VIE_OK) distill_both_kernel<BF16, NT, LT><<<a.N, NT, lds, s>>>(a, keep);
    });
    return e == VIE_OK ? launched("distillation step launch") : e;
}

template <bool BF16> vie_status step(const DistillLaunch &a, hipStream_t s)
{
    // One kernel where its workgroups fill half of the CUs, or where reading
    // the row takes no longer than another launch (8 rows of 64000 bf16: 13.8
    // us so, 14.8 as two kernels; of 128256: 18.6 and 17.2; of 400000: 46 and
    // 17; 256 rows of 400000: 93 and 102).  With the fewest threads that keep
    // the row from its first reading to its second (4096 rows of 8000 bf16:
    // 31 us with 256 threads, 39 with 512, 57 with 1024; of 32000: 107, 99
    // and 106; 512 of 128256: 62, 60 and 51).
    const int64_t bytes = a.V * elem_bytes(a.dtype);
    if (a.N >= 128 || bytes <= 128 * 1024) {
        if (bytes <= 2 * 16 * kStep<256>) return both<BF16, 256>(a, s);
        if (bytes <= 2 * 16 * kStep<512>) return both<BF16, 512>(a, s);
        return both<BF16, 1024>(a, s);
    }
    DistillLaunch b = a;
    b.stats = reinterpret_cast<float *>(static_cast<char *>(a.ws) + parts_bytes(a.N));
    if (vie_status e = forward<BF16>(b, s)) return e;
    return backward<BF16>(b, s);
}

}  // namespace

size_t distill_workspace_bytes(int64_t, int N)  // (enough for fewer rows, which may have parts)
{
    return parts_bytes(std::min(N, 256)) + (size_t)N * 8;
}

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
