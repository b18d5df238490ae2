// Wave and workgroup helpers shared by the operators' kernels.  A workgroup
// is a whole number of 64-lane waves and every lane takes part.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace vie {

constexpr int kLanes = 64;

typedef uint32_t word4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float from_bf16(uint32_t bits) { return __uint_as_float(bits << 16); }

__device__ __forceinline__ uint16_t to_bf16(float v)  // nearest, ties to even
{
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

__device__ __forceinline__ uint32_t to_bf16x2(float lo, float hi)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), b2));
}

// Element types of rows: fp32, and bf16 as raw bits.
template <bool BF16> struct Elem {
    typedef float T;
    static constexpr int kVec = 4;  // elements of 16 bytes
    static __device__ __forceinline__ float get(T v) { return v; }
    static __device__ __forceinline__ T put(float v) { return v; }
    static __device__ __forceinline__ void unpack(word4 w, float *f)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
    }
    static __device__ __forceinline__ word4 pack(const float *f)
    {
        word4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[i]);
        return w;
    }
};
template <> struct Elem<true> {
    typedef uint16_t T;
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float get(T v) { return from_bf16(v); }
    static __device__ __forceinline__ T put(float v) { return to_bf16(v); }
    static __device__ __forceinline__ void unpack(word4 w, float *f)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ word4 pack(const float *f)
    {
        word4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = to_bf16x2(f[2 * i], f[2 * i + 1]);
        return w;
    }
};

// n elements from p on: `head` of them up to the first 16-byte boundary, then
// `vecs` groups of 16 bytes, then the rest.
template <typename T> struct Span {
    int64_t head, vecs, tail0;
    __device__ __forceinline__ Span(const T *p, int64_t n)
    {
        const int64_t h = (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / (int64_t)sizeof(T);
        head = h < n ? h : n;
        vecs = (n - head) / (16 / (int64_t)sizeof(T));
        tail0 = head + vecs * (16 / (int64_t)sizeof(T));
    }
};

// The value held by lane (lane ^ s), s = 1, 2, 4, 8, 16 or 32, without an LDS
// round trip: quad permutes for 1 and 2, row shifts for 4, a row rotation for
// 8, permlane swaps across rows.  Every lane of the wave is active, and s a
// compile-time constant.
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int s)
{
    const int lane = threadIdx.x & (kLanes - 1);
    switch (s) {
    case 1: return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);
    case 2: return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);
    case 4: {
        const uint32_t up = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x104, 0xF, 0xF, true);
        const uint32_t dn = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x114, 0xF, 0xF, true);
        return (lane & 4) ? dn : up;
    }
    case 8: return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true);
    case 16: {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return (lane & 16) ? r[0] : r[1];
    }
    default: {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return (lane & 32) ? r[0] : r[1];
    }
    }
}
__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int s)
{
    return ((uint64_t)lane_xor((uint32_t)(v >> 32), s) << 32) | lane_xor((uint32_t)v, s);
}

// lane_xor of values of any type of 4 or 8 bytes.
template <typename T> __device__ __forceinline__ T lane_xor_as(T v, int s)
{
    if constexpr (sizeof(T) == 8) return __builtin_bit_cast(T, lane_xor(__builtin_bit_cast(uint64_t, v), s));
    else return __builtin_bit_cast(T, lane_xor(__builtin_bit_cast(uint32_t, v), s));
}
// What `combine` (of any order) makes of the lanes' values, in every lane.
template <typename T, typename F> __device__ __forceinline__ T wave_reduce(T v, F combine)
{
    v = combine(v, lane_xor_as(v, 32));
    v = combine(v, lane_xor_as(v, 16));
    v = combine(v, lane_xor_as(v, 8));
    v = combine(v, lane_xor_as(v, 4));
    v = combine(v, lane_xor_as(v, 2));
    return combine(v, lane_xor_as(v, 1));
}
template <typename T> __device__ __forceinline__ T wave_sum(T v)
{
    return wave_reduce(v, [](T a, T b) { return a + b; });
}
template <typename T> __device__ __forceinline__ T wave_max(T v)
{
    return wave_reduce(v, [](T a, T b) { return b > a ? b : a; });
}

// The value of the lane that the DPP pattern CTRL names, 0 where there is
// none and in the rows of 16 lanes outside ROWS.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t lane_from(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, ROWS == 0xF);
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t lane_from(uint64_t v)
{
    return (uint64_t)lane_from<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | lane_from<CTRL, ROWS>((uint32_t)v);
}
// Inclusive sums over each row of 16 lanes, and over the wave: shifts by 1,
// 2, 4 and 8 within a row, then each row's last lane into the rows after it.
template <typename T> __device__ __forceinline__ T row_scan(T v)
{
    v += lane_from<0x111, 0xF>(v);
    v += lane_from<0x112, 0xF>(v);
    v += lane_from<0x114, 0xF>(v);
    return v + lane_from<0x118, 0xF>(v);
}
template <typename T> __device__ __forceinline__ T wave_scan(T v)
{
    v = row_scan(v);
    v += lane_from<0x142, 0xA>(v);
    return v + lane_from<0x143, 0xC>(v);
}
__device__ __forceinline__ uint32_t read_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ uint64_t read_lane(uint64_t v, int lane)
{
    return (uint64_t)read_lane((uint32_t)(v >> 32), lane) << 32 | read_lane((uint32_t)v, lane);
}
// Inclusive sums over a workgroup of `waves` (at most 16) waves, and the
// total, from each wave's inclusive sums.  `tmp`: 16 values of LDS, free
// again after the next barrier.
template <typename T> struct Sums {
    T upto, total;
};
template <typename T> __device__ __forceinline__ void wave_total(T upto, T *tmp)
{
    if ((threadIdx.x & (kLanes - 1)) == kLanes - 1) tmp[threadIdx.x / kLanes] = upto;
}
template <typename T> __device__ __forceinline__ Sums<T> after_waves(T upto, const T *tmp, int waves)
{
    const int at = threadIdx.x & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    const T v = row_scan(at < waves ? tmp[at] : T(0));
    return {upto + (wave ? read_lane(v, wave - 1) : T(0)), read_lane(v, 15)};
}

// The value `combine` makes of every thread's v, in every thread; the order
// of combination is fixed.  `tmp`: NT / 64 values of LDS, free again after the
// next barrier.
template <int NT, typename T, typename F> __device__ __forceinline__ T block_reduce(T v, T *tmp, F combine)
{
    constexpr int W = NT / kLanes;
    v = wave_reduce(v, combine);
    if constexpr (W > 1) {
        __syncthreads();
        if ((threadIdx.x & (kLanes - 1)) == 0) tmp[threadIdx.x / kLanes] = v;
        __syncthreads();
        v = tmp[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = combine(v, tmp[w]);
    }
    return v;
}

}  // namespace vie
