// The int8 head (gfx950): full-vocabulary logits of the int8 rows of W_out.
//
// A token h is quantized by the rule of the rows (scale xs = fp32(max |h| /
// 127), x = rint(fp32(h / xs)) clamped to [-127, 127]; all zeros: scale 0, x
// = 0; a NaN or an infinity among the values: scale NaN), and
//
//   z[b][v] = fp32(fp32(fp32(sum_j q[v][j] x[b][j]) scale[v]) xs[b])
//
// with an exact integer sum (at most 8192 127^2 < 2^31), rounded once more
// if the logits are stored in bf16.  The products run on the matrix cores
// (v_mfma_i32_16x16x64_i8: 16 rows, 16 tokens, 64 columns).
#include <hip/hip_runtime.h>

#include "block.hpp"
#include "operators.hpp"

namespace vie {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;  // columns of a matrix instruction

__host__ __device__ inline int padded(int d) { return (d + kStep - 1) / kStep * kStep; }

__device__ __forceinline__ int quantized(float x, float scale)
{
    return scale == 0.0f ? 0 : (int)fminf(fmaxf(rintf(__fdiv_rn(x, scale)), -127.0f), 127.0f);
}

// The tokens' int8 values [B][padded(d)] (zero past d) and their scales: one
// wave per token.
template <bool BF16>
__global__ __launch_bounds__(256) void tokens_kernel(const typename Elem<BF16>::T *__restrict__ h, int B, int d,
                                                     int8_t *__restrict__ x, float *__restrict__ xs)
{
    typedef Elem<BF16> E;
    const int b = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes, lane = threadIdx.x & (kLanes - 1);
    if (b >= B) return;
    const typename E::T *row = h + (int64_t)b * d;
    float top = 0.0f;
    bool bad = false;
    for (int j = lane; j < d; j += kLanes) {
        const float v = fabsf(E::get(row[j]));
        bad |= !(v < __builtin_inff());
        top = fmaxf(top, v);
    }
    top = wave_max(top);
    bad = __any(bad);
    const float scale = bad ? 0.0f : __fdiv_rn(top, 127.0f);
    for (int j = lane; j < padded(d); j += kLanes)
        x[(int64_t)b * padded(d) + j] = j < d ? (int8_t)quantized(E::get(row[j]), scale) : 0;
    if (lane == 0) xs[b] = bad ? __builtin_nanf("") : scale;
}

// 16 int8 values from p on, as far as they lie before `end`; the bytes past
// a row meet zeros of the token.
__device__ __forceinline__ word4 load16(const int8_t *p, const int8_t *end)
{
    word4 w = {0, 0, 0, 0};
    if (end - p >= 16) {
        __builtin_memcpy(&w, p, 16);
    } else {
        for (int i = 0; i < 16; ++i)
            if (p + i < end) w[i / 4] |= (uint32_t)(uint8_t)p[i] << 8 * (i % 4);
    }
    return w;
}

// One wave: 16 rows and 16 tokens.  Lane (r, g) = (lane % 16, lane / 16)
// holds columns 16 g .. + 15 of a step of row r and of token r, and of the
// result rows 4 g + i for token r.
template <bool OUT_BF16>
__global__ __launch_bounds__(256) void int8_simple_kernel(const int8_t *__restrict__ q, const float *__restrict__ scale,
                                                          int64_t V, int d, const int8_t *__restrict__ x,
                                                          const float *__restrict__ xs, int B,
                                                          typename Elem<OUT_BF16>::T *__restrict__ out, int64_t ld)
{
    const int lane = threadIdx.x & (kLanes - 1), r = lane & 15, g = lane >> 4;
    const int64_t v0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / kLanes) * 16;
    const int b0 = blockIdx.y * 16;
    const int8_t *end = q + V * d;
    const int8_t *row = q + min(v0 + r, V - 1) * d;
    const int8_t *tok = x + (int64_t)min(b0 + r, B - 1) * padded(d);
    i32x4 acc = {0, 0, 0, 0};
    for (int c = 16 * g; c < padded(d); c += kStep) {
        const word4 w = load16(row + c, end), t = *reinterpret_cast<const word4 *>(tok + c);
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, t), acc, 0, 0, 0);
    }
    const int b = b0 + r;
    if (b >= B) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t v = v0 + 4 * g + i;
        if (v < V) out[(int64_t)b * ld + v] = Elem<OUT_BF16>::put((float)acc[i] * scale[v] * xs[b]);
    }
}

vie_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

size_t tokens_bytes(int d, int B) { return ((size_t)B * padded(d) + 255) & ~(size_t)255; }

}  // namespace

// The tokens' int8 values and scales.
size_t int8_workspace_bytes(int64_t, int d, int B) { return tokens_bytes(d, B) + (size_t)B * 4; }

vie_status launch_int8_logits(const Int8Launch &a, hipStream_t s)
{
    int8_t *x = static_cast<int8_t *>(a.ws);
    float *xs = reinterpret_cast<float *>(x + tokens_bytes(a.d, a.B));
    const unsigned tg = (unsigned)((a.B + 3) / 4);
    if (a.h_dtype == VIE_BF16) tokens_kernel<true><<<tg, 256, 0, s>>>(static_cast<const uint16_t *>(a.h), a.B, a.d, x, xs);
    else tokens_kernel<false><<<tg, 256, 0, s>>>(static_cast<const float *>(a.h), a.B, a.d, x, xs);
    if (vie_status e = launched("token quantization launch")) return e;
    const dim3 grid((unsigned)((a.V + 63) / 64), (unsigned)((a.B + 15) / 16));
    if (a.out_dtype == VIE_BF16)
        int8_simple_kernel<true><<<grid, 256, 0, s>>>(a.q, a.scale, a.V, a.d, x, xs, a.B, static_cast<uint16_t *>(a.out), a.ld);
    else
        int8_simple_kernel<false><<<grid, 256, 0, s>>>(a.q, a.scale, a.V, a.d, x, xs, a.B, static_cast<float *>(a.out), a.ld);
    return launched("int8 head launch");
}

}  // namespace vie
