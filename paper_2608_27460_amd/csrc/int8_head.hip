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

#include <algorithm>
#include <type_traits>

#include "block.hpp"
#include "operators.hpp"

namespace vie {

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;   // columns of a matrix instruction
constexpr int kPad = 128;   // tokens are padded to whole stages

__host__ __device__ inline int padded(int d) { return (d + kPad - 1) / kPad * kPad; }

// rint(fp32(x / scale)) clamped to [-127, 127], 0 for scale 0.  The product
// with the reciprocal is off by 4e-5 at most here, so that the division
// itself is only needed near the middle between two integers (and where the
// reciprocal is no number to use).
struct Quantizer {
    float scale, inverse;
    __device__ __forceinline__ explicit Quantizer(float scale)
        : scale(scale), inverse(scale == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(scale))
    {
    }
    __device__ __forceinline__ int operator()(float x) const
    {
        const float q = x * inverse;
        float n = rintf(q);
        if (!(fabsf(q - n) < 0.499f)) n = rintf(__fdiv_rn(x, scale));
        return (int)fminf(fmaxf(n, -127.0f), 127.0f);
    }
};

// The tokens' int8 values [B][padded(d)] (zero past d) and their scales: a
// workgroup per token, whose values it holds in registers, eight to a chunk.
constexpr int kTokenThreads = 256;
constexpr int kChunks = kMaxD / 8 / kTokenThreads;

template <bool BF16>
__global__ __launch_bounds__(kTokenThreads) void tokens_kernel(const typename Elem<BF16>::T *__restrict__ h, int d,
                                                               int8_t *__restrict__ x, float *__restrict__ xs)
{
    typedef Elem<BF16> E;
    __shared__ float s_top[kTokenThreads / kLanes];
    const int b = blockIdx.x, tid = threadIdx.x;
    const typename E::T *row = h + (int64_t)b * d;
    float v[kChunks][8], top = 0.0f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int j = (i * kTokenThreads + tid) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
        if (j + 8 <= d) {
            word4 w[8 / E::kVec];
            __builtin_memcpy(w, row + j, sizeof w);  // (at any alignment)
#pragma unroll
            for (int k = 0; k < 8 / E::kVec; ++k) E::unpack(w[k], &v[i][k * E::kVec]);
        } else if (j < d) {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (j + e < d) v[i][e] = E::get(row[j + e]);
        }
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bad |= !(fabsf(v[i][e]) < __builtin_inff());
            top = fmaxf(top, fabsf(v[i][e]));
        }
    top = bad ? __builtin_inff() : top;
    top = block_reduce<kTokenThreads>(top, s_top, [](float a, float b) { return fmaxf(a, b); });
    bad = top == __builtin_inff();
    const float scale = bad ? 0.0f : __fdiv_rn(top, 127.0f);
    const Quantizer quantized(scale);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int j = (i * kTokenThreads + tid) * 8;
        if (j >= padded(d)) break;
        uint64_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= (uint64_t)(uint8_t)quantized(v[i][e]) << 8 * e;
        *reinterpret_cast<uint64_t *>(x + (int64_t)b * padded(d) + j) = w;
    }
    if (tid == 0) xs[b] = bad ? __builtin_nanf("") : scale;
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
    const int b0 = blockIdx.y * 16, b = b0 + r;
    const int8_t *end = q + V * d;
    const int8_t *tok = x + (int64_t)min(b0 + r, B - 1) * padded(d);
    for (int64_t v0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / kLanes) * 16; v0 < V; v0 += (int64_t)gridDim.x * 64) {
        const int8_t *row = q + min(v0 + r, V - 1) * d;
        i32x4 acc = {0, 0, 0, 0};
        for (int c = 16 * g; c < padded(d); c += kStep) {
            const word4 w = load16(row + c, end), t = *reinterpret_cast<const word4 *>(tok + c);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, t), acc, 0, 0, 0);
        }
        if (b >= B) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t v = v0 + 4 * g + i;
            if (v < V) out[(int64_t)b * ld + v] = Elem<OUT_BF16>::put((float)acc[i] * scale[v] * xs[b]);
        }
    }
}

// ---------------------------------------------------------------------------
// tiles through LDS
// ---------------------------------------------------------------------------
//
// A workgroup of eight waves takes tiles of up to VT = 256 rows and BT tokens.
// Columns go by stages of KC bytes: the rows' and the tokens' bytes of a stage
// go from memory straight to LDS (16 bytes a lane), NBUF stages ahead and
// across the ends of tiles, and a wave reads the operands of the next stage
// from LDS into registers while it multiplies those of the present one, so
// that the matrix cores wait for neither.  A wave multiplies 16 MT rows by 16
// NT tokens.
//
// Piece p (16 bytes) of staged row x sits in slot p ^ swizzle(x) of that row,
// so that the operand reads (16 rows, one piece each) hit every LDS bank
// once.  Pieces past a row re-read its last one, against zeros of the token;
// rows and tokens past the tile re-read its last one, and their results are
// not stored.
//
// A few tokens (HELD) stay in LDS throughout, quantized there by every
// workgroup while its first rows are on their way, which saves the launch of
// tokens_kernel and the tokens' staging.  Rows that are not 16-byte aligned
// (DMA false) go to LDS by way of registers, two stages ahead.
//
// The logits leave through LDS of each wave's own, 16 tokens at a time, so
// that a store covers runs of up to 256 bytes of a token's row; the stages of
// the next tile go on arriving meanwhile.
//
// The waits count the loads and stores (vmcnt) that this source issues: a
// kernel of these that spilled vector registers would wait for its own too.
// (None does; those of the held tokens spill some 60 scalar registers, to
// lanes of vector ones, which takes no load.)
//
// What bounds it: up to 128 tokens the reading of the rows (151936 x 1024, 1
// token: 33 us or 4.8 TB/s where each call has other rows, 28 where the
// last-level cache holds some of them; 128256 x 2048, 64 tokens: 55 us and 5
// of the tokens' own kernel, 5.1 TB/s of rows and logits together).  With
// more, a compute unit's loads and its products: 301 and 318 us of 2048
// tokens' 506 if each is alone, at the clock (1.9 GHz) that the matrix cores
// leave.  It takes 500 to 560 us from call to call, 1.9e15 to 2.1e15
// operations a second; the library's product of 8192^3 reaches 2.0e15 to
// 2.1e15.  Four waves of 128 x 128, which read a third less from LDS and whose
// matrix instructions follow each other without a pause, are no faster (562 us
// beside 506).

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kLanes;
constexpr int kWorkgroups = 256;  // one per CU
constexpr int kTileRows = 256;

template <int KC> __device__ __forceinline__ int swizzle(int x) { return KC == 64 ? x >> 2 & 3 : x >> 1 & 7; }

__device__ __forceinline__ void load_lds16(const int8_t *src, char *dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                     (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
}

// 16 bytes to any alignment.  PAST: past the caches' keeping, for logits of
// many tokens, which would push the rows and tokens out of L2 (2048 tokens, in
// turn: 528 to 535 us without, 509 to 520 with).
template <bool PAST> __device__ __forceinline__ void store16(char *o, word4 w)
{
    typedef word4 any_word4 __attribute__((aligned(2)));
    if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<any_word4 *>(o));
    else __builtin_memcpy(o, &w, 16);
}

constexpr int kHeldLds = 56 * 1024;  // for the held tokens and their scales
constexpr int kHeldPad = 16;         // bytes between them: 16 rows' reads hit every bank once
constexpr int tile_stage(int BT, int KC) { return (kTileRows + BT) * KC; }
constexpr int tile_out(int MT) { return 512 * MT; }  // of a wave, for its logits on their way out
constexpr int tile_lds(int stage, int NBUF, int MT, bool held) { return stage * NBUF + kWaves * tile_out(MT) + (held ? kHeldLds : 0); }
// Whether the tokens are held.  Rows that are not aligned: wherever they fit
// (there is nothing as fast for these rows), if there are 16 bytes of rows, a
// load.  Aligned ones: as long as every workgroup's quantization takes less
// than tokens_kernel's launch, held and apart in us: 32000 x 256, 4 tokens
// 6.5 and 8.1, 16 tokens 8.6 and 8.5; 151936 x 1024, 4 tokens 33.6 and 35.6,
// 12 tokens 35.6 and 36.2, 16 tokens 37.4 and 36.8; 128256 x 2048, 4 tokens
// 51.1 and 52.4, 12 tokens 55.0 and 53.8.  Wider rows gain nothing: 128256 x
// 2304, 1 token 50.0 and 50.4; x 2560, 1 token 59.0 and 59.6, 6 tokens 61.5
// and 61.3; 32000 x 2560, 1 token 18.8 and 18.6; x 4096 27.4 and 24.6; x 8192
// 53 and 46.
inline bool hold_tokens(int64_t V, int B, int d, bool aligned)
{
    if (aligned) return B <= 12 && d <= 2048 && B * padded(d) <= 12 * 1024;
    return B <= 16 && B * (padded(d) + kHeldPad) + 64 <= kHeldLds && V * d >= 16;
}

// The tokens' int8 values at tok + b (padded(d) + kHeldPad) and their scales
// behind them, by tokens_kernel's rule: a wave per token at a time.  A wave's
// first token is fetched before the first rows are, so that it does not wait
// for them, and up to 2048 values of a token are held in registers between
// the search for their largest and their quantization.
constexpr int kTokenChunks = 4;  // of eight values a lane
template <bool BF16> struct Chunk {  // eight values as they are stored
    static constexpr int kWords = 8 / Elem<BF16>::kVec;
    word4 w[kWords];
    // (without branches of the lanes, which would wait for the loads: what
    // lies past d is loaded from before it, and dropped by `values`)
    __device__ __forceinline__ void fetch(const typename Elem<BF16>::T *row, int d, int j)
    {
        if (d % 8 == 0) {
            __builtin_memcpy(w, row + min(j, d - 8), sizeof w);  // (at any alignment)
        } else {
            typename Elem<BF16>::T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = row[min(j + i, d - 1)];
            __builtin_memcpy(w, e, sizeof w);
        }
    }
    __device__ __forceinline__ void values(float *v, int d, int j) const
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k) Elem<BF16>::unpack(w[k], v + k * Elem<BF16>::kVec);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = j + e < d ? v[e] : 0.0f;
    }
};
template <bool BF16> struct Token {
    Chunk<BF16> c[kTokenChunks];
    __device__ __forceinline__ void fetch(const void *h, int b, int d)
    {
        const typename Elem<BF16>::T *row = static_cast<const typename Elem<BF16>::T *>(h) + (int64_t)b * d;
#pragma unroll
        for (int i = 0; i < kTokenChunks; ++i)
            if (8 * i * kLanes < d) c[i].fetch(row, d, 8 * (i * kLanes + (threadIdx.x & (kLanes - 1))));
    }
    // All tokens; the wave's first one is fetched.
    __device__ void hold(const void *h, int B, int d, char *tok, float *s_xs)
    {
        const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes, dp = padded(d);
        constexpr int kHeld = 8 * kTokenChunks * kLanes;
        for (int b = wave; b < B; b += kWaves) {
            const typename Elem<BF16>::T *row = static_cast<const typename Elem<BF16>::T *>(h) + (int64_t)b * d;
            if (b != wave) fetch(h, b, d);
            float top = 0.0f;
            bool bad = false;
            auto look = [&](int j, const Chunk<BF16> &x) {
                float v[8];
                x.values(v, d, j);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bad |= !(fabsf(v[e]) < __builtin_inff());
                    top = fmaxf(top, fabsf(v[e]));
                }
            };
#pragma unroll
            for (int i = 0; i < kTokenChunks; ++i)
                if (8 * i * kLanes < d) look(8 * (i * kLanes + lane), c[i]);
            for (int j = kHeld + 8 * lane; j < d; j += 8 * kLanes) {
                Chunk<BF16> x;
                x.fetch(row, d, j);
                look(j, x);
            }
            top = wave_max(top);
            bad = __any(bad);
            const Quantizer quantized(bad ? 0.0f : __fdiv_rn(top, 127.0f));
            auto write = [&](int j, const Chunk<BF16> &x) {
                float v[8];
                x.values(v, d, j);
                uint64_t w = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) w |= (uint64_t)(uint8_t)quantized(v[e]) << 8 * e;
                if (j < dp) *reinterpret_cast<uint64_t *>(tok + b * (dp + kHeldPad) + j) = w;
            };
#pragma unroll
            for (int i = 0; i < kTokenChunks; ++i)
                if (8 * i * kLanes < d) write(8 * (i * kLanes + lane), c[i]);
            for (int j = kHeld + 8 * lane; j < dp; j += 8 * kLanes) {
                Chunk<BF16> x;
                x.fetch(row, d, j);
                write(j, x);
            }
            if (lane == 0) s_xs[b] = bad ? __builtin_nanf("") : quantized.scale;
        }
    }
};

// Tile t of a workgroup: XCD blockIdx.x % 8 takes a run of the tiles, its
// workgroups take every 32nd of them, and the order goes over up to eight
// token tiles first, so that an XCD's workgroups share rows and tokens in L2.
struct Tiles {
    int rows;          // rows of a tile (at most kTileRows)
    int nv, nb;        // tiles of rows, of tokens
    int per_xcd, step; // tiles of an XCD's run, its workgroups
};

template <int MT, int NT, int WB, int KC, int NBUF, bool AHEAD, bool HELD, bool H_BF16, bool DMA, bool OUT_BF16>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void int8_tile_kernel(
    const int8_t *__restrict__ q, int pitch, const float *__restrict__ scale, int64_t V, const int8_t *__restrict__ x,
    int dp, const float *__restrict__ xs, const void *__restrict__ h, int d, int B, typename Elem<OUT_BF16>::T *__restrict__ out, int64_t ld, Tiles tiles)
{
    typedef Elem<OUT_BF16> E;
    extern __shared__ __align__(16) char smem[];
    constexpr int BT = 16 * NT * WB;
    static_assert(kWaves / WB * MT * 16 == kTileRows, "the waves cover a tile");
    static_assert(DMA || (HELD && !AHEAD && NBUF == 2), "rows by way of registers take two buffers");
    static_assert(!HELD || BT == 16, "held tokens are one operand");
    constexpr int kStage = tile_stage(HELD ? 0 : BT, KC), P = KC / 16, LR = kLanes / P, KS = KC / kStep;
    constexpr int WL = kTileRows / kWaves / LR;                              // loads of a wave's rows per stage
    constexpr int XR = BT / kWaves, XL = HELD ? 0 : (XR + LR - 1) / LR;      // tokens a wave stages, their loads
    constexpr int L = WL + XL;
    char *tok = smem + NBUF * kStage + kWaves * tile_out(MT);                // (HELD)
    float *s_xs = reinterpret_cast<float *>(tok + B * (dp + kHeldPad));
    const int tid = threadIdx.x, lane = tid & (kLanes - 1), r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kLanes);
    const int wv = wave / WB, wb = wave % WB;
    const int nstage = dp / KC;

    // this workgroup's tiles: first, first + step, .. below end
    const int xcd = blockIdx.x % 8;
    const int first = xcd * tiles.per_xcd + blockIdx.x / 8;
    const int end = min((xcd + 1) * tiles.per_xcd, tiles.nv * tiles.nb);
    if (first >= end) return;
    auto place = [&](int t, int64_t &v0, int &b0) {
        const int group = t / (8 * tiles.nv), in = min(8, tiles.nb - 8 * group), k = t - group * 8 * tiles.nv;
        v0 = (int64_t)(k / in) * tiles.rows;
        b0 = (8 * group + k % in) * BT;
    };

    const int lrow = lane / P, slot = lane % P;
    const int8_t *wsrc[WL], *xsrc[XL + 1];
    int wcol[WL], xcol[XL + 1];
#pragma unroll
    for (int t = 0; t < WL; ++t) wcol[t] = 16 * (slot ^ swizzle<KC>(LR * t + lrow));
#pragma unroll
    for (int t = 0; t < XL; ++t) xcol[t] = 16 * (slot ^ swizzle<KC>(wave * XR + LR * t + lrow));
    auto set_tile = [&](int t) {
        int64_t v0;
        int b0;
        place(t, v0, b0);
        const int64_t vlast = min<int64_t>(V, v0 + tiles.rows) - 1;
#pragma unroll
        for (int i = 0; i < WL; ++i)
            wsrc[i] = q + min<int64_t>(v0 + wave * (kTileRows / kWaves) + LR * i + lrow, vlast) * pitch;
#pragma unroll
        for (int i = 0; i < XL; ++i) xsrc[i] = x + (int64_t)min(b0 + wave * XR + LR * i + lrow, B - 1) * dp;
    };
    int lt = first, lst = 0;  // the stage to load next
    word4 hold[DMA ? 1 : 2][WL];
    auto load_next = [&](int buf) {
        char *dst = smem + buf * kStage;
        const int c = lst * KC;
        if constexpr (DMA) {
#pragma unroll
            for (int i = 0; i < WL; ++i)
                load_lds16(wsrc[i] + min(c + wcol[i], pitch - 16), dst + (wave * (kTileRows / kWaves) + LR * i) * KC);
#pragma unroll
            for (int i = 0; i < XL; ++i)
                if (XR >= LR || lane < XR * P)
                    load_lds16(xsrc[i] + c + xcol[i], dst + (kTileRows + wave * XR + LR * i) * KC);
        } else {  // (pieces past a row: any bytes)
#pragma unroll
            for (int i = 0; i < WL; ++i) {
                const int8_t *p = wsrc[i] + (c + wcol[i] < pitch ? c + wcol[i] : 0), *last = q + V * pitch - 16;
                __builtin_memcpy(&hold[buf][i], p < last ? p : last, 16);
            }
        }
        if (++lst == nstage) {  // past the last tile: its stages again, unused
            lst = 0;
            if (lt + tiles.step < end) lt += tiles.step;
            set_tile(lt);
        }
    };
    struct Operands {
        word4 a[KS][MT], b[KS][NT];
    };
    int rst = 0;  // the stage to read next
    auto read = [&](int buf, Operands &o) {
        const char *A = smem + buf * kStage + (wv * MT * 16 + r) * KC;
        const char *X = HELD ? tok + min(r, B - 1) * (dp + kHeldPad) + rst * KC
                             : smem + buf * kStage + (kTileRows + wb * NT * 16 + r) * KC;
        rst = rst == nstage - 1 ? 0 : rst + 1;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int at = 16 * ((4 * k + g) ^ swizzle<KC>(r));
#pragma unroll
            for (int n = 0; n < NT; ++n)
                o.b[k][n] = *reinterpret_cast<const word4 *>(X + (HELD ? kStep * k + 16 * g : n * 16 * KC + at));
#pragma unroll
            for (int m = 0; m < MT; ++m) o.a[k][m] = *reinterpret_cast<const word4 *>(A + m * 16 * KC + at);
        }
    };
    i32x4 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
    auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, o.a[k][m]),
                                                                      __builtin_bit_cast(i32x4, o.b[k][n]), acc[m][n], 0, 0, 0);
    };

    // What the logits of tile t need besides: the scales of the wave's rows
    // (lane, lane + 64) and of its tokens.
    constexpr int kScales = (16 * MT + kLanes - 1) / kLanes;
    float sc[kScales], xf[NT];
    auto load_scales = [&](int t) {
        int64_t v0;
        int b0;
        place(t, v0, b0);
#pragma unroll
        for (int i = 0; i < kScales; ++i) sc[i] = scale[min<int64_t>(v0 + wv * MT * 16 + i * kLanes + lane, V - 1)];
#pragma unroll
        for (int n = 0; n < NT; ++n) xf[n] = HELD ? s_xs[min(r, B - 1)] : xs[min(b0 + (wb * NT + n) * 16 + r, B - 1)];
    };
    // lane (r, g) holds rows 4 g + i of row tile m for token 16 n + r
    constexpr int kHalves = OUT_BF16 ? 1 : 2, kPer = MT / kHalves;  // a token's run: kPer row tiles
    constexpr int kUnits = kPer * 16 / E::kVec;                      // 16-byte units of it
    constexpr int kStores = kHalves * NT * 16 * kUnits / kLanes;
    auto store = [&](int t) {  // whether every store of the wave was made
        int64_t v0;
        int b0;
        place(t, v0, b0);
        const int64_t vend = min<int64_t>(V, v0 + tiles.rows);
        v0 += wv * MT * 16;
        b0 += wb * NT * 16;
        char *tmp = smem + NBUF * kStage + wave * tile_out(MT);
        // (this lane's addresses are made here: kept over the stages they
        // would take the registers that the operands need)
        int lane = threadIdx.x & (kLanes - 1);
        asm volatile("" : "+v"(lane));
        const int r = lane & 15, g = lane >> 4;
        // (a whole tile's stores: one offset a lane, the rest is the wave's)
        const bool full = v0 + MT * 16 <= vend && b0 + 16 * NT <= B && ld < (1 << 24);
        char *to = reinterpret_cast<char *>(out + (int64_t)b0 * ld + v0);
        const uint32_t lane_to = (uint32_t)((lane / kUnits) * (int)ld + lane % kUnits * E::kVec) * (uint32_t)sizeof(typename E::T);
        // the scales to their lanes; the sums become logits in place
#pragma unroll
        for (int i = 0; i < kScales; ++i) reinterpret_cast<float *>(tmp)[i * kLanes + lane] = sc[i];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's own writes, read by its other lanes)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float f[4];
            Elem<false>::unpack(*reinterpret_cast<const word4 *>(tmp + 64 * m + 16 * g), f);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][n][i] = __float_as_int((float)acc[m][n][i] * f[i] * xf[n]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
#pragma unroll
                for (int m = 0; m < kPer; ++m) {
                    float f[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = __int_as_float(acc[h * kPer + m][n][i]);
                    if constexpr (OUT_BF16) {
                        const uint32_t w[2] = {to_bf16x2(f[0], f[1]), to_bf16x2(f[2], f[3])};
                        char *p = tmp + r * (kUnits * 16) + 16 * ((2 * m + g / 2) ^ (r & (kUnits - 1))) + 8 * (g & 1);
                        *reinterpret_cast<uint64_t *>(p) = (uint64_t)w[1] << 32 | w[0];
                    } else {
                        *reinterpret_cast<word4 *>(tmp + r * (kUnits * 16) + 16 * ((4 * m + g) ^ (r & (kUnits - 1)))) =
                            Elem<false>::pack(f);
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < 16 * kUnits / kLanes; ++i) {
                    const int row = (i * kLanes + lane) / kUnits, unit = lane % kUnits;
                    const char *from = tmp + row * (kUnits * 16) + 16 * (unit ^ (row & (kUnits - 1)));
                    const word4 w = *reinterpret_cast<const word4 *>(from);
                    if (full) {
                        char *o = to + ((int64_t)(16 * n + i * (kLanes / kUnits)) * ld + h * kPer * 16) * (int)sizeof(typename E::T);
                        store16<(WB > 1)>(o + lane_to, w);
                        continue;
                    }
                    const int b = b0 + 16 * n + row;
                    const int64_t v = v0 + h * kPer * 16 + unit * E::kVec;
                    typename E::T *o = out + (int64_t)b * ld + v;
                    if (b < B && v + E::kVec <= vend) {
                        store16<false>(reinterpret_cast<char *>(o), w);
                    } else if (b < B) {
                        for (int e = 0; e < E::kVec && v + e < vend; ++e) {
                            typename E::T val;
                            __builtin_memcpy(&val, from + e * sizeof val, sizeof val);
                            o[e] = val;
                        }
                    }
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
        return full;
    };

    Token<H_BF16> token;
    if constexpr (HELD)
        if (wave < B) token.fetch(h, wave, d);
    set_tile(first);
#pragma unroll
    for (int i = 0; i < (DMA ? NBUF - !AHEAD : 2); ++i) load_next(i);
    if constexpr (HELD) {
        token.hold(h, B, d, tok, s_xs);
        __syncthreads();
    }
    int buf = 0, stored = 0, t = first, st = 0;
    Operands now, next;
    if constexpr (!DMA) {
        // Stage s is read from buffer s % 2 while stage s + 1 goes from its
        // registers to the other one and s + 3 is loaded into them.
        int pt = first, pst = 0;  // the stage to put
        auto put = [&](int to) {
            char *dst = smem + to * kStage + wave * (kTileRows / kWaves) * KC + 16 * lane;
            int64_t v0;
            int b0;
            place(pt, v0, b0);
            if ((v0 + tiles.rows) * pitch + 16 > V * pitch) {
                // Pieces that would end past the matrix were loaded before its
                // end: their bytes move to where they belong.  (Rows of a few
                // bytes have such pieces before the last tile, too.)
#pragma unroll
                for (int i = 0; i < WL; ++i) {
                    const int64_t v = min<int64_t>(v0 + wave * (kTileRows / kWaves) + LR * i + lrow, V - 1);
                    const int col = pst * KC + wcol[i];
                    const int64_t by = v * pitch + (col < pitch ? col : 0) - (V * pitch - 16);
                    if (by <= 0) continue;
                    word4 w = hold[to][i];
                    for (int64_t k = 0; k < by; ++k) {
                        w.x = w.x >> 8 | w.y << 24;
                        w.y = w.y >> 8 | w.z << 24;
                        w.z = w.z >> 8 | w.w << 24;
                        w.w >>= 8;
                    }
                    hold[to][i] = w;
                }
            }
#pragma unroll
            for (int i = 0; i < WL; ++i) *reinterpret_cast<word4 *>(dst + LR * i * KC) = hold[to][i];
            if (++pst == nstage) pst = 0, pt += tiles.step;
        };
        put(0);
        load_next(0);
        auto step = [&](int b) {
            __syncthreads();
            if (st == nstage - 1) load_scales(t);
            read(b, now);
            put(1 - b);
            load_next(1 - b);
            multiply(now);
            if (++st == nstage) {
                store(t);
                st = 0;
                t += tiles.step;
                return t < end;
            }
            return true;
        };
        while (step(0) && step(1)) {
        }
        return;
    }
    if constexpr (AHEAD) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NBUF - 1) * L) : "memory");
        __builtin_amdgcn_s_barrier();
        read(0, now);
    }
    auto step = [&](Operands &cur, Operands &nxt) {  // false past the last stage
        // The stage to be read has landed, and the operands of the stage
        // before it are read, in every wave past the barrier.  (The first
        // stages after a tile's end were issued before its stores, which may
        // be in flight too.)
        __builtin_amdgcn_sched_barrier(0);
        if (stored > 0) {
            --stored;
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NBUF - 2) * L + kStores) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NBUF - 2) * L) : "memory");
        }
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if (st == nstage - 1) load_scales(t);
        if constexpr (AHEAD) {
            load_next(buf);
            buf = buf == NBUF - 1 ? 0 : buf + 1;
            read(buf, nxt);
        } else {
            load_next(buf == 0 ? NBUF - 1 : buf - 1);
            read(buf, cur);
            buf = buf == NBUF - 1 ? 0 : buf + 1;
        }
        multiply(cur);
        if constexpr (!AHEAD && KS == 2) {
            // The operands of the first products, then one of the second ones
            // with every two products (2048 tokens of 128256 x 2048, in turn:
            // 538 to 543 us as the compiler orders them, 509 to 520 so).
            constexpr int kReads = MT + NT, kProducts = MT * NT;
            __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
#pragma unroll
            for (int i = 0; i < kReads; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 2 * kProducts - 2 * kReads, 0);
        }
        if (++st == nstage) {
            stored = store(t) ? NBUF - 1 : 0;
            st = 0;
            t += tiles.step;
            return t < end;
        }
        return true;
    };
    if constexpr (AHEAD)
        while (step(now, next) && step(next, now)) {
        }
    else
        while (step(now, now)) {
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the workgroup
}

vie_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

size_t tokens_bytes(int d, int B) { return ((size_t)B * padded(d) + 255) & ~(size_t)255; }

}  // namespace

namespace {
// `q`: rows of `pitch` bytes, a.q's own or copies of them.
template <int MT, int NT, int WB, int KC, int NBUF, bool AHEAD, bool HELD, bool H_BF16, bool DMA, bool OUT_BF16>
hipError_t tile_launch(const Int8Launch &a, const int8_t *q, int pitch, const int8_t *x, const float *xs, bool even, hipStream_t s)
{
    constexpr int BT = 16 * NT * WB, lds = tile_lds(tile_stage(HELD ? 0 : BT, KC), NBUF, MT, HELD);
    static_assert(lds <= 160 * 1024, "a tile's stages fit LDS");
    auto kern = int8_tile_kernel<MT, NT, WB, KC, NBUF, AHEAD, HELD, H_BF16, DMA, OUT_BF16>;
    hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    Tiles t;
    t.nb = (a.B + BT - 1) / BT;
    t.rows = kTileRows;
    if (even) {  // every workgroup as many rows as the others, to eight
        const int64_t rounds = (a.V + kTileRows * kWorkgroups - 1) / (kTileRows * kWorkgroups);
        const int64_t rows = (a.V + rounds * kWorkgroups - 1) / (rounds * kWorkgroups);
        t.rows = (int)((rows + 7) / 8 * 8);
    }
    t.nv = (int)((a.V + t.rows - 1) / t.rows);
    const int64_t n = (int64_t)t.nv * t.nb;
    t.per_xcd = (int)((n + 7) / 8);
    t.step = std::min(kWorkgroups / 8, t.per_xcd);
    kern<<<8 * t.step, kThreads, lds, s>>>(q, pitch, a.scale, a.V, x, padded(a.d), xs, a.h, a.d, a.B,
                                           static_cast<typename Elem<OUT_BF16>::T *>(a.out), a.ld, t);
    return hipGetLastError();
}

// The tile that takes all tokens at once, up to 128 of them: a larger one has
// products of nothing, a smaller one reads the rows more than once.  In us at
// 128256 x 2048 to bf16, with the tiles of 16, 32, 64, 128 and 256 tokens:
//    16 tokens   53   53   54   60   77
//    17          62   53   54   61   76
//    32          64   54   55   62   77
//    33          77   64   55   61   77
//    64          98   67   57   64   77
//    65         111   80   69   64   77
//   128         171  103   75   68   80
//   129         226  118   89   95   80
//   512         628  348  219  194  143
// Where the rows bound it, the tiles are as even as the rows allow.
template <bool OUT_BF16>
hipError_t tiles_launch(const Int8Launch &a, const int8_t *q, int pitch, const int8_t *x, const float *xs, hipStream_t s)
{
    if (a.B <= 16) return tile_launch<2, 1, 1, 128, 3, true, false, false, true, OUT_BF16>(a, q, pitch, x, xs, true, s);
    if (a.B <= 32) return tile_launch<2, 2, 1, 128, 3, true, false, false, true, OUT_BF16>(a, q, pitch, x, xs, true, s);
    if (a.B <= 64) return tile_launch<2, 4, 1, 128, 3, true, false, false, true, OUT_BF16>(a, q, pitch, x, xs, true, s);
    if (a.B <= 128) return tile_launch<4, 4, 2, 64, 4, true, false, false, true, OUT_BF16>(a, q, pitch, x, xs, false, s);
    return tile_launch<8, 4, 4, 128, 2, false, false, false, true, OUT_BF16>(a, q, pitch, x, xs, false, s);
}
template <bool H_BF16, bool OUT_BF16> hipError_t few_launch(const Int8Launch &a, bool aligned, hipStream_t s)
{
    if (aligned) return tile_launch<2, 1, 1, 128, 3, true, true, H_BF16, true, OUT_BF16>(a, a.q, a.d, nullptr, nullptr, true, s);
    return tile_launch<2, 1, 1, 128, 2, false, true, H_BF16, false, OUT_BF16>(a, a.q, a.d, nullptr, nullptr, true, s);
}
template <bool H_BF16> hipError_t few_launch(const Int8Launch &a, bool aligned, hipStream_t s)
{
    return a.out_dtype == VIE_BF16 ? few_launch<H_BF16, true>(a, aligned, s) : few_launch<H_BF16, false>(a, aligned, s);
}

// Rows of d bytes copied to rows of `pitch` bytes, a multiple of 16 (what
// lies past d meets zeros of the tokens): a wave per row.
__global__ __launch_bounds__(256) void repack_kernel(const int8_t *__restrict__ q, int64_t V, int d, int8_t *__restrict__ to, int pitch)
{
    for (int64_t v = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes; v < V; v += (int64_t)gridDim.x * (256 / kLanes))
        for (int c = 16 * (threadIdx.x & (kLanes - 1)); c < pitch; c += 16 * kLanes)
            *reinterpret_cast<word4 *>(to + v * pitch + c) = load16(q + v * d + c, q + V * d);
}
// Workgroups of 256 threads for n pieces of work: a launch holds fewer than
// 2^32 threads, so that those of the largest matrices take more than one.
unsigned grid_of(int64_t n) { return (unsigned)std::min<int64_t>(n, 1 << 22); }
int row_pitch(int d) { return (d + 15) / 16 * 16; }
// Whether unaligned rows are copied first: read and written once for it,
// where int8_simple_kernel reads them for every 16 tokens, and the worse the
// longer they are.  In us copied and not: 50257 x 1000, 32 tokens 34 and 31,
// 33 tokens 35 and 40, 64 tokens 35 and 52; 151936 x 1001, 32 tokens 87 and
// 98; 20000 x 4097, 17 tokens 51 and 110.
bool copy_rows(int B, int d) { return d % 16 != 0 && (B > 32 || d > 2048); }
}  // namespace

// The tokens' int8 values and scales, and unaligned rows copied.
size_t int8_workspace_bytes(int64_t V, int d, int B)
{
    // (rows at an odd address, of a multiple of 16 bytes, ask for less)
    if (hold_tokens(V, B, d, d % 16 == 0)) return 0;
    const size_t tokens = (tokens_bytes(d, B) + (size_t)B * 4 + 255) & ~(size_t)255;
    return tokens + (copy_rows(B, d) ? (size_t)V * row_pitch(d) : 0);
}

vie_status launch_int8_logits(const Int8Launch &a, hipStream_t s)
{
    auto done = [](hipError_t e) {
        return e == hipSuccess ? VIE_OK : fail(VIE_EHIP, "int8 head launch: %s", hipGetErrorString(e));
    };
    const bool bf16 = a.out_dtype == VIE_BF16, aligned = a.d % 16 == 0 && (uintptr_t)a.q % 16 == 0;
    if (hold_tokens(a.V, a.B, a.d, aligned))
        return done(a.h_dtype == VIE_BF16 ? few_launch<true>(a, aligned, s) : few_launch<false>(a, aligned, s));
    int8_t *x = static_cast<int8_t *>(a.ws);
    float *xs = reinterpret_cast<float *>(x + tokens_bytes(a.d, a.B));
    if (a.h_dtype == VIE_BF16) tokens_kernel<true><<<a.B, kTokenThreads, 0, s>>>(static_cast<const uint16_t *>(a.h), a.d, x, xs);
    else tokens_kernel<false><<<a.B, kTokenThreads, 0, s>>>(static_cast<const float *>(a.h), a.d, x, xs);
    if (vie_status e = launched("token quantization launch")) return e;
    const int8_t *q = a.q;
    int pitch = a.d;
    if (copy_rows(a.B, a.d)) {
        int8_t *to = x + ((tokens_bytes(a.d, a.B) + (size_t)a.B * 4 + 255) & ~(size_t)255);
        pitch = row_pitch(a.d);
        repack_kernel<<<grid_of((a.V + 3) / 4), 256, 0, s>>>(a.q, a.V, a.d, to, pitch);
        if (vie_status e = launched("int8 row copy launch")) return e;
        q = to;
    } else if (!aligned) {
        const dim3 grid(grid_of((a.V + 63) / 64), (unsigned)((a.B + 15) / 16));
        if (bf16)
            int8_simple_kernel<true><<<grid, 256, 0, s>>>(a.q, a.scale, a.V, a.d, x, xs, a.B, static_cast<uint16_t *>(a.out), a.ld);
        else
            int8_simple_kernel<false><<<grid, 256, 0, s>>>(a.q, a.scale, a.V, a.d, x, xs, a.B, static_cast<float *>(a.out), a.ld);
        return launched("int8 head launch");
    }
    return done(bf16 ? tiles_launch<true>(a, q, pitch, x, xs, s) : tiles_launch<false>(a, q, pitch, x, xs, s));
}

}  // namespace vie
