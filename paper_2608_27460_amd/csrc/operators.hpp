// Internal declarations of the operators around the head's logits: the int8
// head, sampling and distillation (operators.cpp checks their arguments; the
// kernels are in int8_head.hip, sample.hip and distill.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "index.hpp"
#include "vie.h"

namespace vie {

constexpr int kMaxList = kMaxK + kMaxForced;  // longest candidate list a head returns

// ---- int8 head (int8_head.hip) -----------------------------------------

struct Int8Launch {
    const int8_t *q;     // [V][d]
    const float *scale;  // [V]
    int64_t V;
    int d;
    const void *h;       // [B][d] of h_dtype
    int h_dtype;
    int B;
    void *out;           // [B][ld] of out_dtype
    int out_dtype;
    int64_t ld;
    void *ws;
};
size_t int8_workspace_bytes(int64_t V, int d, int B);
vie_status launch_int8_logits(const Int8Launch &a, hipStream_t s);

// ---- sampling (sample.hip) ---------------------------------------------

struct SampleLaunch {
    const int32_t *ids;  // [B][n] for lists, nullptr for full rows
    const void *logits;  // [B][ld]
    int dtype;
    int64_t n, ld;       // candidates of a row, row stride
    int B;
    vie_sample_params prm;
    const float *u;
    int32_t *token;
    float *prob;         // may be nullptr
    int32_t *kept;       // may be nullptr
    void *ws;
};
size_t sample_rows_workspace_bytes(int64_t V, int B);
vie_status launch_sample_lists(const SampleLaunch &a, hipStream_t s);
vie_status launch_sample_rows(const SampleLaunch &a, hipStream_t s);

// ---- distillation (distill.hip) ----------------------------------------

struct DistillLaunch {
    const void *logits;  // [N][ld] of dtype
    int dtype;
    int N;
    int64_t V, ld;
    const int32_t *ids;  // [N][k]
    const float *teacher;
    int k;
    float tau;
    float *loss;         // [N]
    float *stats;        // [N][2]
    const float *gloss;  // [N] or nullptr
    float weight;
    void *grad;          // [N][grad_ld] of dtype
    int64_t grad_ld;
    void *ws;
};
size_t distill_workspace_bytes(int64_t V, int N);
vie_status launch_distill(const DistillLaunch &a, hipStream_t s);
vie_status launch_distill_grad(const DistillLaunch &a, hipStream_t s);
vie_status launch_distill_step(const DistillLaunch &a, hipStream_t s);

}  // namespace vie
