// Root-mean-square norm (gfx950): arguments of its kernels.
#pragma once
#include "dfa_scaled.h"

namespace dfa {

constexpr int64_t kNormMaxCols = 32768;     // a row is held in registers: 1024 threads of 32 elements

struct NormParams {
    const void *x, *residual, *weight;      // [M][C] with row pitches; residual and weight may be NULL
    int64_t ldx, ldr;
    int64_t M, C;
    float eps;
    void *h, *y;                            // may be NULL
    int64_t ldh, ldy;
    uint8_t *values, *scales;               // may be NULL: y in blocks of 128 (dfa_scaled.h)
    int64_t ldv, lds;
};
// The forward's launch.  (The gradients' workgroups walk along the rows: any number of them.)
struct NormGrid {
    int64_t workgroups;
    int32_t threads;                        // of each
};
NormGrid norm_grid(int64_t M, int64_t C);
hipError_t launch_norm(const NormParams& p, bool f32, bool weight_f32, hipStream_t st);

struct NormBackwardParams {
    const void *dy, *h, *weight, *dh;       // dh and weight may be NULL
    int64_t lddy, ldh, lddh;
    int64_t M, C;
    float eps;
    void* dx;
    int64_t lddx;
    float* dw;                              // [C] or NULL
    float* parts;                           // [workgroups][C] workspace where there is more than one
    int32_t workgroups;
};
int32_t norm_backward_workgroups(int64_t M, int64_t C, bool f32, const ChipShape& chip);
hipError_t launch_norm_backward(const NormBackwardParams& p, bool f32, bool weight_f32, hipStream_t st);

}  // namespace dfa
