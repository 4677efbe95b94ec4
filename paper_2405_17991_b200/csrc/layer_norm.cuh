// Layer norm of rows, with a residual added in front, and its gradients (layer_norm.cu).
#pragma once

#include "common.cuh"

namespace velora {

struct NormArgs {
    const void* X;
    int64_t ldx;
    const void* R;                  // NULL: nothing is added
    int64_t ldr;
    const void* w;                  // NULL: ones
    const void* b;                  // NULL: zeros
    int p_dtype;                    // of w and b
    float eps;
    void* H;                        // X + R; may be NULL
    int64_t ldh;
    void* Y;
    int64_t ldy;
    float* mean;                    // may be NULL, as rstd
    float* rstd;
    int dtype;
    int64_t N;
    int D;
};

struct NormGradArgs {
    const void* dY;
    int64_t lddy;
    const void* H;
    int64_t ldh;
    const float* mean;
    const float* rstd;
    const void* w;
    int p_dtype;
    const void* dH;                 // added to dX; may be NULL
    int64_t lddh;
    void* dX;                       // may be NULL, as dw and db
    int64_t lddx;
    void* dw;
    void* db;
    int dw_dtype;                   // of dw and db
    int beta;
    int dtype;
    int64_t N;
    int D;
    float* partials;                // [2][slices][D]: sums of some rows each, for dw and for db
};

// Rows of `partials`, at most.
constexpr int kNormSlices = 296;
inline int64_t norm_slices(int64_t N) { return N < kNormSlices ? N : kNormSlices; }

int launch_layer_norm(const NormArgs& a, cudaStream_t stream);
int launch_layer_norm_backward(const NormGradArgs& a, cudaStream_t stream);

}  // namespace velora
