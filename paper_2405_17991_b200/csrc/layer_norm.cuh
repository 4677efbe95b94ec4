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
    float* partials;                // [2][slices][norm_pitch(D)]: sums of some rows each, for dw and for db
};

#ifdef __CUDACC__
__host__ __device__
#endif
inline int64_t norm_pitch(int64_t D) { return (D + 7) / 8 * 8; }
// Rows of `partials`, at most.
constexpr int kNormSlices = 296;
inline int64_t norm_slices(int64_t N) { return N < kNormSlices ? N : kNormSlices; }
// Blocks of `teams` rows at a time, up to `most`.  Where dw or db is asked for, each leaves a row of sums that is written and read: then one for four rows at
// the most, once there are 64 of them.
inline int64_t norm_grad_blocks(const NormGradArgs& a, int teams, int64_t most)
{
    const int64_t rounds = ceil_div64(a.N, teams), few = a.dw || a.db ? ceil_div64(rounds, 4) : rounds, blocks = few > 64 ? few : (rounds < 64 ? rounds : 64);
    if (most > kNormSlices) most = kNormSlices;
    return blocks < most ? blocks : most;
}

// Rows of any length (layer_norm_any.cu).
int launch_layer_norm_any(const NormArgs& a, int sm_count, cudaStream_t stream);
int launch_layer_norm_backward_any(const NormGradArgs& a, int sm_count, cudaStream_t stream);
// Rows that do not all start on 16-byte boundaries (layer_norm_odd.cu, layer_norm_backward_odd.cu).
int launch_layer_norm_odd(const NormArgs& a, int sm_count, cudaStream_t stream);
int launch_layer_norm_backward_odd(const NormGradArgs& a, int sm_count, cudaStream_t stream);
// dw and db = beta .. + the sums of `partials` over so many slices.
int launch_norm_slices(const NormGradArgs& a, int slices, cudaStream_t stream);

#ifdef __CUDACC__
__device__ __forceinline__ float load_param(const void* p, int dtype, int d, float none)
{
    if (!p) return none;
    return dtype == VELORA_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[d]) : static_cast<const float*>(p)[d];
}
__device__ __forceinline__ void store_param(void* p, int dtype, int d, float x, int beta)
{
    if (dtype == VELORA_BF16) {
        __nv_bfloat16* q = static_cast<__nv_bfloat16*>(p) + d;
        *q = __float2bfloat16_rn(beta ? __bfloat162float(*q) + x : x);
    } else {
        float* q = static_cast<float*>(p) + d;
        *q = beta ? *q + x : x;
    }
}

template <typename T> __device__ __forceinline__ float rounded(float x) { T t; Elem<T>::store(&t, x); return Elem<T>::load(&t); }
#endif

int launch_layer_norm(const NormArgs& a, cudaStream_t stream);
int launch_layer_norm_backward(const NormGradArgs& a, cudaStream_t stream);

}  // namespace velora
