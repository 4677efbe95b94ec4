// Softmax cross entropy of a linear head without its logits, and its gradients: layout of the workspace and the pieces.
#pragma once

#include "common.cuh"

namespace velora {

// Where things lie in a call's workspace, in bytes from its start.  Rows of the arrays below are the tokens in another order: those with
// a target first, in their own order, then the others; `order` says which token a row is.
struct HeadLayout {
    size_t live;            // int32: how many rows have a target
    size_t order;           // int32[N]
    size_t target;          // int32[N]: column, -1 without one, -2 where it is no column
    size_t common;          // fp32: the largest |dloss| of a row with a target, a factor taken out of all of them (backward)
    size_t scale, lse;      // fp32[N]: what is left of the row's dloss, log sum exp (backward)
    size_t at_target;       // fp32[N]: logit of the target (forward)
    size_t running;         // float2[N], or float2[parts of the vocabulary][N]: maximum, and the sum of exponentials relative to it (forward)
    size_t x;               // the rows of X, pitch ldx elements; zeros for rows without a target
    size_t w;               // W with a pitch that tensor maps take, where W's own is not
    size_t sum;             // fp32, pitch ldx: dX so far, `splits` partial sums (backward)
    size_t piece;           // a piece of the vocabulary: logits or their gradient, pitch `piece_cols` elements
    int64_t ldx, piece_cols;
    int rows;               // copies of the rows of X, and rows of the logits' gradients for each (backward)
    int splits, parts;      // partial sums of dX; of the logits (fp32), one piece behind another
    size_t bytes;
};

struct HeadArgs {
    const void* X;
    int64_t ldx;
    const void* W;
    int64_t ldw;
    const int64_t* target;
    int dtype;
    int64_t N, D, V;
    char* ws;
    size_t ws_bytes;
    cudaStream_t stream;
};

// A product's worth of logits, columns v0 .. v0 + cols of the vocabulary; arrays as in HeadLayout.
struct HeadTile {
    const int* live;
    const int* target;
    const float* scale;
    const float* lse;
    float* at_target;
    float2* running;
    int N, D, cols, v0;
};
// G == nullptr: statistics of bf16 x W^T; otherwise its gradient to G [N, ldg].  W: its row v0.  (head_loss_tc.cu)
int launch_head_tiles(const void* x, int64_t ldx, const void* W, int64_t ldw, void* G, int64_t ldg, const HeadTile& h, int* status, cudaStream_t stream);

// The same for up to kHeadFew tokens; `twice`: what the gradient's rounding to bf16 leaves of it goes to rows N .. 2 N - 1.  (head_loss_few.cu)
constexpr int kHeadFew = 128;
constexpr int kHeadFewHeight = 64;                  // least height of its tiles
int head_few_height(int64_t cols);                  // columns of the vocabulary in a tile: a row of `running` each
int launch_head_few(const void* x, int64_t ldx, const void* W, int64_t ldw, void* G, int64_t ldg, int twice, const HeadTile& h, int* status, cudaStream_t stream);

// k-blocks of 64 whose products an accumulator of the tensor cores adds up; segments are added in registers, rounded to nearest.  The same for both
// kernels and both passes: G's 1 - p of a token that the head is sure of has no other source than logits equal to those in lse.
constexpr int kHeadSegment = 8;

#ifdef __CUDACC__
constexpr float kHeadLog2e = 1.4426950408889634f;
constexpr float kHeadLost = 0x1p-8f;                // rounding of a maximum times log2 e that a first-order term makes up for (to 4e-6 of the sum)
__device__ __forceinline__ float head_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
#endif

// What velora_workspace_bytes reports.
size_t head_loss_bytes(bool backward, int dtype, int64_t N, int64_t D, int64_t V, bool any_rows);
int launch_head_loss(const HeadArgs& a, float* loss, float* lse);
int launch_head_loss_backward(const HeadArgs& a, const float* lse, const float* dloss, void* dX, int64_t lddx,
                              void* dW, int dw_dtype, int64_t lddw, int beta);

}  // namespace velora
