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
    size_t common;          // fp32: the largest |dloss| of a row with a target, over the temperature, a factor taken out of all of them (backward)
    size_t scale, lse;      // fp32[N]: what is left of the row's dloss over the temperature, log sum exp (backward)
    size_t at_target;       // fp32[N]: logit of the target (forward)
    size_t running;         // float2[N], or float2[parts of the vocabulary][N]: maximum, and the sum of exponentials relative to it (forward)
    size_t x;               // the rows of X, pitch ldx elements; zeros for rows without a target
    size_t w;               // W with a pitch that tensor maps take, where W's own is not
    size_t sum;             // fp32, pitch ldx: dX so far, `splits` partial sums (backward)
    // Distillation, by token: a target for the arrays above, entries and their probabilities in the order of their columns, where each 128
    // columns' entries start, the probabilities' sum, the entries' logits (forward)
    size_t mark, entries, starts, mass, at_entries;
    size_t piece;           // a piece of the vocabulary: logits or their gradient, pitch `piece_cols` elements
    int64_t ldx, piece_cols;
    int rows;               // copies of the rows of X, and rows of the logits' gradients for each (backward)
    int splits, parts;      // partial sums of dX; of the logits (fp32), one piece behind another
    size_t bytes;
};

// What a teacher says of the next token: K columns and logits a token (distill.cu).
struct Teacher {
    const int64_t* index;
    int64_t ldi;
    const void* logits;
    int t_dtype;
    int64_t ldt;
    const float* lse;               // NULL: of the K entries
    float temperature;
    int K;
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
    const Teacher* teacher;         // NULL: a target a token
};

// An entry of a teacher's list: the column and its probability.
struct Entry {
    int column;
    float p;
};
constexpr int kEntryColumns = 128;                  // of `starts`: entries of columns 128 b .. are entries[starts[b]] .. before entries[starts[b + 1]]
struct Entries {
    const Entry* entries;                           // [token][K], in the order of their columns
    const unsigned short* starts;                   // [token][pitch]
    const float* mass;                              // [token]
    const int* order;                               // token of a row
    float* at;                                      // [token][K]: logits over the temperature (forward)
    int K, pitch;
    float inverse_t;                                // 1 / temperature
};
inline int entry_pitch(int64_t V) { return static_cast<int>(ceil_div64(V, kEntryColumns)) + 1; }

// A product's worth of logits, columns v0 .. v0 + cols of the vocabulary; arrays as in HeadLayout.
struct HeadTile {
    const int* live;
    const int* target;
    const float* scale;
    const float* lse;
    float* at_target;
    float2* running;
    int N, D, cols, v0;
    Entries e;                      // entries == nullptr: a target a row
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
__device__ __forceinline__ float warp_max(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// In a fixed order; up to 16, all under way at once.
__device__ __forceinline__ float sum_of_parts(const float* p, int parts, int64_t stride)
{
    float x[16];
#pragma unroll
    for (int s = 0; s < 16; ++s) x[s] = s < parts ? p[s * stride] : 0.f;
    float y = x[0];
#pragma unroll
    for (int s = 1; s < 16; ++s)
        if (s < parts) y += x[s];
    return y;
}

constexpr int kNoColumn = 1 << 30;
// The entries of a row that lie in some columns from `first` on, one after the other; the one behind the current is on its way.
struct EntryWalk {
    const Entry* list;
    int j, end, first;
    int column, next_column;                        // from `first` on; kNoColumn behind the last
    float p, next_p;
    __device__ __forceinline__ void fetch(int at)
    {
        next_column = kNoColumn;
        if (at < end) {
            const Entry e = list[at];
            next_column = e.column - first;
            next_p = e.p;
        }
    }
    __device__ __forceinline__ void next()
    {
        ++j;
        column = next_column;
        p = next_p;
        fetch(j + 1);
    }
    // Entries j0 .. before j1 of a token's list, counted from column `from` on (negative: in front of it).
    __device__ __forceinline__ void begin(const Entries& e, int token, int j0, int j1, int from)
    {
        list = e.entries + static_cast<int64_t>(token) * e.K;
        j = j0;
        end = j1;
        first = from;
        fetch(j);
        column = next_column;
        p = next_p;
        fetch(j + 1);
    }
    // The first of which, where there is one, has been loaded.
    __device__ __forceinline__ void begin(const Entries& e, int token, int j0, int j1, int from, Entry head)
    {
        list = e.entries + static_cast<int64_t>(token) * e.K;
        j = j0;
        end = j1;
        first = from;
        column = j < end ? head.column - first : kNoColumn;
        p = head.p;
        fetch(j + 1);
    }
    __device__ __forceinline__ void none()
    {
        list = nullptr;
        j = end = 0;
        column = next_column = kNoColumn;
    }
};
// Where a row's entries of a tile's 128 columns are; looked up a tile ahead in two steps, since each waits for memory.
struct EntryPlace {
    int token;                                      // negative: the row has no part in it
    int j, end;
    __device__ __forceinline__ void find_token(const Entries& e, const int* target, int row, bool is)
    {
        token = -1;
        if (is && target[row] >= 0) token = e.order[row];
    }
    __device__ __forceinline__ void find_entries(const Entries& e, int column)
    {
        j = end = 0;
        if (token >= 0) {
            const unsigned short* s = e.starts + static_cast<int64_t>(token) * e.pitch + column / kEntryColumns;
            j = s[0];
            end = s[1];
        }
    }
};
#endif

// What velora_workspace_bytes reports.
size_t head_loss_bytes(bool backward, int dtype, int64_t N, int64_t D, int64_t V, bool any_rows, int K = 0);      // K > 0: distillation
// Distillation's own kernels (distill.cu).
Entries distill_entries(const HeadArgs& a, const HeadLayout& l);
int launch_distill_lists(const HeadArgs& a, const HeadLayout& l);
// fp32: parts of the rows' statistics to `running`, from row *part on, which moves behind them; never more than one for 256 columns.
int launch_distill_stats(const float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile& h, int* part, cudaStream_t stream);
int launch_distill_gradient(float* logits, int64_t ld, int parts, int64_t part_stride, const HeadTile& h, cudaStream_t stream);
int launch_distill_merge(const HeadTile& h, int parts, float* loss, float* lse, cudaStream_t stream);
// Its fp32 products for up to kDistillFew tokens (distill_few.cu): logits, and slices of dX's sums, N lds apart, that are added to what is there (`add`) or
// written; then those to dX.
constexpr int kDistillFew = 16;
int distill_few_slices(int64_t D);
int launch_distill_few_logits(const float* x, int64_t ldx, const float* W, int64_t ldw, float* C, int64_t ldc, int64_t N, int64_t D, int64_t V, cudaStream_t stream);
int launch_distill_few_rows_back(const float* sum, int64_t lds, int slices, int64_t N, int64_t D, const int* live, const int* order, float* dX, int64_t lddx,
                                 cudaStream_t stream);
int launch_distill_few_grad(const float* G, int64_t ldg, const float* W, int64_t ldw, float* sum, int64_t lds, int slices, int add, int64_t N, int64_t D, int64_t V,
                            cudaStream_t stream);
// dW or, with beta, more of it, from the piece's gradients and the rows of X.
int launch_distill_few_weight_grad(const float* G, int64_t ldg, const float* x, int64_t ldx, void* dW, int dw_dtype, int64_t lddw, int beta, int64_t N, int64_t D,
                                   int64_t V, cudaStream_t stream);
int launch_head_loss(const HeadArgs& a, float* loss, float* lse);
int launch_head_loss_backward(const HeadArgs& a, const float* lse, const float* dloss, void* dX, int64_t lddx,
                              void* dW, int dw_dtype, int64_t lddw, int beta);

}  // namespace velora
