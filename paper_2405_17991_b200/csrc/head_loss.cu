// Softmax cross entropy of a linear head without its logits, and its gradients.
//   l[n, v] = sum_d X[n, d] W[v, d],  lse[n] = log sum_v exp l[n, v],  loss[n] = lse[n] - l[n, t[n]]
//   G[n, v] = g[n] (exp(l[n, v] - lse[n]) - [v = t[n]]),   dX = G W,   dW = beta dW + G^T X
// The logits exist a piece of the vocabulary at a time.  Tokens without a target have no part in any of it; they are moved behind the
// others and their rows of X taken as zeros, so nothing that stands there (a NaN of an unused buffer) can reach dW through 0 * NaN.
#include "head_loss.cuh"

#include "gemm_store.cuh"
#include "gemm_tc.cuh"

namespace velora {

namespace {

constexpr int kRowThreads = 256;
// Logits that exist at a time where the workspace has the room: 128 MB in bf16 (fp32: half as many), but never fewer than 1024 columns of them.
constexpr int64_t kPieceElements = 1 << 26;
// Of the gradients' products: the operands are larger than L2 (backward pass of 8192 x 4096 of 32000: 5.38 ms in bands of 4, 5.26 in bands of 8).
constexpr int kBand = 8;
constexpr int kPieceStep = 256;                     // pieces are multiples of this

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
int64_t round_up(int64_t x, int64_t to) { return ceil_div64(x, to) * to; }

// Pieces of equal width, as few as fit the room but for up to two more where those fill the last wave of tiles better.  What a piece
// costs, in k-blocks of 256 x 256 tiles on 74 pairs: its products, and the sums of dX that each but the first reads and writes (about 9 k-blocks
// of a tile).
int64_t piece_width(int64_t N, int64_t D, int64_t V, int64_t room_cols)
{
    const int64_t tm = ceil_div64(N, 256), td = ceil_div64(D, 256), least = ceil_div64(V, room_cols);
    int64_t best = 0, best_cost = 0;
    for (int64_t p = least; p <= least + 2; ++p) {
        const int64_t cols = round_up(ceil_div64(V, p), kPieceStep), tv = cols / 256;
        const int64_t cost = p * (ceil_div64(tm * tv, 74) * ceil_div64(D, 64) + ceil_div64(tv * td, 74) * ceil_div64(N, 64) + ceil_div64(tm * td, 74) * (4 * tv + 9));
        if (best == 0 || cost < best_cost) {
            best = cols;
            best_cost = cost;
        }
    }
    return best;
}

int64_t room_wanted(int dtype, int64_t N, int64_t V)          // in columns
{
    const int64_t cols = (dtype == VELORA_BF16 ? kPieceElements : kPieceElements / 2) / N / kPieceStep * kPieceStep, all = round_up(V, kPieceStep);
    const int64_t least = cols < 4 * kPieceStep ? 4 * kPieceStep : cols;
    return least < all ? least : all;
}

// Up to 64 tokens the logits' gradients take two rows of bf16 each, the second what the first leaves: few of them do not average their
// roundings out (one token: dX and dW off by up to 4e-3), and the products' tiles have the rows to spare.
int gradient_rows(int dtype, int64_t N) { return dtype == VELORA_BF16 && N <= 64 ? 2 : 1; }

// Bytes of a token and column of the piece, one part.
size_t piece_element(int dtype, bool backward, int64_t N) { return dtype == VELORA_BF16 && backward ? 2 * static_cast<size_t>(gradient_rows(dtype, N)) : 4; }

// fp32 products of few tiles are cut into parts on the CUDA cores where that is estimated to be faster than either form of the whole
// product: 64 x 768 of 1000, whose four products took 51 us of its 59 in clusters.
int fp32_parts(int64_t M, int64_t N, int64_t K)
{
    if (M > 4096) return 1;                                     // the parts' sums would be large
    const SimtParts p = simt_parts(M, N, K);
    return p.parts > 1 && p.us < 0.9 * gemm_f32_us(M, N, K, 148) ? p.parts : 1;
}

// Parts of the contraction that dX's products are cut into, where its tiles are few: waves of units on 74 pairs, each its k-blocks and about
// 4 more for its sums' way.
int gradient_splits(int dtype, int64_t N, int64_t D, int64_t V)
{
    if (dtype != VELORA_BF16) return fp32_parts(N, D, piece_width(N, D, V, room_wanted(dtype, N, V)));
    if (N <= kHeadFew) return gradient_rows(dtype, N);          // the rows' sums, one behind the other
    const int64_t tiles = ceil_div64(N, 256) * ceil_div64(D, 256), kblocks = ceil_div64(piece_width(N, D, V, room_wanted(dtype, N, V)), 64);
    int best = 1;
    int64_t best_cost = 0;
    for (int s = 1; s <= 8 && s * 8 <= kblocks; ++s) {
        const int64_t cost = ceil_div64(tiles * s, 74) * (ceil_div64(kblocks, s) + 4);
        if (best_cost == 0 || cost < best_cost) {
            best = s;
            best_cost = cost;
        }
    }
    return best;
}

// The arrays in front of the piece; bf16 needs none for the forward pass.
HeadLayout head_front(bool backward, int dtype, int64_t N, int64_t D, int64_t V, bool pack_w, int splits)
{
    HeadLayout l{};
    const size_t n = static_cast<size_t>(N);
    size_t at = kStatusBytes;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    l.ldx = round_up(D, 8);
    l.live = take(4);
    l.order = take(4 * n);
    l.target = take(4 * n);
    if (backward) {
        l.common = take(4);
        l.scale = take(4 * n);
        l.lse = take(4 * n);
        l.splits = splits;
        l.sum = take(n * static_cast<size_t>(l.ldx) * 4 * static_cast<size_t>(l.splits));
    } else {
        l.at_target = take(4 * n);
        // fp32: one of a row; bf16: one of each 128 columns (of 256 rounded up), of a tile for few tokens.
        const size_t parts = dtype != VELORA_BF16 ? 1 : static_cast<size_t>(N <= kHeadFew ? ceil_div64(V, kHeadFewHeight) : 2 * ceil_div64(V, 256));
        l.running = take(8 * n * parts);
    }
    l.rows = backward ? gradient_rows(dtype, N) : 1;
    l.x = take(n * static_cast<size_t>(l.rows) * static_cast<size_t>(l.ldx) * dtype_size(dtype));
    if (pack_w) l.w = take(pack_rows_bytes(V, D));
    l.piece = at;
    return l;
}

int logit_parts(int dtype, int64_t N, int64_t D, int64_t V) { return dtype == VELORA_BF16 ? 1 : fp32_parts(N, piece_width(N, D, V, room_wanted(dtype, N, V)), D); }

// As many columns a piece as there is room for.
int head_layout(HeadLayout* l, bool backward, const HeadArgs& a)
{
    const bool pack_w = a.dtype == VELORA_BF16 && !tc_operand_ok(a.W, a.ldw);
    size_t column = piece_element(a.dtype, backward, a.N) * static_cast<size_t>(a.N);
    *l = head_front(backward, a.dtype, a.N, a.D, a.V, pack_w, backward ? gradient_splits(a.dtype, a.N, a.D, a.V) : 1);
    l->parts = logit_parts(a.dtype, a.N, a.D, a.V);
    if (a.ws_bytes < l->piece + column * l->parts * kPieceStep) {             // less room than asked for: no partial sums
        *l = head_front(backward, a.dtype, a.N, a.D, a.V, pack_w, backward ? gradient_rows(a.dtype, a.N) : 1);
        l->parts = 1;
    }
    column *= static_cast<size_t>(l->parts);
    if (a.ws_bytes < l->piece) return VELORA_ERR_WORKSPACE;
    if (a.dtype == VELORA_BF16 && !backward) return VELORA_OK;
    const int64_t fit = static_cast<int64_t>((a.ws_bytes - l->piece) / column) / kPieceStep * kPieceStep;
    if (fit < kPieceStep) return VELORA_ERR_WORKSPACE;
    const int64_t want = room_wanted(a.dtype, a.N, a.V);
    l->piece_cols = piece_width(a.N, a.D, a.V, fit < want ? fit : want);
    if (a.dtype != VELORA_BF16 || l->rows > 1) return VELORA_OK;
    // In every piece, the last and narrower one too, each part has k-blocks.
    const int64_t last = a.V - (ceil_div64(a.V, l->piece_cols) - 1) * l->piece_cols;
    auto fills = [](int64_t cols, int parts) { const int64_t kb = ceil_div64(cols, 64); return ceil_div64(kb, ceil_div64(kb, parts)) == parts; };
    while (l->splits > 1 && !(fills(last, l->splits) && (last == a.V || fills(l->piece_cols, l->splits)))) --l->splits;
    return VELORA_OK;
}

// ---- rows in order of having a target ----
// Every CTA counts all targets (8 bytes a token, from L2) rather than wait for another CTA's count, then moves its own rows.
struct RowsArgs {
    const void* X;
    int64_t ldx;
    const int64_t* target;
    const float* dloss;             // backward only
    const float* lse;
    int take_common;                // whether a factor is taken out of the dloss
    int N, V, D, rows_per_cta, copies;
    int* live;
    int* order;
    int* target_out;
    float* common;
    float* scale_out;
    float* lse_out;
    void* x_out;
    int64_t ldx_out;
    int* status;
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(kRowThreads)
head_rows_kernel(const RowsArgs a)
{
    __shared__ int counts[3];                         // live rows before this CTA's, all of them, bits of the largest |dloss|
    __shared__ int warp_live[kRowThreads / 32];
    __shared__ int row_to[kRowThreads];               // where a row goes; negative: -1 - that, and zeros are written
    pdl_wait();
    pdl_trigger();
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int r0 = blockIdx.x * a.rows_per_cta, r1 = min(a.N, r0 + a.rows_per_cta);
    if (t < 3) counts[t] = 0;
    __syncthreads();
    int before = 0, total = 0;
    float top = 0.f;
    for (int i0 = 0; i0 < a.N; i0 += kRowThreads * 8) {
        int64_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * kRowThreads + t;
            v[j] = i < a.N ? a.target[i] : -1;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int is = v[j] >= 0 && v[j] < a.V;
            total += is;
            before += is && i0 + j * kRowThreads + t < r0;
            if (is && a.take_common) top = fmaxf(top, fabsf(a.dloss[i0 + j * kRowThreads + t]));
        }
    }
    before = __reduce_add_sync(0xffffffffu, before);
    total = __reduce_add_sync(0xffffffffu, total);
    const int top_bits = static_cast<int>(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
    if (lane == 0) {
        atomicMax(&counts[2], top_bits);
        atomicAdd(&counts[0], before);
        atomicAdd(&counts[1], total);
    }
    __syncthreads();
    before = counts[0];
    total = counts[1];
    // The common factor: none where it could not be divided by.
    float common = __int_as_float(counts[2]);
    if (!(common >= 1.17549435e-38f && common <= 3.4e38f)) common = 1.f;
    if (blockIdx.x == 0 && blockIdx.y == 0 && t == 0) {
        *a.live = total;
        if (a.scale_out) *a.common = common;
    }
    for (int b0 = r0; b0 < r1; b0 += kRowThreads) {
        const int n = b0 + t;
        const int64_t v = n < r1 ? a.target[n] : -1;
        const bool is = v >= 0 && v < a.V;
        const unsigned votes = __ballot_sync(0xffffffffu, is);
        if (lane == 0) warp_live[warp] = __popc(votes);
        __syncthreads();
        int first = before, all = 0;
        for (int w = 0; w < kRowThreads / 32; ++w) {
            if (w < warp) first += warp_live[w];
            all += warp_live[w];
        }
        first += __popc(votes & ((1u << lane) - 1u));              // live rows before this one
        if (n < r1) {
            const int to = is ? first : total + (n - first);
            row_to[t] = is ? to : -1 - to;
            if (blockIdx.y == 0) {
                a.order[to] = n;
                a.target_out[to] = is ? static_cast<int>(v) : (v < 0 ? -1 : -2);
                if (a.scale_out) {
                    a.scale_out[to] = is ? a.dloss[n] / common : 0.f;
                    a.lse_out[to] = is ? a.lse[n] : 0.f;
                }
                if (v >= a.V && a.status) atomicCAS(a.status, 0, VELORA_ERR_INVALID_ARG);
            }
        }
        __syncthreads();
        // Few rows: the columns of each are shared out over the blocks of the grid's other direction.
        for (int i = warp; i < min(kRowThreads, r1 - b0); i += kRowThreads / 32) {
            const int code = row_to[i];
            const bool zero = code < 0;
            const T* src = static_cast<const T*>(a.X) + static_cast<int64_t>(b0 + i) * a.ldx;
            T* dst = static_cast<T*>(a.x_out) + static_cast<int64_t>(zero ? -1 - code : code) * a.ldx_out;
            const int64_t copy = static_cast<int64_t>(a.N) * a.ldx_out;
            if (VEC) {
                constexpr int per = 16 / sizeof(T);
                const int chunks = a.D / per;                      // D is a multiple of 8
#pragma unroll 4
                for (int c = lane + 32 * blockIdx.y; c < chunks; c += 32 * gridDim.y) {
                    const uint4 x = ld_stream_if(src + c * per, !zero);
                    reinterpret_cast<uint4*>(dst)[c] = x;
                    if (a.copies > 1) reinterpret_cast<uint4*>(dst + copy)[c] = x;
                }
            } else {
                for (int c = lane + 32 * blockIdx.y; c < a.ldx_out; c += 32 * gridDim.y) {
                    const float x = zero || c >= a.D ? 0.f : Elem<T>::load(src + c);
                    Elem<T>::store(dst + c, x);
                    if (a.copies > 1) Elem<T>::store(dst + copy + c, x);
                }
            }
        }
        before += all;
        __syncthreads();
    }
}

int launch_rows(const HeadArgs& a, const HeadLayout& l, const float* lse, const float* dloss, bool take_common)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    RowsArgs r{};
    r.X = a.X;
    r.ldx = a.ldx;
    r.target = a.target;
    r.N = static_cast<int>(a.N);
    r.V = static_cast<int>(a.V);
    r.D = static_cast<int>(a.D);
    r.live = reinterpret_cast<int*>(a.ws + l.live);
    r.order = reinterpret_cast<int*>(a.ws + l.order);
    r.target_out = reinterpret_cast<int*>(a.ws + l.target);
    if (dloss) {
        r.dloss = dloss;
        r.lse = lse;
        r.take_common = take_common ? 1 : 0;
        r.common = reinterpret_cast<float*>(a.ws + l.common);
        r.scale_out = reinterpret_cast<float*>(a.ws + l.scale);
        r.lse_out = reinterpret_cast<float*>(a.ws + l.lse);
    }
    r.x_out = a.ws + l.x;
    r.ldx_out = l.ldx;
    r.copies = l.rows;
    r.status = reinterpret_cast<int*>(a.ws);
    // Eight rows a CTA (one a warp) as long as that leaves no more than four CTAs per SM.
    const int64_t most = static_cast<int64_t>(di.sm_count) * 4;
    r.rows_per_cta = static_cast<int>(round_up(ceil_div64(a.N, most), 8));
    const int64_t ctas = ceil_div64(a.N, r.rows_per_cta), slices = ceil_div64(a.D, 512);          // of two chunks a lane and more
    const dim3 grid(static_cast<unsigned>(ctas), static_cast<unsigned>(ctas * slices <= di.sm_count ? slices : 1));
    const bool vec = a.D % 8 == 0 && aligned16(a.X) && (a.ldx * dtype_size(a.dtype)) % 16 == 0;
    if (a.dtype == VELORA_BF16)
        return vec ? launch_chained(head_rows_kernel<__nv_bfloat16, true>, grid, kRowThreads, 0, a.stream, r)
                   : launch_chained(head_rows_kernel<__nv_bfloat16, false>, grid, kRowThreads, 0, a.stream, r);
    return vec ? launch_chained(head_rows_kernel<float, true>, grid, kRowThreads, 0, a.stream, r)
               : launch_chained(head_rows_kernel<float, false>, grid, kRowThreads, 0, a.stream, r);
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

// A row's loss and log sum exp to where its token is.
__device__ __forceinline__ void write_loss(float* loss, float* lse, int n, int target, float m, float s, float at_target)
{
    const float l = m + logf(s);
    loss[n] = target >= 0 ? l - at_target : (target == -1 ? 0.f : __int_as_float(0x7fc00000));
    lse[n] = target >= 0 ? l : 0.f;
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

// A block per row takes the piece's maximum, then its exponentials, into what the pieces before have left; behind the last one the loss.  (A warp
// per row: 29 us for 64 rows of 8000, 4 us here.)
__global__ void __launch_bounds__(kRowThreads)
head_stats_kernel(float* logits, int64_t ld, int parts, int64_t part_stride, int cols, int v0, const int* live, const int* order, const int* target, float* at_target,
                  float2* running, int first, int last, float* loss, float* lse)
{
    __shared__ float part[2][kRowThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = target[row];
    float2 ms = make_float2(0.f, 1.f);
    float hit = 0.f;
    if (row < *live) {                                                // the same for the block
        float* l = logits + row * ld;
        float m = -INFINITY;
        if (parts > 1) {
            for (int c = threadIdx.x; c < cols; c += kRowThreads) {
                const float x = sum_of_parts(l + c, parts, part_stride);
                l[c] = x;                                             // read again by this thread, the target's behind a barrier
                m = fmaxf(m, x);
            }
        } else {
#pragma unroll 4
            for (int c = threadIdx.x; c < cols; c += kRowThreads) m = fmaxf(m, l[c]);
        }
        m = warp_max(m);
        if (lane == 0) part[0][warp] = m;
        __syncthreads();
        for (int w = 0; w < kRowThreads / 32; ++w) m = fmaxf(m, part[0][w]);
        const float2 old = first ? make_float2(-INFINITY, 0.f) : running[row];
        if (!first) hit = at_target[row];
        m = fmaxf(m, old.x);
        const float ref = m == -INFINITY ? 0.f : m;                  // nothing but minus infinities so far: their sum is 0
        const float before = old.y * expf(old.x - ref);
        float s = 0.f;
#pragma unroll 4
        for (int c = threadIdx.x; c < cols; c += kRowThreads) s += expf(l[c] - ref);
        s = warp_sum(s);
        if (lane == 0) part[1][warp] = s;
        __syncthreads();
        s = before;
        for (int w = 0; w < kRowThreads / 32; ++w) s += part[1][w];
        ms = make_float2(m, s);
        if (t >= v0 && t < v0 + cols) hit = l[t - v0];
        if (threadIdx.x == 0) {
            running[row] = ms;
            at_target[row] = hit;
        }
    }
    if (last && threadIdx.x == 0) write_loss(loss, lse, order[row], t, ms.x, ms.y, hit);
}

// A block takes 32 rows: eight slices of their parts (128 columns each), then the eight together.
__global__ void __launch_bounds__(kRowThreads)
head_merge_kernel(const float2* running, int parts, int N, const int* live, const int* order, const int* target, const float* at_target, float* loss, float* lse)
{
    __shared__ float2 slice[kRowThreads / 32][32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * 32 + lane;
    float m = -INFINITY, s = 0.f;
    if (row < *live) {
        for (int p0 = warp; p0 < parts; p0 += kRowThreads / 32 * 8) {        // eight loads in flight
            float2 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int p = p0 + kRowThreads / 32 * i;
                x[i] = p < parts ? running[static_cast<int64_t>(p) * N + row] : make_float2(-INFINITY, 0.f);
            }
            float both = m;
#pragma unroll
            for (int i = 0; i < 8; ++i) both = x[i].x > both ? x[i].x : (x[i].x == x[i].x ? both : x[i].x);      // a NaN stays one
            const float ref = both == -INFINITY ? 0.f : both;
            s *= expf(m - ref);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += x[i].y * expf(x[i].x - ref);
            m = both;
        }
    }
    slice[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (warp != 0 || row >= N) return;
    m = -INFINITY;
    bool nan = false;
    for (int w = 0; w < kRowThreads / 32; ++w) {
        m = fmaxf(m, slice[w][lane].x);
        nan |= slice[w][lane].x != slice[w][lane].x;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    s = nan ? __int_as_float(0x7fc00000) : 0.f;
    for (int w = 0; w < kRowThreads / 32; ++w) s += slice[w][lane].y * expf(slice[w][lane].x - ref);
    const int t = target[row];
    write_loss(loss, lse, order[row], t, m, s, t >= 0 ? at_target[row] : 0.f);
}

// Logits to their gradients, in place; a warp takes 128 columns of a row at a time, dealt over the blocks of its row.
__global__ void __launch_bounds__(kRowThreads)
head_gradient_kernel(float* logits, int64_t ld, int parts, int64_t part_stride, int cols, int v0, const int* target, const float* scale, const float* lse)
{
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* l = logits + row * ld;
    const int t = target[row] - v0;
    const bool is = target[row] >= 0;
    const float g = scale[row], z = lse[row];
    for (int c0 = (static_cast<int>(blockIdx.y) * (kRowThreads / 32) + warp) * 128; c0 < cols; c0 += static_cast<int>(gridDim.y) * (kRowThreads / 32) * 128) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = is && c0 + lane + 32 * i < cols ? sum_of_parts(l + c0 + lane + 32 * i, parts, part_stride) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = c0 + lane + 32 * i;
            if (c < cols) l[c] = is ? g * (expf(x[i] - z) - (c == t ? 1.f : 0.f)) : 0.f;
        }
    }
}

// dX from its fp32 sums, rows back to their tokens; eight columns a lane where dX's rows start on 16-byte boundaries.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kRowThreads)
head_rows_back_kernel(const float* sum, int64_t ld, int splits, int N, int D, const int* live, const int* order, const float* common, T* dX, int64_t lddx)
{
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= N) return;
    T* dst = dX + order[row] * lddx;
    const bool is = row < *live;
    const float f = *common;
    const int64_t stride = static_cast<int64_t>(N) * ld;
    if (VEC) {                                           // D is a multiple of 8
#pragma unroll 2
        for (int c = 8 * lane; c < D; c += 256) {
            float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int s = 0; s < splits; ++s) {
                const float* p = sum + s * stride + row * ld + c;
                const uint4 x = ld_stream_if(p, is), z = ld_stream_if(p + 4, is);
                y[0] += __uint_as_float(x.x); y[1] += __uint_as_float(x.y); y[2] += __uint_as_float(x.z); y[3] += __uint_as_float(x.w);
                y[4] += __uint_as_float(z.x); y[5] += __uint_as_float(z.y); y[6] += __uint_as_float(z.z); y[7] += __uint_as_float(z.w);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= f;
            if (sizeof(T) == 2)
                __stcs(reinterpret_cast<uint4*>(dst + c), make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])));
            else
                store_f32x8(reinterpret_cast<float*>(dst + c), y);
        }
    } else {
        for (int c = lane; c < D; c += 32) {
            float y = 0.f;
            for (int s = 0; is && s < splits; ++s) y += sum[s * stride + row * ld + c];
            Elem<T>::store(dst + c, y * f);
        }
    }
}

// C = beta C + op(A) op(B): the tensor cores where they take the operands.
int product(int kind, const void* A, int a_dtype, int64_t lda, const void* B, int b_dtype, int64_t ldb, void* C, int c_dtype, int64_t ldc, int beta,
            int64_t M, int64_t N, int64_t K, int* status, const GemmMore& more, cudaStream_t stream)
{
    if (a_dtype == b_dtype) {
        const int rc = launch_gemm_tc(kind, A, lda, B, ldb, C, c_dtype, ldc, beta, M, N, K, a_dtype, status, stream, more);
        if (rc != VELORA_ERR_UNSUPPORTED) return rc;
    }
    if (more.alpha) return VELORA_ERR_UNSUPPORTED;
    const bool a_t = kind == GEMM_TN_MN_MN, b_t = kind == GEMM_NT_K_K;
    return launch_gemm_simt(A, a_dtype, a_t ? 1 : lda, a_t ? lda : 1, B, b_dtype, b_t ? ldb : 1, b_t ? 1 : ldb, C, c_dtype, ldc, beta, M, N, K, stream);
}

}  // namespace

size_t head_loss_bytes(bool backward, int dtype, int64_t N, int64_t D, int64_t V, bool any_rows)
{
    if (N < 1) return kStatusBytes;
    const size_t front = head_front(backward, dtype, N, D, V, any_rows && dtype == VELORA_BF16, backward ? gradient_splits(dtype, N, D, V) : 1).piece;
    if (dtype == VELORA_BF16 && !backward) return front;
    return front + up256(piece_element(dtype, backward, N) * static_cast<size_t>(logit_parts(dtype, N, D, V)) * static_cast<size_t>(N) *
                         static_cast<size_t>(room_wanted(dtype, N, V)));
}

namespace {

// W as the tensor cores take it: a copy in the workspace where its rows do not start on 16-byte boundaries.
int head_weights(const HeadArgs& a, const HeadLayout& l, const char** W, int64_t* ldw)
{
    *W = static_cast<const char*>(a.W);
    *ldw = a.ldw;
    if (l.w == 0) return VELORA_OK;
    const PackJob job{a.W, a.ldw, a.V, a.D, a.ws + l.w};
    *W = a.ws + l.w;
    *ldw = pack_rows_pitch(a.D);
    return launch_pack_rows(&job, 1, a.stream);
}

// fp32 logits of a piece, in as many parts as it returns (up to the layout's).
int fp32_logits(const HeadArgs& a, const HeadLayout& l, const char* w, int64_t ldw, int64_t cols, int* rc)
{
    const float* x = reinterpret_cast<const float*>(a.ws + l.x);
    float* c = reinterpret_cast<float*>(a.ws + l.piece);
    const int parts = l.parts > 1 ? fp32_parts(a.N, cols, a.D) : 1;
    if (parts > 1 && parts <= l.parts) {
        *rc = launch_gemm_simt_parts(simt_parts(a.N, cols, a.D), x, l.ldx, 1, reinterpret_cast<const float*>(w), ldw, 1, c, l.piece_cols,
                                     a.N * l.piece_cols, 0, a.N, cols, a.D, a.stream);
        return parts;
    }
    *rc = product(GEMM_NT_K_K, x, VELORA_F32, l.ldx, w, VELORA_F32, ldw, c, VELORA_F32, l.piece_cols, 0, a.N, cols, a.D,
                  reinterpret_cast<int*>(a.ws), GemmMore{}, a.stream);
    return 1;
}

HeadTile head_tile(const HeadArgs& a, const HeadLayout& l, int64_t v0, int64_t cols)
{
    HeadTile h{};
    h.live = reinterpret_cast<const int*>(a.ws + l.live);
    h.target = reinterpret_cast<const int*>(a.ws + l.target);
    h.scale = reinterpret_cast<const float*>(a.ws + l.scale);
    h.lse = reinterpret_cast<const float*>(a.ws + l.lse);
    h.at_target = reinterpret_cast<float*>(a.ws + l.at_target);
    h.running = reinterpret_cast<float2*>(a.ws + l.running);
    h.N = static_cast<int>(a.N);
    h.D = static_cast<int>(a.D);
    h.cols = static_cast<int>(cols);
    h.v0 = static_cast<int>(v0);
    return h;
}

}  // namespace

int launch_head_loss(const HeadArgs& a, float* loss, float* lse)
{
    HeadLayout l;
    int rc = head_layout(&l, false, a);
    if (rc != VELORA_OK) return rc;
    const char* W;
    int64_t ldw;
    rc = head_weights(a, l, &W, &ldw);
    if (rc != VELORA_OK) return rc;
    rc = launch_rows(a, l, nullptr, nullptr, false);
    if (rc != VELORA_OK) return rc;
    int* status = reinterpret_cast<int*>(a.ws);
    const int n = static_cast<int>(a.N);
    if (a.dtype == VELORA_BF16) {
        const HeadTile h = head_tile(a, l, 0, a.V);
        const bool few = a.N <= kHeadFew;
        rc = few ? launch_head_few(a.ws + l.x, l.ldx, W, ldw, nullptr, 0, 0, h, status, a.stream)
                 : launch_head_tiles(a.ws + l.x, l.ldx, W, ldw, nullptr, 0, h, status, a.stream);
        if (rc != VELORA_OK) return rc;
        return launch_chained(head_merge_kernel, dim3(static_cast<unsigned>(ceil_div64(a.N, 32))), kRowThreads, 0, a.stream, h.running,
                              static_cast<int>(ceil_div64(a.V, few ? head_few_height(a.V) : 128)), n, h.live,
                              reinterpret_cast<int*>(a.ws + l.order), h.target, h.at_target, loss, lse);
    }
    float* piece = reinterpret_cast<float*>(a.ws + l.piece);
    for (int64_t v0 = 0; v0 < a.V; v0 += l.piece_cols) {
        const int64_t cols = a.V - v0 < l.piece_cols ? a.V - v0 : l.piece_cols;
        const int64_t part_stride = a.N * l.piece_cols;
        const int parts = fp32_logits(a, l, W + static_cast<size_t>(v0) * ldw * 4, ldw, cols, &rc);
        if (rc != VELORA_OK) return rc;
        rc = launch_chained(head_stats_kernel, dim3(static_cast<unsigned>(a.N)), kRowThreads, 0, a.stream, piece, l.piece_cols, parts,
                            part_stride, static_cast<int>(cols), static_cast<int>(v0),
                            reinterpret_cast<int*>(a.ws + l.live), reinterpret_cast<int*>(a.ws + l.order), reinterpret_cast<int*>(a.ws + l.target),
                            reinterpret_cast<float*>(a.ws + l.at_target), reinterpret_cast<float2*>(a.ws + l.running), v0 == 0 ? 1 : 0,
                            v0 + cols == a.V ? 1 : 0, loss, lse);
        if (rc != VELORA_OK) return rc;
    }
    return VELORA_OK;
}

int launch_head_loss_backward(const HeadArgs& a, const float* lse, const float* dloss, void* dX, int64_t lddx,
                              void* dW, int dw_dtype, int64_t lddw, int beta)
{
    HeadLayout l;
    int rc = head_layout(&l, true, a);
    if (rc != VELORA_OK) return rc;
    const char* W;
    int64_t ldw;
    rc = head_weights(a, l, &W, &ldw);
    if (rc != VELORA_OK) return rc;
    // In bf16 the logits' gradients are rounded once (more than 64 tokens), for the tensor cores: by half a step each.  A mean's 1 / count in
    // all of them would be the same rounding again and again, which does not average out (relative error of dX and dW up to 4e-3 by the
    // count alone); so the largest dloss is taken out and multiplied back in fp32, wherever the product that writes dW takes a factor.
    const bool take_common = a.dtype == VELORA_BF16 && (!dW || dw_dtype == VELORA_BF16 || c_rows_vec(dW, lddw, sizeof(float)));
    rc = launch_rows(a, l, lse, dloss, take_common);
    if (rc != VELORA_OK) return rc;
    int* status = reinterpret_cast<int*>(a.ws);
    const int n = static_cast<int>(a.N);
    const dim3 grid(static_cast<unsigned>(ceil_div64(a.N, kRowThreads / 32)));
    const int* live = reinterpret_cast<const int*>(a.ws + l.live);
    const float* common = reinterpret_cast<const float*>(a.ws + l.common);
    char* G = a.ws + l.piece;
    for (int64_t v0 = 0; v0 < a.V; v0 += l.piece_cols) {
        const int64_t cols = a.V - v0 < l.piece_cols ? a.V - v0 : l.piece_cols;
        const char* w = W + static_cast<size_t>(v0) * ldw * dtype_size(a.dtype);
        if (a.dtype == VELORA_BF16) {
            const HeadTile h = head_tile(a, l, v0, cols);
            rc = a.N <= kHeadFew ? launch_head_few(a.ws + l.x, l.ldx, w, ldw, G, l.piece_cols, l.rows > 1, h, status, a.stream)
                                 : launch_head_tiles(a.ws + l.x, l.ldx, w, ldw, G, l.piece_cols, h, status, a.stream);
        } else {
            const int parts = fp32_logits(a, l, w, ldw, cols, &rc);
            if (rc != VELORA_OK) return rc;
            const int64_t blocks = ceil_div64(cols, 128 * (kRowThreads / 32));
            rc = launch_chained(head_gradient_kernel, dim3(static_cast<unsigned>(a.N), static_cast<unsigned>(blocks < 16 ? blocks : 16)), kRowThreads,
                                0, a.stream, reinterpret_cast<float*>(G), l.piece_cols, parts, a.N * l.piece_cols, static_cast<int>(cols),
                                static_cast<int>(v0), reinterpret_cast<int*>(a.ws + l.target), reinterpret_cast<float*>(a.ws + l.scale),
                                reinterpret_cast<float*>(a.ws + l.lse));
        }
        if (rc != VELORA_OK) return rc;
        if (dW) {
            char* dw = static_cast<char*>(dW) + static_cast<size_t>(v0) * lddw * dtype_size(dw_dtype);
            rc = product(GEMM_TN_MN_MN, G, a.dtype, l.piece_cols, a.ws + l.x, a.dtype, l.ldx, dw, dw_dtype, lddw, beta, cols, a.D, a.N * l.rows, status,
                         GemmMore{l.rows > 1 ? nullptr : live, take_common ? common : nullptr, 1, 0, kBand}, a.stream);
            if (rc != VELORA_OK) return rc;
        }
        if (dX && a.dtype != VELORA_BF16 && l.splits > 1) {
            SimtParts shape = simt_parts(a.N, a.D, l.piece_cols);
            shape.parts = l.splits;
            rc = launch_gemm_simt_parts(shape, reinterpret_cast<float*>(G), l.piece_cols, 1, reinterpret_cast<const float*>(w), 1, ldw,
                                        reinterpret_cast<float*>(a.ws + l.sum), l.ldx, a.N * l.ldx, v0 > 0 ? 1 : 0, a.N, a.D, cols, a.stream);
            if (rc != VELORA_OK) return rc;
        } else if (dX) {
            rc = product(GEMM_NN_K_MN, G, a.dtype, l.piece_cols, w, a.dtype, ldw, a.ws + l.sum, VELORA_F32, l.ldx, v0 > 0 ? 1 : 0, a.N * l.rows, a.D, cols, status,
                         l.rows > 1 ? GemmMore{} : GemmMore{live, nullptr, l.splits, a.N * l.ldx, kBand}, a.stream);
            if (rc != VELORA_OK) return rc;
        }
    }
    if (!dX) return VELORA_OK;
    const float* sum = reinterpret_cast<float*>(a.ws + l.sum);
    const int d = static_cast<int>(a.D);
    const int* order = reinterpret_cast<const int*>(a.ws + l.order);
    const bool vec = a.D % 8 == 0 && c_rows_vec(dX, lddx, dtype_size(a.dtype));
    if (a.dtype == VELORA_BF16) {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(dX);
        return vec ? launch_chained(head_rows_back_kernel<__nv_bfloat16, true>, grid, kRowThreads, 0, a.stream, sum, l.ldx, l.splits, n, d, live, order, common, out, lddx)
                   : launch_chained(head_rows_back_kernel<__nv_bfloat16, false>, grid, kRowThreads, 0, a.stream, sum, l.ldx, l.splits, n, d, live, order, common, out, lddx);
    }
    float* out = static_cast<float*>(dX);
    return vec ? launch_chained(head_rows_back_kernel<float, true>, grid, kRowThreads, 0, a.stream, sum, l.ldx, l.splits, n, d, live, order, common, out, lddx)
               : launch_chained(head_rows_back_kernel<float, false>, grid, kRowThreads, 0, a.stream, sum, l.ldx, l.splits, n, d, live, order, common, out, lddx);
}

}  // namespace velora
