// fp32 products of a head's distillation for up to 16 tokens, which tiles of more rows waste most of themselves on: two read W once and are bound by that.
//   l[n, v] = sum_d X[n, d] W[v, d]      a warp takes four rows of W against all tokens, whose rows lie in shared memory; 64 sums a warp, halved from lane to lane
//   dW[v, d] = sum_n G[n, v] X[n, d]     bound by writing it, see there
//   dX[n, d] = sum_v G[n, v] W[v, d]     a thread takes four columns of a slice of W's rows; the slices' sums are added where rows go back to their tokens
// Calls for 4096 columns and a vocabulary of 32000 (W alone 80 us): forward 101 us for 1 token, 123 for 8, 225 for 16, dX 196, 251, 345, dW 209, 225, 349 (all with
// the logits).  4095 columns, 16 tokens: 255, 443, 367.  (Tiles of the CUDA-core product: 109 and 208 us for the first two of 12 x 656 of 45362, now 48 and
// 43; dW calls of 1 x 4096 287, of 16 x 4095 506.)
#include "head_loss.cuh"

namespace velora {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 26624;                              // floats of X in shared memory at most: columns of a chunk times tokens; two blocks fit an SM
constexpr int kStep = 128;                                 // columns that a warp takes at a time
constexpr int kColumnThreads = 128, kRows = 64;            // of dX: columns (or fours) of a block, rows of W whose gradients are in shared memory at a time

template <int V> struct Wide;
template <> struct Wide<4> {
    static __device__ __forceinline__ float4 load(const float* p) { return *reinterpret_cast<const float4*>(p); }
};
template <> struct Wide<1> {
    static __device__ __forceinline__ float4 load(const float* p) { return make_float4(*p, 0.f, 0.f, 0.f); }
};

// VEC 4: a lane takes four neighbouring columns (rows of W on 16-byte boundaries, D a multiple of four); 1: four that are 32 apart.
template <int TOKENS, int VEC>
__global__ void __launch_bounds__(kThreads, 2)
few_logits_kernel(const float* x, int64_t ldx, const float* W, int64_t ldw, float* C, int64_t ldc, int N, int D, int V, int pitch)
{
    constexpr int kSums = 4 * TOKENS;
    extern __shared__ __align__(16) float rows[];          // [TOKENS][pitch], zeros where there is nothing
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), warps = gridDim.x * (kThreads / 32);
    for (int d0 = 0; d0 < D; d0 += pitch) {
        const int columns = min(pitch, D - d0), padded = (columns + kStep - 1) / kStep * kStep;
        __syncthreads();                                   // the last chunk has been read
        for (int d = threadIdx.x; d < padded; d += kThreads) {
            float y[TOKENS];
#pragma unroll
            for (int n = 0; n < TOKENS; ++n) y[n] = x[min(n, N - 1) * ldx + d0 + min(d, columns - 1)];          // no branch: all under way
#pragma unroll
            for (int n = 0; n < TOKENS; ++n) rows[n * pitch + d] = n < N && d < columns ? y[n] : 0.f;
        }
        __syncthreads();
        for (int v = 4 * warp; v < V; v += 4 * warps) {
            const float* w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] = W + static_cast<int64_t>(min(v + r, V - 1)) * ldw + d0;
            float s[kSums];
#pragma unroll
            for (int i = 0; i < kSums; ++i) s[i] = 0.f;
#pragma unroll (TOKENS == 16 ? 1 : 2)
            for (int d = VEC * lane; d < padded; d += kStep) {          // 16 tokens leave no registers for a second step's loads (225 us -> 247)
                float y[4][4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {              // columns that are not there: the last ones, no branch
                    if (VEC == 4) {
                        const float4 u = *reinterpret_cast<const float4*>(w[r] + min(d, columns - 4));
                        y[r][0] = u.x; y[r][1] = u.y; y[r][2] = u.z; y[r][3] = u.w;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[r][e] = w[r][min(d + 32 * e, columns - 1)];
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[r][e] = d + (VEC == 4 ? e : 32 * e) < columns ? y[r][e] : 0.f;
#pragma unroll
                for (int n = 0; n < TOKENS; ++n) {
                    float z[4];
                    if (VEC == 4) {
                        const float4 u = *reinterpret_cast<const float4*>(rows + n * pitch + d);
                        z[0] = u.x; z[1] = u.y; z[2] = u.z; z[3] = u.w;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[e] = rows[n * pitch + d + 32 * e];
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[4 * n + r] = fmaf(y[r][e], z[e], s[4 * n + r]);
                }
            }
            // Lanes halve the sums that they carry until each has kSums / 32, or one that several share.
            int first = 0, o = 16;
#pragma unroll
            for (int k = kSums / 2; k > 0 && k >= kSums / 32; k /= 2, o /= 2) {
                const bool upper = (lane & o) != 0;
#pragma unroll
                for (int i = 0; i < k; ++i) {
                    const float give = upper ? s[i] : s[i + k], keep = upper ? s[i + k] : s[i];
                    s[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
                if (upper) first += k;
            }
#pragma unroll
            for (; o > 0; o /= 2) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
#pragma unroll
            for (int i = 0; i < (kSums >= 32 ? kSums / 32 : 1); ++i) {
                const int n = (first + i) / 4, r = (first + i) % 4;
                const bool mine = kSums >= 32 || (lane & (32 / (kSums < 32 ? kSums : 32) - 1)) == 0;          // one of those that share it
                if (mine && n < N && v + r < V) {
                    float* c = C + n * ldc + v + r;
                    *c = d0 > 0 ? *c + s[i] : s[i];
                }
            }
        }
    }
}

template <int TOKENS, int VEC>
__global__ void __launch_bounds__(kColumnThreads)
few_input_grad_kernel(const float* G, int64_t ldg, const float* W, int64_t ldw, float* sum, int64_t lds, int64_t slice_stride, int add, int N, int D, int V)
{
    __shared__ __align__(16) float g[kRows][TOKENS];
    pdl_wait();
    pdl_trigger();
    const int d = (blockIdx.x * kColumnThreads + threadIdx.x) * VEC, slice = blockIdx.y, slices = gridDim.y;
    const int v0 = static_cast<int>(static_cast<int64_t>(V) * slice / slices), v1 = static_cast<int>(static_cast<int64_t>(V) * (slice + 1) / slices);
    float s[TOKENS][VEC];
#pragma unroll
    for (int n = 0; n < TOKENS; ++n)
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[n][e] = 0.f;
    for (int v = v0; v < v1; v += kRows) {
        const int count = min(kRows, v1 - v);
        __syncthreads();                                   // the last rows have been read
        for (int i = threadIdx.x; i < kRows * TOKENS; i += kColumnThreads) {
            const int n = i / kRows, r = i % kRows;
            g[r][n] = n < N && r < count ? G[n * ldg + v + r] : 0.f;
        }
        __syncthreads();
        if (d < D) {
            const float* w = W + static_cast<int64_t>(v) * ldw + d;
#pragma unroll 8
            for (int r = 0; r < count; ++r, w += ldw) {
                const float4 y = Wide<VEC>::load(w);
#pragma unroll
                for (int n = 0; n < TOKENS; n += 4) {
                    const float4 z = *reinterpret_cast<const float4*>(&g[r][n]);
                    const float zs[4] = {z.x, z.y, z.z, z.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) s[n + k][e] = fmaf(zs[k], ys[e], s[n + k][e]);
                }
            }
        }
    }
    if (d >= D) return;
    float* out = sum + slice * slice_stride + d;
#pragma unroll
    for (int n = 0; n < TOKENS; ++n)
        if (n < N)
#pragma unroll
            for (int e = 0; e < VEC; ++e) out[n * lds + e] = add ? out[n * lds + e] + s[n][e] : s[n][e];
}

// A thread has four columns, VEC 4: neighbouring ones (rows of dW on 16-byte boundaries, D a multiple of four), 1: every 128th of the block's 512, and all
// tokens' X there in registers; a block walks along a slice of dW's rows.
template <int TOKENS, int VEC, typename T>
__global__ void __launch_bounds__(kColumnThreads)
few_weight_grad_kernel(const float* G, int64_t ldg, const float* x, int64_t ldx, T* dW, int64_t lddw, int beta, int N, int D, int V)
{
    constexpr int kApart = VEC == 4 ? 1 : kColumnThreads;
    __shared__ __align__(16) float g[kRows][TOKENS];
    pdl_wait();
    pdl_trigger();
    const int d = blockIdx.x * 4 * kColumnThreads + threadIdx.x * VEC, slice = blockIdx.y, slices = gridDim.y;
    const int v0 = static_cast<int>(static_cast<int64_t>(V) * slice / slices), v1 = static_cast<int>(static_cast<int64_t>(V) * (slice + 1) / slices);
    float y[TOKENS][4];
#pragma unroll
    for (int n = 0; n < TOKENS; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[n][e] = x[min(n, N - 1) * ldx + min(d + e * kApart, D - 1)];       // no branch: all under way; tokens that are not there have g = 0
#pragma unroll
    for (int n = 0; n < TOKENS; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) y[n][e] = n < N ? y[n][e] : 0.f;
    for (int v = v0; v < v1; v += kRows) {
        const int count = min(kRows, v1 - v);
        __syncthreads();                                   // the last rows have been read
        for (int i = threadIdx.x; i < kRows * TOKENS; i += kColumnThreads) {
            const int n = i / kRows, r = i % kRows;
            g[r][n] = n < N && r < count ? G[n * ldg + v + r] : 0.f;
        }
        __syncthreads();
        if (d >= D) continue;
        T* out = dW + static_cast<int64_t>(v) * lddw + d;
#pragma unroll 2
        for (int r = 0; r < count; ++r, out += lddw) {
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < TOKENS; n += 4) {
                const float4 z = *reinterpret_cast<const float4*>(&g[r][n]);
                const float zs[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[e] = fmaf(zs[k], y[n + k][e], s[e]);
            }
            if (beta) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (VEC == 4 || d + e * kApart < D) s[e] += Elem<T>::load(out + e * kApart);
            }
            if (VEC == 4 && sizeof(T) == 4) {
                *reinterpret_cast<float4*>(out) = make_float4(s[0], s[1], s[2], s[3]);
            } else if (VEC == 4) {
                *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (d + e * kApart < D) Elem<T>::store(out + e * kApart, s[e]);
            }
        }
    }
}

// The slices' sums, in order, to where the rows' tokens are: a block takes 32 columns of a row, a warp every eighth slice, 16 of them under way at once.
__global__ void __launch_bounds__(kThreads)
few_rows_back_kernel(const float* sum, int64_t lds, int64_t slice_stride, int slices, int D, const int* live, const int* order, float* dX, int64_t lddx)
{
    constexpr int kWarps = kThreads / 32;
    __shared__ float part[kWarps][32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.y, d = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (row < *live && d < D)
        for (int first = warp; first < slices; first += 16 * kWarps) {
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = sum[min(first + kWarps * i, slices - 1) * slice_stride + row * lds + d];       // no branch: all under way
#pragma unroll
            for (int i = 0; i < 16; ++i) s += first + kWarps * i < slices ? x[i] : 0.f;
        }
    part[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || d >= D) return;
    s = 0.f;
    for (int w = 0; w < kWarps; ++w) s += part[w][lane];
    dX[order[row] * lddx + d] = s;
}

bool four(const void* W, int64_t ldw, int64_t D) { return aligned16(W) && ldw % 4 == 0 && D % 4 == 0; }

template <int TOKENS, int VEC>
int launch_logits(const float* x, int64_t ldx, const float* W, int64_t ldw, float* C, int64_t ldc, int64_t N, int64_t D, int64_t V, int sm_count, cudaStream_t stream)
{
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    auto kern = few_logits_kernel<TOKENS, VEC>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kChunk * 4) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    const int64_t steps = ceil_div64(D, kStep), chunks = ceil_div64(steps, kChunk / TOKENS / kStep), pitch = ceil_div64(steps, chunks) * kStep;
    const size_t smem = static_cast<size_t>(TOKENS) * static_cast<size_t>(pitch) * 4;
    const int64_t fit = static_cast<int64_t>(216 * 1024 / smem), blocks = ceil_div64(V, 4 * (kThreads / 32)), most = static_cast<int64_t>(sm_count) * (fit < 2 ? fit : 2);
    return launch_chained(kern, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), kThreads, smem, stream, x, ldx, W, ldw, C, ldc,
                          static_cast<int>(N), static_cast<int>(D), static_cast<int>(V), static_cast<int>(pitch));
}

template <int TOKENS, int VEC>
int launch_grad(const float* G, int64_t ldg, const float* W, int64_t ldw, float* sum, int64_t lds, int slices, int add, int64_t N, int64_t D, int64_t V,
                cudaStream_t stream)
{
    return launch_chained(few_input_grad_kernel<TOKENS, VEC>, dim3(static_cast<unsigned>(ceil_div64(D, kColumnThreads * VEC)), static_cast<unsigned>(slices)),
                          kColumnThreads, 0, stream, G, ldg, W, ldw, sum, lds, N * lds, add, static_cast<int>(N), static_cast<int>(D), static_cast<int>(V));
}

template <int TOKENS, int VEC, typename T>
int launch_weight_grad(const float* G, int64_t ldg, const float* x, int64_t ldx, void* dW, int64_t lddw, int beta, int64_t N, int64_t D, int64_t V, int sm_count,
                       cudaStream_t stream)
{
    const int64_t across = ceil_div64(D, 4 * kColumnThreads), most = ceil_div64(V, kRows), fill = ceil_div64(static_cast<int64_t>(sm_count) * 8, across);
    return launch_chained(few_weight_grad_kernel<TOKENS, VEC, T>, dim3(static_cast<unsigned>(across), static_cast<unsigned>(fill < most ? fill : most)),
                          kColumnThreads, 0, stream, G, ldg, x, ldx, static_cast<T*>(dW), lddw, beta, static_cast<int>(N), static_cast<int>(D), static_cast<int>(V));
}
template <int VEC, typename T>
int launch_weight_grad(const float* G, int64_t ldg, const float* x, int64_t ldx, void* dW, int64_t lddw, int beta, int64_t N, int64_t D, int64_t V, int sm_count,
                       cudaStream_t stream)
{
    return N <= 4   ? launch_weight_grad<4, VEC, T>(G, ldg, x, ldx, dW, lddw, beta, N, D, V, sm_count, stream)
           : N <= 8 ? launch_weight_grad<8, VEC, T>(G, ldg, x, ldx, dW, lddw, beta, N, D, V, sm_count, stream)
                    : launch_weight_grad<16, VEC, T>(G, ldg, x, ldx, dW, lddw, beta, N, D, V, sm_count, stream);
}

}  // namespace

int launch_distill_few_weight_grad(const float* G, int64_t ldg, const float* x, int64_t ldx, void* dW, int dw_dtype, int64_t lddw, int beta, int64_t N, int64_t D,
                                   int64_t V, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    const bool vec = D % 4 == 0 && aligned16(dW) && lddw * static_cast<int64_t>(dtype_size(dw_dtype)) % 16 == 0;
    if (dw_dtype == VELORA_BF16)
        return vec ? launch_weight_grad<4, __nv_bfloat16>(G, ldg, x, ldx, dW, lddw, beta, N, D, V, di.sm_count, stream)
                   : launch_weight_grad<1, __nv_bfloat16>(G, ldg, x, ldx, dW, lddw, beta, N, D, V, di.sm_count, stream);
    return vec ? launch_weight_grad<4, float>(G, ldg, x, ldx, dW, lddw, beta, N, D, V, di.sm_count, stream)
               : launch_weight_grad<1, float>(G, ldg, x, ldx, dW, lddw, beta, N, D, V, di.sm_count, stream);
}

int distill_few_slices(int64_t D)
{
    const int64_t slices = 1184 / ceil_div64(D, 4 * kColumnThreads);          // eight blocks on each of 148 SMs
    return static_cast<int>(slices < 1 ? 1 : (slices > 256 ? 256 : slices));
}

int launch_distill_few_logits(const float* x, int64_t ldx, const float* W, int64_t ldw, float* C, int64_t ldc, int64_t N, int64_t D, int64_t V, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    if (four(W, ldw, D))
        return N <= 4   ? launch_logits<4, 4>(x, ldx, W, ldw, C, ldc, N, D, V, di.sm_count, stream)
               : N <= 8 ? launch_logits<8, 4>(x, ldx, W, ldw, C, ldc, N, D, V, di.sm_count, stream)
                        : launch_logits<16, 4>(x, ldx, W, ldw, C, ldc, N, D, V, di.sm_count, stream);
    return N <= 4   ? launch_logits<4, 1>(x, ldx, W, ldw, C, ldc, N, D, V, di.sm_count, stream)
           : N <= 8 ? launch_logits<8, 1>(x, ldx, W, ldw, C, ldc, N, D, V, di.sm_count, stream)
                    : launch_logits<16, 1>(x, ldx, W, ldw, C, ldc, N, D, V, di.sm_count, stream);
}

int launch_distill_few_grad(const float* G, int64_t ldg, const float* W, int64_t ldw, float* sum, int64_t lds, int slices, int add, int64_t N, int64_t D, int64_t V,
                            cudaStream_t stream)
{
    if (four(W, ldw, D))
        return N <= 4   ? launch_grad<4, 4>(G, ldg, W, ldw, sum, lds, slices, add, N, D, V, stream)
               : N <= 8 ? launch_grad<8, 4>(G, ldg, W, ldw, sum, lds, slices, add, N, D, V, stream)
                        : launch_grad<16, 4>(G, ldg, W, ldw, sum, lds, slices, add, N, D, V, stream);
    return N <= 4   ? launch_grad<4, 1>(G, ldg, W, ldw, sum, lds, slices, add, N, D, V, stream)
           : N <= 8 ? launch_grad<8, 1>(G, ldg, W, ldw, sum, lds, slices, add, N, D, V, stream)
                    : launch_grad<16, 1>(G, ldg, W, ldw, sum, lds, slices, add, N, D, V, stream);
}

int launch_distill_few_rows_back(const float* sum, int64_t lds, int slices, int64_t N, int64_t D, const int* live, const int* order, float* dX, int64_t lddx,
                                 cudaStream_t stream)
{
    return launch_chained(few_rows_back_kernel, dim3(static_cast<unsigned>(ceil_div64(D, 32)), static_cast<unsigned>(N)), kThreads, 0, stream, sum, lds, N * lds,
                          slices, static_cast<int>(D), live, order, dX, lddx);
}

}  // namespace velora
