// Layer norm and its gradients (formulas: layer_norm.cu) of rows of any length, one element at a time, each row read several times (from L1 or L2 but for
// the first): for rows that are too long to be held.  And the sum of the slices of dw and db, for these and the others.
#include "layer_norm.cuh"

namespace velora {

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;

// Sums over the block, the same in every thread.
__device__ __forceinline__ float2 block_sum(float x, float y, float2* part)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        x += __shfl_xor_sync(0xffffffffu, x, o);
        y += __shfl_xor_sync(0xffffffffu, y, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = make_float2(x, y);
    __syncthreads();
    float2 s = make_float2(0.f, 0.f);
    for (int w = 0; w < kWarps; ++w) {
        s.x += part[w].x;
        s.y += part[w].y;
    }
    return s;
}

// A block per row, three times over it.
template <typename T>
__global__ void __launch_bounds__(kThreads)
norm_any_kernel(const NormArgs a)
{
    __shared__ float2 part[kWarps];
    pdl_wait();
    pdl_trigger();
    const float inverse = 1.f / static_cast<float>(a.D);
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
        const T* x = static_cast<const T*>(a.X) + n * a.ldx;
        const T* r = a.R ? static_cast<const T*>(a.R) + n * a.ldr : nullptr;
        T* h = a.H ? static_cast<T*>(a.H) + n * a.ldh : nullptr;
        T* y = static_cast<T*>(a.Y) + n * a.ldy;
        auto value = [&](int d) { return r ? rounded<T>(Elem<T>::load(x + d) + Elem<T>::load(r + d)) : Elem<T>::load(x + d); };
        float sum = 0.f;
        for (int d = threadIdx.x; d < a.D; d += kThreads) sum += value(d);
        const float m = block_sum(sum, 0.f, part).x * inverse;
        sum = 0.f;
        for (int d = threadIdx.x; d < a.D; d += kThreads) {
            const float c = value(d) - m;
            sum += c * c;
        }
        const float s = 1.f / sqrtf(block_sum(sum, 0.f, part).x * inverse + a.eps);
        for (int d = threadIdx.x; d < a.D; d += kThreads) {
            const float v = value(d);
            if (h) Elem<T>::store(h + d, v);
            Elem<T>::store(y + d, (v - m) * s * load_param(a.w, a.p_dtype, d, 1.f) + load_param(a.b, a.p_dtype, d, 0.f));
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[n] = m;
            if (a.rstd) a.rstd[n] = s;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
norm_grad_any_kernel(const NormGradArgs a)
{
    __shared__ float2 part[kWarps];
    pdl_wait();
    pdl_trigger();
    const float inverse = 1.f / static_cast<float>(a.D);
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
        const T* dy = static_cast<const T*>(a.dY) + n * a.lddy;
        const T* h = static_cast<const T*>(a.H) + n * a.ldh;
        const T* dh = a.dH ? static_cast<const T*>(a.dH) + n * a.lddh : nullptr;
        T* dx = static_cast<T*>(a.dX) + n * a.lddx;
        const float m = a.mean[n], s = a.rstd[n];
        float sum = 0.f, along = 0.f;
        for (int d = threadIdx.x; d < a.D; d += kThreads) {
            const float c = Elem<T>::load(dy + d) * load_param(a.w, a.p_dtype, d, 1.f);
            sum += c;
            along += c * ((Elem<T>::load(h + d) - m) * s);
        }
        const float2 t = block_sum(sum, along, part);
        const float mean_c = t.x * inverse, mean_cx = t.y * inverse;
        for (int d = threadIdx.x; d < a.D; d += kThreads) {
            const float c = Elem<T>::load(dy + d) * load_param(a.w, a.p_dtype, d, 1.f);
            const float g = s * (c - mean_c - (Elem<T>::load(h + d) - m) * s * mean_cx);
            Elem<T>::store(dx + d, dh ? Elem<T>::load(dh + d) + g : g);
        }
    }
}

// Sums over a slice of the rows: a thread a column.
template <typename T>
__global__ void __launch_bounds__(kThreads)
norm_columns_kernel(const NormGradArgs a, int slices)
{
    pdl_wait();
    pdl_trigger();
    const int d = blockIdx.x * kThreads + threadIdx.x, slice = blockIdx.y;
    if (d >= a.D) return;
    const int64_t n0 = a.N * slice / slices, n1 = a.N * (slice + 1) / slices;
    float dw = 0.f, db = 0.f;
    for (int64_t n = n0; n < n1; ++n) {
        const float dy = Elem<T>::load(static_cast<const T*>(a.dY) + n * a.lddy + d);
        dw += dy * ((Elem<T>::load(static_cast<const T*>(a.H) + n * a.ldh + d) - a.mean[n]) * a.rstd[n]);
        db += dy;
    }
    a.partials[static_cast<int64_t>(slice) * norm_pitch(a.D) + d] = dw;
    a.partials[static_cast<int64_t>(slices + slice) * norm_pitch(a.D) + d] = db;
}

// The slices' sums in a fixed order: a block takes 32 columns of dw or db, a warp every 32nd slice, ten loads under way at once, which all of kNormSlices are.
constexpr int kSliceWarps = 32, kSliceLoads = 10;
static_assert(kSliceWarps * kSliceLoads >= kNormSlices, "one round");
__global__ void __launch_bounds__(32 * kSliceWarps)
norm_slices_kernel(const float* partials, int slices, int D, void* dw, void* db, int dtype, int beta)
{
    __shared__ float part[kSliceWarps][33];
    pdl_wait();
    pdl_trigger();
    void* out = blockIdx.y ? db : dw;
    if (!out) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = blockIdx.x * 32 + lane;
    const int64_t pitch = norm_pitch(D);
    const float* p = partials + blockIdx.y * slices * pitch + d;
    float x[kSliceLoads];
#pragma unroll
    for (int i = 0; i < kSliceLoads; ++i) x[i] = d < D && warp + kSliceWarps * i < slices ? p[(warp + kSliceWarps * i) * pitch] : 0.f;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kSliceLoads; ++i) s += x[i];
    part[warp][lane] = s;
    __syncthreads();
    s = part[lane][warp];                                     // column blockIdx.x * 32 + warp, of warp `lane`
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0 && blockIdx.x * 32 + warp < D) store_param(out, dtype, blockIdx.x * 32 + warp, s, beta);
}

template <typename T>
int norm_any(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    const int64_t most = static_cast<int64_t>(sm_count) * 4;
    return launch_chained(norm_any_kernel<T>, dim3(static_cast<unsigned>(a.N < most ? a.N : most)), kThreads, 0, stream, a);
}

template <typename T>
int norm_grad_any(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    if (a.dw || a.db) {                                       // first: dX may lie where dY or H does
        const int slices = static_cast<int>(norm_slices(a.N));
        int rc = launch_chained(norm_columns_kernel<T>, dim3(static_cast<unsigned>(ceil_div64(a.D, kThreads)), static_cast<unsigned>(slices)), kThreads, 0,
                                stream, a, slices);
        if (rc != VELORA_OK) return rc;
        rc = launch_norm_slices(a, slices, stream);
        if (rc != VELORA_OK) return rc;
    }
    if (!a.dX) return VELORA_OK;
    const int64_t most = static_cast<int64_t>(sm_count) * 4;
    return launch_chained(norm_grad_any_kernel<T>, dim3(static_cast<unsigned>(a.N < most ? a.N : most)), kThreads, 0, stream, a);
}

}  // namespace

int launch_layer_norm_any(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    return a.dtype == VELORA_BF16 ? norm_any<__nv_bfloat16>(a, sm_count, stream) : norm_any<float>(a, sm_count, stream);
}

int launch_layer_norm_backward_any(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    return a.dtype == VELORA_BF16 ? norm_grad_any<__nv_bfloat16>(a, sm_count, stream) : norm_grad_any<float>(a, sm_count, stream);
}

int launch_norm_slices(const NormGradArgs& a, int slices, cudaStream_t stream)
{
    return launch_chained(norm_slices_kernel, dim3(static_cast<unsigned>(ceil_div64(a.D, 32)), 2), 32 * kSliceWarps, 0, stream, a.partials, slices, a.D,
                          a.dw, a.db, a.dw_dtype, a.beta);
}

}  // namespace velora
