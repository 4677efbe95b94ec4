// Layer norm of rows, with a residual added in front, and its gradients.
//   h = x + r (rounded to the rows' type),  m = mean h,  s = 1 / sqrt(mean (h - m)^2 + eps),  xhat = (h - m) s,  y = xhat w + b
//   c = dy w,  dx = dh + s (c - mean c - xhat mean(c xhat)),  dw = sum_n dy xhat,  db = sum_n dy
// Statistics and sums are fp32; the variance is taken about the mean.
#include "layer_norm.cuh"

namespace velora {

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;

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

template <typename T> __device__ __forceinline__ float rounded(float x) { T t; Elem<T>::store(&t, x); return Elem<T>::load(&t); }

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
    a.partials[static_cast<int64_t>(slice) * a.D + d] = dw;
    a.partials[static_cast<int64_t>(slices + slice) * a.D + d] = db;
}

// The slices' sums in a fixed order: a block takes 32 columns of dw or db, a warp every eighth slice.
__global__ void __launch_bounds__(256)
norm_slices_kernel(const float* partials, int slices, int D, void* dw, void* db, int dtype, int beta)
{
    __shared__ float part[8][32];
    pdl_wait();
    pdl_trigger();
    void* out = blockIdx.y ? db : dw;
    if (!out) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = blockIdx.x * 32 + lane;
    const float* p = partials + static_cast<int64_t>(blockIdx.y) * slices * D + d;
    float s = 0.f;
    if (d < D)
#pragma unroll 8
        for (int i = warp; i < slices; i += 8) s += p[static_cast<int64_t>(i) * D];
    part[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || d >= D) return;
    s = 0.f;
    for (int w = 0; w < 8; ++w) s += part[w][lane];
    store_param(out, dtype, d, s, beta);
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
        rc = launch_chained(norm_slices_kernel, dim3(static_cast<unsigned>(ceil_div64(a.D, 32)), 2), 256, 0, stream, a.partials, slices, a.D, a.dw, a.db,
                            a.dw_dtype, a.beta);
        if (rc != VELORA_OK) return rc;
    }
    if (!a.dX) return VELORA_OK;
    const int64_t most = static_cast<int64_t>(sm_count) * 4;
    return launch_chained(norm_grad_any_kernel<T>, dim3(static_cast<unsigned>(a.N < most ? a.N : most)), kThreads, 0, stream, a);
}

}  // namespace

int launch_layer_norm(const NormArgs& a, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    return a.dtype == VELORA_BF16 ? norm_any<__nv_bfloat16>(a, di.sm_count, stream) : norm_any<float>(a, di.sm_count, stream);
}

int launch_layer_norm_backward(const NormGradArgs& a, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    return a.dtype == VELORA_BF16 ? norm_grad_any<__nv_bfloat16>(a, di.sm_count, stream) : norm_grad_any<float>(a, di.sm_count, stream);
}

}  // namespace velora
