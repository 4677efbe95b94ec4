// Layer norm and its gradients (formulas: layer_norm.cu) of rows of any length, one element at a time, each row read several times (from L1 or L2 but for
// the first): for rows that are too long to be held.  And the sum of the slices of dw and db, for these and the others.  8192 x 14336 bf16: 351 us forward, 458
// backward (1.3 and 1.5 TB/s of x, y and dy, h, dx; 12288 columns, which are held: 71 and 113).
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

// The slices' sums in a fixed order: a block takes 32 V columns of dw or db, a warp every WARPS-th slice, LOADS of them under way at once.  Two shapes:
// eight warps of two columns a lane for up to 160 slices, which are one round (64 x 4096: 1.7 us, 32 warps 4.0); 32 warps of one for more (behind the kernel
// that writes them, 296 x 4096: 5.1 us for both together, 7.7 with eight warps).
template <int WARPS, int LOADS, int V>
__global__ void __launch_bounds__(32 * WARPS)
norm_slices_kernel(const float* partials, int slices, int D, void* dw, void* db, int dtype, int beta)
{
    __shared__ float part[WARPS][32 * V];
    pdl_wait();
    pdl_trigger();
    void* out = blockIdx.y ? db : dw;
    if (!out) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t pitch = norm_pitch(D), d = (static_cast<int64_t>(blockIdx.x) * 32 + lane) * V;          // the pitch is a multiple of eight
    const float* p = partials + blockIdx.y * slices * pitch + (d < pitch ? d : 0);                       // columns behind the last: any, nobody has their sums
    float2 s = make_float2(0.f, 0.f);
    for (int first = warp; first < slices; first += WARPS * LOADS) {
        float2 x[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const float* q = p + min(first + WARPS * i, slices - 1) * pitch;          // no branch: all under way
            if (V == 2) x[i] = *reinterpret_cast<const float2*>(q);
            else x[i].x = *q;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const bool is = first + WARPS * i < slices;
            s.x += is ? x[i].x : 0.f;
            if (V == 2) s.y += is ? x[i].y : 0.f;
        }
    }
    if (V == 2) *reinterpret_cast<float2*>(&part[warp][2 * lane]) = s;
    else part[warp][lane] = s.x;
    __syncthreads();
    const int c = blockIdx.x * 32 * V + threadIdx.x;
    if (threadIdx.x >= 32 * V || c >= D) return;
    float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) t[w & 3] += part[w][threadIdx.x];
    store_param(out, dtype, c, (t[0] + t[1]) + (t[2] + t[3]), beta);
}

template <int WARPS, int LOADS, int V>
int launch_slices(const NormGradArgs& a, int slices, cudaStream_t stream)
{
    return launch_chained(norm_slices_kernel<WARPS, LOADS, V>, dim3(static_cast<unsigned>(ceil_div64(a.D, 32 * V)), 2), 32 * WARPS, 0, stream, a.partials,
                          slices, a.D, a.dw, a.db, a.dw_dtype, a.beta);
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
    return slices <= 160 ? launch_slices<8, 20, 2>(a, slices, stream) : launch_slices<32, 10, 1>(a, slices, stream);
}

}  // namespace velora
