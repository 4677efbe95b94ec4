// Layer norm of rows, with a residual added in front.
//   h = x + r (rounded to the rows' type),  m = mean h,  s = 1 / sqrt(mean (h - m)^2 + eps),  y = (h - m) s w + b
// Bound by HBM: x (and r) once in, y (and h) once out.  A row is held in the registers of a warp (up to 1024 columns) or of a block while its mean and its
// variance about the mean are taken; blocks walk over rows, the weights stay in registers, and the next rows are on their way to shared memory meanwhile.
// A warp takes its own columns' mean and squares about it, and the block puts those together (n, sum and squares of each warp), so that a row costs one
// barrier and nothing is lost to a mean that is large beside the deviation.
#include "layer_norm_odd.cuh"

namespace velora {

namespace {

// 1 / sqrt(v): the approximation and one step of Newton's method, where that has a meaning.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v), e = fmaf(-v * r, r, 1.f);
    return v > 1e-37f && v < 1e37f ? fmaf(0.5f * r, e, r) : 1.f / sqrtf(v);
}

template <typename T, int WARPS, int C, bool VEC, int BLOCKS>
__global__ void __launch_bounds__((RowShape<WARPS, C>::kThreads), BLOCKS)
norm_rows_kernel(const NormArgs a, const Ring ring)
{
    typedef RowShape<WARPS, C> S;
    constexpr int P = S::kPerRow, kShare = kShareBytes<T, WARPS, C, VEC>;
    extern __shared__ __align__(16) char ring_bytes[];
    __shared__ float4 part[2][WARPS];                          // sum, squares about the warp's mean, that mean, number of columns
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = threadIdx.x % P;
    const int D = a.D;
    const float inverse = 1.f / static_cast<float>(D);
    // This thread's columns, this warp's.
    int mine = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) mine += min(8, max(0, chunk_left<VEC, P>(c, t, D)));
    const float n_warp = static_cast<float>(__reduce_add_sync(0xffffffffu, mine)), inverse_warp = n_warp > 0.f ? 1.f / n_warp : 0.f;
    pdl_wait();
    pdl_trigger();

    const int64_t first = static_cast<int64_t>(blockIdx.x) * S::kRows + (WARPS == 1 ? warp : 0), step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const RowSource<T, WARPS, C, VEC> X{static_cast<const T*>(a.X), a.ldx}, R{static_cast<const T*>(a.R), a.ldr};
    const bool residual = a.R != nullptr;
    char* slots = ring_bytes + (WARPS == 1 ? warp * ring.stages * ring.stage_bytes : 0);
    const uint32_t slots_at = static_cast<uint32_t>(__cvta_generic_to_shared(slots));
    auto fetch = [&](int64_t n, int slot) {
        if (n < a.N) {
            const int at = slot * ring.stage_bytes;
            X.copy(slots + at, slots_at + at, n, D, t);
            if (residual) R.copy(slots + at + kShare, slots_at + at + kShare, n, D, t);
        }
        copies_commit();                                       // a row that is not there is an empty one
    };
    for (int s = 0; s < ring.stages - 1; ++s) fetch(first + s * step, s);
    F2 w[C][4], b[C][4];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_params<VEC, P>(w[c], a.w, a.p_dtype, ring.wide, c, t, D, 1.f);
        load_params<VEC, P>(b[c], a.b, a.p_dtype, ring.wide, c, t, D, 0.f);
    }
    int slot = 0, buffer = 0;
    for (int64_t n = first; n < a.N; n += step, slot = slot + 1 == ring.stages ? 0 : slot + 1, buffer ^= 1) {
        const int before = slot == 0 ? ring.stages - 1 : slot - 1;
        if (VEC) {
            fetch(n + (ring.stages - 1) * step, before);
            copies_wait(ring.stages - 1);
        } else {
            copies_wait(ring.stages - 2);
            row_barrier<WARPS>();
            fetch(n + (ring.stages - 1) * step, before);
        }
        const char* row = slots + slot * ring.stage_bytes;
        T* h = a.H ? static_cast<T*>(a.H) + n * a.ldh : nullptr;
        F2 x[C][4];
        float sum = 0.f;                                       // columns that are not there hold zeros
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D);
            if (left > 0) {                                    // else nothing was copied
                X.load(x[c], row, n, c, t, left);
                if (residual) {
                    F2 r[4];
                    R.load(r, row + kShare, n, c, t, left);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[c][i] = add(x[c][i], r[i]);
                        if (sizeof(T) == 2) x[c][i] = of_bf16(to_bf16(x[c][i]));
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[c][i] = f2(0.f, 0.f);
            }
            sum += sum8(x[c][0], x[c][1], x[c][2], x[c][3]);
        }
        sum = lanes_sum<32>(sum);
        const float m_warp = sum * inverse_warp;
        const F2 minus_warp = f2(-m_warp, -m_warp);
        F2 q[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D);
            if (left < 8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 v = parts(x[c][i]);
                    x[c][i] = f2(2 * i < left ? v.x : m_warp, 2 * i + 1 < left ? v.y : m_warp);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const F2 d = add(x[c][i], minus_warp);
                q[i & 1] = fma(d, d, q[i & 1]);
            }
        }
        const float2 both = parts(add(q[0], q[1]));
        float squares = lanes_sum<32>(both.x + both.y), m = m_warp;
        if (WARPS > 1) {
            if (lane == 0) part[buffer][warp] = make_float4(sum, squares, m_warp, n_warp);
            __syncthreads();                                   // the other buffer's readers are past the barrier before
            const float4 v = part[buffer][lane % WARPS];
            m = lanes_sum<WARPS>(v.x) * inverse;
            squares = lanes_sum<WARPS>(fmaf(v.w * (v.z - m), v.z - m, v.y));
        }
        const float s = inverse_root(fmaf(squares, inverse, a.eps));
        const F2 minus_m = f2(-m, -m), scale = f2(s, s);
        T* y = static_cast<T*>(a.Y) + n * a.ldy;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D);
            if (h) store_chunk<T, VEC, P>(h, x[c], c, t, left);
            F2 o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fma(mul(add(x[c][i], minus_m), scale), w[c][i], b[c][i]);
            store_chunk<T, VEC, P>(y, o, c, t, left);
        }
        if (t == 0) {
            if (a.mean) a.mean[n] = m;
            if (a.rstd) a.rstd[n] = s;
        }
    }
}

template <typename T, int WARPS, int C, bool VEC, int BLOCKS>
int launch_rows(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    typedef RowShape<WARPS, C> S;
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    constexpr int kBudget = 216 * 1024 / BLOCKS;               // shared memory of a block, so that BLOCKS of them fit
    constexpr int kShare = kShareBytes<T, WARPS, C, VEC>;
    static_assert(2 * 2 * kShare * S::kRows <= kBudget, "two rows of both operands");
    auto kern = norm_rows_kernel<T, WARPS, C, VEC, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kBudget) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    Ring ring{};
    ring.stage_bytes = kShare * (a.R ? 2 : 1);
    const int fit = kBudget / (ring.stage_bytes * S::kRows);
    ring.stages = fit > 4 ? 4 : fit;
    ring.wide = aligned16(a.w) && aligned16(a.b);
    const int64_t blocks = ceil_div64(a.N, S::kRows), most = static_cast<int64_t>(sm_count) * BLOCKS;
    return launch_chained(kern, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), S::kThreads,
                          static_cast<size_t>(ring.stages) * ring.stage_bytes * S::kRows, stream, a, ring);
}

template <typename T, bool VEC>
int launch_held(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    if (a.D <= 256) return launch_rows<T, 1, 1, VEC, 4>(a, sm_count, stream);
    if (a.D <= 512) return launch_rows<T, 1, 2, VEC, 3>(a, sm_count, stream);
    if (a.D <= 768) return launch_rows<T, 1, 3, VEC, 2>(a, sm_count, stream);
    if (a.D <= 1024) return launch_rows<T, 1, 4, VEC, sizeof(T) == 2 ? 2 : 1>(a, sm_count, stream);
    if (a.D <= 2048) return launch_rows<T, 4, 2, VEC, 6>(a, sm_count, stream);
    if (a.D <= 4096) return launch_rows<T, 8, 2, VEC, 3>(a, sm_count, stream);
    if (a.D <= 6144) return launch_rows<T, 8, 3, VEC, 2>(a, sm_count, stream);
    if (a.D <= 8192) return launch_rows<T, 16, 2, VEC, 1>(a, sm_count, stream);
    return launch_rows<T, 16, 3, VEC, 1>(a, sm_count, stream);
}

}  // namespace

int launch_layer_norm_odd(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    if (a.D > 12288) return launch_layer_norm_any(a, sm_count, stream);
    return a.dtype == VELORA_BF16 ? launch_held<__nv_bfloat16, false>(a, sm_count, stream) : launch_held<float, false>(a, sm_count, stream);
}

}  // namespace velora
