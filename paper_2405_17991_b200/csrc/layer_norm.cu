// Layer norm of rows, with a residual added in front.
//   h = x + r (rounded to the rows' type),  m = mean h,  s = 1 / sqrt(mean (h - m)^2 + eps),  y = (h - m) s w + b
// Bound by HBM: x (and r) once in, y (and h) once out.  A row is held in the registers of a warp (up to 1024 columns) or of a block while its mean and its
// variance about the mean are taken; blocks walk over rows, the weights stay in registers, and the next rows are on their way to shared memory meanwhile.
// A warp takes its own columns' mean and squares about it, and the block puts those together (n, sum and squares of each warp), so that a row costs one
// barrier and nothing is lost to a mean that is large beside the deviation.
#include "layer_norm_rows.cuh"

namespace velora {

namespace {

struct Rows {
    int stages;                                                // rows on their way or in use
    int stage_bytes;                                           // of a row (of a block's, or of a warp's)
    bool wide;                                                 // weights on 16-byte boundaries
};

template <typename T, int WARPS, int C, bool VEC, int BLOCKS>
__global__ void __launch_bounds__((RowShape<WARPS, C>::kThreads), BLOCKS)
norm_rows_kernel(const NormArgs a, const Rows rows)
{
    typedef RowShape<WARPS, C> S;
    constexpr int P = S::kPerRow;
    extern __shared__ __align__(16) char ring[];
    __shared__ float4 part[2][WARPS];                          // sum, squares about the warp's mean, that mean, number of columns
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = threadIdx.x % P;
    const int D = a.D;
    const float inverse = 1.f / static_cast<float>(D);
    // This thread's columns, this warp's.
    int mine = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) mine += min(8, max(0, chunk_left<VEC, P>(c, t, D)));
    const int count = __reduce_add_sync(0xffffffffu, mine);
    const float n_warp = static_cast<float>(count), inverse_warp = count > 0 ? 1.f / n_warp : 0.f;
    pdl_wait();
    pdl_trigger();

    const int64_t first = static_cast<int64_t>(blockIdx.x) * S::kRows + (WARPS == 1 ? warp : 0), step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const T* X = static_cast<const T*>(a.X);
    const T* R = static_cast<const T*>(a.R);
    constexpr int kShare = Share<T, C>::kWords * P * 16;
    char* own = ring + (WARPS == 1 ? warp * rows.stages * rows.stage_bytes : 0) + t * 16;
    const uint32_t own_at = static_cast<uint32_t>(__cvta_generic_to_shared(own));
    auto fetch = [&](int64_t n, int slot) {
        if (n < a.N) {
            Share<T, C>::template copy<P>(own_at + slot * rows.stage_bytes, X + n * a.ldx, D, t);
            if (R) Share<T, C>::template copy<P>(own_at + slot * rows.stage_bytes + kShare, R + n * a.ldr, D, t);
        }
        copies_commit();                                       // a row that is not there is an empty one
    };
    if (VEC)
        for (int s = 0; s < rows.stages - 1; ++s) fetch(first + s * step, s);
    float w[C][8], b[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_params<VEC, P>(w[c], a.w, a.p_dtype, rows.wide, c, t, D, 1.f);
        load_params<VEC, P>(b[c], a.b, a.p_dtype, rows.wide, c, t, D, 0.f);
    }
    int slot = 0, buffer = 0;
    for (int64_t n = first; n < a.N; n += step, slot = slot + 1 == rows.stages ? 0 : slot + 1, buffer ^= 1) {
        float x[C][8];
        if (VEC) {
            fetch(n + (rows.stages - 1) * step, slot == 0 ? rows.stages - 1 : slot - 1);
            copies_wait(rows.stages - 1);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (chunk_left<VEC, P>(c, t, D) > 0) {          // else nothing was copied

                    Share<T, C>::template load<P>(x[c], own + slot * rows.stage_bytes, c);
                    if (R) {
                        float r[8];
                        Share<T, C>::template load<P>(r, own + slot * rows.stage_bytes + kShare, c);
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[c][e] = rounded<T>(x[c][e] + r[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[c][e] = 0.f;
                }
            }
        } else {
            const T* p = X + n * a.ldx + t;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int left = chunk_left<VEC, P>(c, t, D);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[c][e] = e < left ? Elem<T>::load(p + (c * 8 + e) * P) : 0.f;
            }
            if (R) {
                const T* q = R + n * a.ldr + t;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int left = chunk_left<VEC, P>(c, t, D);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < left) x[c][e] = rounded<T>(x[c][e] + Elem<T>::load(q + (c * 8 + e) * P));
                }
            }
        }
        float sum = 0.f;                                       // columns that are not there hold zeros
#pragma unroll
        for (int c = 0; c < C; ++c) sum += sum8(x[c]);
        sum = lanes_sum(sum);
        const float m_warp = sum * inverse_warp;
        float squares = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D);
            if (left < 8) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e >= left) x[c][e] = m_warp;
            }
            float q[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = x[c][e] - m_warp;
                q[e & 1] = fmaf(d, d, q[e & 1]);
            }
            squares += q[0] + q[1];
        }
        squares = lanes_sum(squares);
        float m = m_warp;
        if (WARPS > 1) {
            if (lane == 0) part[buffer][warp] = make_float4(sum, squares, m_warp, n_warp);
            __syncthreads();                                   // the other buffer's readers are past the barrier before
            float all = 0.f;
#pragma unroll 4
            for (int i = 0; i < WARPS; ++i) all += part[buffer][i].x;
            m = all * inverse;
            squares = 0.f;
#pragma unroll 2
            for (int i = 0; i < WARPS; ++i) {                  // few in registers at a time

                const float4 v = part[buffer][i];
                squares += fmaf(v.w * (v.z - m), v.z - m, v.y);
            }
        }
        const float s = 1.f / sqrtf(squares * inverse + a.eps);
        T* y = static_cast<T*>(a.Y) + n * a.ldy;
        T* h = a.H ? static_cast<T*>(a.H) + n * a.ldh : nullptr;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf((x[c][e] - m) * s, w[c][e], b[c][e]);
            const int left = chunk_left<VEC, P>(c, t, D), col = column_of<VEC, P>(c, 0, t);
            if (VEC) {
                if (left > 0) {
                    if (h) store_chunk(h + col, x[c], left);
                    store_chunk(y + col, o, left);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < left) {
                        if (h) Elem<T>::store(h + col + e * P, x[c][e]);
                        Elem<T>::store(y + col + e * P, o[e]);
                    }
            }
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
    auto kern = norm_rows_kernel<T, WARPS, C, VEC, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kBudget) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    Rows rows{};
    rows.stage_bytes = Share<T, C>::kWords * S::kPerRow * 16 * (a.R ? 2 : 1);
    const int fit = kBudget / (rows.stage_bytes * S::kRows);
    rows.stages = fit < 2 ? 2 : (fit > 4 ? 4 : fit);
    static_assert(2 * Share<T, C>::kWords * S::kPerRow * 16 * S::kRows * 2 <= kBudget, "two rows of both operands");
    rows.wide = aligned16(a.w) && aligned16(a.b);
    const int64_t blocks = ceil_div64(a.N, S::kRows), most = static_cast<int64_t>(sm_count) * BLOCKS;
    return launch_chained(kern, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), S::kThreads,
                          VEC ? static_cast<size_t>(rows.stages) * rows.stage_bytes * S::kRows : 0, stream, a, rows);
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

bool rows_vec(const void* p, int64_t ld, int dtype) { return !p || (aligned16(p) && ld * static_cast<int64_t>(dtype_size(dtype)) % 16 == 0); }

}  // namespace

int launch_layer_norm(const NormArgs& a, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    if (a.D > 12288) return launch_layer_norm_any(a, di.sm_count, stream);
    const bool vec = rows_vec(a.X, a.ldx, a.dtype) && rows_vec(a.R, a.ldr, a.dtype) && rows_vec(a.H, a.ldh, a.dtype) && rows_vec(a.Y, a.ldy, a.dtype);
    if (a.dtype == VELORA_BF16)
        return vec ? launch_held<__nv_bfloat16, true>(a, di.sm_count, stream) : launch_held<__nv_bfloat16, false>(a, di.sm_count, stream);
    return vec ? launch_held<float, true>(a, di.sm_count, stream) : launch_held<float, false>(a, di.sm_count, stream);
}

}  // namespace velora
