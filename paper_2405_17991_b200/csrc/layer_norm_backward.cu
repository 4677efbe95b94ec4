// Gradients of a layer norm.
//   xhat = (h - m) s,  c = dy w,  dx = dh + s (c - mean c - xhat mean(c xhat)),  dw = sum_n dy xhat,  db = sum_n dy
// Bound by HBM: dy, h (and dh) once in, dx once out.  Rows are dealt out as in layer_norm.cu, but stay in shared memory, where each thread reads its columns
// twice: once for the row's two sums and its share of dw and db, which it keeps in registers from row to row, and once for dx.  What a block has of dw and
// db goes to its row of `partials`, and a second kernel adds those up in order.  (One block: it writes dw and db itself.)
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
norm_grad_rows_kernel(const NormGradArgs a, const Rows rows)
{
    typedef RowShape<WARPS, C> S;
    constexpr int P = S::kPerRow;
    constexpr bool kHold = C <= 3;                             // weights in registers
    extern __shared__ __align__(16) char ring[];
    __shared__ float2 part[2][WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = threadIdx.x % P;
    const int D = a.D;
    const float inverse = 1.f / static_cast<float>(D);
    pdl_wait();
    pdl_trigger();

    const int64_t first = static_cast<int64_t>(blockIdx.x) * S::kRows + (WARPS == 1 ? warp : 0), step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const T* dY = static_cast<const T*>(a.dY);
    const T* H = static_cast<const T*>(a.H);
    const T* dH = a.dX ? static_cast<const T*>(a.dH) : nullptr;
    constexpr int kShare = Share<T, C>::kWords * P * 16;
    char* own = ring + (WARPS == 1 ? warp * rows.stages * rows.stage_bytes : 0) + t * 16;
    const uint32_t own_at = static_cast<uint32_t>(__cvta_generic_to_shared(own));
    auto fetch = [&](int64_t n, int slot) {
        if (n < a.N) {
            const uint32_t to = own_at + slot * rows.stage_bytes;
            Share<T, C>::template copy<P>(to, dY + n * a.lddy, D, t);
            Share<T, C>::template copy<P>(to + kShare, H + n * a.ldh, D, t);
            if (dH) Share<T, C>::template copy<P>(to + 2 * kShare, dH + n * a.lddh, D, t);
        }
        copies_commit();
    };
    if (VEC)
        for (int s = 0; s < rows.stages - 1; ++s) fetch(first + s * step, s);
    float w[kHold ? C : 1][8], dw[C][8], db[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (kHold) load_params<VEC, P>(w[kHold ? c : 0], a.w, a.p_dtype, rows.wide, c, t, D, 1.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = db[c][e] = 0.f;
    }
    float m_next = first < a.N ? a.mean[first] : 0.f, s_next = first < a.N ? a.rstd[first] : 0.f;
    int slot = 0, buffer = 0;
    for (int64_t n = first; n < a.N; n += step, slot = slot + 1 == rows.stages ? 0 : slot + 1, buffer ^= 1) {
        const float m = m_next, s = s_next;
        if (n + step < a.N) {
            m_next = a.mean[n + step];
            s_next = a.rstd[n + step];
        }
        if (VEC) {
            fetch(n + (rows.stages - 1) * step, slot == 0 ? rows.stages - 1 : slot - 1);
            copies_wait(rows.stages - 1);
        }
        const char* row = own + slot * rows.stage_bytes;
        // A chunk of dy and h.
        auto load = [&](float (&dy)[8], float (&h)[8], int c, int left) {
            if (VEC) {
                Share<T, C>::template load<P>(dy, row, c);
                Share<T, C>::template load<P>(h, row + kShare, c);
            } else {
                const int col = column_of<VEC, P>(c, 0, t);
                const T* p = dY + n * a.lddy + col;
                const T* q = H + n * a.ldh + col;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dy[e] = e < left ? Elem<T>::load(p + e * P) : 0.f;
                    h[e] = e < left ? Elem<T>::load(q + e * P) : 0.f;
                }
            }
        };
        float sum = 0.f, along = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D);
            if (left <= 0) continue;                           // columns behind the row's end within a chunk are zeros of dy
            float dy[8], h[8], loaded[8];
            load(dy, h, c, left);
            if (!kHold) load_params<VEC, P>(loaded, a.w, a.p_dtype, rows.wide, c, t, D, 1.f);
            float u[2] = {0.f, 0.f}, v[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xhat = (h[e] - m) * s, g = dy[e] * (kHold ? w[kHold ? c : 0][e] : loaded[e]);
                dw[c][e] = fmaf(dy[e], xhat, dw[c][e]);
                db[c][e] += dy[e];
                u[e & 1] += g;
                v[e & 1] = fmaf(g, xhat, v[e & 1]);
            }
            sum += u[0] + u[1];
            along += v[0] + v[1];
        }
        if (!a.dX) continue;
        sum = lanes_sum(sum);
        along = lanes_sum(along);
        if (WARPS > 1) {
            if (lane == 0) part[buffer][warp] = make_float2(sum, along);
            __syncthreads();                                   // the other buffer's readers are past the barrier before
            sum = along = 0.f;
#pragma unroll 4
            for (int i = 0; i < WARPS; ++i) {
                const float2 v = part[buffer][i];
                sum += v.x;
                along += v.y;
            }
        }
        sum *= inverse;
        along *= inverse;
        T* dx = static_cast<T*>(a.dX) + n * a.lddx;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D), col = column_of<VEC, P>(c, 0, t);
            if (left <= 0) continue;
            float dy[8], h[8], o[8], loaded[8];
            load(dy, h, c, left);
            if (!kHold) load_params<VEC, P>(loaded, a.w, a.p_dtype, rows.wide, c, t, D, 1.f);
            if (dH) {
                if (VEC) {
                    Share<T, C>::template load<P>(o, row + 2 * kShare, c);
                } else {
                    const T* p = dH + n * a.lddh + col;
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = e < left ? Elem<T>::load(p + e * P) : 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xhat = (h[e] - m) * s, g = s * (dy[e] * (kHold ? w[kHold ? c : 0][e] : loaded[e]) - sum - xhat * along);
                o[e] = dH ? o[e] + g : g;
            }
            if (VEC) {
                store_chunk(dx + col, o, left);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < left) Elem<T>::store(dx + col + e * P, o[e]);
            }
        }
    }
    if (!a.dw && !a.db) return;
    const bool alone = gridDim.x == 1;
    float* out_w = a.partials + static_cast<int64_t>(blockIdx.x) * norm_pitch(D);
    float* out_b = out_w + static_cast<int64_t>(gridDim.x) * norm_pitch(D);
    auto put = [&](bool bias, int d, float x) {
        if (alone) {
            if (bias ? a.db : a.dw) store_param(bias ? a.db : a.dw, a.dw_dtype, d, x, a.beta);
        } else {
            (bias ? out_b : out_w)[d] = x;
        }
    };
    if (WARPS == 1) {                                          // the eight warps' sums, through the ring's room
        if (VEC) asm volatile("cp.async.wait_all;" ::: "memory");
        float* sums = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[warp * S::kColumns + column_of<VEC, P>(c, e, t)] = which ? db[c][e] : dw[c][e];
            __syncthreads();
            for (int d = threadIdx.x; d < D; d += S::kThreads) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) x += sums[i * S::kColumns + d];
                put(which != 0, d, x);
            }
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int left = chunk_left<VEC, P>(c, t, D), col = column_of<VEC, P>(c, 0, t);
        if (VEC && !alone) {
            if (left > 0) {                                    // the pitch is a multiple of eight
                store_chunk(out_w + col, dw[c], 8);
                store_chunk(out_b + col, db[c], 8);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) {
                    put(false, column_of<VEC, P>(c, e, t), dw[c][e]);
                    put(true, column_of<VEC, P>(c, e, t), db[c][e]);
                }
        }
    }
}

template <typename T, int WARPS, int C, bool VEC, int BLOCKS>
int launch_rows(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    typedef RowShape<WARPS, C> S;
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    constexpr int kBudget = 216 * 1024 / BLOCKS;               // shared memory of a block, so that BLOCKS of them fit
    auto kern = norm_grad_rows_kernel<T, WARPS, C, VEC, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kBudget) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    Rows rows{};
    rows.stage_bytes = Share<T, C>::kWords * S::kPerRow * 16 * (a.dH && a.dX ? 3 : 2);
    const int fit = kBudget / (rows.stage_bytes * S::kRows);
    rows.stages = fit < 2 ? 2 : (fit > 4 ? 4 : fit);
    static_assert(2 * Share<T, C>::kWords * S::kPerRow * 16 * S::kRows * 3 <= kBudget, "two rows of three operands");
    rows.wide = aligned16(a.w);
    size_t smem = VEC ? static_cast<size_t>(rows.stages) * rows.stage_bytes * S::kRows : 0;
    if (WARPS == 1 && smem < 8 * sizeof(float) * S::kColumns) smem = 8 * sizeof(float) * S::kColumns;
    int64_t blocks = ceil_div64(a.N, S::kRows);
    const int64_t most = static_cast<int64_t>(sm_count) * BLOCKS < kNormSlices ? static_cast<int64_t>(sm_count) * BLOCKS : kNormSlices;
    if (blocks > most) blocks = most;
    const int rc = launch_chained(kern, dim3(static_cast<unsigned>(blocks)), S::kThreads, smem, stream, a, rows);
    if (rc != VELORA_OK || blocks == 1 || (!a.dw && !a.db)) return rc;
    return launch_norm_slices(a, static_cast<int>(blocks), stream);
}

template <typename T, bool VEC>
int launch_held(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    constexpr int kPair = sizeof(T) == 2 ? 2 : 1;              // blocks where two rows of three operands take half of an SM's shared memory, or all of it
    if (a.D <= 256) return launch_rows<T, 1, 1, VEC, 2>(a, sm_count, stream);
    if (a.D <= 512) return launch_rows<T, 1, 2, VEC, 2>(a, sm_count, stream);
    if (a.D <= 768) return launch_rows<T, 1, 3, VEC, kPair>(a, sm_count, stream);
    if (a.D <= 1024) return launch_rows<T, 1, 4, VEC, kPair>(a, sm_count, stream);
    if (a.D <= 2048) return launch_rows<T, 4, 2, VEC, 2>(a, sm_count, stream);
    if (a.D <= 4096) return launch_rows<T, 8, 2, VEC, 2>(a, sm_count, stream);
    if (a.D <= 6144) return launch_rows<T, 8, 3, VEC, kPair>(a, sm_count, stream);
    if (a.D <= 8192) return launch_rows<T, 16, 2, VEC, 1>(a, sm_count, stream);
    if (sizeof(T) == 2) return launch_rows<__nv_bfloat16, 16, 3, VEC, 1>(a, sm_count, stream);
    return launch_layer_norm_backward_any(a, sm_count, stream);
}

bool rows_vec(const void* p, int64_t ld, int dtype) { return !p || (aligned16(p) && ld * static_cast<int64_t>(dtype_size(dtype)) % 16 == 0); }

}  // namespace

int launch_layer_norm_backward(const NormGradArgs& a, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    if (a.D > 12288) return launch_layer_norm_backward_any(a, di.sm_count, stream);
    const bool vec = rows_vec(a.dY, a.lddy, a.dtype) && rows_vec(a.H, a.ldh, a.dtype) && rows_vec(a.dX ? a.dH : nullptr, a.lddh, a.dtype) &&
                     rows_vec(a.dX, a.lddx, a.dtype);
    if (a.dtype == VELORA_BF16)
        return vec ? launch_held<__nv_bfloat16, true>(a, di.sm_count, stream) : launch_held<__nv_bfloat16, false>(a, di.sm_count, stream);
    return vec ? launch_held<float, true>(a, di.sm_count, stream) : launch_held<float, false>(a, di.sm_count, stream);
}

}  // namespace velora
