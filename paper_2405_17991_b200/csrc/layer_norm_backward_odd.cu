// Gradients of a layer norm.
//   xhat = (h - m) s,  c = dy w,  dx = dh + s (c - mean c - xhat mean(c xhat)),  dw = sum_n dy xhat,  db = sum_n dy
// Bound by HBM: dy, h (and dh) once in, dx once out.  Rows are dealt out and fetched as in layer_norm.cu.  A thread adds its columns of dw and db up in
// registers from row to row; a block's go to its row of `partials`, and a second kernel adds those up in order.  (One block: it writes dw and db itself.)
#include "layer_norm_odd.cuh"

namespace velora {

namespace {

template <typename T, int WARPS, int C, bool VEC, int BLOCKS>
__global__ void __launch_bounds__((RowShape<WARPS, C>::kThreads), BLOCKS)
norm_grad_rows_kernel(const NormGradArgs a, const Ring ring)
{
    typedef RowShape<WARPS, C> S;
    constexpr int P = S::kPerRow, kShare = kShareBytes<T, WARPS, C, VEC>;
    constexpr bool kHold = C <= 3;                             // weights in registers
    constexpr bool kKeep = C <= 2;                             // xhat and c between the row's sums and dx; else from shared memory again
    extern __shared__ __align__(16) char ring_bytes[];
    __shared__ float2 part[2][WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = threadIdx.x % P;
    const int D = a.D;
    const float inverse = 1.f / static_cast<float>(D);
    pdl_wait();
    pdl_trigger();

    const int64_t first = static_cast<int64_t>(blockIdx.x) * S::kRows + (WARPS == 1 ? warp : 0), step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const RowSource<T, WARPS, C, VEC> dY{static_cast<const T*>(a.dY), a.lddy}, H{static_cast<const T*>(a.H), a.ldh}, dH{static_cast<const T*>(a.dH), a.lddh};
    const bool more = a.dH && a.dX;
    char* slots = ring_bytes + (WARPS == 1 ? warp * ring.stages * ring.stage_bytes : 0);
    const uint32_t slots_at = static_cast<uint32_t>(__cvta_generic_to_shared(slots));
    auto fetch = [&](int64_t n, int slot) {
        if (n < a.N) {
            const int at = slot * ring.stage_bytes;
            dY.copy(slots + at, slots_at + at, n, D, t);
            H.copy(slots + at + kShare, slots_at + at + kShare, n, D, t);
            if (more) dH.copy(slots + at + 2 * kShare, slots_at + at + 2 * kShare, n, D, t);
        }
        copies_commit();                                       // a row that is not there is an empty one
    };
    for (int s = 0; s < ring.stages - 1; ++s) fetch(first + s * step, s);
    F2 w[kHold ? C : 1][4], dw[C][4], db[C][4];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (kHold) load_params<VEC, P>(w[kHold ? c : 0], a.w, a.p_dtype, ring.wide, c, t, D, 1.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[c][i] = db[c][i] = f2(0.f, 0.f);
    }
    float m_next = first < a.N ? a.mean[first] : 0.f, s_next = first < a.N ? a.rstd[first] : 0.f;
    int slot = 0, buffer = 0;
    for (int64_t n = first; n < a.N; n += step, slot = slot + 1 == ring.stages ? 0 : slot + 1, buffer ^= 1) {
        const float s = s_next;
        const F2 minus_m = f2(-m_next, -m_next), scale = f2(s, s);
        if (n + step < a.N) {
            m_next = a.mean[n + step];
            s_next = a.rstd[n + step];
        }
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
        F2 kept_x[kKeep ? C : 1][4], kept_c[kKeep ? C : 1][4];
        F2 sum2 = f2(0.f, 0.f), along2 = f2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D);
            if (left <= 0) continue;                           // columns behind the row's end within a chunk are zeros of dy
            F2 dy[4], h[4], now[4];
            dY.load(dy, row, n, c, t, left);
            H.load(h, row + kShare, n, c, t, left);
            if (!kHold) load_params<VEC, P>(now, a.w, a.p_dtype, ring.wide, c, t, D, 1.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const F2 xhat = mul(add(h[i], minus_m), scale), g = mul(dy[i], kHold ? w[kHold ? c : 0][i] : now[i]);
                dw[c][i] = fma(dy[i], xhat, dw[c][i]);
                db[c][i] = add(db[c][i], dy[i]);
                sum2 = add(sum2, g);
                along2 = fma(g, xhat, along2);
                if (kKeep) {
                    kept_x[c][i] = xhat;
                    kept_c[c][i] = g;
                }
            }
        }
        if (!a.dX) continue;
        const float2 u = parts(sum2), v = parts(along2);
        float sum = lanes_sum<32>(u.x + u.y), along = lanes_sum<32>(v.x + v.y);
        if (WARPS > 1) {
            if (lane == 0) part[buffer][warp] = make_float2(sum, along);
            __syncthreads();                                   // the other buffer's readers are past the barrier before
            const float2 p = part[buffer][lane % WARPS];
            sum = lanes_sum<WARPS>(p.x);
            along = lanes_sum<WARPS>(p.y);
        }
        const F2 minus_sum = f2(-sum * inverse, -sum * inverse), minus_along = f2(-along * inverse, -along * inverse);
        T* dx = static_cast<T*>(a.dX) + n * a.lddx;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int left = chunk_left<VEC, P>(c, t, D);
            if (left <= 0) continue;
            F2 o[4];
            if (!kKeep) {
                F2 dy[4], h[4], now[4];
                dY.load(dy, row, n, c, t, left);
                H.load(h, row + kShare, n, c, t, left);
                if (!kHold) load_params<VEC, P>(now, a.w, a.p_dtype, ring.wide, c, t, D, 1.f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const F2 xhat = mul(add(h[i], minus_m), scale), g = mul(dy[i], kHold ? w[kHold ? c : 0][i] : now[i]);
                    o[i] = mul(add(fma(xhat, minus_along, g), minus_sum), scale);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = mul(add(fma(kept_x[kKeep ? c : 0][i], minus_along, kept_c[kKeep ? c : 0][i]), minus_sum), scale);
            }
            if (more) {
                F2 dh[4];
                dH.load(dh, row + 2 * kShare, n, c, t, left);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = add(o[i], dh[i]);
            }
            store_chunk<T, VEC, P>(dx, o, c, t, left);
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
        copies_wait(0);
        float* sums = reinterpret_cast<float*>(ring_bytes);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 v = parts(which ? db[c][i] : dw[c][i]);
                    float* p = sums + warp * S::kColumns;
                    p[column_of<VEC, P>(c, 2 * i, t)] = v.x;
                    p[column_of<VEC, P>(c, 2 * i + 1, t)] = v.y;
                }
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
        const int left = chunk_left<VEC, P>(c, t, D);
        if (!alone) {
            const int room = VEC && left > 0 ? 8 : left;       // the pitch is a multiple of eight
            store_chunk<float, VEC, P>(out_w, dw[c], c, t, room);
            store_chunk<float, VEC, P>(out_b, db[c], c, t, room);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) {
                    put(false, column_of<VEC, P>(c, e, t), e & 1 ? parts(dw[c][e >> 1]).y : parts(dw[c][e >> 1]).x);
                    put(true, column_of<VEC, P>(c, e, t), e & 1 ? parts(db[c][e >> 1]).y : parts(db[c][e >> 1]).x);
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
    constexpr int kShare = kShareBytes<T, WARPS, C, VEC>;
    static_assert(2 * 3 * kShare * S::kRows <= kBudget, "two rows of three operands");
    auto kern = norm_grad_rows_kernel<T, WARPS, C, VEC, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kBudget) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    Ring ring{};
    ring.stage_bytes = kShare * (a.dH && a.dX ? 3 : 2);
    const int fit = kBudget / (ring.stage_bytes * S::kRows);
    ring.stages = fit > 4 ? 4 : fit;
    ring.wide = aligned16(a.w);
    size_t smem = static_cast<size_t>(ring.stages) * ring.stage_bytes * S::kRows;
    if (WARPS == 1 && smem < 8 * sizeof(float) * S::kColumns) smem = 8 * sizeof(float) * S::kColumns;
    int64_t blocks = ceil_div64(a.N, S::kRows);
    const int64_t most = static_cast<int64_t>(sm_count) * BLOCKS < kNormSlices ? static_cast<int64_t>(sm_count) * BLOCKS : kNormSlices;
    if (blocks > most) blocks = most;
    const int rc = launch_chained(kern, dim3(static_cast<unsigned>(blocks)), S::kThreads, smem, stream, a, ring);
    if (rc != VELORA_OK || blocks == 1 || (!a.dw && !a.db)) return rc;
    return launch_norm_slices(a, static_cast<int>(blocks), stream);
}

template <typename T, bool VEC>
int launch_held(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    constexpr int kPair = sizeof(T) == 2 ? 2 : 1;              // blocks where two rows of three operands take half of an SM's shared memory, or all of it
    if (a.D <= 256) return launch_rows<T, 1, 1, VEC, 2>(a, sm_count, stream);
    if (a.D <= 512) return launch_rows<T, 1, 2, VEC, kPair>(a, sm_count, stream);
    if (a.D <= 768) return launch_rows<T, 1, 3, VEC, kPair>(a, sm_count, stream);
    if (a.D <= 1024) return launch_rows<T, 4, 1, VEC, 2>(a, sm_count, stream);
    if (a.D <= 2048) return launch_rows<T, 4, 2, VEC, 2>(a, sm_count, stream);
    if (a.D <= 4096) return launch_rows<T, 8, 2, VEC, kPair>(a, sm_count, stream);
    if (a.D <= 6144) return launch_rows<T, 8, 3, VEC, kPair>(a, sm_count, stream);
    if (a.D <= 8192) return launch_rows<T, 16, 2, VEC, 1>(a, sm_count, stream);
    if (sizeof(T) == 2) return launch_rows<__nv_bfloat16, 16, 3, VEC, 1>(a, sm_count, stream);
    return launch_layer_norm_backward_any(a, sm_count, stream);
}

}  // namespace

int launch_layer_norm_backward_odd(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    if (a.D > 12288) return launch_layer_norm_backward_any(a, sm_count, stream);
    return a.dtype == VELORA_BF16 ? launch_held<__nv_bfloat16, false>(a, sm_count, stream) : launch_held<float, false>(a, sm_count, stream);
}

}  // namespace velora
