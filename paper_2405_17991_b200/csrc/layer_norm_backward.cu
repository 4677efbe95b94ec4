// Gradients of a layer norm.
//   xhat = (h - m) s,  c = dy w,  dx = dh + s (c - mean c - xhat mean(c xhat)),  dw = sum_n dy xhat,  db = sum_n dy
// Bound by HBM: dy, h (and dh) once in, dx once out.  Rows are dealt out and fetched as in layer_norm.cu.  A thread adds its columns of dw and db up in
// registers from row to row; a block's go to its row of `partials`, and a second kernel adds those up in order.
#include "layer_norm_rows.cuh"

namespace velora {

namespace {

// E columns' sums, at a 16-byte boundary.  WIDE: 16 bytes at a time, for which they have to lie in four neighbouring registers all along: right where there are
// registers to spare (8192 x 4096 bf16: 39 us, two at a time 42), but 8192 x 11008, dX alone, takes 112 us instead of 92.
template <int E, bool WIDE> __device__ __forceinline__ void store_sums(float* p, const F2 (&x)[E / 2])
{
    if (WIDE) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) reinterpret_cast<ulonglong2*>(p)[i] = make_ulonglong2(x[2 * i].v, x[2 * i + 1].v);
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) reinterpret_cast<float2*>(p)[i] = parts(x[i]);
    }
}
// TEAM: the warps that have a row, so that a block of 256 threads has 8 / TEAM at a time; 0: the whole block has one.  KEEP: xhat and c stay in registers between the row's sums and dx; else dy and h are read from shared memory again.
template <typename T, int C, int STAGES, bool MORE, int TEAM, bool KEEP, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS)
norm_grad_rows_kernel(const NormGradArgs a, bool wide)
{
    constexpr int E = Word<T>::E, kTeams = TEAM ? 8 / TEAM : 1, kLanes = TEAM ? TEAM : kWarpLanes<THREADS>;
    extern __shared__ __align__(16) char ring_bytes[];
    __shared__ float2 part[2][kTeams * kLanes];
    const int P = TEAM ? 32 * TEAM : blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int mine = TEAM ? warp / (TEAM ? TEAM : 1) : 0, t = TEAM ? threadIdx.x % (TEAM ? 32 * TEAM : 1) : threadIdx.x;       // team of the block, thread of the team
    const int D = a.D, share = C * P * 16, stage = share * (MORE ? 3 : 2), ring_end = STAGES * stage;
    const bool last = ((C - 1) * P + t) * E < D;               // the last word is there
    const float inverse = 1.f / static_cast<float>(D);
    if (!TEAM && threadIdx.x < 2 * kLanes) part[threadIdx.x / kLanes][threadIdx.x % kLanes] = make_float2(0.f, 0.f);     // warps that are not there
    pdl_wait();
    pdl_trigger();

    const int64_t team = static_cast<int64_t>(blockIdx.x) * kTeams + mine, teams = static_cast<int64_t>(gridDim.x) * kTeams;
    const int64_t each = a.N / teams, over = a.N % teams, first = each * team + (team < over ? team : over), rows = each + (team < over ? 1 : 0);
    const T* dy_at = static_cast<const T*>(a.dY) + first * a.lddy + t * E;
    const T* h_at = static_cast<const T*>(a.H) + first * a.ldh + t * E;
    const T* dh_at = MORE ? static_cast<const T*>(a.dH) + first * a.lddh + t * E : nullptr;
    T* dx_at = a.dX ? static_cast<T*>(a.dX) + first * a.lddx + t * E : nullptr;
    const float* mean_at = a.mean + first;
    const float* rstd_at = a.rstd + first;
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(ring_bytes)) + mine * ring_end + t * 16;
    auto fetch = [&](int at) {
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (c < C - 1 || last) {
                copy_word(ring + at + c * P * 16, dy_at + c * P * E);
                copy_word(ring + at + share + c * P * 16, h_at + c * P * E);
                if (MORE) copy_word(ring + at + 2 * share + c * P * 16, dh_at + c * P * E);
            }
        dy_at += a.lddy;
        h_at += a.ldh;
        if (MORE) dh_at += a.lddh;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        if (s < rows) fetch(s * stage);
        copies_commit();
    }
    F2 w[C][E / 2], dw[C][E / 2], db[C][E / 2];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (c < C - 1 || last) load_columns<E>(w[c], a.w, a.p_dtype, wide, (c * P + t) * E, 1.f);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) dw[c][i] = db[c][i] = f2(0.f);
    }
    float m_next = rows > 0 ? mean_at[0] : 0.f, s_next = rows > 0 ? rstd_at[0] : 0.f;
    if (!TEAM) __syncthreads();
    int at = 0, turn = 0;
    for (int64_t row = 0; row < rows; ++row) {
        const F2 minus_m = f2(-m_next), scale = f2(s_next);
        if (row + 1 < rows) {
            m_next = mean_at[row + 1];
            s_next = rstd_at[row + 1];
        }
        if (row + STAGES - 1 < rows) fetch(at == 0 ? ring_end - stage : at - stage);
        copies_commit();
        copies_wait<STAGES - 1>();
        const uint32_t here = ring + at;
        at = at == ring_end - stage ? 0 : at + stage;
        F2 kept_x[KEEP ? C : 1][E / 2], kept_c[KEEP ? C : 1][E / 2];
        F2 sums = f2(0.f), along = f2(0.f);
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (c < C - 1 || last) {
                Word<T> dy, h;
                dy.load(here + c * P * 16);
                h.load(here + share + c * P * 16);
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const F2 xhat = mul(add(h.x[i], minus_m), scale), g = mul(dy.x[i], w[c][i]);
                    dw[c][i] = fma(dy.x[i], xhat, dw[c][i]);
                    db[c][i] = add(db[c][i], dy.x[i]);
                    sums = add(sums, g);
                    along = fma(g, xhat, along);
                    if (KEEP) {
                        kept_x[KEEP ? c : 0][i] = xhat;
                        kept_c[KEEP ? c : 0][i] = g;
                    }
                }
            }
        if (!dx_at) continue;
        float s1 = warp_total(sum(sums)), s2 = warp_total(sum(along));
        if (TEAM != 1) {
            if (lane == 0) part[turn][warp] = make_float2(s1, s2);
            if (TEAM) asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "n"(32 * TEAM) : "memory");
            else __syncthreads();                              // the other half's readers are past the barrier before
            const float2 v = part[turn][mine * kLanes + lane % kLanes];
            turn ^= 1;
            s1 = warps_total<kLanes>(v.x);
            s2 = warps_total<kLanes>(v.y);
        }
        const F2 minus_sum = f2(-s1 * inverse), minus_along = f2(-s2 * inverse);
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (c < C - 1 || last) {
                Word<T> o;
                if (KEEP) {
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) o.x[i] = mul(add(fma(kept_x[KEEP ? c : 0][i], minus_along, kept_c[KEEP ? c : 0][i]), minus_sum), scale);
                } else {
                    Word<T> dy, h;
                    dy.load(here + c * P * 16);
                    h.load(here + share + c * P * 16);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        const F2 xhat = mul(add(h.x[i], minus_m), scale), g = mul(dy.x[i], w[c][i]);
                        o.x[i] = mul(add(fma(xhat, minus_along, g), minus_sum), scale);
                    }
                }
                if (MORE) {
                    Word<T> dh;
                    dh.load(here + 2 * share + c * P * 16);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) o.x[i] = add(o.x[i], dh.x[i]);
                }
                o.store(dx_at + c * P * E);
            }
        dx_at += a.lddx;
    }
    if (!a.dw && !a.db) return;
    float* out_w = a.partials + static_cast<int64_t>(blockIdx.x) * norm_pitch(D);
    float* out_b = out_w + static_cast<int64_t>(gridDim.x) * norm_pitch(D);
    if (TEAM) {                                                // the teams' sums, through the ring's room
        copies_wait<0>();
        float* sums = reinterpret_cast<float*>(ring_bytes);
        constexpr int kColumns = C * 32 * TEAM * E;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const float2 v = parts(which ? db[c][i] : dw[c][i]);
                    *reinterpret_cast<float2*>(sums + mine * kColumns + (c * P + t) * E + 2 * i) = v;
                }
            __syncthreads();
            for (int d = threadIdx.x; d < D; d += THREADS) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < kTeams; ++i) x += sums[i * kColumns + d];
                (which ? out_b : out_w)[d] = x;
            }
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (c < C - 1 || last) {
            const int d = (c * P + t) * E;
            store_sums<E, KEEP>(out_w + d, dw[c]);
            store_sums<E, KEEP>(out_b + d, db[c]);
        }
}

template <typename T, int C, bool MORE, int TEAM, bool KEEP, int THREADS, int BLOCKS>
int launch_rows(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    constexpr int kTeams = TEAM ? 8 / TEAM : 1;
    // Rows of a full block on their way or in use: up to four of them, in the share of an SM's shared memory that BLOCKS leave.
    constexpr int kRow = C * THREADS * 16 * (MORE ? 3 : 2), kFit = 216 * 1024 / BLOCKS / kRow, kStages = kFit > 4 ? 4 : kFit;
    static_assert(kStages >= 1, "a row");
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    auto kern = norm_grad_rows_kernel<T, C, kStages, MORE, TEAM, KEEP, THREADS, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kStages * kRow) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    static_assert(TEAM == 0 || kStages * kRow >= C * THREADS * Word<T>::E * 4, "room for the teams' sums");
    const int words = row_words(a.D, a.dtype), threads = TEAM ? THREADS : row_threads(words, C), per_row = TEAM ? 32 * TEAM : threads;
    if (threads > THREADS || (C - 1) * per_row >= words || C * per_row < words) return VELORA_ERR_UNSUPPORTED;         // only last words may be missing
    const int64_t blocks = norm_grad_blocks(a, kTeams, sm_count * BLOCKS);
    const int rc = launch_chained(kern, dim3(static_cast<unsigned>(blocks)), threads, static_cast<size_t>(kStages) * kRow / THREADS * threads, stream, a,
                                  aligned16(a.w));
    if (rc != VELORA_OK || (!a.dw && !a.db)) return rc;
    return launch_norm_slices(a, static_cast<int>(blocks), stream);
}

// By the row's words: what was fastest of some forty shapes, in TB/s of dy, h, dx (and dh), dw and db included.  bf16, without and with dh: 16384 x 256 2.6 / 3.2,
// 16384 x 512 3.8 / 4.2, 12608 x 768 3.7 / 4.0 (a warp a row: 3.6 / 4.0), 16384 x 1024 4.8 / 4.7, 8192 x 2048 4.5 / 4.7 (a block a row: 3.3 / 3.9),
// 8192 x 4096 5.1 / 5.4, 4096 x 5464 3.6 / 4.3, 8192 x 8192 5.2 / 5.9, 8192 x 11008 5.2 / 4.8.  fp32: 8192 x 512 4.0 / 4.4, 12608 x 768 4.9 / 5.2,
// 4096 x 2048 4.7 / 5.0, 4096 x 4096 5.5 / 5.9, 4096 x 8192 5.3 / 6.0, 2048 x 11008 4.8 / 5.0.
template <typename T, bool MORE>
int launch_words(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    const int words = row_words(a.D, a.dtype);
    if (words <= 32) return launch_rows<T, 1, MORE, 1, true, 256, 2>(a, sm_count, stream);
    if (words <= 64) return launch_rows<T, 2, MORE, 1, true, 256, 2>(a, sm_count, stream);
    if constexpr (sizeof(T) == 2) {
        if (words <= 128) return launch_rows<T, 2, MORE, 2, true, 256, 2>(a, sm_count, stream);
        if (words <= 256) return launch_rows<T, 2, MORE, 4, true, 256, 2>(a, sm_count, stream);
        if (words <= 512) return launch_rows<T, 2, MORE, 0, true, 256, 2>(a, sm_count, stream);
        if (words <= 768) return launch_rows<T, 3, MORE, 0, true, 256, 1>(a, sm_count, stream);
        if (words <= 1024) return launch_rows<T, 2, MORE, 0, true, 512, 1>(a, sm_count, stream);
        if (words <= 1536) return launch_rows<T, 3, MORE, 0, false, 512, 1>(a, sm_count, stream);
    } else {
        if (words <= 96) return launch_rows<T, 3, MORE, 1, true, 256, 2>(a, sm_count, stream);
        if (words <= 128) return launch_rows<T, 4, MORE, 1, true, 256, 2>(a, sm_count, stream);
        if (words <= 192) return launch_rows<T, 3, MORE, 2, true, 256, 2>(a, sm_count, stream);
        if (words <= 256) return launch_rows<T, 4, MORE, 2, true, 256, 2>(a, sm_count, stream);
        if (words <= 384) return launch_rows<T, 3, MORE, 4, true, 256, 2>(a, sm_count, stream);
        if (words <= 512) return launch_rows<T, 4, MORE, 4, true, 256, 2>(a, sm_count, stream);
        if (words <= 1024) return launch_rows<T, 3, MORE, 0, true, 512, 1>(a, sm_count, stream);
        if (words <= 2048) return launch_rows<T, 4, MORE, 0, true, 512, 1>(a, sm_count, stream);
        if (words <= 6 * 512) return launch_rows<T, 6, MORE, 0, false, 512, 1>(a, sm_count, stream);
    }
    return launch_layer_norm_backward_any(a, sm_count, stream);
}

}  // namespace

int launch_layer_norm_backward(const NormGradArgs& a, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    const void* dH = a.dX ? a.dH : nullptr;
    const bool vec = a.D * static_cast<int64_t>(dtype_size(a.dtype)) % 16 == 0 && rows_vec(a.dY, a.lddy, a.dtype) && rows_vec(a.H, a.ldh, a.dtype) &&
                     rows_vec(dH, a.lddh, a.dtype) && rows_vec(a.dX, a.lddx, a.dtype);
    if (!vec) return launch_layer_norm_backward_odd(a, di.sm_count, stream);
    if (a.dtype == VELORA_BF16)
        return dH ? launch_words<__nv_bfloat16, true>(a, di.sm_count, stream) : launch_words<__nv_bfloat16, false>(a, di.sm_count, stream);
    return dH ? launch_words<float, true>(a, di.sm_count, stream) : launch_words<float, false>(a, di.sm_count, stream);
}

}  // namespace velora
