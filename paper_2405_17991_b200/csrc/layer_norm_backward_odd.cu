// Gradients of a layer norm for rows that start on any boundary (formula and plan: layer_norm_backward.cu).
#include "layer_norm_odd.cuh"

namespace velora {

namespace {

// TEAM: the warps that have a row, so that a block of 256 threads has 8 / TEAM at a time; 0: the whole block of P threads has one.  N columns a thread, of
// which every thread has LEAST.  KEEP: xhat and c stay in registers between the row's sums and dx; else dy and h are read from shared memory again.
template <typename T, int N, int LEAST, bool MORE, int TEAM, int P, bool KEEP, int BLOCKS>
__global__ void __launch_bounds__(TEAM ? 256 : P, BLOCKS)
norm_grad_odd_kernel(const NormGradArgs a, int stages, int share)
{
    constexpr int kTeams = TEAM ? 8 / TEAM : 1, kLanes = TEAM ? TEAM : kWarpLanes<P>;
    extern __shared__ __align__(16) char ring[];
    __shared__ float2 part[2][kTeams * kLanes];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mine = TEAM ? warp / (TEAM ? TEAM : 1) : 0, t = threadIdx.x % P;
    const int D = a.D, stage = share * (MORE ? 3 : 2);
    const OddColumns<LEAST> has = odd_columns<P, LEAST>(D, t);
    const float inverse = 1.f / static_cast<float>(D);
    if (!TEAM && threadIdx.x < 2 * kLanes) part[threadIdx.x / kLanes][threadIdx.x % kLanes] = make_float2(0.f, 0.f);
    pdl_wait();
    pdl_trigger();

    const int64_t team = static_cast<int64_t>(blockIdx.x) * kTeams + mine, teams = static_cast<int64_t>(gridDim.x) * kTeams;
    const int64_t each = a.N / teams, over = a.N % teams, first = each * team + (team < over ? team : over), rows = each + (team < over ? 1 : 0);
    OddRows<T, P> dY(a.dY, a.lddy, first), H(a.H, a.ldh, first), dH(MORE ? a.dH : a.H, MORE ? a.lddh : a.ldh, first);
    T* dx_at = a.dX ? static_cast<T*>(a.dX) + first * a.lddx + t : nullptr;
    const float* mean_at = a.mean + first;
    const float* rstd_at = a.rstd + first;
    char* slots = ring + mine * stages * stage;
    const uint32_t slots_at = static_cast<uint32_t>(__cvta_generic_to_shared(slots));
    auto fetch = [&](int slot) {
        dY.template fetch<N>(slots + slot * stage, D, t);
        H.template fetch<N>(slots + slot * stage + share, D, t);
        if (MORE) dH.template fetch<N>(slots + slot * stage + 2 * share, D, t);
    };
    for (int s = 0; s < stages - 1; ++s) {
        if (s < rows) fetch(s);
        copies_commit();
    }
    F2 w[N / 2], dw[N / 2], db[N / 2];
    odd_params<P, N>(w, a.w, a.p_dtype, has, t, 1.f);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) dw[i] = db[i] = f2(0.f);
    float m_next = rows > 0 ? mean_at[0] : 0.f, s_next = rows > 0 ? rstd_at[0] : 0.f;
    int slot = 0, turn = 0;
    for (int64_t row = 0; row < rows; ++row) {
        const float m = m_next;
        const F2 minus_m = f2(-m), scale = f2(s_next);
        if (row + 1 < rows) {
            m_next = mean_at[row + 1];
            s_next = rstd_at[row + 1];
        }
        copies_wait_behind(stages - 2);
        team_barrier<TEAM>(mine);                              // this row is there; all are done with the one before, whose place is filled again
        if (row + stages - 1 < rows) fetch(slot == 0 ? stages - 1 : slot - 1);
        copies_commit();
        const uint32_t here = slots_at + slot * stage;
        slot = slot + 1 == stages ? 0 : slot + 1;
        const uint32_t dy_row = dY.row(here, t);
        const uint32_t h_row = H.row(here + share, t);
        const uint32_t dh_row = dH.row(here + 2 * share, t);
        dY.step();
        H.step();
        if (MORE) dH.step();
        // Columns that are not there: dy and w are zeros, and h is the mean, since m s may be beyond fp32 where every h - m is zero.
        F2 xhat[N / 2], c[N / 2], sums = f2(0.f), along = f2(0.f);
        {
            F2 dy[N / 2], h[N / 2];
            odd_load<T, P, N>(dy, dy_row, has);
            odd_load<T, P, N>(h, h_row, has, m);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                xhat[i] = mul(add(h[i], minus_m), scale);
                c[i] = mul(dy[i], w[i]);
                dw[i] = fma(dy[i], xhat[i], dw[i]);
                db[i] = add(db[i], dy[i]);
                sums = add(sums, c[i]);
                along = fma(c[i], xhat[i], along);
            }
        }
        if (!dx_at) continue;
        float s1 = warp_total(sum(sums)), s2 = warp_total(sum(along));
        if (TEAM != 1) {
            if (lane == 0) part[turn][warp] = make_float2(s1, s2);
            team_barrier<TEAM>(mine);
            const float2 v = part[turn][mine * kLanes + lane % kLanes];
            turn ^= 1;
            s1 = warps_total<kLanes>(v.x);
            s2 = warps_total<kLanes>(v.y);
        }
        const F2 minus_sum = f2(-s1 * inverse), minus_along = f2(-s2 * inverse);
        if (!KEEP) {
            F2 dy[N / 2], h[N / 2];
            odd_load<T, P, N>(dy, dy_row, has);
            odd_load<T, P, N>(h, h_row, has, m);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                xhat[i] = mul(add(h[i], minus_m), scale);
                c[i] = mul(dy[i], w[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) c[i] = mul(add(fma(xhat[i], minus_along, c[i]), minus_sum), scale);
        if (MORE) {
            F2 dh[N / 2];
            odd_load<T, P, N>(dh, dh_row, has);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) c[i] = add(c[i], dh[i]);
        }
        odd_store<T, P, N>(dx_at, c, has);
        dx_at += a.lddx;
    }
    if (!a.dw && !a.db) return;
    float* out_w = a.partials + static_cast<int64_t>(blockIdx.x) * norm_pitch(D);
    float* out_b = out_w + static_cast<int64_t>(gridDim.x) * norm_pitch(D);
    if (TEAM) {                                                // the teams' sums, through the ring's room
        copies_wait<0>();
        float* all = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float2 v = parts(which ? db[i] : dw[i]);
                all[mine * (N * P) + 2 * i * P + t] = v.x;
                all[mine * (N * P) + (2 * i + 1) * P + t] = v.y;
            }
            __syncthreads();
            for (int d = threadIdx.x; d < D; d += 256) {
                float x = 0.f;
#pragma unroll
                for (int i = 0; i < kTeams; ++i) x += all[i * (N * P) + d];
                (which ? out_b : out_w)[d] = x;
            }
        }
        return;
    }
    odd_store<float, P, N>(out_w + t, dw, has);
    odd_store<float, P, N>(out_b + t, db, has);
}

template <typename T, int N, int LEAST, bool MORE, int TEAM, int P, bool KEEP, int BLOCKS>
int launch_rows(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    static_assert(TEAM == 0 || P == 32 * TEAM, "a team's threads");
    constexpr int kTeams = TEAM ? 8 / TEAM : 1, kRoom = 216 * 1024 / BLOCKS;
    const int share = odd_share(a.D, a.dtype), row = share * (MORE ? 3 : 2) * kTeams, stages = kRoom / row < 4 ? kRoom / row : 4;
    if (a.D > N * P || a.D < LEAST * P || stages < 2) return VELORA_ERR_UNSUPPORTED;
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    auto kern = norm_grad_odd_kernel<T, N, LEAST, MORE, TEAM, P, KEEP, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    size_t smem = static_cast<size_t>(stages) * row;
    if (TEAM && smem < sizeof(float) * N * 256) smem = sizeof(float) * N * 256;
    const int64_t blocks = norm_grad_blocks(a, kTeams, sm_count * BLOCKS);
    const int rc = launch_chained(kern, dim3(static_cast<unsigned>(blocks)), TEAM ? 256 : P, smem, stream, a, stages, share);
    if (rc != VELORA_OK || (!a.dw && !a.db)) return rc;
    return launch_norm_slices(a, static_cast<int>(blocks), stream);
}

// Longest rows of which two fit a block's 216 KB: with dH three operands of fp32, (ceil(4 D / 16) + 1) 16 bytes each.
template <typename T, bool MORE> constexpr int kOddHeld = sizeof(T) == 4 && MORE ? 9212 : 12288;

// 4096 x 5461 bf16 46 us (the same rows on 16-byte boundaries 37), 12608 x 769 25, 8192 x 10001 143.
template <typename T, bool MORE>
int launch_width(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    if (a.D <= 256) return launch_rows<T, 8, 0, MORE, 1, 32, true, 2>(a, sm_count, stream);
    if (a.D <= 512) return launch_rows<T, 16, 8, MORE, 1, 32, true, 2>(a, sm_count, stream);
    if (a.D <= 1024) return launch_rows<T, 8, 4, MORE, 4, 128, true, 2>(a, sm_count, stream);
    if (a.D <= 2048) return launch_rows<T, 16, 8, MORE, 4, 128, true, 2>(a, sm_count, stream);
    if (a.D <= 2560) return launch_rows<T, 16, 12, MORE, 0, 160, true, 2>(a, sm_count, stream);
    if (a.D <= 4096) return launch_rows<T, 16, 10, MORE, 0, 256, true, 2>(a, sm_count, stream);
    if (a.D <= 5632) return launch_rows<T, 16, 11, MORE, 0, 352, true, 1>(a, sm_count, stream);
    if (a.D <= 8192) return launch_rows<T, 16, 11, MORE, 0, 512, true, 1>(a, sm_count, stream);
    if (a.D <= 10240 && a.D <= kOddHeld<T, MORE>) return launch_rows<T, 20, 16, MORE, 0, 512, false, 1>(a, sm_count, stream);
    if constexpr (kOddHeld<T, MORE> > 10240)
        if (a.D <= 12288) return launch_rows<T, 24, 20, MORE, 0, 512, false, 1>(a, sm_count, stream);
    return launch_layer_norm_backward_any(a, sm_count, stream);
}

}  // namespace

int launch_layer_norm_backward_odd(const NormGradArgs& a, int sm_count, cudaStream_t stream)
{
    const bool more = a.dH && a.dX;
    if (a.dtype == VELORA_BF16)
        return more ? launch_width<__nv_bfloat16, true>(a, sm_count, stream) : launch_width<__nv_bfloat16, false>(a, sm_count, stream);
    return more ? launch_width<float, true>(a, sm_count, stream) : launch_width<float, false>(a, sm_count, stream);
}

}  // namespace velora
