// Layer norm of rows that start on any boundary (formula and plan: layer_norm.cu).  4096 x 5461 bf16: one element a load and a store, so bound by instructions.
#include "layer_norm_odd.cuh"

namespace velora {

namespace {

// TEAM: 1, a warp has a row, eight of them a block; 0: the block of P threads has one.  N columns a thread, of which every thread has
// LEAST.
template <typename T, int N, int LEAST, bool RESIDUAL, int TEAM, int P, int BLOCKS>
__global__ void __launch_bounds__(TEAM ? 256 : P, BLOCKS)
norm_odd_kernel(const NormArgs a, int stages, int share)
{
    constexpr int kTeams = TEAM ? 8 : 1, kLanes = TEAM ? 1 : kWarpLanes<P>;
    extern __shared__ __align__(16) char ring[];
    __shared__ float4 part[2][kLanes];                         // sum, squares about the warp's mean, that mean, number of columns
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mine = TEAM ? warp : 0, t = TEAM ? lane : threadIdx.x;
    const int D = a.D, stage = share * (RESIDUAL ? 2 : 1);
    const OddColumns<LEAST> has = odd_columns<P, LEAST>(D, t);
    const float inverse = 1.f / static_cast<float>(D);
    if (!TEAM && threadIdx.x < 2 * kLanes) part[threadIdx.x / kLanes][threadIdx.x % kLanes] = make_float4(0.f, 0.f, 0.f, 0.f);
    pdl_wait();
    pdl_trigger();

    const int64_t team = static_cast<int64_t>(blockIdx.x) * kTeams + mine, teams = static_cast<int64_t>(gridDim.x) * kTeams;
    const int64_t each = a.N / teams, over = a.N % teams, first = each * team + (team < over ? team : over), rows = each + (team < over ? 1 : 0);
    OddRows<T, P> X(a.X, a.ldx, first), R(RESIDUAL ? a.R : a.X, RESIDUAL ? a.ldr : a.ldx, first);
    T* y_at = static_cast<T*>(a.Y) + first * a.ldy + t;
    T* h_at = a.H ? static_cast<T*>(a.H) + first * a.ldh + t : nullptr;
    char* slots = ring + mine * stages * stage;
    const uint32_t slots_at = static_cast<uint32_t>(__cvta_generic_to_shared(slots));
    auto fetch = [&](int slot) {
        X.template fetch<N>(slots + slot * stage, D, t);
        if (RESIDUAL) R.template fetch<N>(slots + slot * stage + share, D, t);
    };
    for (int s = 0; s < stages - 1; ++s) {
        if (s < rows) fetch(s);
        copies_commit();                                       // a row that is not there is an empty one
    }
    F2 w[N / 2], b[N / 2];
    odd_params<P, N>(w, a.w, a.p_dtype, has, t, 1.f);
    odd_params<P, N>(b, a.b, a.p_dtype, has, t, 0.f);
    const int count = __reduce_add_sync(0xffffffffu, min(N, has.full) + (has.more ? 1 : 0));
    const float n_warp = static_cast<float>(count), inverse_warp = TEAM ? inverse : (count > 0 ? 1.f / n_warp : 0.f);
    int slot = 0, turn = 0;
    for (int64_t row = 0; row < rows; ++row) {
        copies_wait_behind(stages - 2);
        team_barrier<TEAM>(mine);                              // this row is there; all are done with the one before, whose place is filled again
        if (row + stages - 1 < rows) fetch(slot == 0 ? stages - 1 : slot - 1);
        copies_commit();
        const uint32_t here = slots_at + slot * stage;
        slot = slot + 1 == stages ? 0 : slot + 1;
        F2 x[N / 2];
        odd_load<T, P, N>(x, X.row(here, t), has);
        X.step();
        if (RESIDUAL) {
            F2 r[N / 2];
            odd_load<T, P, N>(r, R.row(here + share, t), has);
            R.step();
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                x[i] = add(x[i], r[i]);
                if (sizeof(T) == 2) x[i] = of_bf16(to_bf16(x[i]));
            }
        }
        F2 total[2] = {f2(0.f), f2(0.f)}, q[2] = {f2(0.f), f2(0.f)};
#pragma unroll
        for (int i = 0; i < N / 2; ++i) total[i & 1] = add(total[i & 1], x[i]);
        const float s1 = warp_total(sum(add(total[0], total[1])));
        float m = s1 * inverse_warp;
        F2 minus_m = f2(-m);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            F2 d = add(x[i], minus_m);
            if (2 * i + 1 >= LEAST && 2 * i + 1 >= has.full) {
                const float2 v = parts(d);
                d = f2(has.has(2 * i) ? v.x : 0.f, has.has(2 * i + 1) ? v.y : 0.f);
            }
            q[i & 1] = fma(d, d, q[i & 1]);
        }
        float s2 = warp_total(sum(add(q[0], q[1])));
        if (!TEAM) {
            if (lane == 0) part[turn][warp] = make_float4(s1, s2, m, n_warp);
            __syncthreads();
            const float4 v = part[turn][lane % kLanes];
            turn ^= 1;
            m = warps_total<kLanes>(v.x) * inverse;
            s2 = warps_total<kLanes>(fmaf(v.w * (v.z - m), v.z - m, v.y));
            minus_m = f2(-m);
        }
        const float s = inverse_root(fmaf(s2, inverse, a.eps));
        const F2 scale = f2(s);
        if (h_at) {
            odd_store<T, P, N>(h_at, x, has);
            h_at += a.ldh;
        }
#pragma unroll
        for (int i = 0; i < N / 2; ++i) x[i] = fma(mul(add(x[i], minus_m), scale), w[i], b[i]);
        odd_store<T, P, N>(y_at, x, has);
        y_at += a.ldy;
        if (t == 0) {
            if (a.mean) a.mean[first + row] = m;
            if (a.rstd) a.rstd[first + row] = s;
        }
    }
}

template <typename T, int N, int LEAST, bool RESIDUAL, int TEAM, int P, int BLOCKS>
int launch_rows(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    constexpr int kTeams = TEAM ? 8 : 1, kRoom = 216 * 1024 / BLOCKS;
    const int share = odd_share(a.D, a.dtype), row = share * (RESIDUAL ? 2 : 1) * kTeams, stages = kRoom / row < 4 ? kRoom / row : 4;
    if (a.D > N * P || a.D < LEAST * P || stages < 2) return VELORA_ERR_UNSUPPORTED;
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    auto kern = norm_odd_kernel<T, N, LEAST, RESIDUAL, TEAM, P, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRoom) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    const int64_t blocks = ceil_div64(a.N, kTeams), most = static_cast<int64_t>(sm_count) * BLOCKS;
    return launch_chained(kern, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), TEAM ? 256 : P, static_cast<size_t>(stages) * row, stream, a, stages,
                          share);
}

// 4096 x 5461 bf16 31 us (the same rows on 16-byte boundaries 22), 12608 x 769 15, 8192 x 10001 109.
template <typename T, bool RESIDUAL>
int launch_width(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    if (a.D <= 256) return launch_rows<T, 8, 0, RESIDUAL, 1, 32, 3>(a, sm_count, stream);
    if (a.D <= 512) return launch_rows<T, 16, 8, RESIDUAL, 1, 32, 2>(a, sm_count, stream);
    if (a.D <= 1024) return launch_rows<T, 16, 8, RESIDUAL, 0, 64, 10>(a, sm_count, stream);
    if (a.D <= 2048) return launch_rows<T, 16, 8, RESIDUAL, 0, 128, 5>(a, sm_count, stream);
    if (a.D <= 2560) return launch_rows<T, 16, 12, RESIDUAL, 0, 160, 4>(a, sm_count, stream);
    if (a.D <= 4096) return launch_rows<T, 16, 10, RESIDUAL, 0, 256, 3>(a, sm_count, stream);
    if (a.D <= 5632) return launch_rows<T, 16, 11, RESIDUAL, 0, 352, 2>(a, sm_count, stream);
    if (a.D <= 7168) return launch_rows<T, 16, 12, RESIDUAL, 0, 448, 1>(a, sm_count, stream);
    if (a.D <= 8192) return launch_rows<T, 16, 14, RESIDUAL, 0, 512, 1>(a, sm_count, stream);
    if (a.D <= 10240) return launch_rows<T, 16, 12, RESIDUAL, 0, 640, 1>(a, sm_count, stream);
    if (a.D <= 12288) return launch_rows<T, 16, 13, RESIDUAL, 0, 768, 1>(a, sm_count, stream);
    return launch_layer_norm_any(a, sm_count, stream);
}

}  // namespace

int launch_layer_norm_odd(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    if (a.dtype == VELORA_BF16)
        return a.R ? launch_width<__nv_bfloat16, true>(a, sm_count, stream) : launch_width<__nv_bfloat16, false>(a, sm_count, stream);
    return a.R ? launch_width<float, true>(a, sm_count, stream) : launch_width<float, false>(a, sm_count, stream);
}

}  // namespace velora
