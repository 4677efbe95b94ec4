// Layer norm of rows, with a residual added in front.
//   h = x + r (rounded to the rows' type),  m = mean h,  s = 1 / sqrt(mean (h - m)^2 + eps),  y = (h - m) s w + b
// Bound by HBM: x (and r) once in, y (and h) once out.  A row is held in the registers of a warp or of a block while its mean and its variance about the
// mean are taken; blocks walk over neighbouring rows, the weights stay in registers, and the next rows are on their way to shared memory meanwhile.
// A warp takes its own columns' mean and squares about it, and the block puts those together (sum, squares, mean and number of each warp), so that a row
// costs one barrier and nothing is lost to a mean that is large beside the deviation.
#include "layer_norm_rows.cuh"

namespace velora {

namespace {

// R: rows that a team works on side by side.
template <typename T, int C, int R, int STAGES, bool RESIDUAL, bool ONE, int THREADS, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS)
norm_rows_kernel(const NormArgs a, bool wide)
{
    constexpr int E = Word<T>::E, kTeams = ONE ? 8 : 1, kLanes = kWarpLanes<THREADS>;
    extern __shared__ __align__(16) char ring_bytes[];
    __shared__ float4 part[2][R][ONE ? 1 : kLanes];               // sum, squares about the warp's mean, that mean, number of columns
    const int P = ONE ? 32 : blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = ONE ? lane : threadIdx.x;
    const int D = a.D, share = C * P * 16, row_bytes = share * (RESIDUAL ? 2 : 1), stage = R * row_bytes, ring_end = STAGES * stage;
    const bool last = ((C - 1) * P + t) * E < D;               // the last word is there
    const float inverse = 1.f / static_cast<float>(D);
    if (!ONE)                                                  // warps that are not there
        for (int i = threadIdx.x; i < 2 * R * kLanes; i += blockDim.x) (&part[0][0][0])[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    pdl_wait();
    pdl_trigger();

    // This team's rows.
    const int64_t team = static_cast<int64_t>(blockIdx.x) * kTeams + (ONE ? warp : 0), teams = static_cast<int64_t>(gridDim.x) * kTeams;
    const int64_t each = a.N / teams, over = a.N % teams, first = each * team + (team < over ? team : over), rows = each + (team < over ? 1 : 0);
    const T* x_at = static_cast<const T*>(a.X) + first * a.ldx + t * E;
    const T* r_at = RESIDUAL ? static_cast<const T*>(a.R) + first * a.ldr + t * E : nullptr;
    T* y_at = static_cast<T*>(a.Y) + first * a.ldy + t * E;
    T* h_at = a.H ? static_cast<T*>(a.H) + first * a.ldh + t * E : nullptr;
    const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(ring_bytes)) + (ONE ? warp * ring_end : 0) + t * 16;
    auto fetch = [&](int at, int64_t row) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (row + r < rows) {
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (c < C - 1 || last) {
                        copy_word(ring + at + r * row_bytes + c * P * 16, x_at + c * P * E);
                        if (RESIDUAL) copy_word(ring + at + r * row_bytes + share + c * P * 16, r_at + c * P * E);
                    }
                x_at += a.ldx;
                if (RESIDUAL) r_at += a.ldr;
            }
        copies_commit();                                       // rows that are not there are none
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(s * stage, s * R);
    F2 w[C][E / 2], b[C][E / 2];
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (c < C - 1 || last) {
            load_columns<E>(w[c], a.w, a.p_dtype, wide, (c * P + t) * E, 1.f);
            load_columns<E>(b[c], a.b, a.p_dtype, wide, (c * P + t) * E, 0.f);
        }
    const int words = __reduce_add_sync(0xffffffffu, C - 1 + (last ? 1 : 0));
    const float n_warp = static_cast<float>(words * E), inverse_warp = ONE ? inverse : (words > 0 ? 1.f / n_warp : 0.f);
    if (!ONE) __syncthreads();
    int at = 0, turn = 0;
    for (int64_t row = 0; row < rows; row += R) {
        fetch(at == 0 ? ring_end - stage : at - stage, row + (STAGES - 1) * R);
        copies_wait<STAGES - 1>();
        Word<T> x[R][C];                                       // of a row that is not there: whatever was
        float s1[R], s2[R], m[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            F2 total = f2(0.f);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c < C - 1 || last) {
                    x[r][c].load(ring + at + r * row_bytes + c * P * 16);
                    if (RESIDUAL) {
                        Word<T> y;
                        y.load(ring + at + r * row_bytes + share + c * P * 16);
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) x[r][c].x[i] = add(x[r][c].x[i], y.x[i]);
                        x[r][c].round();
                    }
                    total = add(total, x[r][c].total());
                }
            s1[r] = sum(total);
        }
        at = at == ring_end - stage ? 0 : at + stage;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s1[r] = warp_total(s1[r]);
            m[r] = s1[r] * inverse_warp;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const F2 minus_m = f2(-m[r]);
            F2 q[2] = {f2(0.f), f2(0.f)};
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c < C - 1 || last)
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        const F2 d = add(x[r][c].x[i], minus_m);
                        q[i & 1] = fma(d, d, q[i & 1]);
                    }
            s2[r] = sum(add(q[0], q[1]));
        }
#pragma unroll
        for (int r = 0; r < R; ++r) s2[r] = warp_total(s2[r]);
        if (!ONE) {
            if (lane == 0)
#pragma unroll
                for (int r = 0; r < R; ++r) part[turn][r][warp] = make_float4(s1[r], s2[r], m[r], n_warp);
            __syncthreads();                                   // the other half's readers are past the barrier before
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 v = part[turn][r][lane % kLanes];
                m[r] = warps_total<kLanes>(v.x) * inverse;
                s2[r] = warps_total<kLanes>(fmaf(v.w * (v.z - m[r]), v.z - m[r], v.y));
            }
            turn ^= 1;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (R > 1 && row + r >= rows) break;
            const float s = inverse_root(fmaf(s2[r], inverse, a.eps));
            const F2 minus_m = f2(-m[r]), scale = f2(s);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c < C - 1 || last) {
                    if (h_at) x[r][c].store(h_at + c * P * E);
                    Word<T> y;
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) y.x[i] = fma(mul(add(x[r][c].x[i], minus_m), scale), w[c][i], b[c][i]);
                    y.store(y_at + c * P * E);
                }
            y_at += a.ldy;
            if (h_at) h_at += a.ldh;
            if (t == 0) {
                if (a.mean) a.mean[first + row + r] = m[r];
                if (a.rstd) a.rstd[first + row + r] = s;
            }
        }
    }
}

template <typename T, int C, bool RESIDUAL, bool ONE, int THREADS, int BLOCKS, int R = 1>
int launch_rows(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    constexpr int kTeams = ONE ? 8 : 1;
    // R rows of a full block on their way or in use: two, up to four times, in the share of an SM's shared memory that BLOCKS leave.
    constexpr int kRow = R * C * THREADS * 16 * (RESIDUAL ? 2 : 1), kFit = 216 * 1024 / BLOCKS / kRow, kStages = kFit > 4 ? 4 : kFit;
    static_assert(kStages >= 2, "two rows");
    static DeviceOnce configured;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VELORA_ERR_CUDA;
    auto kern = norm_rows_kernel<T, C, R, kStages, RESIDUAL, ONE, THREADS, BLOCKS>;
    if (!configured.get(dev)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kStages * kRow) != cudaSuccess) return VELORA_ERR_CUDA;
        configured.set(dev);
    }
    const int words = row_words(a.D, a.dtype), threads = ONE ? THREADS : row_threads(words, C), per_row = ONE ? 32 : threads;
    if (threads > THREADS || (C - 1) * per_row >= words || C * per_row < words) return VELORA_ERR_UNSUPPORTED;         // only last words may be missing
    const int64_t blocks = ceil_div64(a.N, kTeams), most = static_cast<int64_t>(sm_count) * BLOCKS;
    return launch_chained(kern, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), threads, static_cast<size_t>(kStages) * kRow / THREADS * threads,
                          stream, a, aligned16(a.w) && aligned16(a.b));
}

// By the row's words: what was fastest of some forty shapes, in TB/s of x, y (and r, h).  bf16, without and with a residual: 16384 x 256 2.6 / 4.1, 16384 x 512
// 4.2 / 5.2, 12608 x 768 4.0 / 5.0, 16384 x 1024 4.5 / 5.2, 8192 x 2048 4.5 / 5.3, 8192 x 4096 5.0 / 5.8 (256 threads with a residual: 5.2), 4096 x 5464
// 4.1 / 5.3 (256 threads: 5.1), 8192 x 8192 5.2 (512 threads: 4.6) / 6.2, 8192 x 11008 5.7 (a row at a time: 5.0) / 5.5.  fp32: 8192 x
// 512 3.9 / 5.0, 12608 x 768 5.0 (a warp a row: 4.7) / 5.1, 4096 x 2048 4.9 / 5.1, 4096 x 4096 5.4 / 5.3, 4096 x 5464 5.3 (a row at a time: 5.0) / 5.1, 4096 x
// 8192 5.7 / 5.4, 2048 x 11008 5.4 / 5.2.
// Two rows side by side pay where one block of an SM is left and its row is 17 to 24 KB, so that a dozen warps wait at each barrier and sum; with a residual
// (131 -> 136 us at 8192 x 11008), in smaller rows, which have other blocks to run meanwhile, and in rows over 24 KB (fp32 4096 x 8192: 47 -> 50 us) they do not.
template <typename T, bool RESIDUAL>
int launch_words(const NormArgs& a, int sm_count, cudaStream_t stream)
{
    const int words = row_words(a.D, a.dtype);
    if (words <= 32) return launch_rows<T, 1, RESIDUAL, true, 256, 3>(a, sm_count, stream);
    if (words <= 64) return launch_rows<T, 2, RESIDUAL, true, 256, 2>(a, sm_count, stream);
    if constexpr (sizeof(T) == 2) {
        if (words <= 96) return launch_rows<T, 3, RESIDUAL, true, 256, 2>(a, sm_count, stream);
        if (words <= 128) return launch_rows<T, 2, RESIDUAL, false, 64, 10>(a, sm_count, stream);
        if (words <= 256) return launch_rows<T, 2, RESIDUAL, false, 128, 5>(a, sm_count, stream);
        if (words <= 512) return RESIDUAL ? launch_rows<T, 1, true, false, 512, 2>(a, sm_count, stream) : launch_rows<T, 2, false, false, 256, 3>(a, sm_count, stream);
        if (words <= 704) return launch_rows<T, 2, RESIDUAL, false, 352, 2>(a, sm_count, stream);
        if (RESIDUAL) return words <= 1408 ? launch_rows<T, 2, true, false, 704, 1>(a, sm_count, stream) : words <= 1536 ? launch_rows<T, 3, true, false, 512, 1>(a, sm_count, stream) : launch_layer_norm_any(a, sm_count, stream);
        if (words <= 1024) return launch_rows<T, 4, false, false, 256, 2>(a, sm_count, stream);
        if (words <= 1536) return launch_rows<T, 4, false, false, 384, 1, 2>(a, sm_count, stream);
    } else {
        if (words <= 96) return launch_rows<T, 3, RESIDUAL, true, 256, 2>(a, sm_count, stream);
        if (words <= 128) return launch_rows<T, 4, RESIDUAL, true, 256, 2>(a, sm_count, stream);
        if (words <= 192) return launch_rows<T, 2, RESIDUAL, false, 96, 8>(a, sm_count, stream);
        if (words <= 384) return launch_rows<T, 3, RESIDUAL, false, 128, 5>(a, sm_count, stream);
        if (words <= 512) return launch_rows<T, 4, RESIDUAL, false, 128, 4>(a, sm_count, stream);
        if (words <= 1024) return launch_rows<T, 2, RESIDUAL, false, 512, 2>(a, sm_count, stream);
        if (!RESIDUAL && words <= 1536) return launch_rows<T, 4, false, false, 384, 1, 2>(a, sm_count, stream);
        if (words <= 2048) return launch_rows<T, 4, RESIDUAL, false, 512, 1>(a, sm_count, stream);
        if (words <= 4 * 768) return launch_rows<T, 4, RESIDUAL, false, 768, 1>(a, sm_count, stream);
    }
    return launch_layer_norm_any(a, sm_count, stream);
}

}  // namespace

int launch_layer_norm(const NormArgs& a, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    const bool vec = a.D * static_cast<int64_t>(dtype_size(a.dtype)) % 16 == 0 && rows_vec(a.X, a.ldx, a.dtype) && rows_vec(a.R, a.ldr, a.dtype) &&
                     rows_vec(a.H, a.ldh, a.dtype) && rows_vec(a.Y, a.ldy, a.dtype);
    if (!vec) return launch_layer_norm_odd(a, di.sm_count, stream);
    if (a.dtype == VELORA_BF16)
        return a.R ? launch_words<__nv_bfloat16, true>(a, di.sm_count, stream) : launch_words<__nv_bfloat16, false>(a, di.sm_count, stream);
    return a.R ? launch_words<float, true>(a, di.sm_count, stream) : launch_words<float, false>(a, di.sm_count, stream);
}

}  // namespace velora
