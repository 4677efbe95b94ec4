// 8-bit checkpoints of a layer's input: for the layers that a rank-1 projection is not used on, the array that the backward pass needs
// is kept as one byte per element and one exponent per block of 32 columns of a row.
//   a = max |x| over the block,  s = 2^e the smallest power of two with a <= 127 s  (-126 <= e <= 121),
//   q = round(x / s), ties to even, at most 127 in size,  E = e + 127,      Xhat = q 2^(E - 127).
// A power of two costs half a bit against a step of a / 127 and buys three things: x / s is exact, so the code is the nearest one
// whatever the order of operations; q s has seven significant bits and so is exact in bf16, fp32 and for the tensor cores;
// and the step takes a byte.  E = 255 marks a block with an infinity or a NaN; its codes are zero, and 0 * 2^128 reads back as
// NaN.  Both are bound by HBM: N D (b + 1 + 1/32) bytes each way.
#include "checkpoint.cuh"
#include "gemm_store.cuh"

namespace velora {

namespace {

constexpr int kSegment = 256;                       // columns of a row that a warp takes at a time: 8 per lane, 4 lanes a block

// Units (row, segment) dealt to warps U at a time; one division at the start, then steps.
struct UnitWalk {
    int64_t row;
    int seg;
    __device__ __forceinline__ void start(int64_t unit, int segs)
    {
        row = unit / segs;
        seg = static_cast<int>(unit - row * segs);
    }
    __device__ __forceinline__ void step(int64_t rows, int by, int segs)
    {
        row += rows;
        seg += by;
        if (seg >= segs) {
            seg -= segs;
            ++row;
        }
    }
};

// Eight elements at a 16-byte boundary as loaded.
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool take) { w = ld_stream_if(p, take); }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    }
};
template <> struct Raw8<float> {
    uint4 w[2];
    __device__ __forceinline__ void load(const float* p, bool take)
    {
        w[0] = ld_stream_if(p, take);
        w[1] = ld_stream_if(p + 4, take);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        x[0] = __uint_as_float(w[0].x); x[1] = __uint_as_float(w[0].y); x[2] = __uint_as_float(w[0].z); x[3] = __uint_as_float(w[0].w);
        x[4] = __uint_as_float(w[1].x); x[5] = __uint_as_float(w[1].y); x[6] = __uint_as_float(w[1].z); x[7] = __uint_as_float(w[1].w);
    }
};

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&y)[8])
{
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])));
}
__device__ __forceinline__ void store8(float* p, const float (&y)[8]) { store_f32x8(p, y); }

// Rows of X on 16-byte boundaries, rows of Q on 8-byte ones.
template <typename T, int U>
__global__ void __launch_bounds__(kStreamThreads)
checkpoint_store_vec_kernel(const T* X, int64_t ldx, int64_t N, int D, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, int segs)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * (kStreamThreads / 32) + (threadIdx.x >> 5);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * (kStreamThreads / 32) * U;
    const int64_t step_rows = stride / segs;
    const int step_segs = static_cast<int>(stride - step_rows * segs);
    UnitWalk at;
    for (at.start(warp * U, segs); at.row < N; at.step(step_rows, step_segs, segs)) {
        Raw8<T> raw[U];
        UnitWalk u = at;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int col = u.seg * kSegment + lane * 8;
            raw[i].load(X + u.row * ldx + col, u.row < N && col + 8 <= D);
            u.step(0, 1, segs);
        }
        u = at;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int col = u.seg * kSegment + lane * 8;
            float x[8];
            raw[i].get(x);
            const bool tail = u.row < N && col < D && col + 8 > D;
            if (tail) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < D) x[e] = Elem<T>::load(X + u.row * ldx + col + e);
            }
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t exponent = checkpoint_exponent(top);
            uint32_t q[2];
            checkpoint_codes(x, exponent, q);
            if (u.row < N && col < D) {
                int8_t* dst = Q + u.row * ldq + col;
                if (!tail) {
                    __stcs(reinterpret_cast<uint2*>(dst), make_uint2(q[0], q[1]));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col + e < D) dst[e] = static_cast<int8_t>(q[e / 4] >> (8 * (e % 4)));
                }
                if ((lane & 3) == 0) E[u.row * lde + col / kCheckpointBlock] = static_cast<uint8_t>(exponent);
            }
            u.step(0, 1, segs);
        }
    }
}

// Any rows: one element per lane, so a warp reads and writes consecutive ones; the block's maximum over the warp's lanes.
template <typename T>
__global__ void __launch_bounds__(kStreamThreads)
checkpoint_store_elem_kernel(const T* X, int64_t ldx, int64_t N, int D, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, int segs)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * (kStreamThreads / 32);
    const int64_t step_rows = stride / segs;
    const int step_segs = static_cast<int>(stride - step_rows * segs);
    UnitWalk at;
    for (at.start(static_cast<int64_t>(blockIdx.x) * (kStreamThreads / 32) + (threadIdx.x >> 5), segs); at.row < N;
         at.step(step_rows, step_segs, segs)) {
        const int col0 = at.seg * kSegment + lane;
        const T* src = X + at.row * ldx + col0;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = col0 + 32 * i < D ? Elem<T>::load(src + 32 * i) : 0.f;
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t exponent = checkpoint_exponent(__reduce_max_sync(0xffffffffu, __float_as_uint(x[i]) & 0x7fffffffu));
            if (lane == i) mine = exponent;
            if (col0 + 32 * i < D) Q[at.row * ldq + col0 + 32 * i] = static_cast<int8_t>(checkpoint_code(x[i], exponent));
        }
        if (lane < 8 && at.seg * kSegment + 32 * lane < D) E[at.row * lde + at.seg * (kSegment / 32) + lane] = static_cast<uint8_t>(mine);
    }
}

template <typename T, int U>
__global__ void __launch_bounds__(kStreamThreads)
checkpoint_load_vec_kernel(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int D, T* Xhat, int64_t ldx, int segs)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * (kStreamThreads / 32) + (threadIdx.x >> 5);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * (kStreamThreads / 32) * U;
    const int64_t step_rows = stride / segs;
    const int step_segs = static_cast<int>(stride - step_rows * segs);
    UnitWalk at;
    for (at.start(warp * U, segs); at.row < N; at.step(step_rows, step_segs, segs)) {
        uint2 q[U];
        uint32_t exponent[U];
        UnitWalk u = at;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int col = u.seg * kSegment + lane * 8;
            const bool in = u.row < N && col < D;
            q[i] = make_uint2(0, 0);
            exponent[i] = 0;
            if (in) {
                exponent[i] = E[u.row * lde + col / kCheckpointBlock];
                const int8_t* src = Q + u.row * ldq + col;
                if (col + 8 <= D) {
                    q[i] = __ldcs(reinterpret_cast<const uint2*>(src));
                } else {
                    for (int e = 0; e < D - col; ++e) {
                        const uint32_t byte = static_cast<uint8_t>(src[e]);
                        if (e < 4) q[i].x |= byte << (8 * e);
                        else q[i].y |= byte << (8 * e - 32);
                    }
                }
            }
            u.step(0, 1, segs);
        }
        u = at;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int col = u.seg * kSegment + lane * 8;
            if (u.row < N && col < D) {
                const float s = checkpoint_step(exponent[i]);
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = static_cast<float>(static_cast<int8_t>((e < 4 ? q[i].x : q[i].y) >> (8 * (e % 4)))) * s;
                T* dst = Xhat + u.row * ldx + col;
                if (col + 8 <= D) {
                    store8(dst, y);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col + e < D) Elem<T>::store(dst + e, y[e]);
                }
            }
            u.step(0, 1, segs);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kStreamThreads)
checkpoint_load_elem_kernel(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int D, T* Xhat, int64_t ldx, int segs)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * (kStreamThreads / 32);
    const int64_t step_rows = stride / segs;
    const int step_segs = static_cast<int>(stride - step_rows * segs);
    UnitWalk at;
    for (at.start(static_cast<int64_t>(blockIdx.x) * (kStreamThreads / 32) + (threadIdx.x >> 5), segs); at.row < N;
         at.step(step_rows, step_segs, segs)) {
        const int col0 = at.seg * kSegment + lane;
        float q[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = col0 + 32 * i < D;
            q[i] = in ? static_cast<float>(Q[at.row * ldq + col0 + 32 * i]) : 0.f;
            s[i] = in ? checkpoint_step(E[at.row * lde + at.seg * (kSegment / 32) + i]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col0 + 32 * i < D) Elem<T>::store(Xhat + at.row * ldx + col0 + 32 * i, q[i] * s[i]);
    }
}

// CTAs for `units` warps' worth of work, U units a warp and step.
unsigned grid_for(int64_t units, int u, int sm_count)
{
    const int64_t ctas = ceil_div64(units, static_cast<int64_t>(kStreamThreads / 32) * u), most = static_cast<int64_t>(sm_count) * kStreamCtasPerSm;
    return static_cast<unsigned>(ctas < most ? ctas : most);
}

template <typename T>
int store_typed(const void* X, int64_t N, int64_t D, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, int sm_count, cudaStream_t stream)
{
    const int d = static_cast<int>(D), segs = static_cast<int>(ceil_div64(D, kSegment));
    const int64_t units = N * segs;
    const T* x = static_cast<const T*>(X);
    if (c_rows_vec(X, ldx, sizeof(T)) && reinterpret_cast<uintptr_t>(Q) % 8 == 0 && ldq % 8 == 0) {
        if (units > static_cast<int64_t>(sm_count) * kStreamCtasPerSm * (kStreamThreads / 32))
            return launch_chained(checkpoint_store_vec_kernel<T, 4>, dim3(grid_for(units, 4, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
        return launch_chained(checkpoint_store_vec_kernel<T, 1>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
    }
    return launch_chained(checkpoint_store_elem_kernel<T>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
}

template <typename T>
int load_typed(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int64_t D, void* Xhat, int64_t ldx, int sm_count, cudaStream_t stream)
{
    const int d = static_cast<int>(D), segs = static_cast<int>(ceil_div64(D, kSegment));
    const int64_t units = N * segs;
    T* x = static_cast<T*>(Xhat);
    if (c_rows_vec(Xhat, ldx, sizeof(T)) && reinterpret_cast<uintptr_t>(Q) % 8 == 0 && ldq % 8 == 0) {
        if (units > static_cast<int64_t>(sm_count) * kStreamCtasPerSm * (kStreamThreads / 32))
            return launch_chained(checkpoint_load_vec_kernel<T, 4>, dim3(grid_for(units, 4, sm_count)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, segs);
        return launch_chained(checkpoint_load_vec_kernel<T, 1>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, segs);
    }
    return launch_chained(checkpoint_load_elem_kernel<T>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, segs);
}

}  // namespace

int launch_checkpoint_store(const void* X, int x_dtype, int64_t N, int64_t D, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    return x_dtype == VELORA_BF16 ? store_typed<__nv_bfloat16>(X, N, D, ldx, Q, ldq, E, lde, di.sm_count, stream)
                                  : store_typed<float>(X, N, D, ldx, Q, ldq, E, lde, di.sm_count, stream);
}

int launch_checkpoint_load(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int64_t D, void* Xhat, int x_dtype, int64_t ldx, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    return x_dtype == VELORA_BF16 ? load_typed<__nv_bfloat16>(Q, ldq, E, lde, N, D, Xhat, ldx, di.sm_count, stream)
                                  : load_typed<float>(Q, ldq, E, lde, N, D, Xhat, ldx, di.sm_count, stream);
}

}  // namespace velora
