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
#include "row_chunks.cuh"

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

// Eight consecutive elements of a row as loaded, rows on 16-byte boundaries.  `begin` and `end` bound the matrix.
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int col, int D, bool in, int, const char*, const char*) { w = ld_stream_if(row + col, in && col + 8 <= D); }
    // The elements, zeros behind the row's end; the largest of their bits without signs.
    __device__ __forceinline__ uint32_t get(float (&x)[8], const __nv_bfloat16* row, int col, int D, bool in, int)
    {
        if (in && col < D && col + 8 > D) {
            uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < D) v[e >> 1] |= static_cast<uint32_t>(__bfloat16_as_ushort(row[col + e])) << (16 * (e & 1));
            w = make_uint4(v[0], v[1], v[2], v[3]);
        }
        return unpack(x, w);
    }
    static __device__ __forceinline__ uint32_t unpack(float (&x)[8], const uint4& w)
    {
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
        const uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
        return max(m << 16, m & 0xffff0000u);
    }
};
template <> struct Raw8<float> {
    uint4 w[2];
    __device__ __forceinline__ void load(const float* row, int col, int D, bool in, int, const char*, const char*)
    {
        w[0] = ld_stream_if(row + col, in && col + 8 <= D);
        w[1] = ld_stream_if(row + col + 4, in && col + 8 <= D);
    }
    __device__ __forceinline__ uint32_t get(float (&x)[8], const float* row, int col, int D, bool in, int) const
    {
        x[0] = __uint_as_float(w[0].x); x[1] = __uint_as_float(w[0].y); x[2] = __uint_as_float(w[0].z); x[3] = __uint_as_float(w[0].w);
        x[4] = __uint_as_float(w[1].x); x[5] = __uint_as_float(w[1].y); x[6] = __uint_as_float(w[1].z); x[7] = __uint_as_float(w[1].w);
        if (in && col < D && col + 8 > D) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < D) x[e] = row[col + e];
        }
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
        return top;
    }
};
// bf16 rows on any boundary: a lane loads the aligned 16 bytes that its first element lies in, its neighbour has the rest.
struct Raw8Odd {
    uint4 w, over;
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int col, int D, bool in, int lane, const char* begin, const char* end)
    {
        const char* a = reinterpret_cast<const char*>(reinterpret_cast<uintptr_t>(row + col) & ~static_cast<uintptr_t>(15));
        const char* row_end = reinterpret_cast<const char*>(row + D);
        w = over = make_uint4(0u, 0u, 0u, 0u);
        if (in && a < row_end) w = load_aligned_chunk(a, begin, end);
        if (in && lane == 31 && a + 16 < row_end) over = load_aligned_chunk(a + 16, begin, end);
    }
    __device__ __forceinline__ uint32_t get(float (&x)[8], const __nv_bfloat16* row, int col, int D, bool, int lane)
    {
        uint4 next = make_uint4(__shfl_down_sync(0xffffffffu, w.x, 1), __shfl_down_sync(0xffffffffu, w.y, 1),
                                __shfl_down_sync(0xffffffffu, w.z, 1), __shfl_down_sync(0xffffffffu, w.w, 1));
        if (lane == 31) next = over;
        w = shift_chunks(w, next, static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row + col) & 15));
        if (col + 8 > D) {                                             // what follows is the next row's
            uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e >= D) v[e >> 1] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
            w = make_uint4(v[0], v[1], v[2], v[3]);
        }
        return Raw8<__nv_bfloat16>::unpack(x, w);
    }
};

__device__ __forceinline__ uint4 pack8(const float (&y)[8])
{
    return make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&y)[8]) { __stcs(reinterpret_cast<uint4*>(p), pack8(y)); }
__device__ __forceinline__ void store8(float* p, const float (&y)[8]) { store_f32x8(p, y); }

// Rows of Q on 8-byte boundaries; RAW says which rows of X.
template <typename T, typename RAW, int U>
__global__ void __launch_bounds__(kStreamThreads)
checkpoint_store_vec_kernel(const T* X, int64_t ldx, int64_t N, int D, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, int segs)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const char* begin = reinterpret_cast<const char*>(X);
    const char* end = reinterpret_cast<const char*>(X + (N - 1) * ldx + D);
    const int64_t warp = static_cast<int64_t>(blockIdx.x) * (kStreamThreads / 32) + (threadIdx.x >> 5);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * (kStreamThreads / 32) * U;
    const int64_t step_rows = stride / segs;
    const int step_segs = static_cast<int>(stride - step_rows * segs);
    UnitWalk at;
    for (at.start(warp * U, segs); at.row < N; at.step(step_rows, step_segs, segs)) {
        RAW raw[U];
        UnitWalk u = at;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            raw[i].load(X + u.row * ldx, u.seg * kSegment + lane * 8, D, u.row < N, lane, begin, end);
            u.step(0, 1, segs);
        }
        u = at;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int col = u.seg * kSegment + lane * 8;
            float x[8];
            uint32_t top = raw[i].get(x, X + u.row * ldx, col, D, u.row < N, lane);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t exponent = checkpoint_exponent(top);
            const uint2 q = checkpoint_codes(x, exponent);
            if (u.row < N && col < D) {
                int8_t* dst = Q + u.row * ldq + col;
                if (col + 8 <= D) {
                    __stcs(reinterpret_cast<uint2*>(dst), q);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col + e < D) dst[e] = static_cast<int8_t>((e < 4 ? q.x : q.y) >> (8 * (e % 4)));
                }
                if ((lane & 3) == 0) E[u.row * lde + col / kCheckpointBlock] = static_cast<uint8_t>(exponent);
            }
            u.step(0, 1, segs);
        }
    }
}

// Everything else: one element per lane, so a warp reads and writes consecutive ones; the block's maximum over the warp's lanes.
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

// Eight values of a bf16 row on any boundary.  A lane puts the aligned 16 bytes that its first element lies in together with its
// neighbour's last elements; what has no such neighbour is written one element at a time.
__device__ __forceinline__ void store8_odd(__nv_bfloat16* p, const float (&y)[8], int count, int lane)
{
    const uint4 v = pack8(y);
    const uint32_t s = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) & 15);        // bytes of the chunk that are the neighbour's
    const uint4 before = make_uint4(__shfl_up_sync(0xffffffffu, v.x, 1), __shfl_up_sync(0xffffffffu, v.y, 1),
                                    __shfl_up_sync(0xffffffffu, v.z, 1), __shfl_up_sync(0xffffffffu, v.w, 1));
    const int mine = static_cast<int>(16 - s) / 2;                                        // elements in the chunk
    const bool whole = (lane > 0 || s == 0) && count >= mine;
    const bool next_whole = __shfl_down_sync(0xffffffffu, static_cast<int>(whole), 1) != 0 && lane < 31;
    if (whole) __stcs(reinterpret_cast<uint4*>(reinterpret_cast<char*>(p) - s), s == 0 ? v : shift_chunks(before, v, 16 - s));
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < count && (e < mine ? !whole : !next_whole)) p[e] = __float2bfloat16_rn(y[e]);
}

// Rows of Q on 8-byte boundaries, rows of Xhat on 16-byte ones unless ODD.
template <typename T, int U, bool ODD = false>
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
            float y[8];
            checkpoint_values(q[i], exponent[i], y);
            T* dst = Xhat + u.row * ldx + col;
            if constexpr (ODD) {
                store8_odd(dst, y, u.row < N ? min(max(D - col, 0), 8) : 0, lane);
            } else if (u.row < N && col < D) {
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
    const bool many = units > static_cast<int64_t>(sm_count) * kStreamCtasPerSm * (kStreamThreads / 32);
    if (reinterpret_cast<uintptr_t>(Q) % 8 == 0 && ldq % 8 == 0) {
        if (c_rows_vec(X, ldx, sizeof(T))) {
            if (many) return launch_chained(checkpoint_store_vec_kernel<T, Raw8<T>, 4>, dim3(grid_for(units, 4, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
            return launch_chained(checkpoint_store_vec_kernel<T, Raw8<T>, 1>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
        }
        if constexpr (sizeof(T) == 2) {
            if (many) return launch_chained(checkpoint_store_vec_kernel<T, Raw8Odd, 4>, dim3(grid_for(units, 4, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
            return launch_chained(checkpoint_store_vec_kernel<T, Raw8Odd, 1>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
        }
    }
    return launch_chained(checkpoint_store_elem_kernel<T>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, segs);
}

template <typename T>
int load_typed(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int64_t D, void* Xhat, int64_t ldx, int sm_count, cudaStream_t stream)
{
    const int d = static_cast<int>(D), segs = static_cast<int>(ceil_div64(D, kSegment));
    const int64_t units = N * segs;
    T* x = static_cast<T*>(Xhat);
    const bool many = units > static_cast<int64_t>(sm_count) * kStreamCtasPerSm * (kStreamThreads / 32);
    if (reinterpret_cast<uintptr_t>(Q) % 8 == 0 && ldq % 8 == 0) {
        if (c_rows_vec(Xhat, ldx, sizeof(T))) {
            if (many) return launch_chained(checkpoint_load_vec_kernel<T, 4>, dim3(grid_for(units, 4, sm_count)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, segs);
            return launch_chained(checkpoint_load_vec_kernel<T, 1>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, segs);
        }
        if constexpr (sizeof(T) == 2) {
            if (many) return launch_chained(checkpoint_load_vec_kernel<T, 4, true>, dim3(grid_for(units, 4, sm_count)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, segs);
            return launch_chained(checkpoint_load_vec_kernel<T, 1, true>, dim3(grid_for(units, 1, sm_count)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, segs);
        }
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
