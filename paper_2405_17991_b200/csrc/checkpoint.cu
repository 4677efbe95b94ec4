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

// Runs of `U` segments of a row dealt to warps; one division at the start, then steps.  Both streams were held up by instructions before
// HBM (16 an element and 70 % of the issue slots with the addresses of every segment worked out anew): a run works out its
// addresses once, its segments are constant offsets.
struct RunWalk {
    int64_t row, step_rows;
    int run, step_runs, runs;
    __device__ __forceinline__ RunWalk(int runs_a_row) : runs(runs_a_row)
    {
        const int64_t warp = static_cast<int64_t>(blockIdx.x) * (kStreamThreads / 32) + (threadIdx.x >> 5);
        const int64_t warps = static_cast<int64_t>(gridDim.x) * (kStreamThreads / 32);
        row = warp / runs;
        run = static_cast<int>(warp - row * runs);
        step_rows = warps / runs;
        step_runs = static_cast<int>(warps - step_rows * runs);
    }
    __device__ __forceinline__ void next()
    {
        row += step_rows;
        run += step_runs;
        if (run >= runs) {
            run -= runs;
            ++row;
        }
    }
};

// Eight elements of a row as loaded, from p on, of which `left` (may be negative, or more than 8) belong to the row.
// Rows on 16-byte boundaries:
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left, bool, int) { w = ld_stream_if(p, left >= 8); }
    // The elements, zeros behind the row's end; the largest of their bits without signs.
    __device__ __forceinline__ uint32_t get(float (&x)[8], const __nv_bfloat16* p, int left, int)
    {
        if (left > 0 && left < 8) {
            uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) v[e >> 1] |= static_cast<uint32_t>(__bfloat16_as_ushort(p[e])) << (16 * (e & 1));
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
    __device__ __forceinline__ void load(const float* p, int left, bool, int)
    {
        w[0] = ld_stream_if(p, left >= 8);
        w[1] = ld_stream_if(p + 4, left >= 8);
    }
    __device__ __forceinline__ uint32_t get(float (&x)[8], const float* p, int left, int) const
    {
        x[0] = __uint_as_float(w[0].x); x[1] = __uint_as_float(w[0].y); x[2] = __uint_as_float(w[0].z); x[3] = __uint_as_float(w[0].w);
        x[4] = __uint_as_float(w[1].x); x[5] = __uint_as_float(w[1].y); x[6] = __uint_as_float(w[1].z); x[7] = __uint_as_float(w[1].w);
        if (left > 0 && left < 8) {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < left) x[e] = p[e];
        }
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
        return top;
    }
};
// bf16 rows on any boundary: a lane loads the aligned 16 bytes that its first element lies in, its neighbour has the rest.  Element by element
// where the aligned bytes of a row may lie outside the matrix (`edge`: the first and last rows).
struct Raw8Odd {
    uint4 w, over;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left, bool edge, int lane)
    {
        w = over = make_uint4(0u, 0u, 0u, 0u);
        if (edge) return;
        const int s = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15);
        const char* a = reinterpret_cast<const char*>(p) - s;
        w = ld_stream_if(a, left + s / 2 > 0);
        over = ld_stream_if(a + 16, lane == 31 && left + s / 2 > 8);
    }
    __device__ __forceinline__ uint32_t get(float (&x)[8], const __nv_bfloat16* p, int left, int lane)
    {
        uint4 next = make_uint4(__shfl_down_sync(0xffffffffu, w.x, 1), __shfl_down_sync(0xffffffffu, w.y, 1),
                                __shfl_down_sync(0xffffffffu, w.z, 1), __shfl_down_sync(0xffffffffu, w.w, 1));
        if (lane == 31) next = over;
        w = shift_chunks(w, next, static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) & 15));
        if (left < 8) {                                               // what follows is the next row's
            uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= left) v[e >> 1] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
            w = make_uint4(v[0], v[1], v[2], v[3]);
        }
        return Raw8<__nv_bfloat16>::unpack(x, w);
    }
    static __device__ __forceinline__ uint32_t get_edge(float (&x)[8], const __nv_bfloat16* p, int left)
    {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = e < left ? __bfloat162float(p[e]) : 0.f;
            top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
        }
        return top;
    }
};

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&y)[8])
{
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])));
}
__device__ __forceinline__ void store8(float* p, const float (&y)[8]) { store_f32x8(p, y); }

// CTAs on an SM, by the registers that four segments in flight take.
template <typename RAW> constexpr int kResident = sizeof(RAW) == 16 ? 5 : 4;
constexpr int kResidentLoad = 5;

// Rows of Q on 8-byte boundaries; RAW says which rows of X.
template <typename T, typename RAW, int U>
__global__ void __launch_bounds__(kStreamThreads, kResident<RAW>)
checkpoint_store_vec_kernel(const T* X, int64_t ldx, int64_t N, int D, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, int runs)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    for (RunWalk at(runs); at.row < N; at.next()) {
        const int col0 = at.run * (U * kSegment) + lane * 8, left0 = D - col0;
        const T* src = X + at.row * ldx + col0;
        const bool edge = at.row * ldx < 8 || (N - 1 - at.row) * ldx < 8;      // fewer than 16 bytes of the matrix before or behind the row
        RAW raw[U];
#pragma unroll
        for (int i = 0; i < U; ++i) raw[i].load(src + i * kSegment, left0 - i * kSegment, edge, lane);
        int8_t* dst = Q + at.row * ldq + col0;
        uint8_t* exps = E + at.row * lde + col0 / kCheckpointBlock;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int left = left0 - i * kSegment;
            if (D - at.run * (U * kSegment) <= i * kSegment) break;            // for the whole warp
            float x[8];
            uint32_t top = raw[i].get(x, src + i * kSegment, left, lane);
            if constexpr (sizeof(RAW) == sizeof(Raw8Odd) && sizeof(T) == 2)
                if (edge) top = Raw8Odd::get_edge(x, src + i * kSegment, left);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t exponent = checkpoint_exponent(top);
            const uint2 q = checkpoint_codes(x, exponent);
            if (left >= 8) {
                __stcs(reinterpret_cast<uint2*>(dst + i * kSegment), q);
            } else if (left > 0) {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < left) dst[i * kSegment + e] = static_cast<int8_t>((e < 4 ? q.x : q.y) >> (8 * (e % 4)));
            }
            if ((lane & 3) == 0 && left > 0) exps[i * (kSegment / kCheckpointBlock)] = static_cast<uint8_t>(exponent);
        }
    }
}

// Everything else: one element per lane, so a warp reads and writes consecutive ones; the block's maximum over the warp's lanes.
template <typename T>
__global__ void __launch_bounds__(kStreamThreads)
checkpoint_store_elem_kernel(const T* X, int64_t ldx, int64_t N, int D, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, int runs)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    for (RunWalk at(runs); at.row < N; at.next()) {
        const int col0 = at.run * kSegment + lane;
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
        if (lane < 8 && at.run * kSegment + 32 * lane < D) E[at.row * lde + at.run * (kSegment / 32) + lane] = static_cast<uint8_t>(mine);
    }
}

// A run of bf16 segments of a row that starts on any boundary.  A lane puts the aligned 16 bytes that its first element lies in together
// with its neighbour's last elements, the first lane of a segment with those of the segment before; what has no such neighbour, at the ends of
// the run, is written one element at a time.
struct OddRun {
    uint32_t s;                                                 // bytes of a chunk that are the neighbour's
    uint4 carried = {0u, 0u, 0u, 0u};                           // of lane 0: the last lane's values of the segment before
    bool begun = false;
    __device__ __forceinline__ OddRun(const __nv_bfloat16* p) : s(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) & 15)) {}
    // count: how many of this lane's eight there are; next: the same of the next segment's first lane, 0 behind the run's last.
    __device__ __forceinline__ void store(__nv_bfloat16* p, const uint4& v, int count, int next, int lane)
    {
        const int from_lane = (lane + 31) & 31;
        const uint4 turned = make_uint4(__shfl_sync(0xffffffffu, v.x, from_lane), __shfl_sync(0xffffffffu, v.y, from_lane),
                                        __shfl_sync(0xffffffffu, v.z, from_lane), __shfl_sync(0xffffffffu, v.w, from_lane));
        const uint4 before = lane == 0 ? carried : turned;
        carried = turned;
        const int mine = static_cast<int>(16 - s) / 2;           // elements in the chunk
        const bool whole = (lane > 0 || begun || s == 0) && count >= mine;
        bool next_whole = __shfl_down_sync(0xffffffffu, static_cast<int>(whole), 1) != 0;
        if (lane == 31) next_whole = next >= mine;
        if (whole) __stcs(reinterpret_cast<uint4*>(reinterpret_cast<char*>(p) - s), s == 0 ? v : shift_chunks(before, v, 16 - s));
        const int from = whole ? mine : 0, to = next_whole ? mine : count;
        if (from < to && count > 0) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= from && e < to && e < count)
                    p[e] = __ushort_as_bfloat16(static_cast<unsigned short>(w[e >> 1] >> (16 * (e & 1))));
        }
        begun = true;
    }
};

// Rows of Q on 8-byte boundaries, rows of Xhat on 16-byte ones unless ODD.
template <typename T, int U, bool ODD>
__global__ void __launch_bounds__(kStreamThreads, kResidentLoad)
checkpoint_load_vec_kernel(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int D, T* Xhat, int64_t ldx, int runs, uint32_t* zeros)
{
    pdl_wait();
    pdl_trigger();
    if (zeros && blockIdx.x == 0 && threadIdx.x < kLoadZeros) zeros[threadIdx.x] = 0u;
    const int lane = threadIdx.x & 31;
    for (RunWalk at(runs); at.row < N; at.next()) {
        const int col0 = at.run * (U * kSegment) + lane * 8, left0 = D - col0;
        const int8_t* src = Q + at.row * ldq + col0;
        const uint8_t* exps = E + at.row * lde + col0 / kCheckpointBlock;
        uint2 q[U];
        uint32_t exponent[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int left = left0 - i * kSegment;
            q[i] = make_uint2(0, 0);
            exponent[i] = 0;
            if (left > 0) {
                exponent[i] = exps[i * (kSegment / kCheckpointBlock)];
                if (left >= 8) {
                    q[i] = __ldcs(reinterpret_cast<const uint2*>(src + i * kSegment));
                } else {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < left) (e < 4 ? q[i].x : q[i].y) |= static_cast<uint32_t>(static_cast<uint8_t>(src[i * kSegment + e])) << (8 * (e % 4));
                }
            }
        }
        T* dst = Xhat + at.row * ldx + col0;
        OddRun odd(reinterpret_cast<const __nv_bfloat16*>(dst));
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int left = left0 - i * kSegment;
            if (D - at.run * (U * kSegment) <= i * kSegment) break;            // for the whole warp
            if constexpr (ODD) {
                // The next segment's first lane has D - its first column left.
                const int next = i + 1 < U ? D - at.run * (U * kSegment) - (i + 1) * kSegment : 0;
                odd.store(dst + i * kSegment, checkpoint_values_bf16(q[i], exponent[i]), min(max(left, 0), 8), min(max(next, 0), 8), lane);
            } else {
                float y[8];                                   // before the branches: within them 107 us instead of 99 for 8192 x 11008
                checkpoint_values(q[i], exponent[i], y);
                if (left >= 8) {
                    store8(dst + i * kSegment, y);
                } else if (left > 0) {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < left) Elem<T>::store(dst + i * kSegment + e, y[e]);
                }
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kStreamThreads)
checkpoint_load_elem_kernel(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int D, T* Xhat, int64_t ldx, int runs, uint32_t* zeros)
{
    pdl_wait();
    pdl_trigger();
    if (zeros && blockIdx.x == 0 && threadIdx.x < kLoadZeros) zeros[threadIdx.x] = 0u;
    const int lane = threadIdx.x & 31;
    for (RunWalk at(runs); at.row < N; at.next()) {
        const int col0 = at.run * kSegment + lane;
        float q[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = col0 + 32 * i < D;
            q[i] = in ? static_cast<float>(Q[at.row * ldq + col0 + 32 * i]) : 0.f;
            s[i] = in ? checkpoint_step(E[at.row * lde + at.run * (kSegment / 32) + i]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col0 + 32 * i < D) Elem<T>::store(Xhat + at.row * ldx + col0 + 32 * i, q[i] * s[i]);
    }
}

// As many CTAs as are resident at a time and no more than there is work for.
unsigned grid_for(int64_t runs, int sm_count, int resident)
{
    const int64_t ctas = ceil_div64(runs, kStreamThreads / 32), most = static_cast<int64_t>(sm_count) * resident;
    return static_cast<unsigned>(ctas < most ? ctas : most);
}

// Segments in a run: four, or fewer where the rows have fewer or the warps of the chip would not all get a run.
int run_segments(int64_t N, int64_t D, int sm_count)
{
    const int64_t segs = ceil_div64(D, kSegment), warps = static_cast<int64_t>(sm_count) * kResidentLoad * (kStreamThreads / 32);
    if (segs <= 1 || N * ceil_div64(segs, 2) < warps) return 1;
    return segs <= 2 || N * ceil_div64(segs, 4) < warps ? 2 : 4;
}

#define VELORA_BY_SEGMENTS(LAUNCH) (u == 1 ? LAUNCH(1) : (u == 2 ? LAUNCH(2) : LAUNCH(4)))

template <typename T>
int store_typed(const void* X, int64_t N, int64_t D, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, int sm_count, cudaStream_t stream)
{
    const int d = static_cast<int>(D);
    const T* x = static_cast<const T*>(X);
    if (reinterpret_cast<uintptr_t>(Q) % 8 == 0 && ldq % 8 == 0) {
        const int u = run_segments(N, D, sm_count), runs = static_cast<int>(ceil_div64(D, u * kSegment));
#define VELORA_STORE(U) launch_chained(checkpoint_store_vec_kernel<T, Raw8<T>, U>, dim3(grid_for(N * runs, sm_count, kResident<Raw8<T>>)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, runs)
        if (c_rows_vec(X, ldx, sizeof(T))) return VELORA_BY_SEGMENTS(VELORA_STORE);
#undef VELORA_STORE
        if constexpr (sizeof(T) == 2) {
#define VELORA_STORE(U) launch_chained(checkpoint_store_vec_kernel<T, Raw8Odd, U>, dim3(grid_for(N * runs, sm_count, kResident<Raw8Odd>)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, runs)
            return VELORA_BY_SEGMENTS(VELORA_STORE);
#undef VELORA_STORE
        }
    }
    const int runs = static_cast<int>(ceil_div64(D, kSegment));
    return launch_chained(checkpoint_store_elem_kernel<T>, dim3(grid_for(N * runs, sm_count, kStreamCtasPerSm)), kStreamThreads, 0, stream, x, ldx, N, d, Q, ldq, E, lde, runs);
}

template <typename T>
int load_typed(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int64_t D, void* Xhat, int64_t ldx, uint32_t* zeros, int sm_count, cudaStream_t stream)
{
    const int d = static_cast<int>(D);
    T* x = static_cast<T*>(Xhat);
    if (reinterpret_cast<uintptr_t>(Q) % 8 == 0 && ldq % 8 == 0) {
        const int u = run_segments(N, D, sm_count), runs = static_cast<int>(ceil_div64(D, u * kSegment));
        const dim3 grid(grid_for(N * runs, sm_count, kResidentLoad));
#define VELORA_LOAD(U) launch_chained(checkpoint_load_vec_kernel<T, U, false>, grid, kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, runs, zeros)
        if (c_rows_vec(Xhat, ldx, sizeof(T))) return VELORA_BY_SEGMENTS(VELORA_LOAD);
#undef VELORA_LOAD
        if constexpr (sizeof(T) == 2) {
#define VELORA_LOAD(U) launch_chained(checkpoint_load_vec_kernel<T, U, true>, grid, kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, runs, zeros)
            return VELORA_BY_SEGMENTS(VELORA_LOAD);
#undef VELORA_LOAD
        }
    }
    const int runs = static_cast<int>(ceil_div64(D, kSegment));
    return launch_chained(checkpoint_load_elem_kernel<T>, dim3(grid_for(N * runs, sm_count, kStreamCtasPerSm)), kStreamThreads, 0, stream, Q, ldq, E, lde, N, d, x, ldx, runs, zeros);
}
#undef VELORA_BY_SEGMENTS

}  // namespace

int launch_checkpoint_store(const void* X, int x_dtype, int64_t N, int64_t D, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    return x_dtype == VELORA_BF16 ? store_typed<__nv_bfloat16>(X, N, D, ldx, Q, ldq, E, lde, di.sm_count, stream)
                                  : store_typed<float>(X, N, D, ldx, Q, ldq, E, lde, di.sm_count, stream);
}

int launch_checkpoint_load(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int64_t D, void* Xhat, int x_dtype, int64_t ldx, uint32_t* zeros, cudaStream_t stream)
{
    DeviceInfo di;
    const int rc = device_info(&di);
    if (rc != VELORA_OK) return rc;
    return x_dtype == VELORA_BF16 ? load_typed<__nv_bfloat16>(Q, ldq, E, lde, N, D, Xhat, ldx, zeros, di.sm_count, stream)
                                  : load_typed<float>(Q, ldq, E, lde, N, D, Xhat, ldx, zeros, di.sm_count, stream);
}

}  // namespace velora
