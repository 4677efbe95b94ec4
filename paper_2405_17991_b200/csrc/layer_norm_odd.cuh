// Rows that a warp or a block works on, and how they come in: for layer_norm.cu and layer_norm_backward.cu.
#pragma once

#include "layer_norm.cuh"

namespace velora {

// How a row is dealt out: to a warp (WARPS = 1, eight rows a block) or to a block of WARPS warps, each thread C chunks of eight columns.  Rows that all
// start on 16-byte boundaries (VEC): eight neighbouring columns, chunk c of thread t at 8 (c T + t), T threads a row; others: every T-th column, so that a
// warp's lanes read and write neighbouring elements.
template <int WARPS, int C> struct RowShape {
    static constexpr int kThreads = WARPS == 1 ? 256 : 32 * WARPS;
    static constexpr int kRows = WARPS == 1 ? 8 : 1;              // of a block at a time
    static constexpr int kPerRow = 32 * WARPS;                    // threads of a row
    static constexpr int kColumns = kPerRow * C * 8;              // a row may have
};
// Bytes of shared memory that a row of one operand takes: rows on any boundary start within their first 16.
template <typename T, int WARPS, int C, bool VEC> constexpr int kShareBytes = RowShape<WARPS, C>::kColumns * static_cast<int>(sizeof(T)) + (VEC ? 0 : 16);

struct Ring {
    int stages;                                                   // rows on their way or in use
    int stage_bytes;                                              // of a row of all operands
    bool wide;                                                    // weights on 16-byte boundaries
};

#ifdef __CUDACC__
// Two fp32 numbers in one operation: half the instructions of a row, which is what these kernels are held up by before HBM.
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 f2(float lo, float hi)
{
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 parts(F2 a)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ F2 add(F2 a, F2 b)
{
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 mul(F2 a, F2 b)
{
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c)
{
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ F2 of_bf16(uint32_t w) { return f2(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ uint32_t to_bf16(F2 a) { const float2 p = parts(a); return pack_bf16x2(p.x, p.y); }

// Column of element e (0 .. 7) of a thread's chunk c, and how many of a chunk's eight there are (below one: none).
template <bool VEC, int PER_ROW> __device__ __forceinline__ int column_of(int c, int e, int t) { return VEC ? (c * PER_ROW + t) * 8 + e : (c * 8 + e) * PER_ROW + t; }
template <bool VEC, int PER_ROW> __device__ __forceinline__ int chunk_left(int c, int t, int D)
{
    return VEC ? D - (c * PER_ROW + t) * 8 : (D - c * 8 * PER_ROW - t + PER_ROW - 1) / PER_ROW;
}

// ---- rows on their way: asynchronous copies of 16 bytes ----
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes)       // the rest of the 16 becomes zero
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait(int behind)          // until all but the `behind` latest rows are there
{
    if (behind == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (behind == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (behind == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// One operand's rows.
// VEC: a thread copies what it will read itself, so no barrier goes with it: words of 16 bytes, one of every thread side by side.
// Others: the aligned words that a row lies in, whoever's they are, so a barrier of the row's threads stands between copies and reads, and between reads and
// the slot's next copies.  Bytes in front of the first row are not touched (its first word comes element by element); those in front of another row are its
// neighbour's, and nobody looks at them.
template <typename T, int WARPS, int C, bool VEC> struct RowSource {
    static constexpr int P = RowShape<WARPS, C>::kPerRow, kWords = static_cast<int>(sizeof(T)) / 2;      // 16-byte words a chunk
    const T* base;
    int64_t ld;
    __device__ __forceinline__ void copy(char* slot, uint32_t slot_at, int64_t n, int D, int t) const
    {
        const T* row = base + n * ld;
        if (VEC) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * P + t) * 8;
                if (col >= D) continue;
#pragma unroll
                for (int i = 0; i < kWords; ++i) {
                    const int left = (D - col - i * (8 / kWords)) * static_cast<int>(sizeof(T));
                    copy16(slot_at + ((c * kWords + i) * P + t) * 16, left > 0 ? row + col + i * (8 / kWords) : row, min(16, max(0, left)));
                }
            }
        } else {
            const uintptr_t from = reinterpret_cast<uintptr_t>(row) & ~uintptr_t{15}, end = reinterpret_cast<uintptr_t>(row + D);
            for (uintptr_t w = from + 16 * t; w < end; w += 16 * P) {
                const int at = static_cast<int>(w - from);
                if (w < reinterpret_cast<uintptr_t>(base)) {
                    for (uintptr_t p = reinterpret_cast<uintptr_t>(base); p < w + 16 && p < end; p += sizeof(T))
                        *reinterpret_cast<T*>(slot + at + (p - w)) = *reinterpret_cast<const T*>(p);
                } else {
                    copy16(slot_at + at, reinterpret_cast<const void*>(w), static_cast<int>(end - w < 16 ? end - w : 16));
                }
            }
        }
    }
    // A thread's chunk; elements behind the row's end are zeros within a VEC chunk and elsewhere as well.
    __device__ __forceinline__ void load(F2 (&x)[4], const char* slot, int64_t n, int c, int t, int left) const
    {
        if (VEC) {
            const char* p = slot + (c * kWords * P + t) * 16;
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            if (sizeof(T) == 2) {
                x[0] = of_bf16(w.x); x[1] = of_bf16(w.y); x[2] = of_bf16(w.z); x[3] = of_bf16(w.w);
            } else {
                const uint4 v = *reinterpret_cast<const uint4*>(p + P * 16);
                x[0] = f2(__uint_as_float(w.x), __uint_as_float(w.y)); x[1] = f2(__uint_as_float(w.z), __uint_as_float(w.w));
                x[2] = f2(__uint_as_float(v.x), __uint_as_float(v.y)); x[3] = f2(__uint_as_float(v.z), __uint_as_float(v.w));
            }
        } else {
            const T* p = reinterpret_cast<const T*>(slot + (reinterpret_cast<uintptr_t>(base + n * ld) & 15)) + c * 8 * P + t;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = e < left ? Elem<T>::load(p + e * P) : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = f2(y[2 * i], y[2 * i + 1]);
        }
    }
};

// A thread's chunk of outputs, `left` of them there: to `row` + column_of(c, 0, t).
template <typename T, bool VEC, int PER_ROW>
__device__ __forceinline__ void store_chunk(T* row, const F2 (&x)[4], int c, int t, int left)
{
    T* p = row + column_of<VEC, PER_ROW>(c, 0, t);
    if (VEC && left >= 8) {
        if (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(p) = make_uint4(to_bf16(x[0]), to_bf16(x[1]), to_bf16(x[2]), to_bf16(x[3]));
        } else if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
            asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(p), "l"(x[0].v), "l"(x[1].v), "l"(x[2].v), "l"(x[3].v) : "memory");
        } else {
            reinterpret_cast<ulonglong2*>(p)[0] = make_ulonglong2(x[0].v, x[1].v);
            reinterpret_cast<ulonglong2*>(p)[1] = make_ulonglong2(x[2].v, x[3].v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) Elem<T>::store(p + e * (VEC ? 1 : PER_ROW), e & 1 ? parts(x[e >> 1]).y : parts(x[e >> 1]).x);
    }
}

// Weights or biases of a thread's eight columns; `wide`: they start on 16-byte boundaries.
template <bool VEC, int PER_ROW>
__device__ __forceinline__ void load_params(F2 (&x)[4], const void* p, int dtype, bool wide, int c, int t, int D, float none)
{
    const int col = (c * PER_ROW + t) * 8;
    if (VEC && wide && p && col + 8 <= D) {
        if (dtype == VELORA_BF16) {
            const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + col);
            x[0] = of_bf16(w.x); x[1] = of_bf16(w.y); x[2] = of_bf16(w.z); x[3] = of_bf16(w.w);
        } else {
            const float4 u = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col)[0];
            const float4 v = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col)[1];
            x[0] = f2(u.x, u.y); x[1] = f2(u.z, u.w); x[2] = f2(v.x, v.y); x[3] = f2(v.z, v.w);
        }
        return;
    }
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = column_of<VEC, PER_ROW>(c, e, t);
        y[e] = d < D ? load_param(p, dtype, d, none) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f2(y[2 * i], y[2 * i + 1]);
}

__device__ __forceinline__ float sum8(F2 a, F2 b, F2 c, F2 d)
{
    const float2 s = parts(add(add(a, b), add(c, d)));
    return s.x + s.y;
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float x)          // over groups of so many neighbouring lanes
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// The row's threads meet.
template <int WARPS> __device__ __forceinline__ void row_barrier()
{
    if (WARPS == 1) __syncwarp();
    else __syncthreads();
}
#endif

}  // namespace velora
