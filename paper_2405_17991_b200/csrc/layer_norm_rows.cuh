// Rows that a warp or a block holds in registers, and how they come in: for layer_norm.cu and layer_norm_backward.cu.
#pragma once

#include "layer_norm.cuh"

namespace velora {

// How a row is dealt out: to a warp (WARPS = 1, eight rows a block) or to a block of WARPS warps, each thread C chunks of eight columns.  Rows on 16-byte
// boundaries (VEC): eight neighbouring columns, chunk c of thread t at 8 (c T + t), T threads a row; others: every T-th column, so that a warp's lanes read
// neighbouring elements.
template <int WARPS, int C> struct RowShape {
    static constexpr int kThreads = WARPS == 1 ? 256 : 32 * WARPS;
    static constexpr int kRows = WARPS == 1 ? 8 : 1;              // of a block at a time
    static constexpr int kPerRow = 32 * WARPS;                    // threads of a row
    static constexpr int kColumns = kPerRow * C * 8;              // a row may have
};

#ifdef __CUDACC__
template <bool VEC, int PER_ROW> __device__ __forceinline__ int column_of(int c, int e, int t) { return VEC ? (c * PER_ROW + t) * 8 + e : (c * 8 + e) * PER_ROW + t; }
// How many of a chunk's eight columns there are, below one: none.
template <bool VEC, int PER_ROW> __device__ __forceinline__ int chunk_left(int c, int t, int D)
{
    return VEC ? D - (c * PER_ROW + t) * 8 : (D - c * 8 * PER_ROW - t + PER_ROW - 1) / PER_ROW;
}

// ---- rows on their way: copies of 16 bytes that a thread makes for itself, so no barrier goes with them ----
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes)       // the rest of the 16 becomes zero
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait(int behind)          // until all but the `behind` latest rows are there
{
    if (behind == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (behind == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// A thread's share of a row of one operand, in shared memory: 16-byte words, `stride` bytes apart (a word of every thread of the row lies in between).
template <typename T, int C> struct Share {
    static constexpr int kWords = C * static_cast<int>(sizeof(T)) / 2;      // 16 bytes of bf16, 32 of fp32 a chunk
    // From the row's columns; what is behind its end becomes zero within a chunk and is not read.
    template <int PER_ROW> static __device__ __forceinline__ void copy(uint32_t dst, const T* row, int D, int t)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * PER_ROW + t) * 8;
            if (col >= D) continue;
#pragma unroll
            for (int i = 0; i < kWords / C; ++i) {
                constexpr int per = 16 / sizeof(T);
                const int left = (D - col - i * per) * static_cast<int>(sizeof(T));
                copy16(dst + (c * (kWords / C) + i) * PER_ROW * 16, left > 0 ? row + col + i * per : row, min(16, max(0, left)));
            }
        }
    }
    template <int PER_ROW> static __device__ __forceinline__ void load(float (&x)[8], const char* src, int c)
    {
        const uint4 w = *reinterpret_cast<const uint4*>(src + c * (kWords / C) * PER_ROW * 16);
        if (sizeof(T) == 2) {
            x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
            x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
        } else {
            const uint4 v = *reinterpret_cast<const uint4*>(src + (c * (kWords / C) + 1) * PER_ROW * 16);
            x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
            x[4] = __uint_as_float(v.x); x[5] = __uint_as_float(v.y); x[6] = __uint_as_float(v.z); x[7] = __uint_as_float(v.w);
        }
    }
};

// Eight outputs at a 16-byte boundary, `left` of them there.
__device__ __forceinline__ void store_chunk(__nv_bfloat16* p, const float (&y)[8], int left)
{
    if (left >= 8) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) p[e] = __float2bfloat16_rn(y[e]);
    }
}
__device__ __forceinline__ void store_chunk(float* p, const float (&y)[8], int left)
{
    if (left >= 8) {
        if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(p), "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]) : "memory");
        } else {
            reinterpret_cast<float4*>(p)[0] = make_float4(y[0], y[1], y[2], y[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(y[4], y[5], y[6], y[7]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) p[e] = y[e];
    }
}

// Weights or biases of a thread's eight columns; `wide`: they start on 16-byte boundaries.
template <bool VEC, int PER_ROW>
__device__ __forceinline__ void load_params(float (&y)[8], const void* p, int dtype, bool wide, int c, int t, int D, float none)
{
    const int col = (c * PER_ROW + t) * 8;
    if (VEC && wide && p && col + 8 <= D) {
        if (dtype == VELORA_BF16) {
            const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + col);
            y[0] = bf16_lo(w.x); y[1] = bf16_hi(w.x); y[2] = bf16_lo(w.y); y[3] = bf16_hi(w.y);
            y[4] = bf16_lo(w.z); y[5] = bf16_hi(w.z); y[6] = bf16_lo(w.w); y[7] = bf16_hi(w.w);
        } else {
            const float4 u = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col)[0];
            const float4 v = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col)[1];
            y[0] = u.x; y[1] = u.y; y[2] = u.z; y[3] = u.w;
            y[4] = v.x; y[5] = v.y; y[6] = v.z; y[7] = v.w;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = column_of<VEC, PER_ROW>(c, e, t);
        y[e] = d < D ? load_param(p, dtype, d, none) : 0.f;
    }
}

__device__ __forceinline__ float sum8(const float (&x)[8]) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }
__device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
#endif

}  // namespace velora
