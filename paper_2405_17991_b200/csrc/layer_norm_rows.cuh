// Rows on 16-byte boundaries for the layer norm: how they are dealt out, how they come in, sums over them.  For layer_norm.cu and layer_norm_backward.cu.
#pragma once

#include "layer_norm.cuh"

namespace velora {

// A row is D / E words of 16 bytes (E = 8 columns of bf16, 4 of fp32).  ONE: a warp has a row, eight of them a block; else a block has one.  Thread t of P has
// the words c P + t, c < C, so that a warp's lanes lie side by side; P is chosen so that only a thread's last word may be missing.
inline bool rows_vec(const void* p, int64_t ld, int dtype) { return !p || (aligned16(p) && ld * static_cast<int64_t>(dtype_size(dtype)) % 16 == 0); }
inline int row_words(int D, int dtype) { return D / (16 / static_cast<int>(dtype_size(dtype))); }
inline int row_threads(int words, int C) { return 32 * static_cast<int>(ceil_div64(words, 32 * C)); }          // of a block that has one row

#ifdef __CUDACC__
// Two fp32 numbers in one operation: these kernels are held up by instructions before HBM.
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 f2(float lo, float hi)
{
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ F2 f2(float x) { return f2(x, x); }
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
__device__ __forceinline__ float sum(F2 a) { const float2 p = parts(a); return p.x + p.y; }

// A word of a row.
template <typename T> struct Word;
template <> struct Word<__nv_bfloat16> {
    static constexpr int E = 8;
    F2 x[4];
    __device__ __forceinline__ void load(uint32_t smem)
    {
        uint32_t a, b, c, d;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(smem) : "memory");
        x[0] = of_bf16(a); x[1] = of_bf16(b); x[2] = of_bf16(c); x[3] = of_bf16(d);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const
    {
        *reinterpret_cast<uint4*>(p) = make_uint4(to_bf16(x[0]), to_bf16(x[1]), to_bf16(x[2]), to_bf16(x[3]));
    }
    __device__ __forceinline__ void round()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = of_bf16(to_bf16(x[i]));
    }
    __device__ __forceinline__ F2 total() const { return add(add(x[0], x[1]), add(x[2], x[3])); }
};
template <> struct Word<float> {
    static constexpr int E = 4;
    F2 x[2];
    __device__ __forceinline__ void load(uint32_t smem)
    {
        asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(x[0].v), "=l"(x[1].v) : "r"(smem) : "memory");
    }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(x[0].v, x[1].v); }
    __device__ __forceinline__ void round() {}
    __device__ __forceinline__ F2 total() const { return add(x[0], x[1]); }
};

// Columns col .. col + E of a weight or bias; `wide`: it starts on a 16-byte boundary.
template <int E> __device__ __forceinline__ void load_columns(F2 (&x)[E / 2], const void* p, int dtype, bool wide, int col, float none)
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) x[i] = f2(none);
    } else if (wide && dtype == VELORA_BF16) {
        const uint2* q = reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p) + col);
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
            const uint2 w = q[i];
            x[2 * i] = of_bf16(w.x);
            x[2 * i + 1] = of_bf16(w.y);
        }
    } else if (wide) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col);
#pragma unroll
        for (int i = 0; i < E / 4; ++i) {
            const float4 w = q[i];
            x[2 * i] = f2(w.x, w.y);
            x[2 * i + 1] = f2(w.z, w.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) x[i] = f2(load_param(p, dtype, col + 2 * i, none), load_param(p, dtype, col + 2 * i + 1, none));
    }
}

// ---- rows on their way: a thread copies what it will read itself, so no barrier goes with it ----
__device__ __forceinline__ void copy_word(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int BEHIND> __device__ __forceinline__ void copies_wait()          // until all but the latest BEHIND rows are there
{
    asm volatile("cp.async.wait_group %0;" ::"n"(BEHIND) : "memory");
}

// 1 / sqrt(v): the approximation and one step of Newton's method, where that has a meaning.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v), e = fmaf(-v * r, r, 1.f);
    return v > 1e-37f && v < 1e37f ? fmaf(0.5f * r, e, r) : 1.f / sqrtf(v);
}
__device__ __forceinline__ float warp_total(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// Over the block's warps: the first MOST lanes (a power of two) hold one's each, or 0.
template <int MOST> __device__ __forceinline__ float warps_total(float x)
{
#pragma unroll
    for (int o = MOST / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// Lanes that hold a warp's each, of up to THREADS threads.
template <int THREADS> constexpr int kWarpLanes = THREADS <= 64 ? 2 : THREADS <= 128 ? 4 : THREADS <= 256 ? 8 : THREADS <= 512 ? 16 : 32;
#endif

}  // namespace velora
