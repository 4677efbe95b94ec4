// Rows that start on any boundary for the layer norm: how they come in and are dealt out.  For layer_norm_odd.cu and layer_norm_backward_odd.cu.
#pragma once

#include "layer_norm_rows.cuh"

namespace velora {

// A row comes as the aligned words of 16 bytes that it lies in, whoever copies them, so a barrier of the row's threads stands between the copies and the reads,
// and between the reads and the next copies to the same place.  Thread t of P has the columns i P + t, i < N: a warp's lanes read and write neighbouring elements.
inline int odd_share(int D, int dtype) { return (static_cast<int>(ceil_div64(D * static_cast<int64_t>(dtype_size(dtype)), 16)) + 1) * 16; }

#ifdef __CUDACC__
__device__ __forceinline__ void copies_wait_behind(int behind)          // until all but the `behind` latest rows are there
{
    if (behind == 2) copies_wait<2>();
    else if (behind == 1) copies_wait<1>();
    else copies_wait<0>();
}

// The rows of one operand, one after the other.
template <typename T, int P> struct OddRows {
    const char* base;                                            // of the matrix
    const char* next;                                            // row that is fetched next
    int64_t pitch;                                               // bytes
    uint32_t low;                                                // of the row in use: where it starts within its first word
    __device__ __forceinline__ OddRows(const void* p, int64_t ld, int64_t first)
        : base(static_cast<const char*>(p)), next(base + first * ld * static_cast<int64_t>(sizeof(T))), pitch(ld * static_cast<int64_t>(sizeof(T))),
          low(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(next) & 15)) {}
    // To `slot`; N P columns at most.  Bytes in front of the matrix are not touched (a first word that has some comes element by element), nor any behind the row;
    // those in front of a row are its neighbour's, and nobody looks at them.
    template <int N> __device__ __forceinline__ void fetch(char* slot, int D, int t)
    {
        const int skip = static_cast<int>(reinterpret_cast<uintptr_t>(next) & 15), bytes = skip + D * static_cast<int>(sizeof(T));
        const char* from = next - skip;
        const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(slot));
        const bool whole = from >= base;                         // the same for all threads
#pragma unroll
        for (int k = 0; k < N * static_cast<int>(sizeof(T)) / 16 + 1; ++k) {
            const int at = 16 * (t + k * P);
            if (at < bytes && (whole || at > 0))
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + at), "l"(from + at), "r"(min(16, bytes - at)) : "memory");
        }
        if (!whole && t == 0)
            for (int at = skip; at < 16 && at < bytes; at += sizeof(T)) *reinterpret_cast<T*>(slot + at) = *reinterpret_cast<const T*>(from + at);
        next += pitch;
    }
    __device__ __forceinline__ void step() { low = (low + static_cast<uint32_t>(pitch)) & 15u; }
    __device__ __forceinline__ uint32_t row(uint32_t slot, int t) const { return slot + low + t * static_cast<uint32_t>(sizeof(T)); }
};

// Which of a thread's columns there are: the first `full` of every thread's, LEAST or more, then one more of some threads'.
template <int LEAST> struct OddColumns {
    int full;
    bool more;
    __device__ __forceinline__ bool has(int i) const { return i < LEAST || i < full || (i == full && more); }
};
template <int P, int LEAST> __device__ __forceinline__ OddColumns<LEAST> odd_columns(int D, int t)
{
    OddColumns<LEAST> c;
    c.full = D / P;
    c.more = t < D - c.full * P;
    return c;
}
__device__ __forceinline__ float load_shared(uint32_t at, __nv_bfloat16)
{
    float x;
    asm volatile("{\n\t.reg .b16 h, z;\n\tmov.b16 z, 0;\n\tld.shared.b16 h, [%1];\n\tmov.b32 %0, {z, h};\n\t}" : "=f"(x) : "r"(at) : "memory");
    return x;
}
__device__ __forceinline__ float load_shared(uint32_t at, float)
{
    float x;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
    return x;
}
// `none` stands for missing ones.
template <typename T, int P, int N, int LEAST> __device__ __forceinline__ void odd_load(F2 (&x)[N / 2], uint32_t row, const OddColumns<LEAST>& c, float none = 0.f)
{
    constexpr uint32_t kStep = P * sizeof(T);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        float lo = none, hi = none;
        if (c.has(i)) lo = load_shared(row + i * kStep, T());
        if (c.has(i + 1)) hi = load_shared(row + (i + 1) * kStep, T());
        x[i / 2] = f2(lo, hi);
    }
}
template <typename T, int P, int N, int LEAST> __device__ __forceinline__ void odd_store(T* row, const F2 (&x)[N / 2], const OddColumns<LEAST>& c)
{
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 v = parts(x[i / 2]);
        if (c.has(i)) Elem<T>::store(row + i * P, v.x);
        if (c.has(i + 1)) Elem<T>::store(row + (i + 1) * P, v.y);
    }
}
template <int P, int N, int LEAST>
__device__ __forceinline__ void odd_params(F2 (&x)[N / 2], const void* p, int dtype, const OddColumns<LEAST>& c, int t, float none)
{
#pragma unroll
    for (int i = 0; i < N; i += 2)
        x[i / 2] = f2(c.has(i) ? load_param(p, dtype, i * P + t, none) : 0.f, c.has(i + 1) ? load_param(p, dtype, (i + 1) * P + t, none) : 0.f);
}
// The threads of a row meet: a warp, TEAM warps of the block, or all of it.
template <int TEAM> __device__ __forceinline__ void team_barrier(int team)
{
    if (TEAM == 1) __syncwarp();
    else if (TEAM) asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(32 * TEAM) : "memory");
    else __syncthreads();
}
#endif

}  // namespace velora
