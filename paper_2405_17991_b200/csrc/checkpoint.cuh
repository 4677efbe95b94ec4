// Format of the 8-bit checkpoints (checkpoint.cu): codes, block exponents, and who reads them.
#pragma once

#include "common.cuh"

namespace velora {

constexpr int kCheckpointBlock = 32;                // columns that share an exponent
constexpr uint32_t kCheckpointNaN = 255;            // exponent byte of a block that cannot be represented

int launch_checkpoint_store(const void* X, int x_dtype, int64_t N, int64_t D, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, cudaStream_t stream);
// zeros: NULL, or kLoadZeros words that become zero for the kernel behind it.
constexpr int kLoadZeros = 64;
int launch_checkpoint_load(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int64_t D, void* Xhat, int x_dtype, int64_t ldx, uint32_t* zeros, cudaStream_t stream);

#ifdef __CUDACC__
// E from the bits of a = max |x|.  a = m 2^k with 1 <= m < 2 is at most 127 * 2^(k - 6) where m <= 127 / 64, whose fraction's
// bits are 0x7e0000; above that the sum carries into the exponent.
__device__ __forceinline__ uint32_t checkpoint_exponent(uint32_t a_bits)
{
    if (a_bits >= 0x7f800000u) return kCheckpointNaN;
    const int biased = static_cast<int>((a_bits + 0x1ffffu) >> 23) - 6;
    return static_cast<uint32_t>(min(max(biased, 1), 248));
}
// 2^(E - 127); infinite for E = 255, so that its codes of zero give NaN.
__device__ __forceinline__ float checkpoint_step(uint32_t exponent) { return __uint_as_float(exponent << 23); }

// Low byte: q.  x 2^-e is exact, so adding 3 * 2^22 in the same operation rounds it to an integer, ties to even.  Only under the clamped
// exponent 248 can it be more than 127.
__device__ __forceinline__ uint32_t checkpoint_code(float x, uint32_t exponent)
{
    const float inverse = __uint_as_float((254u - min(exponent, 248u)) << 23);
    if (exponent >= 248u) x = exponent == kCheckpointNaN ? 0.f : fminf(fmaxf(x, -127.f / inverse), 127.f / inverse);
    return __float_as_uint(fmaf(x, inverse, 12582912.f)) & 0xffu;
}
// Eight of them, packed.
__device__ __forceinline__ uint2 checkpoint_codes(float (&x)[8], uint32_t exponent)
{
    const float inverse = __uint_as_float((254u - min(exponent, 248u)) << 23);
    if (exponent >= 248u) {
        const float most = 127.f / inverse;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = exponent == kCheckpointNaN ? 0.f : fminf(fmaxf(x[e], -most), most);
    }
    uint32_t r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = __float_as_uint(fmaf(x[e], inverse, 12582912.f));
    return make_uint2(__byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(r[4], r[5], 0x0040), __byte_perm(r[6], r[7], 0x0040), 0x5410));
}

// Eight codes to their values.  A code with its top bit turned over is q + 128; as the low byte of 2^23 + .. it is exact in fp32.
__device__ __forceinline__ void checkpoint_values(const uint2& q, uint32_t exponent, float (&y)[8])
{
    const float s = checkpoint_step(exponent);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = (h ? q.y : q.x) ^ 0x80808080u;
        y[4 * h] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650)) - 8388736.f) * s;
        y[4 * h + 1] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7651)) - 8388736.f) * s;
        y[4 * h + 2] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7652)) - 8388736.f) * s;
        y[4 * h + 3] = (__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7653)) - 8388736.f) * s;
    }
}
// The same in bf16, two at a time: the low seven bits b of a code as 128 + b, minus 128 or, with the sign bit, 256; exact, as is the product
// with a power of two.
__device__ __forceinline__ uint32_t checkpoint_values_bf16x2(uint32_t halves, uint32_t step)
{
    const uint32_t v = (halves & 0x007f007fu) | 0x43004300u, c = (halves & 0x00800080u) | 0x43004300u;
    uint32_t q, r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(q) : "r"(v), "r"(c));
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(q), "r"(step));
    return r;
}
__device__ __forceinline__ uint4 checkpoint_values_bf16(const uint2& q, uint32_t exponent)
{
    const uint32_t step = (exponent << 7) * 0x00010001u;             // 2^(E - 127) twice; infinite for E = 255, so that 0 becomes NaN
    return make_uint4(checkpoint_values_bf16x2(__byte_perm(q.x, 0, 0x4140), step), checkpoint_values_bf16x2(__byte_perm(q.x, 0, 0x4342), step),
                      checkpoint_values_bf16x2(__byte_perm(q.y, 0, 0x4140), step), checkpoint_values_bf16x2(__byte_perm(q.y, 0, 0x4342), step));
}
#endif

}  // namespace velora
