// Format of the 8-bit checkpoints (checkpoint.cu): codes, block exponents, and who reads them.
#pragma once

#include "common.cuh"

namespace velora {

constexpr int kCheckpointBlock = 32;                // columns that share an exponent
constexpr uint32_t kCheckpointNaN = 255;            // exponent byte of a block that cannot be represented

int launch_checkpoint_store(const void* X, int x_dtype, int64_t N, int64_t D, int64_t ldx, int8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, cudaStream_t stream);
int launch_checkpoint_load(const int8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t N, int64_t D, void* Xhat, int x_dtype, int64_t ldx, cudaStream_t stream);

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

// Low byte: q.  x 2^-e is exact but where it is far below one half; adding 3 * 2^22 rounds it to an integer, ties to even.  Only the clamped
// exponent 248 leaves more than 127.
__device__ __forceinline__ uint32_t checkpoint_code(float x, uint32_t exponent)
{
    const float inverse = __uint_as_float((254u - exponent) << 23);
    const float t = fminf(fmaxf(x * inverse, -127.f), 127.f);
    const uint32_t q = __float_as_uint(__fadd_rn(t, 12582912.f)) & 0xffu;
    return exponent == kCheckpointNaN ? 0u : q;
}
__device__ __forceinline__ void checkpoint_codes(const float (&x)[8], uint32_t exponent, uint32_t (&q)[2])
{
    const float inverse = __uint_as_float((254u - exponent) << 23);
    uint32_t r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = __float_as_uint(__fadd_rn(fminf(fmaxf(x[e] * inverse, -127.f), 127.f), 12582912.f));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __byte_perm(r[4 * h], r[4 * h + 1], 0x0040), hi = __byte_perm(r[4 * h + 2], r[4 * h + 3], 0x0040);
        q[h] = exponent == kCheckpointNaN ? 0u : __byte_perm(lo, hi, 0x5410);
    }
}
#endif

}  // namespace velora
