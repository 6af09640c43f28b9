// Activations in 8 bits: blocks of 32 values along a row share a power of two (tconv.h).
//
// The unit 2^e is a power of two, so that x * 2^-e and code * 2^e are exact: the only rounding is the one to the code,
// codes do not hang on the order of any arithmetic, and a restored value fits bf16 (7 bits of magnitude).
#pragma once
#include "tconv_common.cuh"

namespace tconv {

constexpr int kQ8Block = 32;

__host__ __device__ inline int64_t q8_pitch(int64_t inner) { return (inner + 7) / 8 * 8; }
__host__ __device__ inline int64_t q8_blocks(int64_t inner) { return (inner + kQ8Block - 1) / kQ8Block; }

// Magnitudes are compared as integers, so that a NaN, whose bits lie above those of infinity, is not dropped as fmaxf
// would.
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Scale byte e + 127 of a block whose largest magnitude has the bits `top`: with amax = m * 2^k, 1 <= m < 2, it is k - 6
// where m < 127.5 / 64 and k - 5 elsewhere; adding 2^16 carries into the exponent exactly where m's seven leading bits are
// all ones, that is m >= 127.5 / 64.  Not below 1 (a normal 2^e with a normal inverse); 255 for infinities and NaN.
__device__ __forceinline__ uint32_t q8_scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return 255u;
    const int e = (int)((top + 0x10000u) >> 23) - 6;
    return (uint32_t)(e < 1 ? 1 : e);
}
// 2^-e.  A poisoned block has codes 0.
__device__ __forceinline__ float q8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// 2^e; infinity for 255, which makes every code 0 a NaN.
__device__ __forceinline__ float q8_unit(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ int q8_code(float v, uint32_t byte) {
    return byte == 255u ? 0 : __float2int_rn(v * q8_inverse(byte));
}

// One warp per block.
template <typename T>
__global__ void __launch_bounds__(256) q8_store_kernel(int64_t rows, int64_t inner, const T* __restrict__ x,
                                                       int8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const int64_t nb = q8_blocks(inner), pitch = q8_pitch(inner);
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (blockDim.x >> 5);
    for (int64_t b = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); b < rows * nb; b += warps) {
        const int64_t row = b / nb, at = (b - row * nb) * kQ8Block + lane;
        const float v = at < inner ? to_f32(x[row * inner + at]) : 0.0f;
        const uint32_t byte = q8_scale_byte(__reduce_max_sync(~0u, magnitude_bits(v)));
        if (at < pitch) codes[row * pitch + at] = (int8_t)q8_code(v, byte);
        if (lane == 0) scales[b] = (uint8_t)byte;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) q8_restore_kernel(int64_t rows, int64_t inner, const int8_t* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, T* __restrict__ x) {
    const int64_t nb = q8_blocks(inner), pitch = q8_pitch(inner), n = rows * inner;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = i / inner, at = i - row * inner;
        x[i] = from_f32<T>((float)codes[row * pitch + at] * q8_unit(scales[row * nb + at / kQ8Block]));
    }
}

}  // namespace tconv
