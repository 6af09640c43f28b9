// Activations in 8 bits: blocks of 32 values along a row share a power of two (tconv.h).
//
// The unit 2^e is a power of two, so that x * 2^-e and code * 2^e are exact: the only rounding is the one to the code,
// codes do not hang on the order of any arithmetic, and a restored value fits bf16 (7 bits of magnitude).  Bound by HBM: 58 million
// fp32 values are stored in 50 us and restored in 44 (5.9 and 6.6 TB/s).
#pragma once
#include "tconv_common.cuh"

namespace tconv {

constexpr int kQ8Block = 32;

__host__ __device__ inline int64_t q8_pitch(int64_t inner) { return (inner + 7) / 8 * 8; }
__host__ __device__ inline int64_t q8_blocks(int64_t inner) { return (inner + kQ8Block - 1) / kQ8Block; }

// Scale byte e + 127 of a block whose largest magnitude has the bits `top`: with amax = m * 2^k, 1 <= m < 2, it is k - 6
// where m < 127.5 / 64 and k - 5 elsewhere; adding 2^16 carries into the exponent exactly where m's seven leading bits are
// all ones, that is m >= 127.5 / 64.  Not below 1 (a normal 2^e with a normal inverse), nor above kQ8Top (at e = 122 code 64 would
// stand for 2^128, which neither type has); 255 for infinities and NaN.
constexpr uint32_t kQ8Top = 121 + 127;
__device__ __forceinline__ uint32_t q8_scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return 255u;
    const int e = (int)((top + 0x10000u) >> 23) - 6;
    return (uint32_t)min(max(e, 1), (int)kQ8Top);
}
// 2^-e.  A poisoned block has codes 0.
__device__ __forceinline__ float q8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// 2^e; infinity for 255, which makes every code 0 a NaN.
__device__ __forceinline__ float q8_unit(uint32_t byte) { return __uint_as_float(byte << 23); }

// Largest magnitude of N values; NaN if one of them is.
template <int N> __device__ __forceinline__ float top_of(const float (&v)[N]) {
    float m = fabsf(v[0]);
#pragma unroll
    for (int i = 1; i + 1 < N; i += 2) asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(m), "f"(v[i]), "f"(v[i + 1]));
    if constexpr (N % 2 == 0) asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(m) : "f"(m), "f"(v[N - 1]));
    return fabsf(m);
}
// Scale byte of the block that v is part of: a thread has eight values of it, and its four threads are neighbours (G = 1: a row
// of at most eight values, one thread's).
template <int G> __device__ __forceinline__ uint32_t block_scale(const float (&v)[8]) {
    uint32_t top = __float_as_uint(top_of(v));
    if constexpr (G > 1) {
        top = max(top, __shfl_xor_sync(~0u, top, 1));
        top = max(top, __shfl_xor_sync(~0u, top, 2));
    }
    return q8_scale_byte(top);
}
// v * 2^-e + 1.5 * 2^23: the sum's unit is 1, so that its low byte is the code, rounded half to even.  With the largest unit
// magnitudes from 127.5 units on, all below 128, are held to 127: less than a unit off.
constexpr float kQ8Magic = 12582912.0f;
template <int N> __device__ __forceinline__ void q8_round(const float (&v)[N], uint32_t byte, float (&r)[N]) {
    const float inv = q8_inverse(byte);
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = fmaf(v[i], inv, kQ8Magic);
    if (byte >= kQ8Top)
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = byte == 255u ? kQ8Magic : fminf(fmaxf(r[i], kQ8Magic - 127.0f), kQ8Magic + 127.0f);
}
__device__ __forceinline__ uint32_t four_codes(const float* r) {
    return __byte_perm(__byte_perm(__float_as_uint(r[0]), __float_as_uint(r[1]), 0x0040),
                       __byte_perm(__float_as_uint(r[2]), __float_as_uint(r[3]), 0x0040), 0x5410);
}
// Codes of v, which becomes the values that they stand for.
__device__ __forceinline__ uint2 encode_eight(float (&v)[8], uint32_t byte) {
    float r[8];
    q8_round(v, byte, r);
    const float unit = q8_unit(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(__fadd_rn(r[i], -kQ8Magic), unit);
    return make_uint2(four_codes(r), four_codes(r + 4));
}
// A word's four values: code + 128 as the low byte of a float of unit 1.
__device__ __forceinline__ void decode_four(uint32_t w, float unit, float* v) {
    w ^= 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = __fmul_rn(__fadd_rn(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + i)), -8388736.0f), unit);
}
__device__ __forceinline__ void decode_eight(uint2 c, uint32_t byte, float (&v)[8]) {
    const float unit = q8_unit(byte);
    decode_four(c.x, unit, v);
    decode_four(c.y, unit, v + 4);
}

// A thread has 8 values of a row; four neighbours are a block (a row's last block may have idle ones).  I: the type that counts
// these units.  VEC: every row starts on 16 bytes, so a unit is read as vectors; else value by value (a warp's units lie next to
// each other, so that the sectors come from L1 after the first touch).  Codes are written 8 at a time in any case.
template <typename T, typename I, bool VEC>
__global__ void __launch_bounds__(256) q8_store_kernel(int64_t rows, int64_t inner, const T* __restrict__ x,
                                                       int8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const I nb = (I)q8_blocks(inner), per_row = 4 * nb, units = (I)rows * per_row;
    const int64_t pitch = q8_pitch(inner);
    const I unit = (I)blockIdx.x * 256 + threadIdx.x;
    if (unit - (threadIdx.x & 31) >= units) return;           // (a whole warp; units come in fours)
    const I row = unit / per_row, at = (unit - row * per_row) * 8;
    const bool ok = unit < units;
    const T* px = x + (int64_t)row * inner + at;
    float v[8];
    if (VEC && sizeof(T) == 4 && ok && (int64_t)at + 8 <= inner && (reinterpret_cast<uintptr_t>(px) & 31) == 0) {
        asm volatile("ld.global.nc.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(px));
    } else if constexpr (VEC) {
        constexpr int kWords = sizeof(T) / 2, kPer = 16 / sizeof(T);
        uint4 w[kWords];
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            w[j] = make_uint4(0, 0, 0, 0);
            if (ok && (int64_t)at + j * kPer < inner) w[j] = __ldg(reinterpret_cast<const uint4*>(px) + j);
        }
#pragma unroll
        for (int j = 0; j < kWords; ++j) {
            const uint32_t q[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 4) v[4 * j + i] = __uint_as_float(q[i]);
                else {
                    v[2 * i] = __uint_as_float(q[i] << 16);
                    v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
                }
            }
        }
    } else {
        T s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] = zero_of<T>();
            if (ok && (int64_t)at + i < inner) s[i] = __ldg(px + i);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32(s[i]);
    }
    const uint32_t byte = block_scale<4>(v);
    const uint2 c = encode_eight(v, byte);
    if (ok && (int64_t)at < pitch) {
        *reinterpret_cast<uint2*>(codes + (int64_t)row * pitch + at) = c;
        if (at % kQ8Block == 0) scales[(int64_t)row * nb + at / kQ8Block] = (uint8_t)byte;
    }
}

// Eight values that lie next to each other.  fp32: as 32 bytes where x starts on 32 (two stores of 16 would each reach half of every
// sector).
template <typename T> __device__ __forceinline__ void write_eight(T* x, const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        if ((reinterpret_cast<uintptr_t>(x) & 31) == 0) {
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(x), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                         "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
            return;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) reinterpret_cast<float4*>(x)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&p);
        }
        *reinterpret_cast<uint4*>(x) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Rows of whole units of eight: a thread restores kRestore units, 256 apart (one read of 8 bytes a thread would leave the memory
// waiting: 42 us with one unit, 38 with two, for 67 million bf16 values).
constexpr int kRestore = 2;
template <typename T, typename I>
__global__ void __launch_bounds__(256) q8_restore_kernel(int64_t rows, int64_t inner, const int8_t* __restrict__ codes,
                                                         const uint8_t* __restrict__ scales, T* __restrict__ x) {
    const I nb = (I)q8_blocks(inner), units = (I)(rows * inner / 8), per_row = (I)(inner / 8);
    const I first = (I)blockIdx.x * (256 * kRestore) + threadIdx.x;
    uint2 c[kRestore];
    uint32_t byte[kRestore];
#pragma unroll
    for (int j = 0; j < kRestore; ++j) {
        const I u = first + 256 * j;
        if (u >= units) continue;
        const I row = u / per_row, at = u - row * per_row;
        c[j] = __ldg(reinterpret_cast<const uint2*>(codes) + u);
        byte[j] = __ldg(scales + (int64_t)row * nb + at / (kQ8Block / 8));
    }
#pragma unroll
    for (int j = 0; j < kRestore; ++j) {
        const I u = first + 256 * j;
        if (u >= units) continue;
        float v[8];
        decode_eight(c[j], byte[j], v);
        write_eight(x + (int64_t)u * 8, v);
    }
}

// Other rows: a thread restores eight values that lie next to each other in the result, whose writes are the ones that have to be
// whole, from wherever their codes are.
template <typename T, typename I>
__global__ void __launch_bounds__(256) q8_restore_any_kernel(int64_t rows, int64_t inner, const int8_t* __restrict__ codes,
                                                             const uint8_t* __restrict__ scales, T* __restrict__ x) {
    const I nb = (I)q8_blocks(inner), total = (I)(rows * inner);
    const int64_t pitch = q8_pitch(inner);
    const I first = ((I)blockIdx.x * 256 + threadIdx.x) * 8;
    if (first >= total) return;
    I row = first / (I)inner, at = first - row * (I)inner;
    float v[8];
    if (inner >= 8) {
        // eight values lie in one row, or in the end of one and the start of the next; in a row, in one block or two neighbours.
        // Codes are read as the aligned eights around them (a row's codes are whole eights).
        const int here = (int)(inner - at < 8 ? inner - at : 8);
        const uint64_t* c = reinterpret_cast<const uint64_t*>(codes + (int64_t)row * pitch) + at / 8;
        const int skip = 8 * (int)(at & 7);
        uint64_t w = __ldg(c) >> skip;
        if (skip && here > 8 - (int)(at & 7)) w |= __ldg(c + 1) << (64 - skip);
        const uint8_t* s = scales + (int64_t)row * nb;
        const I block = at / kQ8Block;
        const int to_next = kQ8Block - (int)(at % kQ8Block);          // values left of the block
        const uint32_t b0 = __ldg(s + block), b1 = to_next < here ? __ldg(s + block + 1) : b0;
        uint32_t b2 = b0;
        if (here < 8 && first + here < total) {
            w = (w & ~(~0ull << 8 * here)) | __ldg(reinterpret_cast<const uint64_t*>(codes + (int64_t)(row + 1) * pitch)) << 8 * here;
            b2 = __ldg(s + nb);
        }
        decode_four((uint32_t)w, 1.0f, v);
        decode_four((uint32_t)(w >> 32), 1.0f, v + 4);
        const float u0 = q8_unit(b0), u1 = q8_unit(b1), u2 = q8_unit(b2);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= i >= here ? u2 : i >= to_next ? u1 : u0;
    } else {
        int q[8];
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            q[i] = 0;
            b[i] = 1;
            if (first + i < total) {
                q[i] = __ldg(codes + (int64_t)row * pitch + at);
                b[i] = __ldg(scales + (int64_t)row * nb + at / kQ8Block);
            }
            if (++at == (I)inner) { at = 0; ++row; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)q[i] * q8_unit(b[i]);
    }
    if (first + 8 <= total) write_eight(x + first, v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (first + i < total) x[first + i] = from_f32<T>(v[i]);
}

}  // namespace tconv
