// Root-mean-square norm over the channels of [N][C][P] with the residual's addition (tconv.h), and its gradient.
#pragma once
#include "tconv_q8.cuh"

namespace tconv {

struct NormArgs {
    int N, C;
    int64_t P;
    float eps;
};

struct NormOut {
    void *sum, *y;
    float* rstd;
    int8_t* yc;
    uint8_t* ys;
    int8_t* sc;
    uint8_t* ss;
};

// Writes one value of an 8-bit form whose block the warp's lanes hold; `at` is the lane's place in the row.
__device__ __forceinline__ void q8_put(float v, int64_t row, int64_t at, int64_t inner, int8_t* codes, uint8_t* scales) {
    const uint32_t byte = q8_scale_byte(__reduce_max_sync(~0u, magnitude_bits(v)));
    if (at < q8_pitch(inner)) codes[row * q8_pitch(inner) + at] = (int8_t)q8_code(v, byte);
    if ((threadIdx.x & 31) == 0 && at < inner) scales[row * q8_blocks(inner) + at / kQ8Block] = (uint8_t)byte;
}

// P > 1: a thread has one position, a warp 32 positions of one image, which are one 8-bit block of each channel.
template <typename T>
__global__ void __launch_bounds__(128) norm_fwd_cols_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    const int64_t nb = q8_blocks(a.P), b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (b >= nb * a.N) return;
    const int64_t n = b / nb, p = (b - n * nb) * 32 + (threadIdx.x & 31);
    const bool in = p < a.P;
    const int64_t base = n * a.C * a.P + p;
    T* sum = (T*)o.sum;
    const auto value = [&](int c) {
        if (!in) return 0.0f;
        const int64_t i = base + c * a.P;
        return r ? to_f32(from_f32<T>(to_f32(x[i]) + to_f32(r[i]))) : to_f32(x[i]);
    };
    float sq = 0.0f;
    for (int c = 0; c < a.C; ++c) {
        const float v = value(c);
        sq = fmaf(v, v, sq);
        if (r && in) sum[base + c * a.P] = from_f32<T>(v);
        if (o.sc) q8_put(v, n * a.C + c, p, a.P, o.sc, o.ss);
    }
    const float rstd = 1.0f / sqrtf(sq / (float)a.C + a.eps);
    if (o.rstd && in) o.rstd[n * a.P + p] = rstd;
    for (int c = 0; c < a.C; ++c) {
        const float v = in ? value(c) * rstd * w[c] : 0.0f;
        if (o.y && in) ((T*)o.y)[base + c * a.P] = from_f32<T>(v);
        if (o.yc) q8_put(v, n * a.C + c, p, a.P, o.yc, o.ys);
    }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int k = 16; k; k >>= 1) v += __shfl_xor_sync(~0u, v, k);
    return v;
}

// P = 1: a warp has one row of C values.
template <typename T>
__global__ void __launch_bounds__(128) norm_fwd_rows_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (n >= a.N) return;
    const int lane = threadIdx.x & 31, top = (a.C + 31) & ~31;
    T* sum = (T*)o.sum;
    const auto value = [&](int c) {
        if (c >= a.C) return 0.0f;
        const int64_t i = n * a.C + c;
        return r ? to_f32(from_f32<T>(to_f32(x[i]) + to_f32(r[i]))) : to_f32(x[i]);
    };
    float sq = 0.0f;
    for (int c = lane; c < top; c += 32) {
        const float v = value(c);
        sq = fmaf(v, v, sq);
        if (r && c < a.C) sum[n * a.C + c] = from_f32<T>(v);
        if (o.sc) q8_put(v, n, c, a.C, o.sc, o.ss);
    }
    const float rstd = 1.0f / sqrtf(warp_sum(sq) / (float)a.C + a.eps);
    if (o.rstd && lane == 0) o.rstd[n] = rstd;
    for (int c = lane; c < top; c += 32) {
        const float v = c < a.C ? value(c) * rstd * w[c] : 0.0f;
        if (o.y && c < a.C) ((T*)o.y)[n * a.C + c] = from_f32<T>(v);
        if (o.yc) q8_put(v, n, c, a.C, o.yc, o.ys);
    }
}

struct NormIn {
    const void* s;
    const int8_t* sc;
    const uint8_t* ss;
    const float *rstd, *w;
    const void *gy, *gs;
};

template <typename T>
__device__ __forceinline__ float kept_value(const NormIn& k, int64_t row, int64_t at, int64_t inner) {
    if (k.s) return to_f32(((const T*)k.s)[row * inner + at]);
    return (float)k.sc[row * q8_pitch(inner) + at] * q8_unit(k.ss[row * q8_blocks(inner) + at / kQ8Block]);
}

template <typename T>
__global__ void __launch_bounds__(128) norm_bwd_cols_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                            T* __restrict__ gx) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= a.P * a.N) return;
    const int64_t n = i / a.P, p = i - n * a.P;
    const float rstd = k.rstd[i];
    const T *gy = (const T*)k.gy, *gs = (const T*)k.gs;
    float m = 0.0f;
    for (int c = 0; c < a.C; ++c) {
        const int64_t row = n * a.C + c;
        m = fmaf(k.w[c] * to_f32(gy[row * a.P + p]), kept_value<T>(k, row, p, a.P) * rstd, m);
    }
    m /= (float)a.C;
    for (int c = 0; c < a.C; ++c) {
        const int64_t row = n * a.C + c, at = row * a.P + p;
        const float z = kept_value<T>(k, row, p, a.P) * rstd;
        const float d = rstd * (k.w[c] * to_f32(gy[at]) - z * m);
        gx[at] = from_f32<T>(gs ? d + to_f32(gs[at]) : d);
    }
}

template <typename T>
__global__ void __launch_bounds__(128) norm_bwd_rows_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                            T* __restrict__ gx) {
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (n >= a.N) return;
    const int lane = threadIdx.x & 31;
    const float rstd = k.rstd[n];
    const T *gy = (const T*)k.gy, *gs = (const T*)k.gs;
    float m = 0.0f;
    for (int c = lane; c < a.C; c += 32)
        m = fmaf(k.w[c] * to_f32(gy[n * a.C + c]), kept_value<T>(k, n, c, a.C) * rstd, m);
    m = warp_sum(m) / (float)a.C;
    for (int c = lane; c < a.C; c += 32) {
        const int64_t at = n * a.C + c;
        const float z = kept_value<T>(k, n, c, a.C) * rstd;
        const float d = rstd * (k.w[c] * to_f32(gy[at]) - z * m);
        gx[at] = from_f32<T>(gs ? d + to_f32(gs[at]) : d);
    }
}

// grad_weight: one block per channel.
template <typename T>
__global__ void __launch_bounds__(256) norm_bwd_weight_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                              float* __restrict__ gw) {
    __shared__ float red[256];
    const int c = blockIdx.x;
    const T* gy = (const T*)k.gy;
    float m = 0.0f;
    for (int64_t i = threadIdx.x; i < a.P * a.N; i += 256) {
        const int64_t n = i / a.P, p = i - n * a.P, row = n * a.C + c;
        const float v = a.P > 1 ? kept_value<T>(k, row, p, a.P) : kept_value<T>(k, n, c, a.C);
        m = fmaf(to_f32(gy[row * a.P + p]), v * k.rstd[i], m);
    }
    m = block_sum(m, red);
    if (threadIdx.x == 0) gw[c] = m;
}

}  // namespace tconv
