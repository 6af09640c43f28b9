// Gated linear recurrence (tconv.h): h_t = f_t h_{t-1} + (1 - f_t) x_t along the rows of [N][C][L], and its gradient.
#pragma once
#include "tconv_q8.cuh"

namespace tconv {

constexpr int kScanChunk = 256;      // positions between two saved states

struct ScanArgs {
    int64_t rows, L;
    int C;
    int64_t xb, xr, gb, gr;          // strides of x and gate: batch, row
    int64_t ob;                      // batch stride of grad_x and grad_gate
    const int32_t* lengths;
};

struct Gate {
    float f, u;                      // 1 / (1 + e^-g) and 1 - f
};
// e^-g is held to e^80 (a lesser f adds nothing to a sum in fp32), so that u = e^-g * f stays finite; NaN passes.
__device__ __forceinline__ Gate gate_of(float g) {
    float m;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(-g), "f"(80.0f));
    const float e = __expf(m), f = __fdividef(1.0f, 1.0f + e);
    return {f, e * f};
}

__device__ __forceinline__ int64_t row_length(const ScanArgs& a, int64_t n) {
    if (!a.lengths) return a.L;
    const int64_t len = a.lengths[n];
    return len < 0 ? 0 : len > a.L ? a.L : len;
}

// One thread per row.
template <typename T, bool Q8>
__global__ void __launch_bounds__(64) scan_fwd_row_kernel(const __grid_constant__ ScanArgs a, const T* __restrict__ x,
        const T* __restrict__ gate, const float* h0, T* __restrict__ y, float* h_last, float* __restrict__ states,
        int8_t* __restrict__ xc, uint8_t* __restrict__ xs, int8_t* __restrict__ gc, uint8_t* __restrict__ gs) {
    const int64_t row = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (row >= a.rows) return;
    const int64_t n = row / a.C, c = row - n * a.C, len = row_length(a, n);
    const T *px = x + n * a.xb + c * a.xr, *pg = gate + n * a.gb + c * a.gr;
    const int64_t nb = q8_blocks(a.L), pitch = q8_pitch(a.L), nchunk = (a.L + kScanChunk - 1) / kScanChunk;
    float h = h0 ? h0[row] : 0.0f, hq = h;
    for (int64_t t0 = 0; t0 < a.L; t0 += kQ8Block) {
        if (states && t0 % kScanChunk == 0) states[row * nchunk + t0 / kScanChunk] = Q8 ? hq : h;
        const int m = (int)(a.L - t0 < kQ8Block ? a.L - t0 : kQ8Block);
        uint32_t bx = 0, bg = 0;
        if (Q8) {
            for (int i = 0; i < m && t0 + i < len; ++i) {
                bx = max(bx, magnitude_bits(to_f32(px[t0 + i])));
                bg = max(bg, magnitude_bits(to_f32(pg[t0 + i])));
            }
            bx = q8_scale_byte(bx);
            bg = q8_scale_byte(bg);
            xs[row * nb + t0 / kQ8Block] = (uint8_t)bx;
            gs[row * nb + t0 / kQ8Block] = (uint8_t)bg;
        }
        for (int i = 0; i < m; ++i) {
            const int64_t t = t0 + i;
            const bool live = t < len;
            const float xv = live ? to_f32(px[t]) : 0.0f, gv = live ? to_f32(pg[t]) : 0.0f;
            if (live) {
                const Gate k = gate_of(gv);
                h = fmaf(k.f, h, k.u * xv);
            }
            y[row * a.L + t] = from_f32<T>(live ? h : 0.0f);
            if (Q8) {
                const int cx = q8_code(xv, bx), cg = q8_code(gv, bg);
                xc[row * pitch + t] = (int8_t)cx;
                gc[row * pitch + t] = (int8_t)cg;
                if (live) {
                    const Gate k = gate_of((float)cg * q8_unit(bg));
                    hq = fmaf(k.f, hq, k.u * ((float)cx * q8_unit(bx)));
                }
            }
        }
    }
    if (Q8)
        for (int64_t t = a.L; t < pitch; ++t) xc[row * pitch + t] = gc[row * pitch + t] = 0;
    h_last[row] = h;
}

template <typename T, bool Q8>
__global__ void __launch_bounds__(64) scan_bwd_row_kernel(const __grid_constant__ ScanArgs a, const T* __restrict__ x,
        const T* __restrict__ gate, const int8_t* __restrict__ xc, const uint8_t* __restrict__ xs, const int8_t* __restrict__ gc,
        const uint8_t* __restrict__ gs, const float* __restrict__ states, const T* __restrict__ gy,
        const float* __restrict__ gh, T* __restrict__ gx, T* __restrict__ gg, float* __restrict__ gh0) {
    const int64_t row = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (row >= a.rows) return;
    const int64_t n = row / a.C, c = row - n * a.C, len = row_length(a, n);
    const T *px = x + n * a.xb + c * a.xr, *pg = gate + n * a.gb + c * a.gr;
    T *ox = gx + n * a.ob + c * a.L, *og = gg + n * a.ob + c * a.L;
    const int64_t nb = q8_blocks(a.L), pitch = q8_pitch(a.L), nchunk = (a.L + kScanChunk - 1) / kScanChunk;
    const auto xv = [&](int64_t t) {
        return Q8 ? (float)xc[row * pitch + t] * q8_unit(xs[row * nb + t / kQ8Block]) : to_f32(px[t]);
    };
    const auto gv = [&](int64_t t) {
        return Q8 ? (float)gc[row * pitch + t] * q8_unit(gs[row * nb + t / kQ8Block]) : to_f32(pg[t]);
    };
    float d = gh ? gh[row] : 0.0f;   // f_{t+1} D_{t+1}
    float before[kScanChunk];
    for (int64_t k = nchunk - 1; k >= 0; --k) {
        const int64_t t0 = k * kScanChunk;
        const int m = (int)(a.L - t0 < kScanChunk ? a.L - t0 : kScanChunk);
        float h = states[row * nchunk + k];
        for (int i = 0; i < m && t0 + i < len; ++i) {
            const Gate q = gate_of(gv(t0 + i));
            before[i] = h;
            h = fmaf(q.f, h, q.u * xv(t0 + i));
        }
        for (int i = m - 1; i >= 0; --i) {
            const int64_t t = t0 + i;
            float rx = 0.0f, rg = 0.0f;
            if (t < len) {
                const Gate q = gate_of(gv(t));
                const float D = d + to_f32(gy[row * a.L + t]);
                rx = q.u * D;
                rg = D * (before[i] - xv(t)) * (q.f * q.u);
                d = q.f * D;
            }
            ox[t] = from_f32<T>(rx);
            og[t] = from_f32<T>(rg);
        }
    }
    if (gh0) gh0[row] = d;
}

}  // namespace tconv
