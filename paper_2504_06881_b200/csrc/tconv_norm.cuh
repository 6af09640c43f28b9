// Root-mean-square norm over the channels of [N][C][P] with the residual's addition (tconv.h), and its gradient.
//
// Bound by HBM: in bf16 with a residual 8 bytes a value forward and 8 backward, for some ten and fifteen operations.  So a block
// holds all channels of its positions in registers from the one read to the write, and what has to be summed over channels
// goes through shared memory once.  The backward kernels run as many blocks as are resident and keep grad_weight's sums in
// registers over all their positions; a second kernel adds the blocks' sums in order.
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

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int k = 16; k; k >>= 1) v += __shfl_xor_sync(~0u, v, k);
    return v;
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


// ---- V values of a thread that lie next to each other: 16 bytes, or one value where rows do not start on 16 bytes ----
template <typename T, int V> struct Some { uint4 w; };
template <typename T> struct Some<T, 1> { T w; };

template <typename T, int V> __device__ __forceinline__ Some<T, V> none_of() {
    Some<T, V> s;
    if constexpr (V == 1) s.w = zero_of<T>(); else s.w = make_uint4(0, 0, 0, 0);
    return s;
}
template <typename T, int V> __device__ __forceinline__ Some<T, V> load_some(const void* p, int64_t at) {
    Some<T, V> s;
    if constexpr (V == 1) s.w = __ldg((const T*)p + at); else s.w = __ldg(reinterpret_cast<const uint4*>((const T*)p + at));
    return s;
}
template <typename T, int V> __device__ __forceinline__ void store_some(void* p, int64_t at, const Some<T, V>& s) {
    if constexpr (V == 1) ((T*)p)[at] = s.w; else *reinterpret_cast<uint4*>((T*)p + at) = s.w;
}
template <typename T, int V> __device__ __forceinline__ void spread(const Some<T, V>& s, float (&v)[V]) {
    if constexpr (V == 1) v[0] = to_f32(s.w);
    else {
        const uint32_t w[4] = {s.w.x, s.w.y, s.w.z, s.w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (V == 4) v[i] = __uint_as_float(w[i]);
            else {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
}
template <typename T, int V> __device__ __forceinline__ Some<T, V> gather(const float (&v)[V]) {
    Some<T, V> s;
    if constexpr (V == 1) s.w = from_f32<T>(v[0]);
    else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (V == 4) w[i] = __float_as_uint(v[i]);
            else {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&p);
            }
        }
        s.w = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return s;
}

// Stores V values at place `at` of a row of an 8-bit form; the 32 / V lanes of a block are neighbours, and every lane of the warp
// calls.  ok: the row exists.
template <int V>
__device__ __forceinline__ void q8_put_some(const float (&v)[V], bool ok, int64_t row, int64_t at, int64_t inner, int8_t* codes, uint8_t* scales) {
    uint32_t top = magnitude_bits(v[0]);
#pragma unroll
    for (int i = 1; i < V; ++i) top = max(top, magnitude_bits(v[i]));
    if constexpr (V == 1) top = __reduce_max_sync(~0u, top);
    else
#pragma unroll
        for (int d = 1; d < kQ8Block / V; d <<= 1) top = max(top, __shfl_xor_sync(~0u, top, d));
    const uint32_t byte = q8_scale_byte(top);
    if (!ok || at >= q8_pitch(inner)) return;
    int8_t* to = codes + row * q8_pitch(inner) + at;
    uint32_t b[V];
    const float inv = q8_inverse(byte);
#pragma unroll
    for (int i = 0; i < V; ++i)      // (1.5 * 2^23 has unit 1: the code is the sum's low byte)
        b[i] = byte == 255u ? 0u : __float_as_uint(__fadd_rn(__fmul_rn(v[i], inv), 12582912.0f));
    if constexpr (V == 1) *to = (int8_t)b[0];
    else {
        uint32_t w[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            w[i] = __byte_perm(__byte_perm(b[4 * i], b[4 * i + 1], 0x0040), __byte_perm(b[4 * i + 2], b[4 * i + 3], 0x0040), 0x5410);
        if constexpr (V == 4) *reinterpret_cast<uint32_t*>(to) = w[0];
        else *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    }
    if (at % kQ8Block == 0 && at < inner) scales[row * q8_blocks(inner) + at / kQ8Block] = (uint8_t)byte;
}

// The stream's V values for the backward pass: itself, or its codes and their unit.
template <typename T, int V, bool Q8> struct Kept {
    Some<T, V> s;
    __device__ __forceinline__ void load(const NormIn& k, int64_t row, int64_t at, int64_t inner) { s = load_some<T, V>(k.s, row * inner + at); }
    __device__ __forceinline__ void none() { s = none_of<T, V>(); }
    __device__ __forceinline__ void values(float (&v)[V]) const { spread<T, V>(s, v); }
};
template <typename T, int V> struct Kept<T, V, true> {
    uint32_t w[V == 8 ? 2 : 1], byte;
    __device__ __forceinline__ void load(const NormIn& k, int64_t row, int64_t at, int64_t inner) {
        const int8_t* p = k.sc + row * q8_pitch(inner) + at;
        if constexpr (V == 8) {
            const uint2 c = __ldg(reinterpret_cast<const uint2*>(p));
            w[0] = c.x;
            w[1] = c.y;
        } else if constexpr (V == 4) w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        else w[0] = (uint8_t)__ldg(p);
        byte = __ldg(k.ss + row * q8_blocks(inner) + at / kQ8Block);
    }
    __device__ __forceinline__ void none() {
        w[0] = 0;
        if constexpr (V == 8) w[1] = 0;
        byte = 1;
    }
    __device__ __forceinline__ void values(float (&v)[V]) const {
        const float unit = q8_unit(byte);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i & 3))) * unit;
    }
};

// P > 1.  A warp has LP lanes of V positions each and 32 / LP channels at a time, a thread R channels.
template <int V, int LP> struct Cols {
    static constexpr int kTile = V * LP;       // positions of a block
    static_assert(kTile % kQ8Block == 0, "an 8-bit block is a warp's affair");
    int lp, cg, cs;                            // lane's place among positions; first channel, channels at a time
    __device__ __forceinline__ Cols() {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        lp = lane % LP;
        cg = warp * (32 / LP) + lane / LP;
        cs = (blockDim.x >> 5) * (32 / LP);
    }
    // Sums v over the block's threads that share positions, then lets `last` turn each position's sum into what all of them get.
    template <typename F> __device__ __forceinline__ void sum(float (&v)[V], float (*part)[kTile], float* total, F last) {
#pragma unroll
        for (int d = LP; d < 32; d <<= 1)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += __shfl_xor_sync(~0u, v[i], d);
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
        if (lane < LP)
#pragma unroll
            for (int i = 0; i < V; ++i) part[warp][lp * V + i] = v[i];
        __syncthreads();
        if (threadIdx.x < kTile) {
            float t = 0.0f;
            for (int w = 0; w < warps; ++w) t += part[w][threadIdx.x];
            total[threadIdx.x] = last(t, threadIdx.x);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = total[lp * V + i];
    }
};

template <typename T, int V, int LP, int R>
__global__ void __launch_bounds__(512) norm_fwd_cols_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    using B = Cols<V, LP>;
    __shared__ float part[16][B::kTile], total[B::kTile];
    B b;
    const int64_t tiles = (a.P + B::kTile - 1) / B::kTile, n = blockIdx.x / tiles, p0 = (blockIdx.x - n * tiles) * B::kTile, p = p0 + b.lp * V;
    const bool in = p < a.P;
    Some<T, V> s[R];
    float sq[V];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int c = b.cg + j * b.cs;
        s[j] = none_of<T, V>();
        if (in && c < a.C) s[j] = load_some<T, V>(x, (n * a.C + c) * a.P + p);
    }
    if (r) {
        Some<T, V> t[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = b.cg + j * b.cs;
            t[j] = none_of<T, V>();
            if (in && c < a.C) t[j] = load_some<T, V>(r, (n * a.C + c) * a.P + p);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = b.cg + j * b.cs;
            float u[V], v[V];
            spread<T, V>(s[j], u);
            spread<T, V>(t[j], v);
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] += v[i];
            s[j] = gather<T, V>(u);
            if (in && c < a.C) store_some<T, V>(o.sum, (n * a.C + c) * a.P + p, s[j]);
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sq[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        float v[V];
        spread<T, V>(s[j], v);
#pragma unroll
        for (int i = 0; i < V; ++i) sq[i] = fmaf(v[i], v[i], sq[i]);
        if (o.sc) {
            const int c = b.cg + j * b.cs;
            q8_put_some<V>(v, c < a.C, n * a.C + c, p, a.P, o.sc, o.ss);
        }
    }
    b.sum(sq, part, total, [&](float t, int i) {
        const float rstd = 1.0f / sqrtf(t / (float)a.C + a.eps);
        if (o.rstd && p0 + i < a.P) o.rstd[n * a.P + p0 + i] = rstd;
        return rstd;
    });
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int c = b.cg + j * b.cs;
        const float wc = c < a.C ? __ldg(w + c) : 0.0f;
        float v[V];
        spread<T, V>(s[j], v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = in ? v[i] * sq[i] * wc : 0.0f;
        if (o.y && in && c < a.C) store_some<T, V>(o.y, (n * a.C + c) * a.P + p, gather<T, V>(v));
        if (o.yc) q8_put_some<V>(v, c < a.C, n * a.C + c, p, a.P, o.yc, o.ys);
    }
}

// part: [gridDim.x][C], this block's sums of grad_weight (NULL: not wanted).
template <typename T, int V, int LP, int R, bool Q8>
__global__ void __launch_bounds__(512) norm_bwd_cols_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                            T* __restrict__ gx, float* __restrict__ gw_part) {
    using B = Cols<V, LP>;
    __shared__ float part[16][B::kTile], total[B::kTile];
    B b;
    const int64_t tiles = (a.P + B::kTile - 1) / B::kTile, all = tiles * a.N;
    float gw[R];
#pragma unroll
    for (int j = 0; j < R; ++j) gw[j] = 0.0f;
    for (int64_t tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const int64_t n = tile / tiles, p = (tile - n * tiles) * B::kTile + b.lp * V;
        const bool in = p < a.P;
        Kept<T, V, Q8> s[R];
        Some<T, V> dy[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = b.cg + j * b.cs;
            s[j].none();
            dy[j] = none_of<T, V>();
            if (in && c < a.C) {
                s[j].load(k, n * a.C + c, p, a.P);
                dy[j] = load_some<T, V>(k.gy, (n * a.C + c) * a.P + p);
            }
        }
        float rstd[V], m[V];
#pragma unroll
        for (int i = 0; i < V; ++i) rstd[i] = m[i] = 0.0f;
        if (in) {
            if constexpr (V == 1) rstd[0] = __ldg(k.rstd + n * a.P + p);
            else
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const float4 q = __ldg(reinterpret_cast<const float4*>(k.rstd + n * a.P + p + i));
                    rstd[i] = q.x; rstd[i + 1] = q.y; rstd[i + 2] = q.z; rstd[i + 3] = q.w;
                }
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = b.cg + j * b.cs;
            const float wc = c < a.C ? __ldg(k.w + c) : 0.0f;
            float v[V], d[V];
            s[j].values(v);
            spread<T, V>(dy[j], d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float t = d[i] * (v[i] * rstd[i]);
                gw[j] += t;
                m[i] = fmaf(wc, t, m[i]);
            }
        }
        b.sum(m, part, total, [&](float t, int) { return t / (float)a.C; });
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = b.cg + j * b.cs;
            if (!in || c >= a.C) continue;
            const float wc = __ldg(k.w + c);
            const int64_t at = (n * a.C + c) * a.P + p;
            float v[V], d[V], e[V];
            s[j].values(v);
            spread<T, V>(dy[j], d);
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] = rstd[i] * (wc * d[i] - v[i] * rstd[i] * m[i]);
            if (k.gs) {
                spread<T, V>(load_some<T, V>(k.gs, at), e);
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] += e[i];
            }
            store_some<T, V>(gx, at, gather<T, V>(d));
        }
    }
    if (!gw_part) return;
#pragma unroll
    for (int j = 0; j < R; ++j) {
#pragma unroll
        for (int d = 1; d < LP; d <<= 1) gw[j] += __shfl_xor_sync(~0u, gw[j], d);
        const int c = b.cg + j * b.cs;
        if (b.lp == 0 && c < a.C) gw_part[(int64_t)blockIdx.x * a.C + c] = gw[j];
    }
}

// P = 1.  A warp has a row, a lane V channels in each of R places 32 V apart.
template <typename T, int V, int R>
__global__ void __launch_bounds__(128) norm_fwd_rows_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (n >= a.N) return;
    const int lane = threadIdx.x & 31;
    Some<T, V> s[R];
    float sq = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int c = (j * 32 + lane) * V;
        s[j] = none_of<T, V>();
        if (c < a.C) {
            s[j] = load_some<T, V>(x, n * a.C + c);
            if (r) {
                float u[V], v[V];
                spread<T, V>(s[j], u);
                spread<T, V>(load_some<T, V>(r, n * a.C + c), v);
#pragma unroll
                for (int i = 0; i < V; ++i) u[i] += v[i];
                s[j] = gather<T, V>(u);
                store_some<T, V>(o.sum, n * a.C + c, s[j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int c = (j * 32 + lane) * V;
        float v[V];
        spread<T, V>(s[j], v);
#pragma unroll
        for (int i = 0; i < V; ++i) sq = fmaf(v[i], v[i], sq);
        if (o.sc) q8_put_some<V>(v, true, n, c, a.C, o.sc, o.ss);
    }
    const float rstd = 1.0f / sqrtf(warp_sum(sq) / (float)a.C + a.eps);
    if (o.rstd && lane == 0) o.rstd[n] = rstd;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int c = (j * 32 + lane) * V;
        float v[V];
        spread<T, V>(s[j], v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c < a.C ? v[i] * rstd * __ldg(w + c + i) : 0.0f;
        if (o.y && c < a.C) store_some<T, V>(o.y, n * a.C + c, gather<T, V>(v));
        if (o.yc) q8_put_some<V>(v, true, n, c, a.C, o.yc, o.ys);
    }
}

template <typename T, int V, int R, bool Q8>
__global__ void __launch_bounds__(128) norm_bwd_rows_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                            T* __restrict__ gx, float* __restrict__ gw_part) {
    __shared__ float sums[4][32 * V * R];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float gw[R][V];
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) gw[j][i] = 0.0f;
    for (int64_t n = (int64_t)blockIdx.x * 4 + warp; n < a.N; n += (int64_t)gridDim.x * 4) {
        const float rstd = __ldg(k.rstd + n);
        Kept<T, V, Q8> s[R];
        Some<T, V> dy[R];
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = (j * 32 + lane) * V;
            s[j].none();
            dy[j] = none_of<T, V>();
            if (c < a.C) {
                s[j].load(k, n, c, a.C);
                dy[j] = load_some<T, V>(k.gy, n * a.C + c);
            }
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = (j * 32 + lane) * V;
            float v[V], d[V];
            s[j].values(v);
            spread<T, V>(dy[j], d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float t = d[i] * (v[i] * rstd);
                gw[j][i] += t;
                m = fmaf(c < a.C ? __ldg(k.w + c + i) : 0.0f, t, m);
            }
        }
        m = warp_sum(m) / (float)a.C;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = (j * 32 + lane) * V;
            if (c >= a.C) continue;
            float v[V], d[V], e[V];
            s[j].values(v);
            spread<T, V>(dy[j], d);
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] = rstd * (__ldg(k.w + c + i) * d[i] - v[i] * rstd * m);
            if (k.gs) {
                spread<T, V>(load_some<T, V>(k.gs, n * a.C + c), e);
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] += e[i];
            }
            store_some<T, V>(gx, n * a.C + c, gather<T, V>(d));
        }
    }
    if (!gw_part) return;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) sums[warp][(j * 32 + lane) * V + i] = gw[j][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += 128) gw_part[(int64_t)blockIdx.x * a.C + c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
}

// grad_weight from the blocks' sums: 32 channels a block, eight rows of threads share the blocks.
template <int U>
__global__ void __launch_bounds__(256) norm_weight_sum_kernel(int C, int blocks, const float* __restrict__ part, float* __restrict__ gw) {
    __shared__ float sums[8][32];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, y = threadIdx.x / 32;
    sums[y][threadIdx.x % 32] = c < C ? sum_in_order<U, float>((blocks - y + 7) / 8, [&](int i) { return __ldg(part + (int64_t)(y + 8 * i) * C + c); }) : 0.0f;
    __syncthreads();
    if (y == 0 && c < C) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += sums[i][threadIdx.x];
        gw[c] = t;
    }
}

// What a layer's kernels look like.
struct NormPlan {
    bool held;                       // a block holds all channels of its positions
    bool vec;                        // 16 bytes at a time
    int warps, lp, reps, blocks;     // warps of a block, lanes along positions, channels of a thread, blocks of the backward pass
};

inline NormPlan plan_norm(const NormArgs& a, int dtype) {
    const int V = dtype == TCONV_F32 ? 4 : 8;
    NormPlan p{};
    p.vec = (a.P > 1 ? a.P : a.C) % V == 0;
    const auto reps = [](int need, int least, int most) {
        int r = least;
        while (r < need) r *= 2;
        return r <= most ? r : 0;
    };
    if (a.P == 1) {
        p.warps = 4;
        p.reps = p.vec ? reps((a.C + 32 * V - 1) / (32 * V), 1, 32 / V) : reps((a.C + 31) / 32, 8, 32);
        p.blocks = (a.N + 3) / 4 < 148 * 2 ? (a.N + 3) / 4 : 148 * 2;
    } else {
        if (p.vec) {
            p.lp = kQ8Block / V;
            p.warps = a.C <= 128 ? 8 : 16;
            p.reps = reps((a.C + p.warps * (32 / p.lp) - 1) / (p.warps * (32 / p.lp)), 1, 8);
        } else {
            p.lp = 32;
            p.warps = a.C <= 128 ? 4 : a.C <= 256 ? 8 : 16;
            p.reps = reps((a.C + p.warps - 1) / p.warps, 4, 32);
        }
        const int64_t tile = p.vec ? V * p.lp : 32, tiles = (a.P + tile - 1) / tile * a.N, most = 148 * (16 / p.warps);
        p.blocks = (int)(tiles < most ? tiles : most);
    }
    p.held = p.reps > 0;
    return p;
}

// Any channel count, P > 1: values are read again where they do not stay; a thread has one position, a warp 32 positions of one image, which are one 8-bit block of each channel.
template <typename T>
__global__ void __launch_bounds__(128) norm_fwd_cols_any_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
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

// Any channel count, P = 1: a warp has one row of C values.
template <typename T>
__global__ void __launch_bounds__(128) norm_fwd_rows_any_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
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

template <typename T>
__global__ void __launch_bounds__(128) norm_bwd_cols_any_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
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
__global__ void __launch_bounds__(128) norm_bwd_rows_any_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
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
__global__ void __launch_bounds__(256) norm_bwd_weight_any_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
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
