// Root-mean-square norm over the channels of [N][C][P] with the residual's addition (tconv.h), and its gradient.
//
// Bound by HBM: in bf16 with a residual 8 bytes a value forward and 8 backward, for some ten and fifteen operations.  So a block
// holds all channels of its positions in registers from the one read to the write, and what has to be summed over channels
// goes through shared memory once.  The backward kernels run as many blocks as are resident and keep grad_weight's sums in
// registers over all their positions; a second kernel adds the blocks' sums in order.  8 x 256 x 128 x 256 bf16 with an 8-bit output
// takes 106 us forward (5.7 TB/s) and 101 backward (5.3); 32 x 128 x 3981 fp32, value by value, 45 and 53 us (5.8 and 4.9 TB/s).
#pragma once
#include "tconv_q8.cuh"

#include <type_traits>

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

// ---- V values of a thread that lie next to each other: 16 bytes; 8 or one value where rows do not start on 16 bytes ----
template <typename T, int V> struct Some { uint4 w; };
template <> struct Some<__nv_bfloat16, 4> { uint2 w; };
template <typename T> struct Some<T, 1> { T w; };

template <typename T, int V> using Piece = decltype(Some<T, V>::w);
template <typename T, int V> __device__ __forceinline__ Some<T, V> none_of() {
    if constexpr (V == 1) return {zero_of<T>()};
    else return {};
}
template <typename T, int V> __device__ __forceinline__ Some<T, V> load_some(const void* p, int64_t at) {
    return {__ldg(reinterpret_cast<const Piece<T, V>*>((const T*)p + at))};
}
// What this thread has written before.
template <typename T, int V> __device__ __forceinline__ Some<T, V> load_own(const void* p, int64_t at) {
    return {*reinterpret_cast<const Piece<T, V>*>((const T*)p + at)};
}
template <typename T, int V> __device__ __forceinline__ void store_some(void* p, int64_t at, const Some<T, V>& s) {
    *reinterpret_cast<Piece<T, V>*>((T*)p + at) = s.w;
}
template <typename T, int V> __device__ __forceinline__ void spread(const Some<T, V>& s, float (&v)[V]) {
    if constexpr (V == 1) v[0] = to_f32(s.w);
    else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&s.w);
#pragma unroll
        for (int i = 0; i < (int)sizeof(s.w) / 4; ++i) {
            if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
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
        uint32_t* w = reinterpret_cast<uint32_t*>(&s.w);
#pragma unroll
        for (int i = 0; i < (int)sizeof(s.w) / 4; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v[i]);
            else {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&p);
            }
        }
    }
    return s;
}

// Stores V values of an 8-bit form: codes to `to`, and at a block's first value the scale byte to `scale`; the 32 / V lanes of a block
// are neighbours, and every lane of the warp calls.  ok: the values are there to be stored.
template <int V> __device__ __forceinline__ void q8_put_some(const float (&v)[V], bool ok, int8_t* to, bool head, uint8_t* scale) {
    uint32_t top = __float_as_uint(top_of(v));
    if constexpr (V == 1) top = __reduce_max_sync(~0u, top);
    else
#pragma unroll
        for (int d = 1; d < kQ8Block / V; d <<= 1) top = max(top, __shfl_xor_sync(~0u, top, d));
    const uint32_t byte = q8_scale_byte(top);
    if (!ok) return;
    float r[V];
    q8_round(v, byte, r);
    if constexpr (V == 1) *to = (int8_t)__float_as_uint(r[0]);
    else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(to) = four_codes(r);
    else *reinterpret_cast<uint2*>(to) = make_uint2(four_codes(r), four_codes(r + 4));
    if (head) *scale = (uint8_t)byte;
}

// The stream's V values for the backward pass: itself, or its codes and their unit.
template <typename T, int V, bool Q8> struct Kept {
    Some<T, V> s;
    __device__ __forceinline__ void load(const T* p, const int8_t*, const uint8_t*) { s = load_some<T, V>(p, 0); }
    __device__ __forceinline__ void none() { s = none_of<T, V>(); }
    __device__ __forceinline__ void values(float (&v)[V]) const { spread<T, V>(s, v); }
};
template <typename T, int V> struct Kept<T, V, true> {
    uint32_t w[V == 8 ? 2 : 1], byte;
    __device__ __forceinline__ void load(const T*, const int8_t* c, const uint8_t* scale) {
        if constexpr (V == 8) {
            const uint2 q = __ldg(reinterpret_cast<const uint2*>(c));
            w[0] = q.x;
            w[1] = q.y;
        } else if constexpr (V == 4) w[0] = __ldg(reinterpret_cast<const uint32_t*>(c));
        else w[0] = (uint8_t)__ldg(c);
        byte = __ldg(scale);
    }
    __device__ __forceinline__ void none() {
        w[0] = 0;
        if constexpr (V == 8) w[1] = 0;
        byte = 1;
    }
    __device__ __forceinline__ void values(float (&v)[V]) const {
        const float unit = q8_unit(byte);
        if constexpr (V == 1) v[0] = (float)(int8_t)w[0] * unit;
        else
#pragma unroll
            for (int i = 0; i < V; i += 4) decode_four(w[i / 4], unit, v + i);
    }
};

// P > 1.  A block has WARPS warps and 32 positions of one image, an 8-bit block of every channel; a warp has 32 / V lanes of V
// positions each and V channels at a time, a thread R channels.  Offsets inside an image are 32 bits wide.
template <int V, int WARPS> struct Cols {
    static constexpr int kLanes = kQ8Block / V, kStep = WARPS * V;     // lanes along positions; channels at a time
    const int lp, c0;                                                   // the lane's place among positions; its first channel
    __device__ __forceinline__ Cols() : lp(threadIdx.x % kLanes), c0(threadIdx.x / kLanes) {}
    __device__ __forceinline__ int channels(int C) const { return c0 < C ? (C - c0 + kStep - 1) / kStep : 0; }
    // Sums v over the threads that share positions; `last` turns a position's sum into what all of them get.
    template <typename F> __device__ __forceinline__ void sum(float (&v)[V], float (*part)[kQ8Block], float* total, F last) const {
#pragma unroll
        for (int d = kLanes; d < 32; d <<= 1)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += __shfl_xor_sync(~0u, v[i], d);
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (lane < kLanes)
#pragma unroll
            for (int i = 0; i < V; ++i) part[warp][lane * V + i] = v[i];
        __syncthreads();
        if (threadIdx.x < kQ8Block) {
            float t = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) t += part[w][threadIdx.x];
            total[threadIdx.x] = last(t, threadIdx.x);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = total[lp * V + i];
    }
};

// Blocks of the backward kernel that an SM holds: 128 registers a thread.
constexpr int norm_resident(int warps) { return 16 / warps; }

// RES: with a residual; Q8: some output in 8 bits.
template <typename T, int V, int WARPS, int R, bool RES, bool Q8>
__global__ void __launch_bounds__(WARPS * 32) norm_fwd_cols_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    __shared__ float part[WARPS][kQ8Block], total[kQ8Block];
    const Cols<V, WARPS> b;
    const uint32_t P = (uint32_t)a.P, tiles = (P + kQ8Block - 1) / kQ8Block, pitch = (uint32_t)q8_pitch(a.P);
    const uint32_t n = blockIdx.x / tiles, p0 = (blockIdx.x - n * tiles) * kQ8Block, p = p0 + b.lp * V;
    const int have = b.channels(a.C), live = p < P ? have : 0;          // channels of this thread; with positions in the image
    const int64_t image = (int64_t)n * a.C * P;
    const uint32_t at = b.c0 * P + p, step = b.kStep * P;
    x += image;
    Some<T, V> s[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        s[j] = none_of<T, V>();
        if (j < live) s[j] = load_some<T, V>(x, at + j * step);
    }
    if constexpr (RES) {
        r += image;
        T* sum = (T*)o.sum + image;
        Some<T, V> t[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            t[j] = none_of<T, V>();
            if (j < live) t[j] = load_some<T, V>(r, at + j * step);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            float u[V], v[V];
            spread<T, V>(s[j], u);
            spread<T, V>(t[j], v);
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] += v[i];
            s[j] = gather<T, V>(u);
            if (j < live) store_some<T, V>(sum, at + j * step, s[j]);
        }
    }
    const uint32_t code_at = b.c0 * pitch + p, scale_at = b.c0 * tiles + p0 / kQ8Block;      // (inside the image too)
    const auto put = [&](const float (&v)[V], int j, int8_t* codes, uint8_t* scales) {
        q8_put_some<V>(v, j < have && p < pitch, codes + (code_at + j * b.kStep * pitch), b.lp == 0, scales + (scale_at + j * b.kStep * tiles));
    };
    const int64_t row0 = (int64_t)n * a.C;
    int8_t *sc = o.sc + row0 * pitch, *yc = o.yc + row0 * pitch;
    uint8_t *ss = o.ss + row0 * tiles, *ys = o.ys + row0 * tiles;
    float sq[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sq[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        float v[V];
        spread<T, V>(s[j], v);
#pragma unroll
        for (int i = 0; i < V; ++i) sq[i] = fmaf(v[i], v[i], sq[i]);
        if constexpr (Q8)
            if (o.sc) put(v, j, sc, ss);
    }
    b.sum(sq, part, total, [&](float t, uint32_t i) {
        const float rstd = 1.0f / sqrtf(t / (float)a.C + a.eps);
        if (o.rstd && p0 + i < P) o.rstd[(int64_t)n * P + p0 + i] = rstd;
        return rstd;
    });
    T* y = (T*)o.y + image;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const float wc = j < have ? __ldg(w + b.c0 + j * b.kStep) : 0.0f;
        float v[V];
        spread<T, V>(s[j], v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = v[i] * sq[i] * wc;
        if constexpr (Q8) {
            if (o.y && j < live) store_some<T, V>(y, at + j * step, gather<T, V>(v));
            if (o.yc) {
                if (j >= live)       // (a row's end, where 0 * NaN must not poison the block)
#pragma unroll
                    for (int i = 0; i < V; ++i) v[i] = 0.0f;
                put(v, j, yc, ys);
            }
        } else if (j < live) store_some<T, V>(y, at + j * step, gather<T, V>(v));
    }
}

// gw_part: [gridDim.x][C], each block's sums of grad_weight (NULL: not wanted).  RES: the stream has a gradient of its own.
template <typename T, int V, int WARPS, int R, bool RES, bool Q8>
__global__ void __launch_bounds__(WARPS * 32, norm_resident(WARPS)) norm_bwd_cols_kernel(
        const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k, T* __restrict__ gx, float* __restrict__ gw_part) {
    // the stream's own gradient: read with the rest where registers allow, else in batches when it is added
    constexpr bool kLate = V == 1 ? R > 16 : R > 4;
    constexpr int kBatch = kLate ? R / 4 : R;
    __shared__ float part[WARPS][kQ8Block], total[kQ8Block];
    const Cols<V, WARPS> b;
    const uint32_t P = (uint32_t)a.P, tiles = (P + kQ8Block - 1) / kQ8Block, all = tiles * a.N, pitch = (uint32_t)q8_pitch(a.P);
    const uint32_t step = b.kStep * P;
    const int have = b.channels(a.C);
    float gw[R];
#pragma unroll
    for (int j = 0; j < R; ++j) gw[j] = 0.0f;
    // A tile's place.  The registers of a channel take the next tile's values as soon as this one's are done with, so that the
    // reads go on while the rest is written and summed.
    struct At {
        uint32_t n, p0, p, in_image;
        int live;
    };
    const auto place = [&](uint32_t tile) {
        At t;
        t.n = tile / tiles;
        t.p0 = (tile - t.n * tiles) * kQ8Block;
        t.p = t.p0 + b.lp * V;
        t.in_image = b.c0 * P + t.p;
        t.live = tile < all && t.p < P ? have : 0;
        return t;
    };
    Kept<T, V, Q8> s[R];
    Some<T, V> dy[R], ds[RES ? (kLate ? kBatch : R) : 1];
    const auto load = [&](const At& t, int j) {
        s[j].none();
        dy[j] = none_of<T, V>();
        if constexpr (RES && !kLate) ds[j] = none_of<T, V>();
        if (j < t.live) {
            const int64_t image = (int64_t)t.n * a.C * P, row = (int64_t)t.n * a.C + b.c0 + j * b.kStep;
            const uint32_t at = t.in_image + j * step;
            s[j].load((const T*)k.s + image + at, k.sc + row * pitch + t.p, k.ss + row * tiles + t.p0 / kQ8Block);
            dy[j] = load_some<T, V>((const T*)k.gy + image, at);
            if constexpr (RES && !kLate) ds[j] = load_some<T, V>((const T*)k.gs + image, at);
        }
    };
    At t = place(blockIdx.x);
#pragma unroll
    for (int j = 0; j < R; ++j) load(t, j);
    for (uint32_t tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const At next = place(tile + gridDim.x);
        const int64_t image = (int64_t)t.n * a.C * P;
        float rstd[V], m[V];
#pragma unroll
        for (int i = 0; i < V; ++i) rstd[i] = m[i] = 0.0f;
        if (t.p < P) {
            const float* pr = k.rstd + (int64_t)t.n * P + t.p;
            if constexpr (V == 1) rstd[0] = __ldg(pr);
            else
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const float4 q = __ldg(reinterpret_cast<const float4*>(pr + i));
                    rstd[i] = q.x; rstd[i + 1] = q.y; rstd[i + 2] = q.z; rstd[i + 3] = q.w;
                }
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const float wc = j < have ? __ldg(k.w + b.c0 + j * b.kStep) : 0.0f;
            float v[V], d[V];
            s[j].values(v);
            spread<T, V>(dy[j], d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float u = d[i] * (v[i] * rstd[i]);
                gw[j] += u;
                m[i] = fmaf(wc, u, m[i]);
            }
        }
        b.sum(m, part, total, [&](float u, int) { return u / (float)a.C; });
        T* po = gx + image;
#pragma unroll
        for (int j0 = 0; j0 < R; j0 += kBatch) {
            if constexpr (RES && kLate) {
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    ds[j] = none_of<T, V>();
                    if (j0 + j < t.live) ds[j] = load_some<T, V>((const T*)k.gs + image, t.in_image + (j0 + j) * step);
                }
            }
#pragma unroll
            for (int jj = 0; jj < kBatch; ++jj) {
                const int j = j0 + jj;
                const float wc = j < have ? __ldg(k.w + b.c0 + j * b.kStep) : 0.0f;
                float v[V], d[V];
                s[j].values(v);
                spread<T, V>(dy[j], d);
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = rstd[i] * (wc * d[i] - v[i] * rstd[i] * m[i]);
                if constexpr (RES) {
                    float e[V];
                    spread<T, V>(ds[kLate ? jj : j], e);
#pragma unroll
                    for (int i = 0; i < V; ++i) d[i] += e[i];
                }
                if (j < t.live) store_some<T, V>(po, t.in_image + j * step, gather<T, V>(d));
                if constexpr (!kLate) load(next, j);
            }
        }
        if constexpr (kLate)                                  // (no registers to spare for reads on their way)
#pragma unroll
            for (int j = 0; j < R; ++j) load(next, j);
        t = next;
    }
    if (!gw_part) return;
#pragma unroll
    for (int j = 0; j < R; ++j) {
#pragma unroll
        for (int d = 1; d < b.kLanes; d <<= 1) gw[j] += __shfl_xor_sync(~0u, gw[j], d);
        if (b.lp == 0 && j < have) gw_part[(int64_t)blockIdx.x * a.C + b.c0 + j * b.kStep] = gw[j];
    }
}

// P = 1.  A warp has a row, a lane V channels in each of R places 32 V apart.
template <typename T, int V, int R>
__global__ void __launch_bounds__(128) norm_fwd_rows_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (n >= a.N) return;
    const int lane = threadIdx.x & 31;
    const int pitch = (int)q8_pitch(a.C), nb = (int)q8_blocks(a.C);
    const auto put = [&](const float (&v)[V], int c, int8_t* codes, uint8_t* scales) {
        q8_put_some<V>(v, c < pitch, codes + n * pitch + c, c % kQ8Block == 0 && c < a.C, scales + n * nb + c / kQ8Block);
    };
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
        if (o.sc) put(v, c, o.sc, o.ss);
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
        if (o.yc) put(v, c, o.yc, o.ys);
    }
}

template <typename T, int V, int R, bool Q8>
__global__ void __launch_bounds__(128) norm_bwd_rows_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                            T* __restrict__ gx, float* __restrict__ gw_part) {
    __shared__ float sums[4][32 * V * R];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, pitch = (int)q8_pitch(a.C), nb = (int)q8_blocks(a.C);
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
                s[j].load((const T*)k.s + n * a.C + c, k.sc + n * pitch + c, k.ss + n * nb + c / kQ8Block);
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

// ---- any channel count: the channels go in groups of what registers hold, and are read once more (from L2) after the sums ----
template <typename T, int V, int WARPS, int R, bool RES, bool Q8>
__global__ void __launch_bounds__(WARPS * 32, 2) norm_fwd_loop_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    __shared__ float part[WARPS][kQ8Block], total[kQ8Block];
    const Cols<V, WARPS> b;
    const int64_t P = a.P, tiles = q8_blocks(P), pitch = q8_pitch(P), n = blockIdx.x / tiles, p0 = (blockIdx.x - n * tiles) * kQ8Block, p = p0 + b.lp * V;
    const bool in = p < P;
    const int64_t image = n * a.C * P;
    T* sum = RES ? (T*)o.sum + image : nullptr;
    const auto put = [&](const float (&v)[V], int c, int8_t* codes, uint8_t* scales) {
        const int64_t row = n * a.C + c;
        q8_put_some<V>(v, c < a.C && p < pitch, codes + row * pitch + p, b.lp == 0, scales + row * tiles + p0 / kQ8Block);
    };
    const int64_t step = b.kStep * P;
    float sq[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sq[i] = 0.0f;
    for (int base = b.c0; base - b.c0 < a.C; base += R * b.kStep) {
        const int64_t at = base * P + p;
        Some<T, V> s[R], t[RES ? R : 1];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = base + j * b.kStep;
            s[j] = none_of<T, V>();
            if (in && c < a.C) s[j] = load_some<T, V>(x + image, at + j * step);
            if constexpr (RES) {
                t[j] = none_of<T, V>();
                if (in && c < a.C) t[j] = load_some<T, V>(r + image, at + j * step);
            }
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = base + j * b.kStep;
            float v[V];
            spread<T, V>(s[j], v);
            if constexpr (RES) {
                float u[V];
                spread<T, V>(t[j], u);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += u[i];
                s[j] = gather<T, V>(v);
                spread<T, V>(s[j], v);
                if (in && c < a.C) store_some<T, V>(sum, at + j * step, s[j]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sq[i] = fmaf(v[i], v[i], sq[i]);
            if constexpr (Q8)
                if (o.sc) put(v, c, o.sc, o.ss);
        }
    }
    b.sum(sq, part, total, [&](float t, int i) {
        const float rstd = 1.0f / sqrtf(t / (float)a.C + a.eps);
        if (o.rstd && p0 + i < P) o.rstd[n * P + p0 + i] = rstd;
        return rstd;
    });
    T* y = (T*)o.y + image;
    for (int base = b.c0; base - b.c0 < a.C; base += R * b.kStep) {
        const int64_t at = base * P + p;
        Some<T, V> s[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = base + j * b.kStep;
            s[j] = none_of<T, V>();
            if (in && c < a.C) s[j] = RES ? load_own<T, V>(sum, at + j * step) : load_some<T, V>(x + image, at + j * step);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int c = base + j * b.kStep;
            const float wc = c < a.C ? __ldg(w + c) : 0.0f;
            float v[V];
            spread<T, V>(s[j], v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = in && c < a.C ? v[i] * sq[i] * wc : 0.0f;
            if (o.y && in && c < a.C) store_some<T, V>(y, at + j * step, gather<T, V>(v));
            if constexpr (Q8)
                if (o.yc) put(v, c, o.yc, o.ys);
        }
    }
}

// gw_part as above; a block's sums grow in shared memory where they fit (in place a sum waited for its last write at every
// tile: 151 us against 116 for 8 x 1024 x 8192 bf16), else there, each by one thread.
constexpr int kNormShared = 8192;
template <typename T, int V, int WARPS, int R, bool RES, bool Q8>
__global__ void __launch_bounds__(WARPS * 32, 2) norm_bwd_loop_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                                   T* __restrict__ gx, float* gw_part) {
    __shared__ float part[WARPS][kQ8Block], total[kQ8Block];
    const Cols<V, WARPS> b;
    const int64_t P = a.P, tiles = q8_blocks(P), pitch = q8_pitch(P), all = tiles * a.N;
    extern __shared__ float own[];
    float* out = gw_part ? gw_part + (int64_t)blockIdx.x * a.C : nullptr;
    float* gw = gw_part && a.C <= kNormShared ? own : out;
    if (gw && b.lp == 0)
        for (int c = b.c0; c < a.C; c += b.kStep) gw[c] = 0.0f;
    for (int64_t tile = blockIdx.x; tile < all; tile += gridDim.x) {
        const int64_t n = tile / tiles, p0 = (tile - n * tiles) * kQ8Block, p = p0 + b.lp * V;
        const bool in = p < P;
        const int64_t image = n * a.C * P, step = b.kStep * P;
        Kept<T, V, Q8> s[R];
        Some<T, V> dy[R];
        const auto load = [&](int c, int64_t at, int j) {
            s[j].none();
            dy[j] = none_of<T, V>();
            if (in && c < a.C) {
                const int64_t row = n * a.C + c;
                s[j].load((const T*)k.s + image + at, k.sc + row * pitch + p, k.ss + row * tiles + p0 / kQ8Block);
                dy[j] = load_some<T, V>((const T*)k.gy + image, at);
            }
        };
        float rstd[V], m[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            rstd[i] = in ? __ldg(k.rstd + n * P + p + i) : 0.0f;
            m[i] = 0.0f;
        }
        for (int base = b.c0; base - b.c0 < a.C; base += R * b.kStep) {
#pragma unroll
            for (int j = 0; j < R; ++j) load(base + j * b.kStep, base * P + p + j * step, j);
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int c = base + j * b.kStep;
                const float wc = c < a.C ? __ldg(k.w + c) : 0.0f;
                float v[V], d[V], g = 0.0f;
                s[j].values(v);
                spread<T, V>(dy[j], d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float u = d[i] * (v[i] * rstd[i]);
                    g += u;
                    m[i] = fmaf(wc, u, m[i]);
                }
                if (gw) {
#pragma unroll
                    for (int d2 = 1; d2 < b.kLanes; d2 <<= 1) g += __shfl_xor_sync(~0u, g, d2);
                    if (b.lp == 0 && c < a.C) gw[c] += g;
                }
            }
        }
        b.sum(m, part, total, [&](float u, int) { return u / (float)a.C; });
        for (int base = b.c0; base - b.c0 < a.C; base += R * b.kStep) {
            const int64_t at = base * P + p;
            Some<T, V> ds[RES ? R : 1];
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int c = base + j * b.kStep;
                load(c, at + j * step, j);
                if constexpr (RES) {
                    ds[j] = none_of<T, V>();
                    if (in && c < a.C) ds[j] = load_some<T, V>((const T*)k.gs + image, at + j * step);
                }
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int c = base + j * b.kStep;
                const float wc = c < a.C ? __ldg(k.w + c) : 0.0f;
                float v[V], d[V];
                s[j].values(v);
                spread<T, V>(dy[j], d);
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = rstd[i] * (wc * d[i] - v[i] * rstd[i] * m[i]);
                if constexpr (RES) {
                    float e[V];
                    spread<T, V>(ds[j], e);
#pragma unroll
                    for (int i = 0; i < V; ++i) d[i] += e[i];
                }
                if (in && c < a.C) store_some<T, V>(gx + image, at + j * step, gather<T, V>(d));
            }
        }
    }
    if (gw != out && b.lp == 0)
        for (int c = b.c0; c < a.C; c += b.kStep) out[c] = gw[c];
}

// P = 1: a warp has a row, and its lanes V channels every 32 V.
template <typename T, int V>
__global__ void __launch_bounds__(128) norm_fwd_rows_loop_kernel(const __grid_constant__ NormArgs a, const T* __restrict__ x,
        const T* __restrict__ r, const float* __restrict__ w, const __grid_constant__ NormOut o) {
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (n >= a.N) return;
    const int lane = threadIdx.x & 31, top = (a.C + 31) & ~31;
    const int64_t pitch = q8_pitch(a.C), nb = q8_blocks(a.C);
    const auto put = [&](const float (&v)[V], int64_t c, int8_t* codes, uint8_t* scales) {
        q8_put_some<V>(v, c < pitch, codes + n * pitch + c, c % kQ8Block == 0 && c < a.C, scales + n * nb + c / kQ8Block);
    };
    float sq = 0.0f;
    for (int64_t base = 0; base < top; base += 32 * V) {
        const int64_t c = base + lane * V;
        float v[V];
        Some<T, V> s = none_of<T, V>();
        if (c < a.C) s = load_some<T, V>(x, n * a.C + c);
        spread<T, V>(s, v);
        if (r && c < a.C) {
            float u[V];
            spread<T, V>(load_some<T, V>(r, n * a.C + c), u);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += u[i];
            s = gather<T, V>(v);
            spread<T, V>(s, v);
            store_some<T, V>(o.sum, n * a.C + c, s);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) sq = fmaf(v[i], v[i], sq);
        if (o.sc) put(v, c, o.sc, o.ss);
    }
    const float rstd = 1.0f / sqrtf(warp_sum(sq) / (float)a.C + a.eps);
    if (o.rstd && lane == 0) o.rstd[n] = rstd;
    for (int64_t base = 0; base < top; base += 32 * V) {
        const int64_t c = base + lane * V;
        float v[V];
        Some<T, V> s = none_of<T, V>();
        if (c < a.C) s = r ? load_own<T, V>(o.sum, n * a.C + c) : load_some<T, V>(x, n * a.C + c);
        spread<T, V>(s, v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = c < a.C ? v[i] * rstd * __ldg(w + c + i) : 0.0f;
        if (o.y && c < a.C) store_some<T, V>(o.y, n * a.C + c, gather<T, V>(v));
        if (o.yc) put(v, c, o.yc, o.ys);
    }
}

template <typename T, int V, bool Q8>
__global__ void __launch_bounds__(128) norm_bwd_rows_loop_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                                 T* __restrict__ gx) {
    const int lane = threadIdx.x & 31;
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5), pitch = q8_pitch(a.C), nb = q8_blocks(a.C);
    if (n >= a.N) return;
    const float rstd = __ldg(k.rstd + n);
    Kept<T, V, Q8> s;
    float m = 0.0f;
#pragma unroll 4
    for (int64_t c = lane * V; c < a.C; c += 32 * V) {
        float v[V], d[V];
        s.load((const T*)k.s + n * a.C + c, k.sc + n * pitch + c, k.ss + n * nb + c / kQ8Block);
        s.values(v);
        spread<T, V>(load_some<T, V>(k.gy, n * a.C + c), d);
#pragma unroll
        for (int i = 0; i < V; ++i) m = fmaf(__ldg(k.w + c + i), d[i] * (v[i] * rstd), m);
    }
    m = warp_sum(m) / (float)a.C;
#pragma unroll 4
    for (int64_t c = lane * V; c < a.C; c += 32 * V) {
        float v[V], d[V];
        s.load((const T*)k.s + n * a.C + c, k.sc + n * pitch + c, k.ss + n * nb + c / kQ8Block);
        s.values(v);
        spread<T, V>(load_some<T, V>(k.gy, n * a.C + c), d);
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = rstd * (__ldg(k.w + c + i) * d[i] - v[i] * rstd * m);
        if (k.gs) {
            float e[V];
            spread<T, V>(load_some<T, V>(k.gs, n * a.C + c), e);
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] += e[i];
        }
        store_some<T, V>(gx, n * a.C + c, gather<T, V>(d));
    }
}

// Its grad_weight: a thread has V channels and every gridDim.y-th row.  gw_part: [gridDim.y][C].
template <typename T, int V, bool Q8>
__global__ void __launch_bounds__(128) norm_bwd_rows_weight_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ NormIn k,
                                                                   float* __restrict__ gw_part) {
    const int64_t c = ((int64_t)blockIdx.x * 128 + threadIdx.x) * V, pitch = q8_pitch(a.C), nb = q8_blocks(a.C);
    if (c >= a.C) return;
    float g[V];
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = 0.0f;
#pragma unroll 4
    for (int64_t n = blockIdx.y; n < a.N; n += gridDim.y) {
        const float rstd = __ldg(k.rstd + n);
        Kept<T, V, Q8> s;
        float v[V], d[V];
        s.load((const T*)k.s + n * a.C + c, k.sc + n * pitch + c, k.ss + n * nb + c / kQ8Block);
        s.values(v);
        spread<T, V>(load_some<T, V>(k.gy, n * a.C + c), d);
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = fmaf(d[i], v[i] * rstd, g[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) gw_part[(int64_t)blockIdx.y * a.C + c + i] = g[i];
}

// What a layer's kernels look like.
struct NormPlan {
    int vec;                         // values at a time: 16 bytes' worth, 4 or 1
    int form;                        // which of the kernels with all channels in registers; -1: the one that goes over them in groups
    int blocks, parts;               // blocks of the backward pass, and partial sums of grad_weight
};

// The kernels with P > 1, by values at a time, warps, and channels of a thread, from the smallest that holds all channels on.  The
// last one by single values is at the limit of its registers (its backward from a stream in 8 bits beyond: of a word a code 336 to
// 432 bytes a thread go to local memory, 64 x 512 x 7 x 7 bf16 32 us), and still ahead of the kernel in groups where maps are small
// (64 x 512 x 7 x 7 bf16 forward 7.7 us against 11.6) and even with it where they are large (8 x 512 x 8191 bf16 forward and backward 102 + 206
// against 133 + 183).  Four bf16 values at a time against single ones: 86 + 82 us for 7 x 494 x 13044 (the whole pass 222 against 642).
template <typename F> void with_cols(std::integral_constant<int, 8>, int form, F f) {
    if (form == 0) f.template operator()<8, 4, 2>();
    else if (form == 1) f.template operator()<8, 4, 4>();
    else if (form == 2) f.template operator()<8, 8, 4>();
    else f.template operator()<8, 16, 4>();
}
template <typename F> void with_cols(std::integral_constant<int, 4>, int form, F f) {
    if (form == 0) f.template operator()<4, 4, 4>();
    else if (form == 1) f.template operator()<4, 8, 4>();
    else if (form == 2) f.template operator()<4, 16, 4>();
    else f.template operator()<4, 16, 8>();
}
template <typename F> void with_cols(std::integral_constant<int, 1>, int form, F f) {
    if (form == 0) f.template operator()<1, 4, 8>();
    else if (form == 1) f.template operator()<1, 4, 16>();
    else if (form == 2) f.template operator()<1, 8, 16>();
    else if (form == 3) f.template operator()<1, 16, 16>();
    else f.template operator()<1, 16, 32>();
}
// Calls f with the values at a time as a constant.
template <typename T, typename F> void with_vec(int vec, F f) {
    if constexpr (sizeof(T) == 2)
        if (vec == 8) return f(std::integral_constant<int, 8>{});
    if (vec == 4) f(std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 1>{});
}

inline NormPlan plan_norm(const NormArgs& a, int dtype) {
    NormPlan p{};
    const int64_t inner = a.P > 1 ? a.P : a.C;
    const int most = dtype == TCONV_F32 ? 4 : 8;
    p.vec = inner % most == 0 ? most : a.P > 1 && inner % 4 == 0 ? 4 : 1;
    p.form = -1;
    if (a.P == 1) {
        const int least = p.vec > 1 ? 32 * p.vec : 256;
        for (int k = 0; p.form < 0 && (least << k) <= 1024; ++k)
            if (a.C <= least << k) p.form = k;
        p.blocks = (a.N + 3) / 4 < 148 * 2 ? (a.N + 3) / 4 : 148 * 2;
        const int across = (a.C + 128 * p.vec - 1) / (128 * p.vec), splits = (148 * 8 + across - 1) / across;
        p.parts = p.form >= 0 ? p.blocks : a.N < splits ? a.N : splits;
        return p;
    }
    int warps = 8;                   // of the kernel in groups
    const auto take = [&](auto v) {
        for (int k = decltype(v)::value == 1 ? 4 : 3; k >= 0; --k)
            with_cols(v, k, [&]<int V, int WARPS, int R>() {
                if (a.C > V * WARPS * R) return;
                p.form = k;
                warps = WARPS;
            });
    };
    if ((int64_t)a.C * a.P < (int64_t)1 << 30) {       // (offsets inside an image: 32 bits, in bytes)
        if (p.vec == 8) take(std::integral_constant<int, 8>{});
        else if (p.vec == 4) take(std::integral_constant<int, 4>{});
        else take(std::integral_constant<int, 1>{});
    }
    const int64_t tiles = q8_blocks(a.P) * a.N, resident = 148 * norm_resident(warps);
    p.parts = p.blocks = (int)(tiles < resident ? tiles : resident);
    return p;
}

}  // namespace tconv
