// Gated linear recurrence (tconv.h): h_t = f_t h_{t-1} + (1 - f_t) x_t along the rows of [N][C][L], and its gradient.
//
// A stretch of positions maps the state in front of it to the one behind it by h -> P h + B (P the product of its f,
// B what it makes of a zero state), and two stretches join to (P2 P1, P2 B1 + B2): a thread reduces 8 positions, a warp joins
// its 32 threads' pairs by shuffles (a chunk of 256 positions), a block its warps' through shared memory, and blocks that
// share a row theirs in a pass of their own; then every thread runs its 8 positions once more from its true state.
// The work is bound by HBM: 6 bytes a position forward in bf16, 10 backward, for some 12 and 25 instructions.
#pragma once
#include "tconv_q8.cuh"

namespace tconv {

constexpr int kScanVec = 8;          // positions per thread: 16 bytes of bf16
constexpr int kScanChunk = 256;      // positions per warp and step; between two saved states
constexpr int kScanWarps = 8;        // most warps of a block on one row
constexpr int kScanParts = 64;       // most blocks on one row

// How a thread's positions are read and written: whole vectors where every row starts on 16 bytes; else lane by lane
// through shared memory (8 positions a thread, straight, would touch every sector eight times), straight for short rows.
enum ScanAccess { kVector, kStaged, kStraight };

struct ScanArgs {
    int64_t rows;
    uint32_t L, chunks, per_part;    // chunks of a row, and of one block's part of it (a multiple of the block's warps)
    int C, parts;
    int64_t xb, xr, gb, gr;          // strides of x and gate: batch, row
    int64_t ob;                      // batch stride of grad_x and grad_gate
    const int32_t* lengths;
    float4* joined;                  // [rows][parts]: (P, B) of each part, and those over the restored values
};

struct ScanFwd {
    const void *x, *gate;
    const float* h0;
    void* y;
    float *h_last, *states;
    int8_t *xc, *gc;
    uint8_t *xs, *gs;
};

struct ScanBwd {
    const void *x, *gate;
    const int8_t *xc, *gc;
    const uint8_t *xs, *gs;
    const float* states;
    const void* gy;
    const float* gh;
    void *gx, *gg;
    float* gh0;
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

__device__ __forceinline__ uint32_t row_length(const ScanArgs& a, int64_t n) {
    if (!a.lengths) return a.L;
    const int32_t len = a.lengths[n];
    return len < 0 ? 0u : min((uint32_t)len, a.L);
}

// ---- eight positions of a thread ----
template <typename T> struct Words { static constexpr int n = sizeof(T) * kScanVec / 16, per = 16 / sizeof(T); uint4 w[n]; };

__device__ __forceinline__ void unpack(const Words<float>& r, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        v[4 * j] = __uint_as_float(r.w[j].x); v[4 * j + 1] = __uint_as_float(r.w[j].y);
        v[4 * j + 2] = __uint_as_float(r.w[j].z); v[4 * j + 3] = __uint_as_float(r.w[j].w);
    }
}
__device__ __forceinline__ void unpack(const Words<__nv_bfloat16>& r, float (&v)[8]) {
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void pack(const float (&v)[8], Words<float>& r) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
        r.w[j] = make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
}
__device__ __forceinline__ void pack(const float (&v)[8], Words<__nv_bfloat16>& r) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&p);
    }
    r.w[0] = make_uint4(w[0], w[1], w[2], w[3]);
}

// The values of positions [at, at + 8) of a row below `end` (what a vector holds behind it is not masked).  fetch() starts the loads, take() hands them out.
// Staged: a warp's 256 positions from `chunk_at`, through its `stage` of shared memory.
template <typename T, int ACC> struct Eight {
    Words<T> r;
    T s[ACC == kVector ? 1 : kScanVec];

    __device__ __forceinline__ void fetch(const T* __restrict__ row, uint32_t at, uint32_t end) {
        if constexpr (ACC == kVector) {
#pragma unroll
            for (int j = 0; j < Words<T>::n; ++j) {
                r.w[j] = make_uint4(0, 0, 0, 0);
                if (at + j * Words<T>::per < end) r.w[j] = __ldg(reinterpret_cast<const uint4*>(row + at) + j);
            }
        } else {
            const uint32_t lane = threadIdx.x & 31;
            const uint32_t first = ACC == kStaged ? at - kScanVec * lane + lane : at;
#pragma unroll
            for (int i = 0; i < kScanVec; ++i) {
                const uint32_t p = first + i * (ACC == kStaged ? 32 : 1);
                s[i] = zero_of<T>();
                if (p < end) s[i] = __ldg(row + p);
            }
        }
    }
    __device__ __forceinline__ void take(float (&v)[8], T* stage) {
        if constexpr (ACC == kStraight) {
#pragma unroll
            for (int i = 0; i < kScanVec; ++i) v[i] = to_f32(s[i]);
        } else {
            if constexpr (ACC == kStaged) {
                const uint32_t lane = threadIdx.x & 31;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < kScanVec; ++i) stage[32 * i + lane] = s[i];
                __syncwarp();
#pragma unroll
                for (int j = 0; j < Words<T>::n; ++j) r.w[j] = reinterpret_cast<const uint4*>(stage + kScanVec * lane)[j];
            }
            unpack(r, v);
        }
    }
};

// Writes the values of positions [at, at + 8) below `end`.
template <typename T, int ACC>
__device__ __forceinline__ void put_eight(T* __restrict__ row, uint32_t at, uint32_t end, const float (&v)[8], T* stage) {
    if constexpr (ACC == kStraight) {
#pragma unroll
        for (int i = 0; i < kScanVec; ++i)
            if (at + i < end) row[at + i] = from_f32<T>(v[i]);
    } else {
        Words<T> r;
        pack(v, r);
        if constexpr (ACC == kVector) {
#pragma unroll
            for (int j = 0; j < Words<T>::n; ++j)
                if (at + j * Words<T>::per < end) reinterpret_cast<uint4*>(row + at)[j] = r.w[j];
        } else {
            const uint32_t lane = threadIdx.x & 31, first = at - kScanVec * lane + lane;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < Words<T>::n; ++j) reinterpret_cast<uint4*>(stage + kScanVec * lane)[j] = r.w[j];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kScanVec; ++i)
                if (first + 32 * i < end) row[first + 32 * i] = stage[32 * i + lane];
        }
    }
}

struct Map {
    float P, B;                      // h -> P h + B
};
__device__ __forceinline__ Map then(Map first, Map second) { return {first.P * second.P, fmaf(second.P, first.B, second.B)}; }
__device__ __forceinline__ float apply(Map m, float h) { return fmaf(m.P, h, m.B); }

// Joins the maps of the G threads of a row in order (UP: from the first thread on): a thread gets the map of all before it;
// `all` (valid in the last thread) is the whole group's.
template <int G, bool UP> __device__ __forceinline__ Map before_me(Map m, Map& all) {
    const int sub = (threadIdx.x & 31) % G, me = UP ? sub : G - 1 - sub;
#pragma unroll
    for (int d = 1; d < G; d <<= 1) {
        const Map o{UP ? __shfl_up_sync(~0u, m.P, d, G) : __shfl_down_sync(~0u, m.P, d, G),
                    UP ? __shfl_up_sync(~0u, m.B, d, G) : __shfl_down_sync(~0u, m.B, d, G)};
        if (me >= d) m = then(o, m);
    }
    all = m;
    if constexpr (G == 1) return {1.0f, 0.0f};
    const Map o{UP ? __shfl_up_sync(~0u, m.P, 1, G) : __shfl_down_sync(~0u, m.P, 1, G),
                UP ? __shfl_up_sync(~0u, m.B, 1, G) : __shfl_down_sync(~0u, m.B, 1, G)};
    return me == 0 ? Map{1.0f, 0.0f} : o;
}
template <int G, bool UP> __device__ __forceinline__ Map of_last(Map all) {
    const int src = UP ? G - 1 : 0;
    return {__shfl_sync(~0u, all.P, src, G), __shfl_sync(~0u, all.B, src, G)};
}

// The warps of a block on one row hand their chunks' maps round; double buffered, so that one barrier a step is enough.
template <bool UP> __device__ __forceinline__ void block_carry(Map chunk, Map (&shared)[kScanWarps], int warp, int warps, float c, float& mine, float& next) {
    if ((threadIdx.x & 31) == 0) shared[warp] = chunk;
    __syncthreads();
    for (int k = 0; k < warps; ++k) {
        const int w = UP ? k : warps - 1 - k;
        if (w == warp) mine = c;
        c = apply(shared[w], c);
    }
    next = c;
}

// Forward.  G threads of a row: 32, or fewer for rows of at most 8 G positions (several rows a warp).  MULTI: all warps of a
// block share a row, and gridDim.y blocks may; else a warp has rows of its own.  JOIN: only the maps of the parts.
template <typename T, bool Q8, int ACC, int G, bool MULTI, bool JOIN>
__global__ void __launch_bounds__(MULTI ? kScanWarps * 32 : 128) scan_fwd_kernel(const __grid_constant__ ScanArgs a,
                                                                                 const __grid_constant__ ScanFwd io) {
    __shared__ __align__(16) T stages[ACC == kStaged ? (MULTI ? kScanWarps : 4) : 1][ACC == kStaged ? 2 * kScanChunk : 16];
    __shared__ Map shared[2][MULTI ? kScanWarps : 1], shared_q[2][MULTI && Q8 ? kScanWarps : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = MULTI ? blockDim.x >> 5 : 1, sub = lane % G;
    T* stage = stages[ACC == kStaged ? warp : 0];
    int64_t row = MULTI ? blockIdx.x : ((int64_t)blockIdx.x * (blockDim.x >> 5) + warp) * (32 / G) + lane / G;
    const bool mine = row < a.rows;
    if constexpr (!MULTI) {
        if (row - lane / G >= a.rows) return;                 // (a whole warp)
        if (!mine) row = a.rows - 1;
    }
    const int64_t n = row / a.C, c = row - n * a.C;
    const uint32_t end = mine ? row_length(a, n) : 0u, L = mine ? a.L : 0u;
    const T *px = (const T*)io.x + n * a.xb + c * a.xr, *pg = (const T*)io.gate + n * a.gb + c * a.gr;
    T* py = (T*)io.y + row * a.L;
    const uint32_t part = MULTI ? blockIdx.y : 0, k_begin = MULTI ? part * a.per_part : 0;
    const uint32_t k_end = MULTI ? min(k_begin + a.per_part, a.chunks) : a.chunks;
    const int64_t pitch = q8_pitch(a.L), nb = q8_blocks(a.L);

    Map total{1.0f, 0.0f}, total_q = total;                   // JOIN: the part's maps so far
    float h = 0.0f, hq;
    if constexpr (!JOIN) {
        if (io.h0) h = io.h0[row];
        hq = h;
        if constexpr (MULTI)
            for (uint32_t p = 0; p < part; ++p) {
                const float4 m = __ldg(a.joined + row * a.parts + p);
                h = fmaf(m.x, h, m.y);
                if constexpr (Q8) hq = fmaf(m.z, hq, m.w);
            }
    }
    Eight<T, ACC> rx, rg;
    uint32_t at = (k_begin + (MULTI ? warp : 0)) * kScanChunk + sub * kScanVec;
    rx.fetch(px, at, end);
    rg.fetch(pg, at, end);
    int turn = 0;
    for (uint32_t k = k_begin; k < k_end; k += warps, turn ^= 1) {
        float x[8], g[8], f[8], b[8];
        rx.take(x, stage);
        rg.take(g, stage + (ACC == kStaged ? kScanChunk : 0));
        const uint32_t here = at;
        at += warps * kScanChunk;
        if (G == 32 && k + warps < k_end) {                   // the next chunk is on its way while this one is worked on
            rx.fetch(px, at, end);
            rg.fetch(pg, at, end);
        }
        const int live = end <= here ? 0 : (int)min(end - here, (uint32_t)kScanVec);
        if constexpr (Q8 && ACC == kVector) {                 // what a vector holds behind the row's length is no part of a block
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= live) x[i] = g[i] = 0.0f;
        }
        Map m{1.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Gate q = gate_of(g[i]);
            f[i] = q.f;
            b[i] = __fmul_rn(q.u, x[i]);
            if (i >= live) { f[i] = 1.0f; b[i] = 0.0f; }
            m = then(m, {f[i], b[i]});
        }
        Map all, all_q;
        const Map before = before_me<G, true>(m, all);
        if constexpr (Q8) {
            const uint32_t bx = block_scale<G>(x), bg = block_scale<G>(g);
            const uint2 cx = encode_eight(x, bx), cg = encode_eight(g, bg);
            if constexpr (!JOIN) {
                if (mine && here < (uint32_t)pitch) {
                    *reinterpret_cast<uint2*>(io.xc + row * pitch + here) = cx;
                    *reinterpret_cast<uint2*>(io.gc + row * pitch + here) = cg;
                    if (here % kQ8Block == 0) {
                        io.xs[row * nb + here / kQ8Block] = (uint8_t)bx;
                        io.gs[row * nb + here / kQ8Block] = (uint8_t)bg;
                    }
                }
            }
            Map mq{1.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const Gate q = gate_of(g[i]);
                if (i < live) mq = then(mq, {q.f, __fmul_rn(q.u, x[i])});
            }
            before_me<G, true>(mq, all_q);
            all_q = of_last<G, true>(all_q);
        }
        all = of_last<G, true>(all);
        if constexpr (JOIN) {
            if (lane == 0) { shared[turn][warp] = all; if constexpr (Q8) shared_q[turn][warp] = all_q; }
            __syncthreads();
            for (int w = 0; w < warps; ++w) {
                total = then(total, shared[turn][w]);
                if constexpr (Q8) total_q = then(total_q, shared_q[turn][w]);
            }
        } else {
            float start = h, start_q = hq;
            if constexpr (MULTI) {
                if constexpr (Q8) {
                    if (lane == 0) shared_q[turn][warp] = all_q;
                }
                block_carry<true>(all, shared[turn], warp, warps, h, start, h);
                if constexpr (Q8)
                    for (int w = 0; w < warps; ++w) {
                        if (w == warp) start_q = hq;
                        hq = apply(shared_q[turn][w], hq);
                    }
            } else {
                h = apply(all, h);
                if constexpr (Q8) hq = apply(all_q, hq);
            }
            const uint32_t chunk = k + (MULTI ? warp : 0);
            if (io.states && mine && sub == 0 && chunk < a.chunks) io.states[row * a.chunks + chunk] = Q8 ? start_q : start;
            float v = apply(before, start);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v = fmaf(f[i], v, b[i]);
                y[i] = i < live ? v : 0.0f;
            }
            put_eight<T, ACC>(py, here, L, y, stage);
        }
    }
    if constexpr (JOIN) {
        if (threadIdx.x == 0) a.joined[row * a.parts + part] = make_float4(total.P, total.B, total_q.P, total_q.B);
    } else {
        if (mine && (MULTI ? threadIdx.x == 0 : sub == 0) && k_end == a.chunks) io.h_last[row] = h;
    }
}

// Backward, from a row's end to its front: with E_t = f_t D_t, D_t = dy_t + E_{t+1}, a stretch maps the E behind it to the one in
// front of it, E -> P E + Q, by the same P.  The states of the chunks make the recomputed h of a chunk its own affair.
template <typename T, bool Q8, int ACC, int G, bool MULTI, bool JOIN>
__global__ void __launch_bounds__(MULTI ? kScanWarps * 32 : 128) scan_bwd_kernel(const __grid_constant__ ScanArgs a,
                                                                                 const __grid_constant__ ScanBwd io) {
    __shared__ __align__(16) T stages[ACC == kStaged ? (MULTI ? kScanWarps : 4) : 1][ACC == kStaged ? 3 * kScanChunk : 16];
    __shared__ Map shared[2][MULTI ? kScanWarps : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = MULTI ? blockDim.x >> 5 : 1, sub = lane % G;
    T* stage = stages[ACC == kStaged ? warp : 0];
    constexpr int kOff = ACC == kStaged ? kScanChunk : 0;
    int64_t row = MULTI ? blockIdx.x : ((int64_t)blockIdx.x * (blockDim.x >> 5) + warp) * (32 / G) + lane / G;
    const bool mine = row < a.rows;
    if constexpr (!MULTI) {
        if (row - lane / G >= a.rows) return;                 // (a whole warp)
        if (!mine) row = a.rows - 1;
    }
    const int64_t n = row / a.C, c = row - n * a.C;
    const uint32_t end = mine ? row_length(a, n) : 0u, L = mine ? a.L : 0u;
    const T *px = (const T*)io.x + n * a.xb + c * a.xr, *pg = (const T*)io.gate + n * a.gb + c * a.gr, *py = (const T*)io.gy + row * a.L;
    T *ox = (T*)io.gx + n * a.ob + c * (int64_t)a.L, *og = (T*)io.gg + n * a.ob + c * (int64_t)a.L;
    const uint32_t part = MULTI ? blockIdx.y : 0, k_begin = MULTI ? part * a.per_part : 0;
    const uint32_t k_end = MULTI ? min(k_begin + a.per_part, a.chunks) : a.chunks;
    const int64_t pitch = q8_pitch(a.L), nb = q8_blocks(a.L);
    const int8_t *xc = io.xc + row * pitch, *gc = io.gc + row * pitch;
    const uint8_t *xs = io.xs + row * nb, *gs = io.gs + row * nb;

    Map total{1.0f, 0.0f};
    float E = 0.0f;
    if constexpr (!JOIN) {
        if (io.gh) E = io.gh[row];
        if constexpr (MULTI)
            for (uint32_t p = a.parts - 1; p > part; --p) {
                const float4 m = __ldg(a.joined + row * a.parts + p);
                E = fmaf(m.x, E, m.y);
            }
    }
    Eight<T, ACC> rx, rg, ry;
    uint2 cx, cg;
    uint32_t bx, bg;
    float state;
    const auto fetch = [&](uint32_t k) {
        const uint32_t chunk = k + (MULTI ? warp : 0), at = chunk * kScanChunk + sub * kScanVec;
        ry.fetch(py, at, end);
        if constexpr (Q8) {
            cx = cg = make_uint2(0, 0);
            bx = bg = 1;
            if (at < end) {
                cg = __ldg(reinterpret_cast<const uint2*>(gc + at));
                bg = __ldg(gs + at / kQ8Block);
                if (!JOIN) {
                    cx = __ldg(reinterpret_cast<const uint2*>(xc + at));
                    bx = __ldg(xs + at / kQ8Block);
                }
            }
        } else {
            rg.fetch(pg, at, end);
            if (!JOIN) rx.fetch(px, at, end);
        }
        if (!JOIN) state = chunk < a.chunks ? __ldg(io.states + row * a.chunks + chunk) : 0.0f;
    };
    uint32_t steps = (k_end - k_begin + warps - 1) / warps;
    fetch(k_begin + (steps - 1) * warps);
    int turn = 0;
    for (; steps; --steps, turn ^= 1) {
        const uint32_t here = (k_begin + (steps - 1) * warps + (MULTI ? warp : 0)) * kScanChunk + sub * kScanVec;
        float x[8], g[8], d[8], f[8], u[8];
        ry.take(d, stage);
        if constexpr (Q8) {
            decode_eight(cg, bg, g);
            if (!JOIN) decode_eight(cx, bx, x);
        } else {
            rg.take(g, stage + kOff);
            if (!JOIN) rx.take(x, stage + 2 * kOff);
        }
        const float first = state;
        if (G == 32 && steps > 1) fetch(k_begin + (steps - 2) * warps);
        const int live = end <= here ? 0 : (int)min(end - here, (uint32_t)kScanVec);
        Map m{1.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Gate q = gate_of(g[i]);
            f[i] = q.f;
            u[i] = q.u;
            if (i >= live) { f[i] = 1.0f; u[i] = 0.0f; x[i] = 0.0f; d[i] = 0.0f; }
            if (!JOIN) m = then(m, {f[i], __fmul_rn(u[i], x[i])});
        }
        Map back{1.0f, 0.0f}, all;
#pragma unroll
        for (int i = 7; i >= 0; --i) back = {back.P * f[i], __fmul_rn(f[i], __fadd_rn(d[i], back.B))};
        const Map behind = before_me<G, false>(back, all);
        all = of_last<G, false>(all);
        if constexpr (JOIN) {
            if (lane == 0) shared[turn][warp] = all;
            __syncthreads();
            for (int w = warps - 1; w >= 0; --w) total = then(total, shared[turn][w]);
        } else {
            Map unused;
            const Map before = before_me<G, true>(m, unused);
            float start = E;
            if constexpr (MULTI) block_carry<false>(all, shared[turn], warp, warps, E, start, E);
            else E = apply(all, E);
            float v = apply(before, first), w = apply(behind, start);
            float prev[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                prev[i] = v;
                v = fmaf(f[i], v, __fmul_rn(u[i], x[i]));
            }
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const float D = __fadd_rn(d[i], w);
                w = __fmul_rn(f[i], D);
                g[i] = i < live ? D * (prev[i] - x[i]) * __fmul_rn(f[i], u[i]) : 0.0f;
                x[i] = i < live ? __fmul_rn(u[i], D) : 0.0f;
            }
            put_eight<T, ACC>(ox, here, L, x, stage);
            put_eight<T, ACC>(og, here, L, g, stage + kOff);
        }
    }
    if constexpr (JOIN) {
        if (threadIdx.x == 0) a.joined[row * a.parts + part] = make_float4(total.P, total.B, 0.0f, 0.0f);
    } else {
        if (io.gh0 && mine && (MULTI ? threadIdx.x == 0 : sub == 0) && k_begin == 0) io.gh0[row] = E;
    }
}

// How a row's positions are shared out.
struct ScanPlan {
    int g, warps, parts;             // threads of a row (1, 4, 16, 32); warps of a block on one row (1: one row each); blocks on one row
    uint32_t per_part;               // chunks
};

inline ScanPlan plan_scan(int64_t rows, int64_t L) {
    const int64_t chunks = (L + kScanChunk - 1) / kScanChunk;
    ScanPlan p{32, 1, 1, (uint32_t)chunks};
    if (L <= 8) p.g = 1;
    else if (L <= 32) p.g = 4;
    else if (L <= 128) p.g = 16;
    if (p.g < 32) return p;
    const int64_t enough = 148 * 16;     // warps that keep the memory busy
    while (p.warps < kScanWarps && p.warps < chunks && rows * p.warps < enough) p.warps *= 2;
    if (p.warps > 1 && rows * p.warps < enough) {
        int64_t parts = (2 * enough + rows * p.warps - 1) / (rows * p.warps);
        const int64_t steps = (chunks + p.warps - 1) / p.warps;
        if (parts > kScanParts) parts = kScanParts;
        if (parts > steps / 2) parts = steps / 2;
        if (parts > 1) {
            const int64_t per = (steps + parts - 1) / parts;
            p.per_part = (uint32_t)(per * p.warps);
            p.parts = (int)((steps + per - 1) / per);
        }
    }
    return p;
}

}  // namespace tconv
