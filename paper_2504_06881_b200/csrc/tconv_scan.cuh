// Gated linear recurrence (tconv.h): h_t = f_t h_{t-1} + (1 - f_t) x_t along the rows of [N][C][L], and its gradient.
//
// A stretch of positions maps the state in front of it to the one behind it by h -> P h + B (P the product of its f,
// B what it makes of a zero state), and two stretches join to (P2 P1, P2 B1 + B2): a thread reduces 8 positions, a warp joins
// its 32 threads' pairs by shuffles (a chunk of 256 positions), then every thread runs its 8 positions once more from its true
// state.  Rows go to warps; where there are fewer rows than keep the GPU busy, a block's warps take a row's chunks in turn and
// hand the state round, and where there are very few a first kernel joins the maps of parts of a row.
// HBM would be the bound (6 bytes a position forward in bf16, 10 backward), but at some 25 and 40 instructions a position
// the issue slots are nearly as short, so that what is not arithmetic is kept out of the whole chunks' way.
#pragma once
#include "tconv_q8.cuh"

namespace tconv {

constexpr int kScanVec = 8;          // positions per thread: 16 bytes of bf16
constexpr int kScanChunk = 256;      // positions per warp and step; between two saved states
constexpr int kScanWarps = 8;        // most warps of a block on one row
constexpr int kScanParts = 256;      // most parts of a row

// How a thread's positions are read and written: whole vectors where every row starts on 16 bytes; else lane by lane
// through shared memory (8 positions a thread, straight, would touch every sector eight times), straight for short rows.
enum ScanAccess { kVector, kStaged, kStraight };

struct ScanArgs {
    int64_t rows;
    uint32_t L, chunks, per_part;    // chunks of a row, and of a part
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
// e^-g as 2^(-g log2 e), held to 2^115 (a lesser f adds nothing to a sum in fp32), so that u = e^-g * f stays finite; NaN passes.
__device__ __forceinline__ Gate gate_of(float g) {
    float m, e, f;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(g * -1.4426950408889634f), "f"(115.0f));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(m));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(f) : "f"(1.0f + e));
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
            constexpr int kStride = ACC == kStaged ? 32 : 1;
            const uint32_t lane = threadIdx.x & 31, first = ACC == kStaged ? at - kScanVec * lane + lane : at;
            const T* p = row + first;
            if (ACC == kStaged && first - lane + kScanChunk <= end) {       // (the same for the whole warp)
#pragma unroll
                for (int i = 0; i < kScanVec; ++i) s[i] = __ldg(p + i * kStride);
            } else {
#pragma unroll
                for (int i = 0; i < kScanVec; ++i) {
                    s[i] = zero_of<T>();
                    if (first + i * kStride < end) s[i] = __ldg(p + i * kStride);
                }
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
            T* p = row + first;
            if (first - lane + kScanChunk <= end) {
#pragma unroll
                for (int i = 0; i < kScanVec; ++i) p[32 * i] = stage[32 * i + lane];
            } else {
#pragma unroll
                for (int i = 0; i < kScanVec; ++i)
                    if (first + 32 * i < end) p[32 * i] = stage[32 * i + lane];
            }
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

// The map of the whole warp, in all lanes.
__device__ __forceinline__ Map warp_join(Map m) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Map o{__shfl_xor_sync(~0u, m.P, d), __shfl_xor_sync(~0u, m.B, d)};
        m = (threadIdx.x & d) ? then(o, m) : then(m, o);
    }
    return m;
}

// The warps of a block on one row hand their chunks' maps round; double buffered, so that one barrier a step is enough.
template <bool UP> __device__ __forceinline__ void block_carry(const Map (&shared)[kScanWarps], int warp, int warps, float c, float& mine, float& next) {
#pragma unroll
    for (int k = 0; k < kScanWarps; ++k) {
        const int w = UP ? k : kScanWarps - 1 - k;
        if (w >= warps) continue;
        if (w == warp) mine = c;
        c = apply(shared[w], c);
    }
    next = c;
}

// Who works on a row: a warp (or a part of it, or several rows a warp where G < 32), a block's warps in turn, or a warp a part
// that only leaves the part's maps.
enum ScanMode { kWarp, kBlock, kJoin };

// Where a warp works.
template <int G, int MODE> struct Place {
    int64_t row;
    uint32_t part;
    bool mine, any;                  // this lane's row exists; some row of the warp does
    __device__ __forceinline__ Place(const ScanArgs& a) {
        const int warp = threadIdx.x >> 5;
        if constexpr (MODE == kBlock) {
            row = blockIdx.x;
            part = 0;
            mine = any = true;
        } else {
            const int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + warp;
            part = G == 32 ? (uint32_t)(w % a.parts) : 0;
            row = (G == 32 ? w / a.parts : w * (32 / G)) + (threadIdx.x & 31) / G;
            mine = row < a.rows;
            any = row - (threadIdx.x & 31) / G < a.rows;
            if (!mine) row = a.rows - 1;
        }
    }
};

// Forward.
template <typename T, bool Q8, int ACC, int G, int MODE>
__global__ void __launch_bounds__(MODE == kBlock ? kScanWarps * 32 : 128) scan_fwd_kernel(const __grid_constant__ ScanArgs a,
                                                                                          const __grid_constant__ ScanFwd io) {
    constexpr int kStages = ACC == kStaged ? (MODE == kBlock ? kScanWarps : 4) : 1;
    __shared__ __align__(16) T stages[kStages][ACC == kStaged ? 2 * kScanChunk : 16];
    __shared__ Map shared[MODE == kBlock ? 2 : 1][kScanWarps], shared_q[MODE == kBlock && Q8 ? 2 : 1][kScanWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = MODE == kBlock ? blockDim.x >> 5 : 1, sub = lane % G;
    T *stage = stages[ACC == kStaged ? warp : 0], *stage_g = stage + (ACC == kStaged ? kScanChunk : 0);
    const Place<G, MODE> at_row(a);
    if (!at_row.any) return;
    const int64_t row = at_row.row, n = row / a.C, c = row - n * a.C;
    const bool mine = at_row.mine;
    const uint32_t end = mine ? row_length(a, n) : 0u, L = mine ? a.L : 0u;
    const T *px = (const T*)io.x + n * a.xb + c * a.xr, *pg = (const T*)io.gate + n * a.gb + c * a.gr;
    T* py = (T*)io.y + row * a.L;
    const uint32_t k_begin = G == 32 && MODE != kBlock ? at_row.part * a.per_part : 0;
    const uint32_t k_end = G == 32 && MODE != kBlock ? min(k_begin + a.per_part, a.chunks) : a.chunks;
    const int64_t pitch = q8_pitch(a.L), nb = q8_blocks(a.L);

    Map total{1.0f, 0.0f}, total_q = total;                   // kJoin: the part's maps so far
    float h = 0.0f, hq;
    if constexpr (MODE != kJoin) {
        if (io.h0) h = io.h0[row];
        hq = h;
        if constexpr (G == 32 && MODE == kWarp)
            for (uint32_t p = 0; p < at_row.part; p += 32) {
                float4 m = make_float4(1.0f, 0.0f, 1.0f, 0.0f);
                if (p + lane < at_row.part) m = __ldg(a.joined + row * a.parts + p + lane);
                h = apply(warp_join({m.x, m.y}), h);
                if constexpr (Q8) hq = apply(warp_join({m.z, m.w}), hq);
            }
    }
    Eight<T, ACC> rx, rg;
    uint32_t at = (k_begin + (MODE == kBlock ? warp : 0)) * kScanChunk + sub * kScanVec;
    rx.fetch(px, at, end);
    rg.fetch(pg, at, end);
    int turn = 0;
    for (uint32_t k = k_begin; k < k_end; k += warps, turn ^= 1) {
        const uint32_t here = at, chunk = k + (MODE == kBlock ? warp : 0);
        at += warps * kScanChunk;
        if (G == 32 && MODE != kBlock && k * kScanChunk >= end) {          // behind the row's length, with all that follows
            if constexpr (MODE == kJoin) break;
            else {
                const float zero[8] = {};
                put_eight<T, ACC>(py, here, L, zero, stage);
                if (io.states && sub == 0) io.states[row * a.chunks + chunk] = Q8 ? hq : h;
                if constexpr (Q8)
                    if (here < (uint32_t)pitch) {
                        *reinterpret_cast<uint2*>(io.xc + row * pitch + here) = *reinterpret_cast<uint2*>(io.gc + row * pitch + here) = make_uint2(0, 0);
                        if (here % kQ8Block == 0) io.xs[row * nb + here / kQ8Block] = io.gs[row * nb + here / kQ8Block] = 1;
                    }
                continue;
            }
        }
        float x[8], g[8], f[8], b[8];
        rx.take(x, stage);
        rg.take(g, stage_g);
        if (G == 32 && k + warps < k_end) {                   // the next chunk is on its way while this one is worked on
            rx.fetch(px, at, end);
            rg.fetch(pg, at, end);
        }
        const int live = end <= here ? 0 : (int)min(end - here, (uint32_t)kScanVec);
        if constexpr (Q8 && ACC == kVector) {                 // what a vector holds behind the row's length is no part of a block
            if (live < 8)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= live) x[i] = g[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Gate q = gate_of(g[i]);
            f[i] = q.f;
            b[i] = __fmul_rn(q.u, x[i]);
        }
        if (live < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= live) { f[i] = 1.0f; b[i] = 0.0f; }
        }
        Map m{f[0], b[0]};
#pragma unroll
        for (int i = 1; i < 8; ++i) m = then(m, {f[i], b[i]});
        Map all, all_q, before;
        if constexpr (MODE == kJoin) all = warp_join(m);
        else {
            before = before_me<G, true>(m, all);
            all = of_last<G, true>(all);
        }
        if constexpr (Q8) {
            const uint32_t bx = block_scale<G>(x), bg = block_scale<G>(g);
            const uint2 cx = encode_eight(x, bx), cg = encode_eight(g, bg);
            if constexpr (MODE != kJoin) {
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
            if (live == 8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const Gate q = gate_of(g[i]);
                    mq = then(mq, {q.f, __fmul_rn(q.u, x[i])});
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const Gate q = gate_of(g[i]);
                    if (i < live) mq = then(mq, {q.f, __fmul_rn(q.u, x[i])});
                }
            }
            if constexpr (G == 32) all_q = warp_join(mq);
            else {
                before_me<G, true>(mq, all_q);
                all_q = of_last<G, true>(all_q);
            }
        }
        if constexpr (MODE == kJoin) {
            total = then(total, all);
            if constexpr (Q8) total_q = then(total_q, all_q);
        } else {
            float start = h, start_q = hq;
            if constexpr (MODE == kBlock) {
                if (lane == 0) {
                    shared[turn][warp] = all;
                    if constexpr (Q8) shared_q[turn][warp] = all_q;
                }
                __syncthreads();
                block_carry<true>(shared[turn], warp, warps, h, start, h);
                if constexpr (Q8) block_carry<true>(shared_q[turn], warp, warps, hq, start_q, hq);
            } else {
                h = apply(all, h);
                if constexpr (Q8) hq = apply(all_q, hq);
            }
            if (io.states && mine && sub == 0 && chunk < a.chunks) io.states[row * a.chunks + chunk] = Q8 ? start_q : start;
            float v = apply(before, start);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v = fmaf(f[i], v, b[i]);
                y[i] = v;
            }
            if (live < 8) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= live) y[i] = 0.0f;
            }
            put_eight<T, ACC>(py, here, L, y, stage);
        }
    }
    if constexpr (MODE == kJoin) {
        if (lane == 0) a.joined[row * a.parts + at_row.part] = make_float4(total.P, total.B, total_q.P, total_q.B);
    } else {
        if (mine && (MODE == kBlock ? threadIdx.x == 0 : sub == 0) && k_end == a.chunks) io.h_last[row] = h;
    }
}

// Backward, from a row's end to its front: with E_t = f_t D_t, D_t = dy_t + E_{t+1}, a stretch maps the E behind it to the one in
// front of it, E -> P E + Q, by the same P.  The states of the chunks make the recomputed h of a chunk its own affair.
template <typename T, bool Q8, int ACC, int G, int MODE>
__global__ void __launch_bounds__(MODE == kBlock ? kScanWarps * 32 : 128) scan_bwd_kernel(const __grid_constant__ ScanArgs a,
                                                                                          const __grid_constant__ ScanBwd io) {
    constexpr int kStages = ACC == kStaged ? (MODE == kBlock ? kScanWarps : 4) : 1;
    __shared__ __align__(16) T stages[kStages][ACC == kStaged ? 3 * kScanChunk : 16];
    __shared__ Map shared[MODE == kBlock ? 2 : 1][kScanWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = MODE == kBlock ? blockDim.x >> 5 : 1, sub = lane % G;
    constexpr int kOff = ACC == kStaged ? kScanChunk : 0;
    T* stage = stages[ACC == kStaged ? warp : 0];
    const Place<G, MODE> at_row(a);
    if (!at_row.any) return;
    const int64_t row = at_row.row, n = row / a.C, c = row - n * a.C;
    const bool mine = at_row.mine;
    const uint32_t end = mine ? row_length(a, n) : 0u, L = mine ? a.L : 0u;
    const T *px = (const T*)io.x + n * a.xb + c * a.xr, *pg = (const T*)io.gate + n * a.gb + c * a.gr, *py = (const T*)io.gy + row * a.L;
    T *ox = (T*)io.gx + n * a.ob + c * (int64_t)a.L, *og = (T*)io.gg + n * a.ob + c * (int64_t)a.L;
    const uint32_t k_begin = G == 32 && MODE != kBlock ? at_row.part * a.per_part : 0;
    const uint32_t k_end = G == 32 && MODE != kBlock ? min(k_begin + a.per_part, a.chunks) : a.chunks;
    const int64_t pitch = q8_pitch(a.L), nb = q8_blocks(a.L);
    const int8_t *xc = io.xc + row * pitch, *gc = io.gc + row * pitch;
    const uint8_t *xs = io.xs + row * nb, *gs = io.gs + row * nb;

    Map total{1.0f, 0.0f};
    float E = 0.0f;
    if constexpr (MODE != kJoin) {
        if (io.gh) E = io.gh[row];
        if constexpr (G == 32 && MODE == kWarp)               // the parts behind this one, from the last on
            for (int p = a.parts - 1; p > (int)at_row.part; p -= 32) {
                float4 m = make_float4(1.0f, 0.0f, 1.0f, 0.0f);
                if (p - lane > (int)at_row.part) m = __ldg(a.joined + row * a.parts + p - lane);
                E = apply(warp_join({m.x, m.y}), E);
            }
    }
    Eight<T, ACC> rx, rg, ry;
    uint2 cx, cg;
    uint32_t bx, bg;
    float state;
    const auto fetch = [&](uint32_t k) {
        const uint32_t chunk = k + (MODE == kBlock ? warp : 0), at = chunk * kScanChunk + sub * kScanVec;
        ry.fetch(py, at, end);
        if constexpr (Q8) {
            cx = cg = make_uint2(0, 0);
            bx = bg = 1;
            if (at < end) {
                cg = __ldg(reinterpret_cast<const uint2*>(gc + at));
                bg = __ldg(gs + at / kQ8Block);
                if (MODE != kJoin) {
                    cx = __ldg(reinterpret_cast<const uint2*>(xc + at));
                    bx = __ldg(xs + at / kQ8Block);
                }
            }
        } else {
            rg.fetch(pg, at, end);
            if (MODE != kJoin) rx.fetch(px, at, end);
        }
        if (MODE != kJoin) state = chunk < a.chunks ? __ldg(io.states + row * a.chunks + chunk) : 0.0f;
    };
    uint32_t steps = (k_end - k_begin + warps - 1) / warps;
    if (G == 32 && MODE != kBlock) {                          // chunks behind the row's length
        for (; steps && (k_begin + steps - 1) * kScanChunk >= end; --steps) {
            if constexpr (MODE != kJoin) {
                const uint32_t here = (k_begin + steps - 1) * kScanChunk + sub * kScanVec;
                const float zero[8] = {};
                put_eight<T, ACC>(ox, here, L, zero, stage);
                put_eight<T, ACC>(og, here, L, zero, stage + kOff);
            }
        }
    }
    if (steps) fetch(k_begin + (steps - 1) * warps);
    int turn = 0;
    for (; steps; --steps, turn ^= 1) {
        const uint32_t here = (k_begin + (steps - 1) * warps + (MODE == kBlock ? warp : 0)) * kScanChunk + sub * kScanVec;
        float x[8], g[8], d[8], f[8], u[8];
        ry.take(d, stage);
        if constexpr (Q8) {
            decode_eight(cg, bg, g);
            if (MODE != kJoin) decode_eight(cx, bx, x);
        } else {
            rg.take(g, stage + kOff);
            if (MODE != kJoin) rx.take(x, stage + 2 * kOff);
        }
        const float first = state;
        if (G == 32 && steps > 1) fetch(k_begin + (steps - 2) * warps);
        const int live = end <= here ? 0 : (int)min(end - here, (uint32_t)kScanVec);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Gate q = gate_of(g[i]);
            f[i] = q.f;
            u[i] = q.u;
        }
        if (live < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= live) { f[i] = 1.0f; u[i] = 0.0f; x[i] = 0.0f; d[i] = 0.0f; }
        }
        Map back{f[7], __fmul_rn(f[7], d[7])}, all;
#pragma unroll
        for (int i = 6; i >= 0; --i) back = {back.P * f[i], __fmul_rn(f[i], __fadd_rn(d[i], back.B))};
        if constexpr (MODE == kJoin) {
            // (from the end of the row on: the maps of later lanes come first)
            const Map mirrored{__shfl_sync(~0u, back.P, 31 - lane), __shfl_sync(~0u, back.B, 31 - lane)};
            total = then(total, warp_join(mirrored));
        } else {
            float b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = __fmul_rn(u[i], x[i]);
            Map m{f[0], b[0]}, unused;
#pragma unroll
            for (int i = 1; i < 8; ++i) m = then(m, {f[i], b[i]});
            const Map behind = before_me<G, false>(back, all), before = before_me<G, true>(m, unused);
            all = of_last<G, false>(all);
            float start = E;
            if constexpr (MODE == kBlock) {
                if (lane == 0) shared[turn][warp] = all;
                __syncthreads();
                block_carry<false>(shared[turn], warp, warps, E, start, E);
            } else E = apply(all, E);
            float v = apply(before, first), w = apply(behind, start);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float prev = v;
                v = fmaf(f[i], v, b[i]);
                b[i] = prev - x[i];
            }
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const float D = __fadd_rn(d[i], w);
                w = __fmul_rn(f[i], D);
                x[i] = __fmul_rn(u[i], D);
                g[i] = __fmul_rn(__fmul_rn(w, b[i]), u[i]);
            }
            if (live < 8) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= live) x[i] = g[i] = 0.0f;
            }
            put_eight<T, ACC>(ox, here, L, x, stage);
            put_eight<T, ACC>(og, here, L, g, stage + kOff);
        }
    }
    if constexpr (MODE == kJoin) {
        if (lane == 0) a.joined[row * a.parts + at_row.part] = make_float4(total.P, total.B, 1.0f, 0.0f);
    } else {
        if (io.gh0 && mine && (MODE == kBlock ? threadIdx.x == 0 : sub == 0) && k_begin == 0) io.gh0[row] = E;
    }
}

// How a row's positions are shared out.
struct ScanPlan {
    int g, warps, parts;             // threads of a row (1, 4, 16, 32); warps of a block on one row; parts of a row, a warp each
    uint32_t per_part;               // chunks
};

inline ScanPlan plan_scan(int64_t rows, int64_t L) {
    const int64_t chunks = (L + kScanChunk - 1) / kScanChunk;
    ScanPlan p{32, 1, 1, (uint32_t)chunks};
    if (L <= 8) p.g = 1;
    else if (L <= 32) p.g = 4;
    else if (L <= 128) p.g = 16;
    if (p.g < 32) return p;
    const int64_t enough = 148 * 16;     // warps that keep the GPU busy
    if (rows * kScanWarps >= enough || chunks < 4 * kScanWarps) {
        while (p.warps < kScanWarps && p.warps < chunks && rows * p.warps < enough) p.warps *= 2;
    } else {
        int64_t parts = 2 * enough / rows;
        if (parts > kScanParts) parts = kScanParts;
        if (parts > chunks / 2) parts = chunks / 2;
        const int64_t per = (chunks + parts - 1) / parts;
        p.per_part = (uint32_t)per;
        p.parts = (int)((chunks + per - 1) / per);
    }
    return p;
}

}  // namespace tconv
