// Gated linear recurrence (tconv.h): h_t = f_t h_{t-1} + (1 - f_t) x_t along the rows of [N][C][L], and its gradient.
//
// A stretch of positions maps the state in front of it to the one behind it by h -> P h + B (P the product of its f,
// B what it makes of a zero state), and two stretches join to (P2 P1, P2 B1 + B2): a thread reduces 8 positions, a warp joins
// its 32 threads' pairs by shuffles (a chunk of 256 positions), then every thread runs its 8 positions once more from its true
// state.  Rows go to warps; where there are fewer rows than keep the GPU busy, a block's warps take a row's chunks in turn and
// hand the state round, and where there are very few a first kernel joins the maps of parts of a row.
// HBM is the bound (6 bytes a position forward in bf16, 10 backward) where rows start on 16 bytes: 64 x 256 x 8192 bf16, half of
// it live, takes 88 and 157 us, 5.8 TB/s.  At 31 and 52 instructions a position the issue slots and, for odd 16-bit rows, the
// shared-memory path are nearly as short (32 x 128 x 3981: 29 and 40 us, 3.3 and 4.1 TB/s), so that whatever is not arithmetic
// is kept out of the whole chunks' way.
#pragma once
#include "tconv_q8.cuh"

namespace tconv {

constexpr int kScanVec = 8;          // positions per thread: 16 bytes of bf16
constexpr int kScanChunk = 256;      // positions per warp and step; between two saved states
constexpr int kScanWarps = 8;        // most warps of a block on one row
constexpr int kScanParts = 256;      // most parts of a row

// How a thread's positions are read and written.  Long rows go chunk by chunk through shared memory, two chunks ahead: in whole
// 16-byte vectors where every row of every tensor starts on 16 bytes (kAligned), in words elsewhere (kWords; see Ring).  Rows of
// at most 128 positions: whole vectors (kVector), or value by value (kStraight).
enum ScanAccess { kVector, kStraight, kAligned, kWords };

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

// Two values an instruction: a thread's positions go in pairs (i, i + 4), its two halves side by side.
struct Pair {
    float lo, hi;
};
__device__ __forceinline__ unsigned long long bits(Pair a) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.lo), "f"(a.hi));
    return r;
}
__device__ __forceinline__ Pair pair(unsigned long long r) {
    Pair a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.lo), "=f"(a.hi) : "l"(r));
    return a;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return pair(r);
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)));
    return pair(r);
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
    return pair(r);
}

struct Gate {
    Pair f, u;                       // 1 / (1 + e^-g) and 1 - f
};
// With z = e^-|g| = 2^-|g log2 e|, z / (1 + z) is the smaller of f and u and 1 / (1 + z) the larger: nothing overflows, and a gate
// at an end of its type gives 0 and 1.  Subnormal z count as 0 (a gate beyond -+87.3 is fully shut or open); NaN passes.  The larger
// is formed as 1 less the smaller: 1 + z is rounded twice as coarsely as what lies below 1, and a gate that hardly decays has
// every step of that come back over 1 / u positions.  Against 1 / (1 + e^-g) with e^-g held to 2^115, and u = e^-g f, this costs two
// to three instructions a gate: nothing where memory bounds, 33 -> 37 us forward where there are two gates a position and half the
// bytes (32 x 128 x 4000 bf16 kept in 8 bits).  By a sign on z and packed sums in place of the selects 36 us there, but 18 for 16
// in parts of a long row; by a Newton step on both packed sides 164 us for 157 backward in 64 x 256 x 8192.
__device__ __forceinline__ Gate gate_of(Pair g) {
    const Pair t = mul2(g, {1.4426950408889634f, 1.4426950408889634f});
    Pair z, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(z.lo) : "f"(-fabsf(t.lo)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(z.hi) : "f"(-fabsf(t.hi)));
    const Pair d = add2(z, {1.0f, 1.0f});
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.lo) : "f"(d.lo));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.hi) : "f"(d.hi));
    const Pair small = mul2(z, r), large = fma2(small, {-1.0f, -1.0f}, {1.0f, 1.0f});
    const bool lo = g.lo < 0.0f, hi = g.hi < 0.0f;
    return {{lo ? small.lo : large.lo, hi ? small.hi : large.hi}, {lo ? large.lo : small.lo, hi ? large.hi : small.hi}};
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

// The values of positions [at, at + 8) of a row below `end` (what a vector holds behind it is not masked).
template <typename T, int ACC> __device__ __forceinline__ void get_eight(const T* __restrict__ row, uint32_t at, uint32_t end, float (&v)[8]) {
    if constexpr (ACC == kVector) {
        Words<T> r;
#pragma unroll
        for (int j = 0; j < Words<T>::n; ++j) {
            r.w[j] = make_uint4(0, 0, 0, 0);
            if (at + j * Words<T>::per < end) r.w[j] = __ldg(reinterpret_cast<const uint4*>(row + at) + j);
        }
        unpack(r, v);
    } else {
        T s[8];
#pragma unroll
        for (int i = 0; i < kScanVec; ++i) {
            s[i] = zero_of<T>();
            if (at + i < end) s[i] = __ldg(row + at + i);
        }
#pragma unroll
        for (int i = 0; i < kScanVec; ++i) v[i] = to_f32(s[i]);
    }
}
template <typename T, int ACC> __device__ __forceinline__ void put_eight(T* __restrict__ row, uint32_t at, uint32_t end, const float (&v)[8]) {
    if constexpr (ACC == kVector) {
        Words<T> r;
        pack(v, r);
#pragma unroll
        for (int j = 0; j < Words<T>::n; ++j)
            if (at + j * Words<T>::per < end) reinterpret_cast<uint4*>(row + at)[j] = r.w[j];
    } else {
#pragma unroll
        for (int i = 0; i < kScanVec; ++i)
            if (at + i < end) row[at + i] = from_f32<T>(v[i]);
    }
}

// A warp's chunks of one row on their way through shared memory.  kWords: copied word by word from the one that holds the first
// value on, so that only the half word of a 16-bit row with an odd start is left to be shifted out (its first word starts in
// front of the chunk, its last one is copied up to the chunk's end).
template <typename T, int ACC> struct Ring {
    static constexpr bool kVec = ACC == kAligned;
    static constexpr int kBytes = kScanChunk * (int)sizeof(T), kSlot = kBytes + 16, kSlots = 2, kUnit = kVec ? 16 : 4;
    const char* next;                // this lane's place in the next chunk to be copied
    uint32_t slots;                  // shared address of slot 0
    uint32_t odd;                    // 16, or 0: bits to be shifted out

    __device__ __forceinline__ Ring(const T* row, uint32_t chunk, const char* to) {
        const uint32_t at = (uint32_t)reinterpret_cast<uintptr_t>(row) & (kUnit - 1);
        odd = !kVec && sizeof(T) == 2 ? at * 8 : 0;
        next = reinterpret_cast<const char*>(row) - (sizeof(T) == 2 && !kVec ? at : 0) + (int64_t)chunk * kBytes + kUnit * (threadIdx.x & 31);
        slots = (uint32_t)__cvta_generic_to_shared(to);
    }
    __device__ __forceinline__ static void copy(uint32_t to, const char* src, uint32_t bytes) {
        if constexpr (kVec) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(src), "r"(bytes) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(src), "r"(bytes) : "memory");
    }
    __device__ __forceinline__ static void copy(uint32_t to, const char* src) {
        if constexpr (kVec) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(src) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(src) : "memory");
    }
    __device__ __forceinline__ void move(int64_t bytes) { next += bytes; }
    // Starts the copies of the chunk that `next` is at, all of it (WHOLE) or its first `count` values with zeros behind them.
    template <bool WHOLE> __device__ __forceinline__ void fetch(int slot, uint32_t count = kScanChunk) const {
        const uint32_t lane = threadIdx.x & 31, to = slots + slot * kSlot + kUnit * lane;
        if constexpr (WHOLE) {
#pragma unroll
            for (int j = 0; j < kBytes / (32 * kUnit); ++j) copy(to + 32 * kUnit * j, next + 32 * kUnit * j);
            if (odd && lane == 0) copy(to + kBytes, next + kBytes, 2);
        } else {
            const uint32_t left = count * (uint32_t)sizeof(T) + odd / 8;
            const char* start = next - kUnit * lane;
#pragma unroll
            for (int j = 0; j < kBytes / (32 * kUnit); ++j) {
                const uint32_t b = kUnit * lane + 32 * kUnit * j, n = b < left ? min(left - b, (uint32_t)kUnit) : 0;
                copy(to + 32 * kUnit * j, n ? start + b : start, n);
            }
            if (lane == 0) {
                const uint32_t n = kBytes < left ? left - kBytes : 0;
                if (odd) copy(to + kBytes, n ? start + kBytes : start, n);
            }
        }
    }
    // This lane's eight values of a chunk that has arrived.
    __device__ __forceinline__ void take(int slot, float (&v)[8]) const {
        const uint32_t from = slots + slot * kSlot + (threadIdx.x & 31) * kScanVec * (uint32_t)sizeof(T);
        Words<T> r;
#pragma unroll
        for (int j = 0; j < Words<T>::n; ++j)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[j].x), "=r"(r.w[j].y), "=r"(r.w[j].z), "=r"(r.w[j].w) : "r"(from + 16 * j) : "memory");
        if constexpr (!kVec && sizeof(T) == 2) {
            uint32_t last;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(last) : "r"(from + 16) : "memory");
            uint4& w = r.w[0];
            w = make_uint4(__funnelshift_r(w.x, w.y, odd), __funnelshift_r(w.y, w.z, odd), __funnelshift_r(w.z, w.w, odd), __funnelshift_r(w.w, last, odd));
        }
        unpack(r, v);
    }
};
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void ring_wait() {      // all but the newest group are there
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncwarp();
}

// Writes a thread's eight values to an address of whole vectors.  fp32: as 32 bytes where they start on 32, since two stores of 16
// would each reach half of every sector.
template <typename T> __device__ __forceinline__ void put_words(T* to, const Words<T>& r) {
    if constexpr (sizeof(T) == 4) {
        if ((reinterpret_cast<uintptr_t>(to) & 31) == 0) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(r.w[0].x), "r"(r.w[0].y), "r"(r.w[0].z),
                         "r"(r.w[0].w), "r"(r.w[1].x), "r"(r.w[1].y), "r"(r.w[1].z), "r"(r.w[1].w) : "memory");
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < Words<T>::n; ++j) reinterpret_cast<uint4*>(to)[j] = r.w[j];
}

// Four words from word S of w on, shifted down by `bits` (0 or 16) across them.
template <int S> __device__ __forceinline__ uint4 four_words(const uint32_t (&w)[8], uint32_t bits) {
    return make_uint4(__funnelshift_r(w[S], w[S + 1], bits), __funnelshift_r(w[S + 1], w[S + 2], bits),
                      __funnelshift_r(w[S + 2], w[S + 3], bits), __funnelshift_r(w[S + 3], w[S + 4], bits));
}
// 16 bytes that start `shift` bytes (even, 2 to 14; the same in the whole warp) into the 32 of lo and hi.
__device__ __forceinline__ uint4 across(uint4 lo, uint4 hi, uint32_t shift) {
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, bits = (shift & 2) * 8;
    if (shift < 8) return shift < 4 ? four_words<0>(w, bits) : four_words<1>(w, bits);
    return shift < 12 ? four_words<2>(w, bits) : four_words<3>(w, bits);
}

// Writes a warp's chunk at `to`, all of it (WHOLE) or its first `count` values.  16-bit rows that do not start on 16 bytes: in whole
// vectors, put together from two threads' in `stage`, and what is left of the first and the last (16 bytes in all) value by
// value.  fp32 rows: word by word, a lane next to the other.
template <typename T, int ACC, bool WHOLE>
__device__ __forceinline__ void put_chunk(T* __restrict__ to, uint32_t count, const float (&v)[8], char* stage) {
    const uint32_t lane = threadIdx.x & 31;
    Words<T> r;
    pack(v, r);
    if constexpr (ACC == kAligned) {
        if constexpr (WHOLE) put_words(to + kScanVec * lane, r);
        else
#pragma unroll
            for (int j = 0; j < Words<T>::n; ++j)
                if (kScanVec * lane + j * Words<T>::per < count) reinterpret_cast<uint4*>(to)[Words<T>::n * lane + j] = r.w[j];
        return;
    }
    const T* values = reinterpret_cast<const T*>(stage);
    const uint32_t at = ((uint32_t)reinterpret_cast<uintptr_t>(to) & 15) / (uint32_t)sizeof(T);      // values into a vector
    if (WHOLE && at == 0) {
        put_words(to + kScanVec * lane, r);
        return;
    }
    __syncwarp();
#pragma unroll
    for (int j = 0; j < Words<T>::n; ++j) reinterpret_cast<uint4*>(stage)[Words<T>::n * lane + j] = r.w[j];
    __syncwarp();
    if constexpr (WHOLE && sizeof(T) == 2) {
        const uint4 w = across(reinterpret_cast<const uint4*>(stage)[lane ? lane - 1 : 0], r.w[0], 16 - 2 * at);
        if (lane) reinterpret_cast<uint4*>(to - at)[lane] = w;
        const uint32_t e = lane + at < kScanVec ? lane : kScanChunk - kScanVec + lane;
        if (lane < kScanVec) to[e] = values[e];
    } else {
        const T* from = values + lane;
        T* p = to + lane;
#pragma unroll
        for (int i = 0; i < kScanVec; ++i)
            if (WHOLE || 32 * i + lane < count) p[32 * i] = from[32 * i];
    }
}

struct Map {
    float P, B;                      // h -> P h + B
};
__device__ __forceinline__ Map then(Map first, Map second) { return {first.P * second.P, fmaf(second.P, first.B, second.B)}; }
__device__ __forceinline__ float apply(Map m, float h) { return fmaf(m.P, h, m.B); }
struct Halves {
    Map lo, hi;                      // of a thread's first and last four positions
};
__device__ __forceinline__ Halves chain(const Pair (&f)[4], const Pair (&b)[4]) {
    Pair P = f[0], B = b[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        B = fma2(f[i], B, b[i]);
        P = mul2(P, f[i]);
    }
    return {{P.lo, B.lo}, {P.hi, B.hi}};
}

// Joins the maps of the G threads of a row in order (UP: from the first thread on): a thread gets the map of all before it;
// `all` (valid in the last thread) is the whole group's.  The shuffle's own predicate says whether there is a thread that far.
template <int G, bool UP> __device__ __forceinline__ Map before_me(Map m, Map& all) {
    constexpr int kBounds = ((32 - G) << 8) | (UP ? 0 : G - 1);
#pragma unroll
    for (int d = 1; d < G; d <<= 1) {
        if constexpr (UP)
            asm volatile("{.reg .pred p; .reg .f32 a, b;\n\tshfl.sync.up.b32 b|p, %1, %2, %3, 0xffffffff;\n\tshfl.sync.up.b32 a, %0, %2, %3, 0xffffffff;\n\t"
                         "@p fma.rn.f32 %1, %0, b, %1;\n\t@p mul.rn.f32 %0, %0, a;}" : "+f"(m.P), "+f"(m.B) : "r"(d), "n"(kBounds));
        else
            asm volatile("{.reg .pred p; .reg .f32 a, b;\n\tshfl.sync.down.b32 b|p, %1, %2, %3, 0xffffffff;\n\tshfl.sync.down.b32 a, %0, %2, %3, 0xffffffff;\n\t"
                         "@p fma.rn.f32 %1, %0, b, %1;\n\t@p mul.rn.f32 %0, %0, a;}" : "+f"(m.P), "+f"(m.B) : "r"(d), "n"(kBounds));
    }
    all = m;
    if constexpr (G == 1) return {1.0f, 0.0f};
    Map o;
    if constexpr (UP)
        asm volatile("{.reg .pred p;\n\tshfl.sync.up.b32 %0|p, %2, 1, %4, 0xffffffff;\n\tshfl.sync.up.b32 %1, %3, 1, %4, 0xffffffff;\n\t"
                     "@!p mov.f32 %0, 0f3f800000;\n\t@!p mov.f32 %1, 0f00000000;}" : "=&f"(o.P), "=&f"(o.B) : "f"(m.P), "f"(m.B), "n"(kBounds));
    else
        asm volatile("{.reg .pred p;\n\tshfl.sync.down.b32 %0|p, %2, 1, %4, 0xffffffff;\n\tshfl.sync.down.b32 %1, %3, 1, %4, 0xffffffff;\n\t"
                     "@!p mov.f32 %0, 0f3f800000;\n\t@!p mov.f32 %1, 0f00000000;}" : "=&f"(o.P), "=&f"(o.B) : "f"(m.P), "f"(m.B), "n"(kBounds));
    return o;
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

// The warp's number, in a form that the compiler knows to be the same in all lanes.
__device__ __forceinline__ int warp_of_block() { return __shfl_sync(~0u, (int)(threadIdx.x >> 5), 0); }

// Where a warp works.
template <int G, int MODE> struct Place {
    int64_t row;
    uint32_t part;
    bool mine, any;                  // this lane's row exists; some row of the warp does
    __device__ __forceinline__ Place(const ScanArgs& a) {
        const int warp = warp_of_block();
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

// Shared memory of a warp: rings, and a chunk to be written.
template <typename T, int ACC> __host__ __device__ constexpr int scan_space(int rings, bool writes) {
    return rings * Ring<T, ACC>::kSlots * Ring<T, ACC>::kSlot + (writes && ACC == kWords ? Ring<T, ACC>::kBytes : 0);
}

// Forward.
template <typename T, bool Q8, int ACC, int G, int MODE>
__global__ void __launch_bounds__(MODE == kBlock ? kScanWarps * 32 : 128, MODE == kWarp && G == 32 ? 7 : 1)
scan_fwd_kernel(const __grid_constant__ ScanArgs a,
                                                                                          const __grid_constant__ ScanFwd io) {
    extern __shared__ __align__(16) char ring_space[];        // a warp's: slots of x, of gate, and a chunk to be written
    __shared__ Map shared[MODE == kBlock ? 2 : 1][kScanWarps], shared_q[MODE == kBlock && Q8 ? 2 : 1][kScanWarps];
    constexpr bool kChunks = ACC == kAligned || ACC == kWords;
    const int lane = threadIdx.x & 31, warp = warp_of_block(), warps = MODE == kBlock ? blockDim.x >> 5 : 1, sub = lane % G;
    const Place<G, MODE> at_row(a);
    if (!at_row.any) return;
    const int64_t row = at_row.row, n = row / a.C, c = row - n * a.C;
    const bool mine = at_row.mine;
    const uint32_t length = mine ? row_length(a, n) : 0u, L = mine ? a.L : 0u;
    const uint32_t end = G == 32 ? __shfl_sync(~0u, length, 0) : length;      // (known to be the same in all lanes)
    const T *px = (const T*)io.x + n * a.xb + c * a.xr, *pg = (const T*)io.gate + n * a.gb + c * a.gr;
    T* py = (T*)io.y + row * a.L;
    const uint32_t k_begin = G == 32 && MODE != kBlock ? at_row.part * a.per_part : 0;
    const uint32_t k_end = G == 32 && MODE != kBlock ? min(k_begin + a.per_part, a.chunks) : a.chunks;
    const uint32_t pitch = (uint32_t)q8_pitch(a.L);
    const int64_t codes_at = row * pitch, scales_at = row * q8_blocks(a.L);
    float* states = io.states ? io.states + row * a.chunks : nullptr;

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
    using R = Ring<T, ACC>;
    char* space = ring_space + (kChunks ? warp * scan_space<T, ACC>(2, MODE != kJoin) : 0);
    const uint32_t mine_first = k_begin + (MODE == kBlock ? warp : 0);
    R rx(px, mine_first, space), rg(pg, mine_first, space + R::kSlots * R::kSlot);
    char* stage = space + 2 * R::kSlots * R::kSlot;
    // chunks of which every position is to be read; of which some are
    const uint32_t whole = end / kScanChunk, some = (end + kScanChunk - 1) / kScanChunk;
    const auto fetch = [&](uint32_t k, int slot) {            // (k goes up by `warps` from call to call)
        const uint32_t chunk = k + (MODE == kBlock ? warp : 0);
        if (k < k_end) {
            if (chunk < whole) {
                rx.template fetch<true>(slot);
                rg.template fetch<true>(slot);
            } else if (chunk < some) {
                rx.template fetch<false>(slot, end - chunk * kScanChunk);
                rg.template fetch<false>(slot, end - chunk * kScanChunk);
            }
            rx.move((int64_t)warps * R::kBytes);
            rg.move((int64_t)warps * R::kBytes);
        }
        ring_commit();
    };
    int turn = 0;
    const auto step = [&]<bool WHOLE>(uint32_t k) {
        const uint32_t chunk = k + (MODE == kBlock ? warp : 0), here = chunk * kScanChunk + sub * kScanVec;
        float x[8], g[8];
        Pair f[4], b[4];
        if constexpr (kChunks) {
            ring_wait();
            rx.take(turn, x);
            rg.take(turn, g);
            __syncwarp();
            fetch(k + 2 * warps, turn);                       // two chunks ahead, into the slot just read
        } else {
            get_eight<T, ACC>(px, here, end, x);
            get_eight<T, ACC>(pg, here, end, g);
        }
        const int live = WHOLE ? 8 : end <= here ? 0 : (int)min(end - here, (uint32_t)kScanVec);
        if constexpr (Q8 && !WHOLE) {                         // what lies behind the row's length is no part of a block
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= live) x[i] = g[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Gate q = gate_of(Pair{g[i], g[i + 4]});
            f[i] = q.f;
            b[i] = mul2(q.u, {x[i], x[i + 4]});
            if (!WHOLE && i >= live) { f[i].lo = 1.0f; b[i].lo = 0.0f; }
            if (!WHOLE && i + 4 >= live) { f[i].hi = 1.0f; b[i].hi = 0.0f; }
        }
        const Halves halves = chain(f, b);
        const Map m = then(halves.lo, halves.hi);
        [[maybe_unused]] Map all, all_q, before;
        if constexpr (MODE == kJoin) all = warp_join(m);
        else {
            before = before_me<G, true>(m, all);
            all = of_last<G, true>(all);
        }
        if constexpr (Q8) {
            const uint32_t bx = block_scale<G>(x), bg = block_scale<G>(g);
            const uint2 cx = encode_eight(x, bx), cg = encode_eight(g, bg);
            if constexpr (MODE != kJoin) {
                if (WHOLE || (mine && here < pitch)) {
                    *reinterpret_cast<uint2*>(io.xc + codes_at + here) = cx;
                    *reinterpret_cast<uint2*>(io.gc + codes_at + here) = cg;
                    if (sub % 4 == 0) {
                        io.xs[scales_at + here / kQ8Block] = (uint8_t)bx;
                        io.gs[scales_at + here / kQ8Block] = (uint8_t)bg;
                    }
                }
            }
            Pair fq[4], bq[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Gate q = gate_of(Pair{g[i], g[i + 4]});
                fq[i] = q.f;
                bq[i] = mul2(q.u, {x[i], x[i + 4]});
                if (!WHOLE && i >= live) { fq[i].lo = 1.0f; bq[i].lo = 0.0f; }
                if (!WHOLE && i + 4 >= live) { fq[i].hi = 1.0f; bq[i].hi = 0.0f; }
            }
            const Halves halves_q = chain(fq, bq);
            const Map mq = then(halves_q.lo, halves_q.hi);
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
            if (states && sub == 0 && (WHOLE || (mine && chunk < a.chunks))) states[chunk] = Q8 ? start_q : start;
            const float v0 = apply(before, start);
            Pair v{v0, apply(halves.lo, v0)};
            float y[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v = fma2(f[i], v, b[i]);
                y[i] = WHOLE || i < live ? v.lo : 0.0f;
                y[i + 4] = WHOLE || i + 4 < live ? v.hi : 0.0f;
            }
            if constexpr (!kChunks) put_eight<T, ACC>(py, here, L, y);
            else if (WHOLE || chunk < a.chunks) put_chunk<T, ACC, WHOLE>(py + (int64_t)chunk * kScanChunk, L - chunk * kScanChunk, y, stage);
        }
        turn ^= 1;
    };
    uint32_t k = k_begin;
    if constexpr (kChunks) {
        fetch(k, 0);
        fetch(k + warps, 1);
    }
    if constexpr (kChunks && MODE != kBlock) {
        for (; k < min(k_end, whole); ++k) step.template operator()<true>(k);
        if (k < min(k_end, some)) step.template operator()<false>(k++);
        if constexpr (MODE != kJoin)
            for (; k < k_end; ++k) {                          // behind the row's length
                const float zero[8] = {};
                const uint32_t here = k * kScanChunk + sub * kScanVec;
                put_chunk<T, ACC, false>(py + (int64_t)k * kScanChunk, L - k * kScanChunk, zero, stage);
                if (states && lane == 0) states[k] = Q8 ? hq : h;
                if constexpr (Q8)
                    if (here < pitch) {
                        *reinterpret_cast<uint2*>(io.xc + codes_at + here) = *reinterpret_cast<uint2*>(io.gc + codes_at + here) = make_uint2(0, 0);
                        if (sub % 4 == 0) io.xs[scales_at + here / kQ8Block] = io.gs[scales_at + here / kQ8Block] = 1;
                    }
            }
    } else {
        if constexpr (kChunks)                                // (all warps of the block alike: they meet in the step)
            for (; k + warps <= whole; k += warps) step.template operator()<true>(k);
        for (; k < k_end; k += warps) step.template operator()<false>(k);
    }
    if constexpr (kChunks) asm volatile("cp.async.wait_all;" ::: "memory");
    if constexpr (MODE == kJoin) {
        if (lane == 0) a.joined[row * a.parts + at_row.part] = make_float4(total.P, total.B, total_q.P, total_q.B);
    } else {
        if (mine && (MODE == kBlock ? threadIdx.x == 0 : sub == 0) && k_end == a.chunks) io.h_last[row] = h;
    }
}

// Backward, from a row's end to its front: with E_t = f_t D_t, D_t = dy_t + E_{t+1}, a stretch maps the E behind it to the one in
// front of it, E -> P E + Q, by the same P.  The states of the chunks make the recomputed h of a chunk its own affair.
template <typename T, bool Q8, int ACC, int G, int MODE>
__global__ void __launch_bounds__(MODE == kBlock ? kScanWarps * 32 : 128, MODE == kWarp && G == 32 ? 7 : 1)
scan_bwd_kernel(const __grid_constant__ ScanArgs a,
                                                                                          const __grid_constant__ ScanBwd io) {
    extern __shared__ __align__(16) char ring_space[];        // a warp's: slots of grad_y and, not kept in 8 bits, gate and x; a chunk
    __shared__ Map shared[MODE == kBlock ? 2 : 1][kScanWarps];
    constexpr bool kChunks = ACC == kAligned || ACC == kWords;
    const int lane = threadIdx.x & 31, warp = warp_of_block(), warps = MODE == kBlock ? blockDim.x >> 5 : 1, sub = lane % G;
    const Place<G, MODE> at_row(a);
    if (!at_row.any) return;
    const int64_t row = at_row.row, n = row / a.C, c = row - n * a.C;
    const bool mine = at_row.mine;
    const uint32_t length = mine ? row_length(a, n) : 0u, L = mine ? a.L : 0u;
    const uint32_t end = G == 32 ? __shfl_sync(~0u, length, 0) : length;      // (known to be the same in all lanes)
    const T *px = (const T*)io.x + n * a.xb + c * a.xr, *pg = (const T*)io.gate + n * a.gb + c * a.gr, *py = (const T*)io.gy + row * a.L;
    T *ox = (T*)io.gx + n * a.ob + c * (int64_t)a.L, *og = (T*)io.gg + n * a.ob + c * (int64_t)a.L;
    const uint32_t k_begin = G == 32 && MODE != kBlock ? at_row.part * a.per_part : 0;
    const uint32_t k_end = G == 32 && MODE != kBlock ? min(k_begin + a.per_part, a.chunks) : a.chunks;
    const int64_t codes_at = row * q8_pitch(a.L), scales_at = row * q8_blocks(a.L);
    const float* states = io.states + row * a.chunks;

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
    constexpr int kRings = Q8 ? 1 : MODE == kJoin ? 2 : 3;
    using R = Ring<T, ACC>;
    char* space = ring_space + (kChunks ? warp * scan_space<T, ACC>(kRings, MODE != kJoin) : 0);
    char* stage = space + kRings * R::kSlots * R::kSlot;
    // step j works on the chunks from k_begin + j * warps on; from the last step down
    const uint32_t steps = (k_end - k_begin + warps - 1) / warps;
    const auto chunk_of = [&](uint32_t j) { return k_begin + j * warps + (MODE == kBlock ? warp : 0); };
    const uint32_t whole = end / kScanChunk, some = (end + kScanChunk - 1) / kScanChunk;
    // steps with something to read, where a warp works alone: those behind are a row's end, all zeros
    const uint32_t busy = kChunks && MODE != kBlock ? min(steps, some > k_begin ? some - k_begin : 0) : steps;
    if constexpr (kChunks && MODE == kWarp)
        for (uint32_t i = busy; i < steps; ++i) {
            const float zero[8] = {};
            put_chunk<T, ACC, false>(ox + (int64_t)chunk_of(i) * kScanChunk, L - chunk_of(i) * kScanChunk, zero, stage);
            put_chunk<T, ACC, false>(og + (int64_t)chunk_of(i) * kScanChunk, L - chunk_of(i) * kScanChunk, zero, stage);
        }
    uint32_t j = busy - 1;                                    // (wraps where there is none)
    R ry(py, chunk_of(j), space), rg(pg, chunk_of(j), space + R::kSlots * R::kSlot), rx(px, chunk_of(j), space + 2 * R::kSlots * R::kSlot);
    const auto fetch = [&](uint32_t i, int slot) {            // (i goes down from call to call, and wraps below zero: beyond steps)
        if (i < steps) {
            const uint32_t chunk = chunk_of(i);
            if (chunk < whole) {
                ry.template fetch<true>(slot);
                if constexpr (!Q8) rg.template fetch<true>(slot);
                if constexpr (!Q8 && MODE != kJoin) rx.template fetch<true>(slot);
            } else if (chunk < some) {
                const uint32_t count = end - chunk * kScanChunk;
                ry.template fetch<false>(slot, count);
                if constexpr (!Q8) rg.template fetch<false>(slot, count);
                if constexpr (!Q8 && MODE != kJoin) rx.template fetch<false>(slot, count);
            }
            ry.move(-(int64_t)warps * R::kBytes);
            if constexpr (!Q8) rg.move(-(int64_t)warps * R::kBytes);
            if constexpr (!Q8 && MODE != kJoin) rx.move(-(int64_t)warps * R::kBytes);
        }
        ring_commit();
    };
    uint2 cx, cg;
    uint32_t bx, bg;
    float state;
    const auto fetch_kept = [&](uint32_t i) {
        const uint32_t chunk = chunk_of(i), at = chunk * kScanChunk + sub * kScanVec;
        if constexpr (Q8) {
            cx = cg = make_uint2(0, 0);
            bx = bg = 1;
            if (at < end) {
                cg = __ldg(reinterpret_cast<const uint2*>(io.gc + codes_at + at));
                bg = __ldg(io.gs + scales_at + at / kQ8Block);
                if (MODE != kJoin) {
                    cx = __ldg(reinterpret_cast<const uint2*>(io.xc + codes_at + at));
                    bx = __ldg(io.xs + scales_at + at / kQ8Block);
                }
            }
        }
        if (MODE != kJoin) state = chunk < a.chunks ? __ldg(states + chunk) : 0.0f;
    };
    int turn = 0;
    const auto step = [&]<bool WHOLE>() {
        const uint32_t chunk = chunk_of(j), here = chunk * kScanChunk + sub * kScanVec;
        float x[8], g[8], d[8];
        Pair f[4], u[4];
        if constexpr (kChunks) {
            ring_wait();
            ry.take(turn, d);
            if constexpr (!Q8) rg.take(turn, g);
            if constexpr (!Q8 && MODE != kJoin) rx.take(turn, x);
            __syncwarp();
            fetch(j - 2, turn);                               // two steps ahead, into the slot just read
        } else {
            get_eight<T, ACC>(py, here, end, d);
            if constexpr (!Q8) {
                get_eight<T, ACC>(pg, here, end, g);
                get_eight<T, ACC>(px, here, end, x);
            }
        }
        if constexpr (Q8) {
            decode_eight(cg, bg, g);
            if (MODE != kJoin) decode_eight(cx, bx, x);
        }
        [[maybe_unused]] const float first = state;
        if (kChunks && j > 0) fetch_kept(j - 1);
        const int live = WHOLE ? 8 : end <= here ? 0 : (int)min(end - here, (uint32_t)kScanVec);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Gate q = gate_of(Pair{g[i], g[i + 4]});
            f[i] = q.f;
            u[i] = q.u;
            if (!WHOLE && i >= live) { f[i].lo = 1.0f; u[i].lo = 0.0f; x[i] = 0.0f; d[i] = 0.0f; }
            if (!WHOLE && i + 4 >= live) { f[i].hi = 1.0f; u[i].hi = 0.0f; x[i + 4] = 0.0f; d[i + 4] = 0.0f; }
        }
        [[maybe_unused]] Map all;
        Pair P = f[3], Q = mul2(f[3], {d[3], d[7]});
#pragma unroll
        for (int i = 2; i >= 0; --i) {
            Q = mul2(f[i], add2({d[i], d[i + 4]}, Q));
            P = mul2(P, f[i]);
        }
        const Map back_hi{P.hi, Q.hi}, back = then(back_hi, {P.lo, Q.lo});
        if constexpr (MODE == kJoin) {
            // (from the end of the row on: the maps of later lanes come first)
            const Map mirrored{__shfl_sync(~0u, back.P, 31 - lane), __shfl_sync(~0u, back.B, 31 - lane)};
            total = then(total, warp_join(mirrored));
        } else {
            Pair b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = mul2(u[i], {x[i], x[i + 4]});
            Pair B = b[0];
#pragma unroll
            for (int i = 1; i < 4; ++i) B = fma2(f[i], B, b[i]);
            const Map lo{P.lo, B.lo};
            [[maybe_unused]] Map unused;
            const Map m{back.P, fmaf(P.hi, B.lo, B.hi)};
            const Map behind = before_me<G, false>(back, all), before = before_me<G, true>(m, unused);
            all = of_last<G, false>(all);
            float start = E;
            if constexpr (MODE == kBlock) {
                if (lane == 0) shared[turn][warp] = all;
                __syncthreads();
                block_carry<false>(shared[turn], warp, warps, E, start, E);
            } else E = apply(all, E);
            const float v0 = apply(before, first), w7 = apply(behind, start);
            Pair v{v0, apply(lo, v0)}, w{apply(back_hi, w7), w7};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Pair prev = v;
                v = fma2(f[i], v, b[i]);
                b[i] = fma2({x[i], x[i + 4]}, {-1.0f, -1.0f}, prev);       // h_{t-1} - x_t
            }
#pragma unroll
            for (int i = 3; i >= 0; --i) {
                const Pair D = add2({d[i], d[i + 4]}, w);
                w = mul2(f[i], D);
                const Pair dx = mul2(u[i], D), dg = mul2(mul2(w, u[i]), b[i]);
                x[i] = WHOLE || i < live ? dx.lo : 0.0f;
                x[i + 4] = WHOLE || i + 4 < live ? dx.hi : 0.0f;
                g[i] = WHOLE || i < live ? dg.lo : 0.0f;
                g[i + 4] = WHOLE || i + 4 < live ? dg.hi : 0.0f;
            }
            if constexpr (!kChunks) {
                put_eight<T, ACC>(ox, here, L, x);
                put_eight<T, ACC>(og, here, L, g);
            } else if (WHOLE || chunk < a.chunks) {
                put_chunk<T, ACC, WHOLE>(ox + (int64_t)chunk * kScanChunk, L - chunk * kScanChunk, x, stage);
                put_chunk<T, ACC, WHOLE>(og + (int64_t)chunk * kScanChunk, L - chunk * kScanChunk, g, stage);
            }
        }
        turn ^= 1;
    };
    if (j < steps) fetch_kept(j);
    if constexpr (kChunks) {
        fetch(j, 0);
        fetch(j - 1, 1);
    }
    if constexpr (kChunks && MODE != kBlock) {
        if (j < steps && chunk_of(j) >= whole) {
            step.template operator()<false>();
            --j;
        }
        for (; j < steps; --j) step.template operator()<true>();
    } else {
        for (; j < steps && (!kChunks || (j + 1) * warps > whole); --j) step.template operator()<false>();
        if constexpr (kChunks)                                // (all warps of the block alike: they meet in the step)
            for (; j < steps; --j) step.template operator()<true>();
    }
    if constexpr (kChunks) asm volatile("cp.async.wait_all;" ::: "memory");
    if constexpr (MODE == kJoin) {
        if (lane == 0) a.joined[row * a.parts + at_row.part] = make_float4(total.P, total.B, 1.0f, 0.0f);
    } else {
        if (io.gh0 && mine && (MODE == kBlock ? threadIdx.x == 0 : sub == 0) && k_begin == 0) io.gh0[row] = E;
    }
}

// How a row's positions are shared out: short rows several to a warp; a row to a warp where there are rows enough; a block's warps
// in turn on a row, up to eight, in one pass; below that parts of a row, a warp each, in two passes (24 rows of 400001 positions:
// 28 us against 52 with the parts in blocks whose warps take turns).
struct ScanPlan {
    int g, warps, parts;             // threads of a row (1, 4, 16, 32); warps of a block on one row; parts of a row, a warp each
    uint32_t per_part;               // chunks
};

// heavy: fp32 kernels of 70 registers or so, which memory bounds (in bf16 a warp a row stays ahead: 46 us against 52 for 4096 rows of
// 3981 positions backward).  (What a row's state is made of does not hang on it: chunk by chunk in order in any case.)
inline ScanPlan plan_scan(int64_t rows, int64_t L, bool heavy) {
    const int64_t chunks = (L + kScanChunk - 1) / kScanChunk;
    ScanPlan p{32, 1, 1, (uint32_t)chunks};
    if (L <= 8) p.g = 1;
    else if (L <= 32) p.g = 4;
    else if (L <= 128) p.g = 16;
    if (p.g < 32) return p;
    const int64_t enough = 148 * 16;     // warps that keep the GPU busy
    const int64_t fit = 148 * 28;        // heavy warps on the GPU at once: a little more of them take twice as long, shared rows do not
    if (heavy && rows > fit && rows < 2 * fit && chunks > 1) p.warps = 2;
    else if (rows * kScanWarps >= enough || chunks < 4 * kScanWarps) {
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
