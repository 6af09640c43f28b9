// C ABI of the operators around the one-dimensional layers: 8-bit activations, gated linear recurrence, RMS norm.
#include "tconv.h"
#include "tconv_internal.h"
#include "tconv_norm.cuh"
#include "tconv_scan.cuh"

#include <type_traits>

namespace tconv {
namespace {

constexpr int64_t kMost = (int64_t)1 << 40;     // elements of a tensor

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
template <typename... P> bool all_aligned(P... p) { return (aligned16(p) && ...); }

int check_q8(int64_t rows, int64_t inner, int dtype) {
    if (rows <= 0 || inner <= 0 || (dtype != TCONV_F32 && dtype != TCONV_BF16)) return TCONV_ERR_INVALID_ARG;
    return rows > kMost / inner || rows > ((int64_t)1 << 36) / q8_blocks(inner) ? TCONV_ERR_TOO_LARGE : TCONV_OK;   // (31 bits of blocks)
}

// Rows of whole blocks are one long row.  Units and values are counted in 32 bits where that is enough.
struct Q8Rows { int64_t rows, inner; };
Q8Rows q8_join(int64_t rows, int64_t inner) { return inner % kQ8Block ? Q8Rows{rows, inner} : Q8Rows{1, rows * inner}; }

template <typename T, typename I> int q8_store_t(Q8Rows q, const void* x, void* codes, void* scales, cudaStream_t st) {
    const unsigned grid = (unsigned)((q.rows * q8_blocks(q.inner) * 4 + 255) / 256);
    const auto kern = q.inner % (16 / sizeof(T)) == 0 ? q8_store_kernel<T, I, true> : q8_store_kernel<T, I, false>;
    kern<<<grid, 256, 0, st>>>(q.rows, q.inner, (const T*)x, (int8_t*)codes, (uint8_t*)scales);
    return launched(1, "q8_store");
}
template <typename T, typename I> int q8_restore_t(Q8Rows q, const void* codes, const void* scales, void* x, cudaStream_t st) {
    const int64_t units = (q.rows * q.inner + 7) / 8;
    if (q.inner % 8 == 0)
        q8_restore_kernel<T, I><<<(unsigned)((units + 256 * kRestore - 1) / (256 * kRestore)), 256, 0, st>>>(q.rows, q.inner, (const int8_t*)codes,
                                                                                                             (const uint8_t*)scales, (T*)x);
    else
        q8_restore_any_kernel<T, I><<<(unsigned)((units + 255) / 256), 256, 0, st>>>(q.rows, q.inner, (const int8_t*)codes, (const uint8_t*)scales, (T*)x);
    return launched(1, "q8_restore");
}
template <typename F> int q8_types(Q8Rows q, int dtype, F f) {
    const bool small = q.rows * (q8_blocks(q.inner) * kQ8Block + 8) < (int64_t)1 << 31;
    if (dtype == TCONV_F32) return small ? f(float{}, uint32_t{}) : f(float{}, int64_t{});
    return small ? f(__nv_bfloat16{}, uint32_t{}) : f(__nv_bfloat16{}, int64_t{});
}

int check_scan(const tconv_scan_desc_t* d, ScanArgs* a, ScanPlan* p, bool heavy = false) {
    if (!d || d->N <= 0 || d->C <= 0 || d->L <= 0 || (d->dtype != TCONV_F32 && d->dtype != TCONV_BF16))
        return TCONV_ERR_INVALID_ARG;
    if (d->x_batch < 0 || d->x_row < 0 || d->gate_batch < 0 || d->gate_row < 0 || d->grad_batch < 0) return TCONV_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)d->N * d->C;
    // (positions of a row are counted in 32 bits, a few chunks beyond its end among them)
    if (rows > kMost / d->L || rows > (int64_t)INT32_MAX || d->L > (int64_t)INT32_MAX) return TCONV_ERR_TOO_LARGE;
    *p = plan_scan(rows, d->L, heavy && d->dtype == TCONV_F32);
    *a = ScanArgs{rows, (uint32_t)d->L, (uint32_t)((d->L + kScanChunk - 1) / kScanChunk), p->per_part, d->C, p->parts,
                  d->x_batch, d->x_row, d->gate_batch, d->gate_row, d->grad_batch, nullptr, nullptr};
    return TCONV_OK;
}

size_t scan_workspace(const ScanArgs& a) { return a.parts > 1 ? (size_t)(a.rows * a.parts) * sizeof(float4) : 0; }

// Rows that all start on 16 bytes, and whose length is whole vectors (so that no vector reaches into the next row).
bool rows_aligned(const void* p, int64_t batch, int64_t row, int64_t L, int64_t per) {
    return aligned16(p) && batch % per == 0 && row % per == 0 && L % per == 0;
}

enum { kFwd, kBwd };

template <int DIR, typename T, bool Q8, int ACC, int G, int MODE, typename IO>
void scan_launch(const ScanArgs& a, const ScanPlan& p, const IO& io, cudaStream_t st) {
    const auto kern = [] {
        if constexpr (DIR == kFwd) return scan_fwd_kernel<T, Q8, ACC, G, MODE>;
        else return scan_bwd_kernel<T, Q8, ACC, G, MODE>;
    }();
    constexpr int kRings = DIR == kFwd ? 2 : Q8 ? 1 : MODE == kJoin ? 2 : 3;
    const int warps = MODE == kBlock ? p.warps : 4, smem = ACC == kAligned || ACC == kWords ? warps * scan_space<T, ACC>(kRings, MODE != kJoin) : 0;
    const int64_t warps_needed = G == 32 ? a.rows * p.parts : (a.rows + 32 / G - 1) / (32 / G);
    if (smem > 48 * 1024 && allow_smem(kern, smem) != cudaSuccess) return;       // (its error is what launched() finds)
    kern<<<(unsigned)(MODE == kBlock ? a.rows : (warps_needed + 3) / 4), warps * 32, smem, st>>>(a, io);
}

template <int DIR, typename T, bool Q8, typename IO>
int scan_run(const ScanArgs& a, const ScanPlan& p, const IO& io, bool vec, cudaStream_t st) {
    const char* name = DIR == kFwd ? "scan_fwd" : "scan_bwd";
    if (p.g < 32) {
        const auto go = [&](auto acc) {
            if (p.g == 1) scan_launch<DIR, T, Q8, decltype(acc)::value, 1, kWarp>(a, p, io, st);
            else if (p.g == 4) scan_launch<DIR, T, Q8, decltype(acc)::value, 4, kWarp>(a, p, io, st);
            else scan_launch<DIR, T, Q8, decltype(acc)::value, 16, kWarp>(a, p, io, st);
        };
        if (vec) go(std::integral_constant<int, kVector>{});
        else go(std::integral_constant<int, kStraight>{});
    } else {
        const auto go = [&](auto acc) {
            constexpr int ACC = decltype(acc)::value;
            if (p.warps > 1) {
                scan_launch<DIR, T, Q8, ACC, 32, kBlock>(a, p, io, st);
                return 0;
            }
            if (p.parts > 1) {
                scan_launch<DIR, T, Q8, ACC, 32, kJoin>(a, p, io, st);
                const int rc = launched(1, name);
                if (rc) return rc;
            }
            scan_launch<DIR, T, Q8, ACC, 32, kWarp>(a, p, io, st);
            return 0;
        };
        const int rc = vec ? go(std::integral_constant<int, kAligned>{}) : go(std::integral_constant<int, kWords>{});
        if (rc) return rc;
    }
    return launched(1, name);
}

template <int DIR, typename IO>
int scan_any(const ScanArgs& a, const ScanPlan& p, const IO& io, int dtype, bool q8, bool vec, cudaStream_t st) {
    const auto go = [&](auto type, auto kept) {
        using T = decltype(type);
        return scan_run<DIR, T, decltype(kept)::value>(a, p, io, vec, st);
    };
    if (dtype == TCONV_F32) return q8 ? go(float{}, std::true_type{}) : go(float{}, std::false_type{});
    return q8 ? go(__nv_bfloat16{}, std::true_type{}) : go(__nv_bfloat16{}, std::false_type{});
}

int check_norm(const tconv_norm_desc_t* d, NormArgs* a) {
    if (!d || d->N <= 0 || d->C <= 0 || d->P <= 0 || (d->dtype != TCONV_F32 && d->dtype != TCONV_BF16) || !(d->eps >= 0))
        return TCONV_ERR_INVALID_ARG;
    if ((int64_t)d->N * d->C > kMost / d->P || (int64_t)d->N > (int64_t)INT32_MAX / q8_blocks(d->P)) return TCONV_ERR_TOO_LARGE;
    // (channels and rows are counted in 32 bits, up to a thousand beyond the last among them)
    if (d->N > INT32_MAX - 4095 || d->C > INT32_MAX - 4095) return TCONV_ERR_TOO_LARGE;
    *a = NormArgs{d->N, d->C, d->P, d->eps};
    return TCONV_OK;
}

// Calls f with R as a constant: LEAST << k.
template <int LEAST, int MOST, typename F> void with_reps(int k, F f) {
    if constexpr (LEAST <= MOST) {
        if (k == 0) f.template operator()<LEAST>();
        else with_reps<2 * LEAST, MOST>(k - 1, f);
    }
}
template <typename F> void with_flags(bool p, bool q, F f) {
    if (p) q ? f.template operator()<true, true>() : f.template operator()<true, false>();
    else q ? f.template operator()<false, true>() : f.template operator()<false, false>();
}

template <typename T>
int norm_fwd_t(const NormArgs& a, const NormPlan& p, const void* x_, const void* r_, const float* w, const NormOut& o, cudaStream_t st) {
    constexpr int kMostV = 16 / sizeof(T);
    const T *x = (const T*)x_, *r = (const T*)r_;
    if (a.P == 1) {
        const unsigned grid = (unsigned)((a.N + 3) / 4);
        const bool vec = p.vec > 1;
        if (p.form < 0) {
            if (vec) norm_fwd_rows_loop_kernel<T, kMostV><<<grid, 128, 0, st>>>(a, x, r, w, o);
            else norm_fwd_rows_loop_kernel<T, 1><<<grid, 128, 0, st>>>(a, x, r, w, o);
        } else if (vec) with_reps<1, 32 / kMostV>(p.form, [&]<int R>() { norm_fwd_rows_kernel<T, kMostV, R><<<grid, 128, 0, st>>>(a, x, r, w, o); });
        else with_reps<8, 32>(p.form, [&]<int R>() { norm_fwd_rows_kernel<T, 1, R><<<grid, 128, 0, st>>>(a, x, r, w, o); });
    } else {
        const unsigned grid = (unsigned)(q8_blocks(a.P) * a.N);
        with_vec<T>(p.vec, [&](auto v) {
            constexpr int V = decltype(v)::value;
            with_flags(r, o.yc || o.sc, [&]<bool RES, bool Q8>() {
                if (p.form < 0) norm_fwd_loop_kernel<T, V, 8, V == 1 ? 8 : 4, RES, Q8><<<grid, 256, 0, st>>>(a, x, r, w, o);
                else with_cols(v, p.form, [&]<int, int WARPS, int R>() {
                    norm_fwd_cols_kernel<T, V, WARPS, R, RES, Q8><<<grid, WARPS * 32, 0, st>>>(a, x, r, w, o);
                });
            });
        });
    }
    return launched(1, "norm_fwd");
}
template <typename T> int norm_bwd_t(const NormArgs& a, const NormPlan& p, const NormIn& k, void* gx_, float* gw, float* part, cudaStream_t st) {
    constexpr int kMostV = 16 / sizeof(T);
    T* gx = (T*)gx_;
    if (!gw) part = nullptr;
    const unsigned grid = (unsigned)p.blocks;
    if (a.P == 1) {
        const auto go = [&]<int V, bool Q8>() {
            if (p.form < 0) {
                norm_bwd_rows_loop_kernel<T, V, Q8><<<(unsigned)((a.N + 3) / 4), 128, 0, st>>>(a, k, gx);
                if (part) norm_bwd_rows_weight_kernel<T, V, Q8><<<dim3((unsigned)((a.C + 128 * V - 1) / (128 * V)), (unsigned)p.parts), 128, 0, st>>>(a, k, part);
            } else if constexpr (V > 1) with_reps<1, 32 / V>(p.form, [&]<int R>() { norm_bwd_rows_kernel<T, V, R, Q8><<<grid, 128, 0, st>>>(a, k, gx, part); });
            else with_reps<8, 32>(p.form, [&]<int R>() { norm_bwd_rows_kernel<T, 1, R, Q8><<<grid, 128, 0, st>>>(a, k, gx, part); });
        };
        if (p.vec > 1) k.s ? go.template operator()<kMostV, false>() : go.template operator()<kMostV, true>();
        else k.s ? go.template operator()<1, false>() : go.template operator()<1, true>();
    } else {
        with_vec<T>(p.vec, [&](auto v) {
            constexpr int V = decltype(v)::value;
            with_flags(k.gs, !k.s, [&]<bool RES, bool Q8>() {
                if (p.form < 0) norm_bwd_loop_kernel<T, V, 8, V == 1 ? 8 : 4, RES, Q8><<<grid, 256, a.C <= kNormShared ? a.C * sizeof(float) : 0, st>>>(a, k, gx, part);
                else with_cols(v, p.form, [&]<int, int WARPS, int R>() {
                    norm_bwd_cols_kernel<T, V, WARPS, R, RES, Q8><<<grid, WARPS * 32, 0, st>>>(a, k, gx, part);
                });
            });
        });
    }
    const int rc = launched(a.P == 1 && p.form < 0 && part ? 2 : 1, "norm_bwd");
    if (rc || !gw) return rc;
    norm_weight_sum_kernel<8><<<(unsigned)((a.C + 31) / 32), 256, 0, st>>>(a.C, p.parts, part, gw);
    return launched(1, "norm_bwd");
}

}  // namespace
}  // namespace tconv

using namespace tconv;

extern "C" {

size_t tconv_q8_codes_bytes(int64_t rows, int64_t inner) {
    return check_q8(rows, inner, TCONV_F32) ? 0 : (size_t)(rows * q8_pitch(inner));
}
size_t tconv_q8_scales_bytes(int64_t rows, int64_t inner) {
    return check_q8(rows, inner, TCONV_F32) ? 0 : (size_t)(rows * q8_blocks(inner));
}

int tconv_q8_store(int64_t rows, int64_t inner, int dtype, const void* x, void* codes, void* scales, void* stream) {
    const int rc = check_q8(rows, inner, dtype);
    if (rc) return rc;
    if (!x || !codes || !scales) return TCONV_ERR_INVALID_ARG;
    if (!all_aligned(x, codes, scales)) return TCONV_ERR_MISALIGNED;
    call_begins();
    const Q8Rows q = q8_join(rows, inner);
    return q8_types(q, dtype, [&](auto t, auto i) { return q8_store_t<decltype(t), decltype(i)>(q, x, codes, scales, (cudaStream_t)stream); });
}

int tconv_q8_restore(int64_t rows, int64_t inner, int dtype, const void* codes, const void* scales, void* x, void* stream) {
    const int rc = check_q8(rows, inner, dtype);
    if (rc) return rc;
    if (!x || !codes || !scales) return TCONV_ERR_INVALID_ARG;
    if (!all_aligned(x, codes, scales)) return TCONV_ERR_MISALIGNED;
    call_begins();
    const Q8Rows q = q8_join(rows, inner);
    return q8_types(q, dtype, [&](auto t, auto i) { return q8_restore_t<decltype(t), decltype(i)>(q, codes, scales, x, (cudaStream_t)stream); });
}

size_t tconv_scan_states_bytes(const tconv_scan_desc_t* desc) {
    ScanArgs a;
    ScanPlan p;
    return check_scan(desc, &a, &p) ? 0 : (size_t)(a.rows * a.chunks) * sizeof(float);
}

size_t tconv_scan_workspace_bytes(const tconv_scan_desc_t* desc, int) {
    ScanArgs a;
    ScanPlan p;
    return check_scan(desc, &a, &p) ? 0 : scan_workspace(a);
}

int tconv_scan_forward(const tconv_scan_desc_t* desc, const void* x, const void* gate, const float* h0, const int32_t* lengths,
                       void* y, float* h_last, float* states, void* x_codes, void* x_scales, void* gate_codes, void* gate_scales,
                       void* workspace, size_t workspace_bytes, void* stream) {
    ScanArgs a;
    ScanPlan p;
    const int rc = check_scan(desc, &a, &p, x_codes != nullptr);
    if (rc) return rc;
    const int kept = !!x_codes + !!x_scales + !!gate_codes + !!gate_scales;
    if (!x || !gate || !y || !h_last || (kept != 0 && kept != 4) || (kept && !states)) return TCONV_ERR_INVALID_ARG;
    if (h_last == h0 && a.L > 1) return TCONV_ERR_INVALID_ARG;
    if (!all_aligned(y, h0, h_last, states, x_codes, x_scales, gate_codes, gate_scales, lengths, workspace)) return TCONV_ERR_MISALIGNED;
    const int es = desc->dtype == TCONV_F32 ? 4 : 2;
    if ((uintptr_t)x % es || (uintptr_t)gate % es) return TCONV_ERR_MISALIGNED;
    const size_t need = scan_workspace(a);
    if (workspace_bytes < need || (need && !workspace)) return TCONV_ERR_WORKSPACE_TOO_SMALL;
    a.lengths = lengths;
    a.joined = (float4*)workspace;
    const int64_t per = 16 / es;
    const bool vec = rows_aligned(x, a.xb, a.xr, a.L, per) && rows_aligned(gate, a.gb, a.gr, a.L, per);
    const ScanFwd io{x, gate, h0, y, h_last, states, (int8_t*)x_codes, (int8_t*)gate_codes, (uint8_t*)x_scales, (uint8_t*)gate_scales};
    call_begins();
    return scan_any<kFwd>(a, p, io, desc->dtype, kept, vec, (cudaStream_t)stream);
}

int tconv_scan_backward(const tconv_scan_desc_t* desc, const void* x, const void* gate, const void* x_codes, const void* x_scales,
                        const void* gate_codes, const void* gate_scales, const int32_t* lengths, const float* states,
                        const void* grad_y, const float* grad_h_last, void* grad_x, void* grad_gate, float* grad_h0,
                        void* workspace, size_t workspace_bytes, void* stream) {
    ScanArgs a;
    ScanPlan p;
    const int rc = check_scan(desc, &a, &p, true);
    if (rc) return rc;
    const int kept = !!x_codes + !!x_scales + !!gate_codes + !!gate_scales;
    if ((kept != 4 && (kept != 0 || !x || !gate)) || !states || !grad_y || !grad_x || !grad_gate) return TCONV_ERR_INVALID_ARG;
    if (desc->grad_batch < desc->C * desc->L && desc->N > 1) return TCONV_ERR_INVALID_ARG;
    if (!all_aligned(x_codes, x_scales, gate_codes, gate_scales, lengths, states, grad_y, grad_h_last, grad_h0, workspace))
        return TCONV_ERR_MISALIGNED;
    const int es = desc->dtype == TCONV_F32 ? 4 : 2;
    if ((uintptr_t)x % es || (uintptr_t)gate % es || (uintptr_t)grad_x % es || (uintptr_t)grad_gate % es) return TCONV_ERR_MISALIGNED;
    const size_t need = scan_workspace(a);
    if (workspace_bytes < need || (need && !workspace)) return TCONV_ERR_WORKSPACE_TOO_SMALL;
    a.lengths = lengths;
    a.joined = (float4*)workspace;
    const int64_t per = 16 / es;
    const bool vec = rows_aligned(grad_x, a.ob, a.L, a.L, per) && rows_aligned(grad_gate, a.ob, a.L, a.L, per) &&
                     (kept || (rows_aligned(x, a.xb, a.xr, a.L, per) && rows_aligned(gate, a.gb, a.gr, a.L, per)));
    const ScanBwd io{x, gate, (const int8_t*)x_codes, (const int8_t*)gate_codes, (const uint8_t*)x_scales, (const uint8_t*)gate_scales,
                     states, grad_y, grad_h_last, grad_x, grad_gate, grad_h0};
    call_begins();
    return scan_any<kBwd>(a, p, io, desc->dtype, kept, vec, (cudaStream_t)stream);
}

size_t tconv_norm_workspace_bytes(const tconv_norm_desc_t* desc) {
    NormArgs a;
    if (check_norm(desc, &a)) return 0;
    return (size_t)plan_norm(a, desc->dtype).parts * a.C * sizeof(float);
}

int tconv_norm_forward(const tconv_norm_desc_t* desc, const void* x, const void* residual, const float* weight, void* sum, void* y,
                       float* rstd, void* y_codes, void* y_scales, void* s_codes, void* s_scales, void* stream) {
    NormArgs a;
    const int rc = check_norm(desc, &a);
    if (rc) return rc;
    if (!x || !weight || !y_codes != !y_scales || !s_codes != !s_scales || (!y && !y_codes) || !residual != !sum)
        return TCONV_ERR_INVALID_ARG;
    if (!all_aligned(x, residual, weight, sum, y, rstd, y_codes, y_scales, s_codes, s_scales)) return TCONV_ERR_MISALIGNED;
    const NormOut o{sum, y, rstd, (int8_t*)y_codes, (uint8_t*)y_scales, (int8_t*)s_codes, (uint8_t*)s_scales};
    call_begins();
    return (desc->dtype == TCONV_F32 ? norm_fwd_t<float> : norm_fwd_t<__nv_bfloat16>)(a, plan_norm(a, desc->dtype), x, residual, weight, o, (cudaStream_t)stream);
}

int tconv_norm_backward(const tconv_norm_desc_t* desc, const void* s, const void* s_codes, const void* s_scales, const float* rstd,
                        const float* weight, const void* grad_y, const void* grad_sum, void* grad_x, float* grad_weight,
                        void* workspace, size_t workspace_bytes, void* stream) {
    NormArgs a;
    const int rc = check_norm(desc, &a);
    if (rc) return rc;
    if (!s_codes != !s_scales || !s == !s_codes || !rstd || !weight || !grad_y || !grad_x) return TCONV_ERR_INVALID_ARG;
    if (!all_aligned(s, s_codes, s_scales, rstd, weight, grad_y, grad_sum, grad_x, grad_weight, workspace)) return TCONV_ERR_MISALIGNED;
    const size_t need = grad_weight ? tconv_norm_workspace_bytes(desc) : 0;
    if (workspace_bytes < need || (need && !workspace)) return TCONV_ERR_WORKSPACE_TOO_SMALL;
    const NormIn k{s, (const int8_t*)s_codes, (const uint8_t*)s_scales, rstd, weight, grad_y, grad_sum};
    call_begins();
    const auto run = desc->dtype == TCONV_F32 ? norm_bwd_t<float> : norm_bwd_t<__nv_bfloat16>;
    return run(a, plan_norm(a, desc->dtype), k, grad_x, grad_weight, (float*)workspace, (cudaStream_t)stream);
}

}  // extern "C"
