// The gated recurrence, the RMS norm and the 8-bit store in native code (see torch_layers.cpp): argument checks,
// allocation, library calls, and autograd nodes.
#include <ATen/TracerMode.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/cuda/CUDAContext.h>
#include <c10/cuda/CUDAGuard.h>
#include <torch/extension.h>

#include <optional>
#include <tuple>
#include <vector>

#include "tconv.h"
#include "torch_common.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::Variable;
using torch::autograd::variable_list;
using tconv_torch::fail;
using OptTensor = std::optional<Tensor>;

Tensor given(const OptTensor& t) { return t ? *t : Tensor(); }
void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float* fptr(const Tensor& t) { return t.defined() ? t.data_ptr<float>() : nullptr; }
void* stream() { return (void*)at::cuda::getCurrentCUDAStream().stream(); }

int dtype_of(const Tensor& t, const char* name) {
    TORCH_CHECK_VALUE(t.is_cuda(), name, ": need a CUDA tensor, got one on ", t.device());
    TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16, name,
                      ": need float32 or bfloat16, got ", t.scalar_type());
    return t.scalar_type() == at::kFloat ? TCONV_F32 : TCONV_BF16;
}
void same(const Tensor& t, const Tensor& like, at::ScalarType type, at::IntArrayRef shape, const char* name) {
    if (!t.defined()) return;
    TORCH_CHECK_VALUE(t.device() == like.device() && t.scalar_type() == type && t.sizes() == shape, name, ": need a ", type,
                      " tensor of shape ", shape, " on ", like.device(), ", got ", t.scalar_type(), " ", t.sizes(), " on ",
                      t.device());
}
// Allocation past the dispatcher, which costs the host more than the allocator does.
Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const Tensor& like) {
    return Tensor(at::detail::empty_cuda(shape, type, like.device(), std::nullopt));
}
Tensor bytes(size_t n, const Tensor& like) {
    const int64_t size[1] = {(int64_t)n};
    return n ? fresh(size, at::kByte, like) : Tensor();
}
// Places in a buffer, each on 256 bytes.
struct Places {
    size_t end = 0;
    size_t add(size_t n) {
        const size_t at = end;
        end += (n + 255) / 256 * 256;
        return at;
    }
};
// t dense and aligned to 16 bytes, copied where it is not.
Tensor dense(const Tensor& t) {
    if (!t.defined()) return t;
    Tensor c = t.contiguous();
    return (reinterpret_cast<uintptr_t>(c.data_ptr()) & 15) ? c.clone(at::MemoryFormat::Contiguous) : c;
}
void no_trace(const char* what) {
    TORCH_CHECK_NOT_IMPLEMENTED(!at::tracer::impl::is_dispatch_enabled(), what, " cannot be traced");
}
void no_tangent(const Tensor& t, const char* what) {
    TORCH_CHECK_NOT_IMPLEMENTED(!t.defined() || !t._fw_grad(0).defined(), what, " has no forward-mode derivative");
}
void once(const char* what) {
    TORCH_CHECK_NOT_IMPLEMENTED(!at::GradMode::is_enabled(), what, " has no second derivative");
}
bool records(std::initializer_list<const Tensor*> ts) {
    if (!at::GradMode::is_enabled()) return false;
    for (const Tensor* t : ts)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}

}  // namespace

// ---- activations in 8 bits ------------------------------------------------------------------------------------
std::pair<int64_t, int64_t> tconv_torch::q8_rows(at::IntArrayRef shape) {
    TORCH_CHECK_VALUE(!shape.empty(), "x: need a tensor of one dimension at least");
    int64_t inner = 1, rows = 1;
    for (size_t i = 2; i < shape.size(); ++i) inner *= shape[i];
    if (inner > 1) return {shape[0] * shape[1], inner};
    if (shape.size() == 1) return {1, shape[0]};
    rows = shape[0];
    return {rows, inner == 1 ? shape[1] : 0};
}
tconv_torch::Q8 tconv_torch::q8_empty(const Tensor& like, int64_t rows, int64_t inner) {
    const int64_t pitch = (inner + 7) / 8 * 8, nb = (inner + 31) / 32;
    const int64_t c[2] = {rows, pitch}, b[2] = {rows, nb};
    return {fresh(c, at::kChar, like), fresh(b, at::kByte, like)};
}
void tconv_torch::q8_check(const Q8& q, const Tensor& like, int64_t rows, int64_t inner) {
    const int64_t c[2] = {rows, (inner + 7) / 8 * 8}, s[2] = {rows, (inner + 31) / 32};
    same(q.codes, like, at::kChar, c, "codes");
    same(q.scales, like, at::kByte, s, "scales");
    TORCH_CHECK_VALUE(q.codes.is_cuda() && q.codes.is_contiguous() && q.scales.is_contiguous(), "codes, scales: need contiguous CUDA tensors");
}

namespace {

using tconv_torch::Q8;
using tconv_torch::q8_check;
using tconv_torch::q8_empty;
using tconv_torch::q8_rows;

std::tuple<Tensor, Tensor> q8_store(const Tensor& x) {
    no_trace("q8_store");
    no_tangent(x, "q8_store");
    const int dt = dtype_of(x, "x");
    c10::cuda::CUDAGuard guard(x.device());
    const auto [rows, inner] = q8_rows(x.sizes());
    at::AutoDispatchBelowADInplaceOrView below;
    const Tensor xc = dense(x);
    const Q8 q = q8_empty(x, rows, inner);
    if (const int rc = tconv_q8_store(rows, inner, dt, ptr(xc), ptr(q.codes), ptr(q.scales), stream())) fail(rc, "tconv_q8_store");
    return {q.codes, q.scales};
}
Tensor q8_restore(const Tensor& codes, const Tensor& scales, std::vector<int64_t> shape, int dtype) {
    no_trace("q8_restore");
    TORCH_CHECK_VALUE(codes.is_cuda(), "codes: need a CUDA tensor, got one on ", codes.device());
    c10::cuda::CUDAGuard guard(codes.device());
    const auto [rows, inner] = q8_rows(shape);
    q8_check({codes, scales}, codes, rows, inner);
    const Tensor c = dense(codes), s = dense(scales);
    Tensor x = fresh(shape, dtype == TCONV_F32 ? at::kFloat : at::kBFloat16, codes);
    if (const int rc = tconv_q8_restore(rows, inner, dtype, ptr(c), ptr(s), ptr(x), stream())) fail(rc, "tconv_q8_restore");
    return x;
}

// ---- gated recurrence -----------------------------------------------------------------------------------------
// x [N, C, L] and gate [N, C, L], or both in one tensor [N, 2C, L].
struct Signals {
    Tensor x, g;          // as the kernels read them: positions next to each other (packed: x alone)
    const void *px, *pg;
    bool packed;
    at::ScalarType type;
    tconv_scan_desc_t d;
    int64_t rows() const { return (int64_t)d.N * d.C; }
};
Tensor row_dense(const Tensor& t) { return t.size(2) == 1 || t.stride(2) == 1 ? t : t.contiguous(); }

Signals signals(const Tensor& x, const Tensor& gate) {
    Signals s;
    const int dt = dtype_of(x, "x");
    s.type = x.scalar_type();
    s.packed = !gate.defined();
    TORCH_CHECK_VALUE(x.dim() == 3, "x: need a tensor of 3 dimensions, got ", x.dim());
    TORCH_CHECK_VALUE(!s.packed || x.size(1) % 2 == 0, "x: without a gate it holds as many gates as values, got ", x.size(1), " channels");
    const int64_t N = x.size(0), C = s.packed ? x.size(1) / 2 : x.size(1), L = x.size(2);
    TORCH_CHECK_VALUE(N <= INT32_MAX && C <= INT32_MAX, "a size exceeds 31 bits");
    if (!s.packed) same(gate, x, s.type, x.sizes(), "gate");
    s.x = row_dense(x);
    s.px = ptr(s.x);
    if (s.packed) s.pg = (const char*)s.px + C * s.x.stride(1) * s.x.element_size();
    else {
        s.g = row_dense(gate);
        s.pg = ptr(s.g);
    }
    const Tensor& g = s.packed ? s.x : s.g;
    s.d = tconv_scan_desc_t{(int32_t)N, (int32_t)C, L, dt, s.x.stride(0), s.x.stride(1), g.stride(0), g.stride(1), (s.packed ? 2 : 1) * C * L};
    return s;
}
Tensor row_lengths(const Tensor& lengths, const Signals& s) {
    if (!lengths.defined()) return lengths;
    const int64_t n[1] = {s.d.N};
    if (lengths.scalar_type() == at::kLong) {
        same(lengths, s.x, at::kLong, n, "lengths");
        return lengths.clamp(0, s.d.L).to(at::kInt);
    }
    same(lengths, s.x, at::kInt, n, "lengths");
    return dense(lengths);
}

// What a backward pass needs, in one buffer: the states, and x and gate in 8 bits.
struct ScanKept {
    size_t states, xc, xs, gc, gs, size;
    ScanKept(const tconv_scan_desc_t& d, bool q8) {
        const int64_t rows = (int64_t)d.N * d.C;
        Places p;
        states = p.add(tconv_scan_states_bytes(&d));
        if (q8) {
            const size_t c = tconv_q8_codes_bytes(rows, d.L), s = tconv_q8_scales_bytes(rows, d.L);
            xc = p.add(c);
            xs = p.add(s);
            gc = p.add(c);
            gs = p.add(s);
        }
        size = p.end;
    }
};

struct ScanOut {
    Tensor y, last, kept, lengths;
};
ScanOut scan_forward(const Signals& s, const Tensor& h0_, const Tensor& lengths, bool keep, bool q8) {
    const int64_t nc[2] = {s.d.N, s.d.C}, ncl[3] = {s.d.N, s.d.C, s.d.L};
    same(h0_, s.x, at::kFloat, nc, "h0");
    const Tensor h0 = dense(h0_);
    ScanOut o;
    o.lengths = row_lengths(lengths, s);
    const ScanKept k(s.d, q8);
    if (keep) o.kept = bytes(k.size, s.x);
    o.y = fresh(ncl, s.type, s.x);
    o.last = fresh(nc, at::kFloat, s.x);
    const size_t n = tconv_scan_workspace_bytes(&s.d, 0);
    const Tensor ws = bytes(n, s.x);
    char* b = keep ? (char*)ptr(o.kept) : nullptr;
    const auto at_place = [&](size_t p) { return keep && q8 ? b + p : nullptr; };
    const int rc = tconv_scan_forward(&s.d, s.px, s.pg, fptr(h0), (const int32_t*)ptr(o.lengths), ptr(o.y), fptr(o.last),
                                      keep ? (float*)(b + k.states) : nullptr, at_place(k.xc), at_place(k.xs), at_place(k.gc), at_place(k.gs),
                                      ptr(ws), n, stream());
    if (rc) fail(rc, "tconv_scan_forward");
    return o;
}

class GatedScan : public torch::autograd::Function<GatedScan> {
public:
    static variable_list forward(AutogradContext* ctx, const Variable& x, const OptTensor& gate_, const OptTensor& h0_,
                                 const OptTensor& lengths, bool q8) {
        at::AutoDispatchBelowADInplaceOrView below;
        const Tensor gate = given(gate_), h0 = given(h0_);
        ctx->set_materialize_grads(false);
        const Signals s = signals(x, gate);
        ScanOut o = scan_forward(s, h0, given(lengths), true, q8);
        ctx->saved_data["sizes"] = std::vector<int64_t>{s.d.N, s.d.C, s.d.L, s.d.dtype, s.packed, q8, h0.defined()};
        if (q8) ctx->save_for_backward({o.kept, o.lengths});
        else ctx->save_for_backward({o.kept, o.lengths, x, gate});
        return {o.y, o.last};
    }
    static variable_list backward(AutogradContext* ctx, variable_list go) {
        once("gated_scan");
        if (!go[0].defined() && !go[1].defined()) return variable_list(5);
        const auto v = ctx->get_saved_variables();
        const auto z = ctx->saved_data["sizes"].toIntVector();
        at::AutoDispatchBelowADInplaceOrView below;
        const int64_t N = z[0], C = z[1], L = z[2];
        const bool packed = z[4], q8 = z[5];
        const at::ScalarType type = z[3] == TCONV_F32 ? at::kFloat : at::kBFloat16;
        const int64_t full[3] = {N, C, L}, wide[3] = {N, 2 * C, L}, nc[2] = {N, C}, nl[1] = {N};
        TORCH_CHECK_VALUE(v[0].defined() && v[0].is_cuda(), "states: need the CUDA tensor that the forward saved");
        c10::cuda::CUDAGuard guard(v[0].device());
        Signals s;
        if (q8) {
            s.px = s.pg = nullptr;
            s.d = tconv_scan_desc_t{(int32_t)N, (int32_t)C, L, (int32_t)z[3], 0, 0, 0, 0, (packed ? 2 : 1) * C * L};
        } else {
            s = signals(v[2], v[3]);
            TORCH_CHECK_VALUE(s.packed == packed, "x, gate: need the tensors that the forward saved");
            same(s.x, v[0], type, packed ? at::IntArrayRef(wide) : at::IntArrayRef(full), "x");
        }
        const ScanKept k(s.d, q8);
        const int64_t size[1] = {(int64_t)k.size};
        same(v[0], v[0], at::kByte, size, "states");
        same(v[1], v[0], at::kInt, nl, "lengths");
        same(go[0], v[0], type, full, "grad_y");
        same(go[1], v[0], at::kFloat, nc, "grad_h_last");
        const Tensor kept = dense(v[0]), len = dense(v[1]), gh = dense(go[1]);
        const Tensor gy = go[0].defined() ? dense(go[0]) : at::zeros(full, kept.options().dtype(type));
        Tensor gx = fresh(packed ? at::IntArrayRef(wide) : at::IntArrayRef(full), type, kept), gg, gh0;
        if (!packed) gg = fresh(full, type, kept);
        if (z[6]) gh0 = fresh(nc, at::kFloat, kept);
        const size_t n = tconv_scan_workspace_bytes(&s.d, 1);
        const Tensor ws = bytes(n, kept);
        const char* b = (const char*)ptr(kept);
        const auto at_place = [&](size_t p) { return q8 ? b + p : nullptr; };
        const int rc = tconv_scan_backward(&s.d, s.px, s.pg, at_place(k.xc), at_place(k.xs), at_place(k.gc), at_place(k.gs),
                                           (const int32_t*)ptr(len), (const float*)(b + k.states), ptr(gy), fptr(gh), ptr(gx),
                                           packed ? (char*)ptr(gx) + C * L * gx.element_size() : ptr(gg), fptr(gh0), ptr(ws), n, stream());
        if (rc) fail(rc, "tconv_scan_backward");
        return {gx, gg, gh0, Tensor(), Tensor()};
    }
};

std::tuple<Tensor, Tensor> gated_scan(const Tensor& x, const OptTensor& gate_, const OptTensor& h0_, const OptTensor& lengths, bool q8) {
    no_trace("gated_scan");
    const Tensor gate = given(gate_), h0 = given(h0_);
    for (const Tensor* t : {&x, &gate, &h0}) no_tangent(*t, "gated_scan");
    TORCH_CHECK_VALUE(x.is_cuda(), "x: need a CUDA tensor, got one on ", x.device());
    c10::cuda::CUDAGuard guard(x.device());
    if (records({&x, &gate, &h0})) {
        const variable_list r = GatedScan::apply(x, gate_, h0_, lengths, q8);
        return {r[0], r[1]};
    }
    at::AutoDispatchBelowADInplaceOrView below;
    ScanOut o = scan_forward(signals(x, gate), h0, given(lengths), false, false);
    return {o.y, o.last};
}

std::tuple<Tensor, Tensor> gated_scan_step(const Tensor& h, const Tensor& x, const OptTensor& gate_, const OptTensor& out_) {
    no_trace("gated_scan_step");
    const Tensor gate = given(gate_), out = given(out_);
    for (const Tensor* t : {&h, &x, &gate}) no_tangent(*t, "gated_scan_step");
    TORCH_CHECK_VALUE(!records({&h, &x, &gate, &out}), "gated_scan_step: records no gradients; use gated_scan, or call it under torch.no_grad()");
    TORCH_CHECK_VALUE(x.is_cuda(), "x: need a CUDA tensor, got one on ", x.device());
    TORCH_CHECK_VALUE(x.dim() == 2, "x: need a tensor of 2 dimensions, got ", x.dim());
    c10::cuda::CUDAGuard guard(x.device());
    at::AutoDispatchBelowADInplaceOrView below;
    const Signals s = signals(x.unsqueeze(2), gate.defined() ? gate.unsqueeze(-1) : gate);
    const int64_t nc[2] = {s.d.N, s.d.C};
    same(h, x, at::kFloat, nc, "h");
    TORCH_CHECK_VALUE(h.defined(), "h: need the state");
    const Tensor h0 = dense(h);
    Tensor last;
    if (out.defined()) {
        same(out, x, at::kFloat, nc, "out");
        TORCH_CHECK_VALUE(out.is_contiguous() && !(reinterpret_cast<uintptr_t>(out.data_ptr()) & 15), "out: need a contiguous tensor aligned to 16 bytes");
        const char *lo = (const char*)out.data_ptr(), *hi = lo + out.nbytes();
        const auto meets = [&](const void* p, int64_t bytes) { return lo < (const char*)p + bytes && (const char*)p < hi; };
        TORCH_CHECK_VALUE(ptr(h0) == lo || !meets(ptr(h0), h0.nbytes()), "out: overlaps h without being it");
        // an input that lies just like out is read before out is written; another one must not share memory with it
        const auto apart = [&](const void* p, int64_t batch, int64_t row, int64_t es) {
            if (p == lo && es == 4 && (s.d.N == 1 || batch == s.d.C) && (s.d.C == 1 || row == 1)) return true;
            const int64_t width = ((s.d.C - 1) * row + 1) * es;
            if (!meets(p, (s.d.N - 1) * batch * es + width)) return true;
            for (int64_t n = 0; n < s.d.N; ++n)
                if (meets((const char*)p + n * batch * es, width)) return false;
            return true;
        };
        const int64_t es = s.x.element_size();
        TORCH_CHECK_VALUE(apart(s.px, s.d.x_batch, s.d.x_row, es), "out: overlaps x");
        TORCH_CHECK_VALUE(apart(s.pg, s.d.gate_batch, s.d.gate_row, es), s.packed ? "out: overlaps x" : "out: overlaps gate");
        last = out;
    } else {
        last = fresh(nc, at::kFloat, h0);
    }
    Tensor y = fresh(nc, s.type, s.x);
    const int rc = tconv_scan_forward(&s.d, s.px, s.pg, fptr(h0), nullptr, ptr(y), fptr(last), nullptr, nullptr, nullptr,
                                      nullptr, nullptr, nullptr, 0, stream());
    if (rc) fail(rc, "tconv_scan_forward");
    if (out.defined()) out.unsafeGetTensorImpl()->bump_version();
    return {y, last};
}

// ---- norm -----------------------------------------------------------------------------------------------------
enum Output { kSame = 0, kQ8 = 1, kBoth = 2 };

tconv_norm_desc_t norm_desc(const Tensor& x, double eps) {
    TORCH_CHECK_VALUE(x.dim() >= 2, "x: need a tensor of 2 dimensions at least, got ", x.dim());
    int64_t P = 1;
    for (int64_t i = 2; i < x.dim(); ++i) P *= x.size(i);
    TORCH_CHECK_VALUE(x.size(0) <= INT32_MAX && x.size(1) <= INT32_MAX, "a size exceeds 31 bits");
    return tconv_norm_desc_t{(int32_t)x.size(0), (int32_t)x.size(1), P, dtype_of(x, "x"), (float)eps};
}

// What a backward pass needs beside the stream: rstd, and where asked for the stream in 8 bits, in one buffer.
struct NormKept {
    size_t rstd, codes, scales, size;
    NormKept(const tconv_norm_desc_t& d, int64_t rows, int64_t inner, bool q8) {
        Places p;
        rstd = p.add((size_t)d.N * d.P * sizeof(float));
        if (q8) {
            codes = p.add(tconv_q8_codes_bytes(rows, inner));
            scales = p.add(tconv_q8_scales_bytes(rows, inner));
        }
        size = p.end;
    }
};
struct NormOut {
    Tensor y, sum, stream, w, kept;
    Q8 q;
};

NormOut norm_forward(const Tensor& x, const Tensor& weight, const Tensor& residual, double eps, int output, bool keep, bool q8) {
    const tconv_norm_desc_t d = norm_desc(x, eps);
    const int64_t c[1] = {d.C};
    TORCH_CHECK_VALUE(weight.device() == x.device() && weight.sizes() == at::IntArrayRef(c), "weight: need a tensor of shape ", at::IntArrayRef(c),
                      " on ", x.device(), ", got ", weight.sizes(), " on ", weight.device());
    same(residual, x, x.scalar_type(), x.sizes(), "residual");
    const auto [rows, inner] = q8_rows(x.sizes());
    const Tensor xc = dense(x), rc_ = dense(residual);
    const at::ScalarType type = x.scalar_type();
    const NormKept k(d, rows, inner, q8);
    NormOut o;
    o.w = dense(weight.scalar_type() == at::kFloat ? weight : weight.to(at::kFloat));
    if (output != kQ8) o.y = fresh(x.sizes(), type, x);
    if (residual.defined()) o.sum = fresh(x.sizes(), type, x);
    if (output != kSame) o.q = q8_empty(x, rows, inner);
    if (keep) o.kept = bytes(k.size, x);
    o.stream = residual.defined() ? o.sum : xc;
    char* b = keep ? (char*)ptr(o.kept) : nullptr;
    const int rc = tconv_norm_forward(&d, ptr(xc), ptr(rc_), fptr(o.w), ptr(o.sum), ptr(o.y), keep ? (float*)(b + k.rstd) : nullptr,
                                      ptr(o.q.codes), ptr(o.q.scales), keep && q8 ? b + k.codes : nullptr, keep && q8 ? b + k.scales : nullptr,
                                      stream());
    if (rc) fail(rc, "tconv_norm_forward");
    return o;
}

class RmsNorm : public torch::autograd::Function<RmsNorm> {
public:
    // y, then the sum where there is a residual, then codes and scales where y is wanted in 8 bits too
    static variable_list forward(AutogradContext* ctx, const Variable& x, const Variable& weight, const OptTensor& residual_, double eps,
                                 int64_t output, bool q8) {
        at::AutoDispatchBelowADInplaceOrView below;
        const Tensor residual = given(residual_);
        ctx->set_materialize_grads(false);
        const NormOut o = norm_forward(x, weight, residual, eps, (int)output, true, q8);
        std::vector<int64_t> how{x.scalar_type() == at::kFloat ? TCONV_F32 : TCONV_BF16, q8, residual.defined()};
        how.insert(how.end(), x.sizes().begin(), x.sizes().end());
        ctx->saved_data["how"] = how;
        variable_list r{o.y};
        if (o.sum.defined()) r.push_back(o.sum);
        if (o.q.codes.defined()) {
            r.push_back(o.q.codes);
            r.push_back(o.q.scales);
            ctx->mark_non_differentiable({o.q.codes, o.q.scales});
        }
        if (q8) ctx->save_for_backward({o.kept, o.w});
        else ctx->save_for_backward({o.kept, o.w, o.stream});
        return r;
    }
    static variable_list backward(AutogradContext* ctx, variable_list go) {
        once("rms_norm");
        const auto v = ctx->get_saved_variables();
        const auto how = ctx->saved_data["how"].toIntVector();
        at::AutoDispatchBelowADInplaceOrView below;
        const at::IntArrayRef shape(how.data() + 3, how.size() - 3);
        const bool q8 = how[1], res = how[2];
        const Tensor gsum = res ? go[1] : Tensor();
        if (!go[0].defined() && !gsum.defined()) return variable_list(6);
        const at::ScalarType type = how[0] == TCONV_F32 ? at::kFloat : at::kBFloat16;
        TORCH_CHECK_VALUE(v[0].defined() && v[0].is_cuda() && v[1].defined(), "rstd, weight: need the CUDA tensors that the forward saved");
        c10::cuda::CUDAGuard guard(v[0].device());
        const auto [rows, inner] = q8_rows(shape);
        int64_t P = 1;
        for (size_t i = 2; i < shape.size(); ++i) P *= shape[i];
        const tconv_norm_desc_t d{(int32_t)shape[0], (int32_t)shape[1], P, (int32_t)how[0], 0.0f};
        const NormKept k(d, rows, inner, q8);
        const int64_t size[1] = {(int64_t)k.size}, c[1] = {shape[1]};
        same(v[0], v[0], at::kByte, size, "rstd");
        same(v[1], v[0], at::kFloat, c, "weight");
        Tensor s;
        if (!q8) {
            TORCH_CHECK_VALUE(v[2].defined(), "s: need the tensor that the forward saved");
            same(v[2], v[0], type, shape, "s");
            s = dense(v[2]);
        }
        same(go[0], v[0], type, shape, "grad_y");
        same(gsum, v[0], type, shape, "grad_sum");
        if (!go[0].defined()) {       // the stream's gradient is passed on, whatever the stream holds
            const Tensor gx = gsum.contiguous();
            return {gx, ctx->needs_input_grad(1) ? at::zeros(c, v[1].options()) : Tensor(), gx, Tensor(), Tensor(), Tensor()};
        }
        const Tensor kept = dense(v[0]), w = dense(v[1]), gs = dense(gsum), gy = dense(go[0]);
        Tensor gx = fresh(shape, type, kept), gw;
        if (ctx->needs_input_grad(1)) gw = fresh(c, at::kFloat, kept);
        const size_t n = gw.defined() ? tconv_norm_workspace_bytes(&d) : 0;
        const Tensor ws = bytes(n, kept);
        const char* b = (const char*)ptr(kept);
        const int rc = tconv_norm_backward(&d, ptr(s), q8 ? b + k.codes : nullptr, q8 ? b + k.scales : nullptr, (const float*)(b + k.rstd),
                                           fptr(w), ptr(gy), ptr(gs), ptr(gx), fptr(gw), ptr(ws), n, stream());
        if (rc) fail(rc, "tconv_norm_backward");
        return {gx, gw, res ? gx : Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

std::tuple<OptTensor, OptTensor, OptTensor, OptTensor> rms_norm(const Tensor& x, const Tensor& weight, const OptTensor& residual_, double eps,
                                                                int64_t output, bool q8) {
    no_trace("rms_norm");
    const Tensor residual = given(residual_);
    for (const Tensor* t : {&x, &weight, &residual}) no_tangent(*t, "rms_norm");
    TORCH_CHECK_VALUE(x.is_cuda(), "x: need a CUDA tensor, got one on ", x.device());
    c10::cuda::CUDAGuard guard(x.device());
    const auto opt = [](const Tensor& t) { return t.defined() ? OptTensor(t) : OptTensor(); };
    if (records({&x, &weight, &residual})) {
        TORCH_CHECK_VALUE(output != kQ8, "rms_norm: an output in 8 bits alone leaves nothing to differentiate; ask for both");
        const variable_list r = RmsNorm::apply(x, weight, residual_, eps, output, q8);
        const size_t at = residual.defined() ? 2 : 1;
        return {opt(r[0]), residual.defined() ? opt(r[1]) : OptTensor(), output == kBoth ? opt(r[at]) : OptTensor(),
                output == kBoth ? opt(r[at + 1]) : OptTensor()};
    }
    at::AutoDispatchBelowADInplaceOrView below;
    const NormOut o = norm_forward(x, weight, residual, eps, (int)output, false, false);
    return {opt(o.y), opt(o.sum), opt(o.q.codes), opt(o.q.scales)};
}

}  // namespace

namespace tconv_torch {

void bind_seq(pybind11::module& m) {
    const auto free = pybind11::call_guard<pybind11::gil_scoped_release>();
    m.def("q8_store", &q8_store, free);
    m.def("q8_restore", &q8_restore, free);
    m.def("gated_scan", &gated_scan, free);
    m.def("gated_scan_step", &gated_scan_step, free);
    m.def("rms_norm", &rms_norm, free);
}

}  // namespace tconv_torch
