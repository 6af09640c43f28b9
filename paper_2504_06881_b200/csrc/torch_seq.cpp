// The gated recurrence, the RMS norm and the 8-bit store in native code (see torch_layers.cpp): argument checks,
// allocation, library calls, and autograd nodes.
#include <ATen/TracerMode.h>
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

// ---- activations in 8 bits ------------------------------------------------------------------------------------
struct Q8 {
    Tensor codes, scales;
};
std::pair<int64_t, int64_t> q8_rows(at::IntArrayRef shape) {
    TORCH_CHECK_VALUE(!shape.empty(), "x: need a tensor of one dimension at least");
    int64_t inner = 1, rows = 1;
    for (size_t i = 2; i < shape.size(); ++i) inner *= shape[i];
    if (inner > 1) return {shape[0] * shape[1], inner};
    if (shape.size() == 1) return {1, shape[0]};
    rows = shape[0];
    return {rows, inner == 1 ? shape[1] : 0};
}
Q8 q8_empty(const Tensor& like, int64_t rows, int64_t inner) {
    const int64_t pitch = (inner + 7) / 8 * 8, nb = (inner + 31) / 32;
    return {at::empty({rows, pitch}, like.options().dtype(at::kChar)), at::empty({rows, nb}, like.options().dtype(at::kByte))};
}
void q8_check(const Q8& q, const Tensor& like, int64_t rows, int64_t inner) {
    const int64_t c[2] = {rows, (inner + 7) / 8 * 8}, s[2] = {rows, (inner + 31) / 32};
    same(q.codes, like, at::kChar, c, "codes");
    same(q.scales, like, at::kByte, s, "scales");
    TORCH_CHECK_VALUE(q.codes.is_cuda() && q.codes.is_contiguous() && q.scales.is_contiguous(), "codes, scales: need contiguous CUDA tensors");
}

std::tuple<Tensor, Tensor> q8_store(const Tensor& x) {
    no_trace("q8_store");
    const int dt = dtype_of(x, "x");
    c10::cuda::CUDAGuard guard(x.device());
    const auto [rows, inner] = q8_rows(x.sizes());
    at::NoGradGuard off;
    const Tensor xc = dense(x.detach());
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
    Tensor x = at::empty(shape, codes.options().dtype(dtype == TCONV_F32 ? at::kFloat : at::kBFloat16));
    if (const int rc = tconv_q8_restore(rows, inner, dtype, ptr(c), ptr(s), ptr(x), stream())) fail(rc, "tconv_q8_restore");
    return x;
}

// ---- gated recurrence -----------------------------------------------------------------------------------------
// x [N, C, L] and gate [N, C, L], or both in one tensor [N, 2C, L].
struct Signals {
    Tensor x, g;          // as the kernels read them: positions next to each other
    bool packed;
    int dt;
    tconv_scan_desc_t d;
    at::ScalarType type() const { return x.scalar_type(); }
    int64_t rows() const { return (int64_t)d.N * d.C; }
};
Tensor row_dense(const Tensor& t) { return t.size(2) == 1 || t.stride(2) == 1 ? t : t.contiguous(); }

Signals signals(const Tensor& x, const Tensor& gate) {
    Signals s;
    s.dt = dtype_of(x, "x");
    s.packed = !gate.defined();
    TORCH_CHECK_VALUE(x.dim() == 3, "x: need a tensor of 3 dimensions, got ", x.dim());
    TORCH_CHECK_VALUE(!s.packed || x.size(1) % 2 == 0, "x: without a gate it holds as many gates as values, got ", x.size(1), " channels");
    const int64_t N = x.size(0), C = s.packed ? x.size(1) / 2 : x.size(1), L = x.size(2);
    TORCH_CHECK_VALUE(N <= INT32_MAX && C <= INT32_MAX, "a size exceeds 31 bits");
    if (!s.packed) same(gate, x, x.scalar_type(), x.sizes(), "gate");
    const Tensor whole = row_dense(x);
    s.x = s.packed ? whole.narrow(1, 0, C) : whole;
    s.g = s.packed ? whole.narrow(1, C, C) : row_dense(gate);
    s.d = tconv_scan_desc_t{(int32_t)N, (int32_t)C, L, s.dt, s.x.stride(0), s.x.stride(1), s.g.stride(0), s.g.stride(1),
                            (s.packed ? 2 : 1) * C * L};
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

struct ScanKept {
    Q8 x, g;
    Tensor states, lengths;
};

std::tuple<Tensor, Tensor> scan_forward(const Signals& s, const Tensor& h0_, const Tensor& lengths, bool keep, bool q8, ScanKept& k) {
    const int64_t nc[2] = {s.d.N, s.d.C};
    same(h0_, s.x, at::kFloat, nc, "h0");
    const Tensor h0 = dense(h0_);
    const auto opt = s.x.options();
    k.lengths = row_lengths(lengths, s);
    Tensor y = at::empty({s.d.N, s.d.C, s.d.L}, opt), last = at::empty(nc, opt.dtype(at::kFloat)), ws;
    if (keep) k.states = at::empty({(int64_t)tconv_scan_states_bytes(&s.d) / 4}, opt.dtype(at::kFloat));
    if (keep && q8) {
        k.x = q8_empty(s.x, s.rows(), s.d.L);
        k.g = q8_empty(s.x, s.rows(), s.d.L);
    }
    const size_t n = tconv_scan_workspace_bytes(&s.d, 0);
    if (n) ws = at::empty({(int64_t)n}, opt.dtype(at::kByte));
    const int rc = tconv_scan_forward(&s.d, ptr(s.x), ptr(s.g), fptr(h0), (const int32_t*)ptr(k.lengths), ptr(y), fptr(last),
                                      fptr(k.states), ptr(k.x.codes), ptr(k.x.scales), ptr(k.g.codes), ptr(k.g.scales), ptr(ws), n,
                                      stream());
    if (rc) fail(rc, "tconv_scan_forward");
    return {y, last};
}

class GatedScan : public torch::autograd::Function<GatedScan> {
public:
    static variable_list forward(AutogradContext* ctx, const Variable& x, const OptTensor& gate_, const OptTensor& h0_,
                                 const OptTensor& lengths, bool q8) {
        const Tensor gate = given(gate_), h0 = given(h0_);
        ctx->set_materialize_grads(false);
        const Signals s = signals(x, gate);
        ScanKept k;
        auto [y, last] = scan_forward(s, h0, given(lengths), true, q8, k);
        ctx->saved_data["sizes"] = std::vector<int64_t>{s.d.N, s.d.C, s.d.L, s.dt, s.packed, q8, h0.defined()};
        if (q8)
            ctx->save_for_backward({k.x.codes, k.x.scales, k.g.codes, k.g.scales, k.states, k.lengths});
        else
            ctx->save_for_backward({x, gate, k.states, k.lengths});
        return {y, last};
    }
    static variable_list backward(AutogradContext* ctx, variable_list go) {
        once("gated_scan");
        if (!go[0].defined() && !go[1].defined()) return variable_list(5);
        const auto v = ctx->get_saved_variables();
        const auto z = ctx->saved_data["sizes"].toIntVector();
        const int64_t N = z[0], C = z[1], L = z[2];
        const bool packed = z[4], q8 = z[5];
        const at::ScalarType type = z[3] == TCONV_F32 ? at::kFloat : at::kBFloat16;
        const Tensor states = v[q8 ? 4 : 2], lengths = v[q8 ? 5 : 3];
        const int64_t full[3] = {N, C, L}, nc[2] = {N, C}, nl[1] = {N};
        TORCH_CHECK_VALUE(states.defined() && states.is_cuda(), "states: need the CUDA tensor that the forward saved");
        c10::cuda::CUDAGuard guard(states.device());
        Signals s;
        Q8 qx, qg;
        if (q8) {
            qx = {v[0], v[1]};
            qg = {v[2], v[3]};
            q8_check(qx, states, N * C, L);
            q8_check(qg, states, N * C, L);
            s.d = tconv_scan_desc_t{(int32_t)N, (int32_t)C, L, (int32_t)z[3], 0, 0, 0, 0, (packed ? 2 : 1) * C * L};
        } else {
            s = signals(v[0], v[1]);
            TORCH_CHECK_VALUE(s.packed == packed && s.type() == type, "x, gate: need the tensors that the forward saved");
            same(s.x, states, type, full, "x");
        }
        const int64_t sn[1] = {(int64_t)tconv_scan_states_bytes(&s.d) / 4};
        same(states, states, at::kFloat, sn, "states");
        same(lengths, states, at::kInt, nl, "lengths");
        same(go[0], states, type, full, "grad_y");
        same(go[1], states, at::kFloat, nc, "grad_h_last");
        const auto opt = states.options().dtype(type);
        const Tensor gy = go[0].defined() ? dense(go[0]) : at::zeros(full, opt), gh = dense(go[1]);
        const Tensor st = dense(states), len = dense(lengths);
        Tensor both, gx, gg, gh0, ws;
        if (packed) {
            both = at::empty({N, 2 * C, L}, opt);
            gx = both.narrow(1, 0, C);
            gg = both.narrow(1, C, C);
        } else {
            gx = at::empty(full, opt);
            gg = at::empty(full, opt);
        }
        if (z[6]) gh0 = at::empty(nc, opt.dtype(at::kFloat));
        const size_t n = tconv_scan_workspace_bytes(&s.d, 1);
        if (n) ws = at::empty({(int64_t)n}, opt.dtype(at::kByte));
        const int rc = tconv_scan_backward(&s.d, ptr(s.x), ptr(s.g), ptr(qx.codes), ptr(qx.scales), ptr(qg.codes), ptr(qg.scales),
                                           (const int32_t*)ptr(len), fptr(st), ptr(gy), fptr(gh), ptr(gx), ptr(gg), fptr(gh0), ptr(ws),
                                           n, stream());
        if (rc) fail(rc, "tconv_scan_backward");
        return {packed ? both : gx, packed ? Tensor() : gg, gh0, Tensor(), Tensor()};
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
    at::NoGradGuard off;
    ScanKept k;
    return scan_forward(signals(x, gate), h0, given(lengths), false, false, k);
}

std::tuple<Tensor, Tensor> gated_scan_step(const Tensor& h, const Tensor& x, const OptTensor& gate_, const OptTensor& out_) {
    no_trace("gated_scan_step");
    const Tensor gate = given(gate_), out = given(out_);
    TORCH_CHECK_VALUE(!records({&h, &x, &gate, &out}), "gated_scan_step: records no gradients; use gated_scan, or call it under torch.no_grad()");
    TORCH_CHECK_VALUE(x.is_cuda(), "x: need a CUDA tensor, got one on ", x.device());
    TORCH_CHECK_VALUE(x.dim() == 2, "x: need a tensor of 2 dimensions, got ", x.dim());
    c10::cuda::CUDAGuard guard(x.device());
    at::NoGradGuard off;
    const Signals s = signals(x.unsqueeze(2), gate.defined() ? gate.unsqueeze(-1) : gate);
    const int64_t nc[2] = {s.d.N, s.d.C};
    same(h, x, at::kFloat, nc, "h");
    TORCH_CHECK_VALUE(h.defined(), "h: need the state");
    const Tensor h0 = dense(h);
    Tensor last;
    if (out.defined()) {
        same(out, x, at::kFloat, nc, "out");
        TORCH_CHECK_VALUE(out.is_contiguous() && !(reinterpret_cast<uintptr_t>(out.data_ptr()) & 15), "out: need a contiguous tensor aligned to 16 bytes");
        const auto lo = [](const Tensor& t) { return (const char*)t.data_ptr(); };
        const auto hi = [&](const Tensor& t) { return lo(t) + t.nbytes(); };
        TORCH_CHECK_VALUE(lo(out) == lo(h0) || hi(out) <= lo(h0) || hi(h0) <= lo(out), "out: overlaps h without being it");
        last = out;
    } else {
        last = at::empty(nc, h0.options());
    }
    Tensor y = at::empty(nc, s.x.options());
    const int rc = tconv_scan_forward(&s.d, ptr(s.x), ptr(s.g), fptr(h0), nullptr, ptr(y), fptr(last), nullptr, nullptr, nullptr,
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

struct NormKept {
    Tensor s, rstd, w;
    Q8 q;
};
struct NormOut {
    Tensor y, sum;
    Q8 q;
};

NormOut norm_forward(const Tensor& x, const Tensor& weight, const Tensor& residual, double eps, int output, bool keep, bool q8, NormKept& k) {
    const tconv_norm_desc_t d = norm_desc(x, eps);
    const int64_t c[1] = {d.C};
    TORCH_CHECK_VALUE(weight.device() == x.device() && weight.sizes() == at::IntArrayRef(c), "weight: need a tensor of shape ", at::IntArrayRef(c),
                      " on ", x.device(), ", got ", weight.sizes(), " on ", weight.device());
    same(residual, x, x.scalar_type(), x.sizes(), "residual");
    const auto [rows, inner] = q8_rows(x.sizes());
    const Tensor xc = dense(x), rc_ = dense(residual);
    k.w = dense(weight.to(at::kFloat));
    const auto opt = xc.options();
    NormOut o;
    if (output != kQ8) o.y = at::empty(x.sizes(), opt);
    if (residual.defined()) o.sum = at::empty(x.sizes(), opt);
    if (output != kSame) o.q = q8_empty(x, rows, inner);
    if (keep) k.rstd = at::empty({d.N * d.P}, opt.dtype(at::kFloat));
    if (keep && q8) k.q = q8_empty(x, rows, inner);
    if (keep && !q8) k.s = residual.defined() ? o.sum : xc;
    const int rc = tconv_norm_forward(&d, ptr(xc), ptr(rc_), fptr(k.w), ptr(o.sum), ptr(o.y), fptr(k.rstd), ptr(o.q.codes),
                                      ptr(o.q.scales), ptr(k.q.codes), ptr(k.q.scales), stream());
    if (rc) fail(rc, "tconv_norm_forward");
    return o;
}

class RmsNorm : public torch::autograd::Function<RmsNorm> {
public:
    // y, then the sum where there is a residual, then codes and scales where y is wanted in 8 bits too
    static variable_list forward(AutogradContext* ctx, const Variable& x, const Variable& weight, const OptTensor& residual_, double eps,
                                 int64_t output, bool q8) {
        const Tensor residual = given(residual_);
        ctx->set_materialize_grads(false);
        NormKept k;
        const NormOut o = norm_forward(x, weight, residual, eps, (int)output, true, q8, k);
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["shape"] = x.sizes().vec();
        ctx->saved_data["how"] = std::vector<int64_t>{x.scalar_type() == at::kFloat ? TCONV_F32 : TCONV_BF16, q8, residual.defined()};
        variable_list r{o.y};
        if (o.sum.defined()) r.push_back(o.sum);
        if (o.q.codes.defined()) {
            r.push_back(o.q.codes);
            r.push_back(o.q.scales);
            ctx->mark_non_differentiable({o.q.codes, o.q.scales});
        }
        if (q8)
            ctx->save_for_backward({k.q.codes, k.q.scales, k.rstd, k.w});
        else
            ctx->save_for_backward({k.s, k.rstd, k.w});
        return r;
    }
    static variable_list backward(AutogradContext* ctx, variable_list go) {
        once("rms_norm");
        const auto v = ctx->get_saved_variables();
        const auto shape = ctx->saved_data["shape"].toIntVector();
        const auto how = ctx->saved_data["how"].toIntVector();
        const bool q8 = how[1], res = how[2];
        const Tensor gsum = res ? go[1] : Tensor();
        if (!go[0].defined() && !gsum.defined()) return variable_list(6);
        const at::ScalarType type = how[0] == TCONV_F32 ? at::kFloat : at::kBFloat16;
        const Tensor rstd = v[q8 ? 2 : 1], w = v[q8 ? 3 : 2];
        TORCH_CHECK_VALUE(rstd.defined() && rstd.is_cuda(), "rstd: need the CUDA tensor that the forward saved");
        c10::cuda::CUDAGuard guard(rstd.device());
        const auto [rows, inner] = q8_rows(shape);
        int64_t P = 1;
        for (size_t i = 2; i < shape.size(); ++i) P *= shape[i];
        const tconv_norm_desc_t d{(int32_t)shape[0], (int32_t)shape[1], P, (int32_t)how[0], (float)ctx->saved_data["eps"].toDouble()};
        const int64_t np[1] = {shape[0] * P}, c[1] = {shape[1]};
        same(rstd, rstd, at::kFloat, np, "rstd");
        same(w, rstd, at::kFloat, c, "weight");
        Tensor s;
        Q8 q;
        if (q8) {
            q = {v[0], v[1]};
            q8_check(q, rstd, rows, inner);
        } else {
            TORCH_CHECK_VALUE(v[0].defined(), "s: need the tensor that the forward saved");
            same(v[0], rstd, type, shape, "s");
            s = dense(v[0]);
        }
        same(go[0], rstd, type, shape, "grad_y");
        same(gsum, rstd, type, shape, "grad_sum");
        const auto opt = rstd.options().dtype(type);
        const Tensor gy = go[0].defined() ? dense(go[0]) : at::zeros(shape, opt), gs = dense(gsum), rs = dense(rstd), wc = dense(w);
        Tensor gx = at::empty(shape, opt), gw, ws;
        if (ctx->needs_input_grad(1)) gw = at::empty(c, opt.dtype(at::kFloat));
        const size_t n = tconv_norm_workspace_bytes(&d);
        if (n) ws = at::empty({(int64_t)n}, opt.dtype(at::kByte));
        const int rc = tconv_norm_backward(&d, ptr(s), ptr(q.codes), ptr(q.scales), fptr(rs), fptr(wc), ptr(gy), ptr(gs), ptr(gx), fptr(gw),
                                           ptr(ws), n, stream());
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
    at::NoGradGuard off;
    NormKept k;
    const NormOut o = norm_forward(x, weight, residual, eps, (int)output, false, false, k);
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
