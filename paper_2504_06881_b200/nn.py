"""PyTorch glue over the C ABI: an autograd Function, a drop-in layer and the
ResNet-18-shaped hybrid network of benchmark configuration 5.

Everything tropical runs in the library's CUDA kernels (forward with winners, winner-routed
backward); PyTorch supplies BatchNorm, the standard convolutions of the stem / stage 1 /
1x1 downsamples, the loss and the optimiser, none of which is on the tropical hot path.
The layer follows the paper's usage (Appendix "Compatibility with PyTorch"): same constructor
arguments as ``nn.Conv2d``; ``mode`` selects max_plus / min_plus / compound / parallel.
"""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import torch
import torch.nn as nn

from . import tconv, tconv3d, tseq  # noqa: F401
try:
    from . import _tconv_torch as _native
except ImportError as err:
    raise ImportError(f"the layers' extension module is missing or does not load ({err}): build it with "
                      f"`python -m paper_2504_06881_b200.build`") from err

_native.set_error(tconv.TconvError)


def _emit_winners(recording, *tensors):
    """Whether a forward has to leave the winners a backward will need.  `recording` is
    ``torch.is_grad_enabled()`` where the layer was called: inside a Function's forward the grad mode is
    always off, and parameters keep ``requires_grad`` under ``torch.no_grad``."""
    return recording and any(t is not None and t.requires_grad for t in tensors)


def _as(t, dtype):
    """t in the given type, dense; None stays None.  (Called with the grad mode off.)"""
    if t is None:
        return None
    if t.dtype != dtype:
        t = t.to(dtype)
    return t if t.is_contiguous() else t.contiguous()


_KINDS = {"dense": 0, "depthwise": 1, "volume": 2}
_geoms = tconv.KeptPlans(lambda kind, mode, chan, dtype, stride, pad, dil: _native.Geom(
    _KINDS[kind], tconv.MODES[mode], tconv.CHANS[chan], tconv.DTYPES[dtype], stride, pad, dil))


def _layer(kind, mode, chan, dtype, stride, pad, dil, x, w, w2, alpha, beta, bias, checkpoint=None, stored=None):
    """One layer through the native autograd path (csrc/torch_layers.cpp).  Under ``torch.jit.trace`` through the
    Python Function, which a trace records as one operation: of the native path it would record the allocations."""
    geom = (kind, mode, chan, dtype, stride, pad, dil)
    try:
        g = _geoms.get(geom, *geom)
    except TypeError:            # (geometry set as lists)
        stride, pad, dil = tuple(stride), tuple(pad), tuple(dil)
        geom = (kind, mode, chan, dtype, stride, pad, dil)
        g = _geoms.get(geom, *geom)
    if checkpoint is None:
        if stored is not None:
            raise ValueError("stored: only a layer with checkpoint='q8' takes its input's 8-bit form")
        y = _native.layer(g, x, w, w2, alpha, beta, bias)
    elif stored is None:
        y = _native.layer(g, x, w, w2, alpha, beta, bias, True)
    else:
        y = _native.layer(g, x, w, w2, alpha, beta, bias, True, stored.codes, stored.scales)
    if y is not None:
        return y
    if checkpoint is not None:
        raise NotImplementedError("a layer with checkpoint='q8' cannot be traced")
    fn = {"dense": TropicalConvFn, "depthwise": TropicalDepthwiseFn, "volume": TropicalConv3dFn}[kind]
    return fn.apply(x, w, w2, alpha, beta, bias, (mode, dtype, stride, pad, dil) if kind == "depthwise" else geom[1:])


class TropicalConvFn(torch.autograd.Function):
    """y = tconv_forward(x, w, w2, alpha, beta, bias); backward = tconv_backward with the stored winners.
    The layers take the native path (csrc/torch_layers.cpp) unless one of the two settings below is on or a trace is
    recorded.  geom: mode, channel combine, type, stride, padding, dilation and optionally whether gradients are
    recorded where the layer was called (inside a Function's forward the grad mode is always off).

    Master parameters may be fp32 while the layer computes in bf16: the cast happens here and the
    parameter gradients come back in fp32.  When ``TropicalConvFn.events`` is a list, every library
    call is bracketed by a pair of CUDA events appended to it (for the benchmark's per-layer times)."""

    events = None
    # True: bf16 layers read a float x directly (x_dtype) instead of a converted copy.  Off by default:
    # the conversion while staging rules out the copy-engine path, which costs more than the cast
    # kernel saves on the ResNet-18 shape (tropical forward 21.5 -> 23.9 ms per step).
    fuse_cast = False

    @staticmethod
    def forward(ctx, x, w, w2, alpha, beta, bias, geom):
        mode, chan, dtype, stride, pad, dil = geom[:6]
        recording = geom[6] if len(geom) > 6 else True
        dt = tconv.TORCH_DTYPE[dtype]
        N, C, H, W = x.shape
        K, _, R, S = w.shape
        d = dict(N=N, C=C, H=H, W=W, K=K, R=R, S=S, stride_h=stride[0], stride_w=stride[1],
                 pad_h=pad[0], pad_w=pad[1], dil_h=dil[0], dil_w=dil[1], mode=mode, chan=chan, dtype=dtype)
        # a float x for a bf16 layer is rounded by the kernel while it stages x (no cast kernel, no
        # bf16 copy); layers the tiled kernels do not serve fall back to the explicit cast
        fused_cast = TropicalConvFn.fuse_cast and dtype == "bf16" and x.dtype == torch.float32
        if fused_cast:
            d["x_dtype"] = "f32"
        xc = _as(x, x.dtype if fused_cast else dt)
        wc, w2c = _as(w, dt), _as(w2, dt)
        al, be, bi = _as(alpha, torch.float32), _as(beta, torch.float32), _as(bias, torch.float32)
        need_grad = _emit_winners(recording, x, w, w2, alpha, beta, bias)
        ev = TropicalConvFn.events
        if ev is not None:
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
        try:
            y, winners = tconv.forward(d, xc, wc, w2c, al, be, bi, want_winners=need_grad)
        except tconv.TconvError as err:
            if not fused_cast or err.status != -2:
                raise
            del d["x_dtype"]
            xc = _as(x, dt)
            y, winners = tconv.forward(d, xc, wc, w2c, al, be, bi, want_winners=need_grad)
        if ev is not None:
            e1.record()
            ev.append(("fwd", d, e0, e1))
        ctx.d = d
        ctx.in_dtype = x.dtype
        ctx.save_for_backward(xc, wc, w2c, al, be, winners)
        ctx.has = (w2 is not None, alpha is not None, beta is not None, bias is not None)
        return y.to(x.dtype) if x.dtype != dt else y

    @staticmethod
    def backward(ctx, gy):
        xc, wc, w2c, al, be, winners = ctx.saved_tensors
        d = ctx.d
        dt = tconv.TORCH_DTYPE[d["dtype"]]
        g = _as(gy, dt)
        ev = TropicalConvFn.events
        if ev is not None:
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
        need = ["grad_w", "grad_w2", "grad_alpha", "grad_beta", "grad_bias"]
        if ctx.needs_input_grad[0]:
            need.append("grad_x")          # a first layer's input needs none: the kernel is skipped
        try:
            grads = tconv.backward(d, xc, wc, g, w2c, al, be, winners, need=tuple(need))
        except tconv.TconvError as err:
            if d.get("x_dtype") != "f32" or err.status != -2:
                raise
            d = {k: v for k, v in d.items() if k != "x_dtype"}      # a path that reads x itself: convert first
            grads = tconv.backward(d, xc.to(dt), wc, g, w2c, al, be, winners, need=tuple(need))
        if ev is not None:
            e1.record()
            ev.append(("bwd", d, e0, e1))
        has_w2, has_a, has_b, has_bias = ctx.has
        gx = grads["grad_x"].to(ctx.in_dtype) if "grad_x" in grads else None
        return (gx, grads["grad_w"], grads.get("grad_w2") if has_w2 else None,
                grads.get("grad_alpha") if has_a else None, grads.get("grad_beta") if has_b else None,
                grads["grad_bias"] if has_bias else None, None)


class TropicalConvBNFn(torch.autograd.Function):
    """Tropical layer followed by training-mode batch normalisation, the pair the paper's residual
    blocks are made of (section "ResNet Models").  The layer's kernel leaves the per-channel sums of
    y and y^2 (tconv_forward_stats), so the normalisation reads y once (scale and shift) instead of
    twice (statistics, then scale and shift).  Backward: the usual batch-normalisation gradient
    (channel reductions of grad and grad * y, then one elementwise pass), then tconv_backward."""

    @staticmethod
    def forward(ctx, x, w, w2, alpha, beta, gamma, bn_bias, geom, eps):
        mode, chan, dtype, stride, pad, dil = geom
        dt = tconv.TORCH_DTYPE[dtype]
        N, C, H, W = x.shape
        K, _, R, S = w.shape
        d = dict(N=N, C=C, H=H, W=W, K=K, R=R, S=S, stride_h=stride[0], stride_w=stride[1],
                 pad_h=pad[0], pad_w=pad[1], dil_h=dil[0], dil_w=dil[1], mode=mode, chan=chan, dtype=dtype)
        fused_cast = TropicalConvFn.fuse_cast and dtype == "bf16" and x.dtype == torch.float32
        xc = x.detach().contiguous() if fused_cast else x.detach().to(dt).contiguous()
        if fused_cast:
            d["x_dtype"] = "f32"
        wc = w.detach().to(dt).contiguous()
        w2c = w2.detach().to(dt).contiguous() if w2 is not None else None
        al = alpha.detach().float().contiguous() if alpha is not None else None
        be = beta.detach().float().contiguous() if beta is not None else None
        ev = TropicalConvFn.events
        if ev is not None:
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
        try:
            y, winners, s1, s2 = tconv.forward_stats(d, xc, wc, w2c, al, be, None, want_winners=True)
        except tconv.TconvError as err:
            if not fused_cast or err.status != -2:
                raise
            d.pop("x_dtype")
            xc = x.detach().to(dt).contiguous()
            y, winners, s1, s2 = tconv.forward_stats(d, xc, wc, w2c, al, be, None, want_winners=True)
        if ev is not None:
            e1.record()
            ev.append(("fwd", d, e0, e1))
        cnt = float(y.shape[0] * y.shape[2] * y.shape[3])
        mean = s1 / cnt
        var = (s2 / cnt - mean * mean).clamp_min_(0.0)          # biased variance of the batch
        invstd = torch.rsqrt(var + eps)
        scale = gamma.detach().float() * invstd
        shift = bn_bias.detach().float() - mean * scale
        out = torch.addcmul(shift.view(1, -1, 1, 1), y, scale.view(1, -1, 1, 1))    # one pass over y, fp32 result
        ctx.d, ctx.in_dtype, ctx.cnt = d, x.dtype, cnt
        ctx.save_for_backward(xc, wc, w2c, al, be, winners, y, mean, invstd, gamma.detach().float())
        ctx.has = (w2 is not None, alpha is not None, beta is not None)
        ctx.mark_non_differentiable(mean, var)
        return out.to(x.dtype), mean, var

    @staticmethod
    def backward(ctx, go, _gm, _gv):
        xc, wc, w2c, al, be, winners, y, mean, invstd, gamma = ctx.saved_tensors
        d, cnt = ctx.d, ctx.cnt
        dt = tconv.TORCH_DTYPE[d["dtype"]]
        go = go.float()
        yf = y.float()
        sum_go = go.sum(dim=(0, 2, 3))
        sum_go_y = (go * yf).sum(dim=(0, 2, 3))
        sum_go_xmu = sum_go_y - mean * sum_go
        g_gamma = sum_go_xmu * invstd
        g_bias = sum_go
        # dy = gamma * invstd * (go - sum_go / cnt - (y - mean) * invstd^2 * sum_go_xmu / cnt)
        k1 = (gamma * invstd).view(1, -1, 1, 1)
        k2 = (invstd * invstd * sum_go_xmu / cnt).view(1, -1, 1, 1)
        k3 = (sum_go / cnt - mean * invstd * invstd * sum_go_xmu / cnt).view(1, -1, 1, 1)
        gy = (k1 * (go - yf * k2 - k3)).to(dt).contiguous()
        ev = TropicalConvFn.events
        if ev is not None:
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
        need = ["grad_w", "grad_w2", "grad_alpha", "grad_beta"]
        if ctx.needs_input_grad[0]:
            need.append("grad_x")
        try:
            grads = tconv.backward(d, xc, wc, gy, w2c, al, be, winners, need=tuple(need))
        except tconv.TconvError as err:
            if d.get("x_dtype") != "f32" or err.status != -2:
                raise
            d = {k: v for k, v in d.items() if k != "x_dtype"}
            grads = tconv.backward(d, xc.to(dt), wc, gy, w2c, al, be, winners, need=tuple(need))
        if ev is not None:
            e1.record()
            ev.append(("bwd", d, e0, e1))
        has_w2, has_a, has_b = ctx.has
        gx = grads["grad_x"].to(ctx.in_dtype) if "grad_x" in grads else None
        return (gx, grads["grad_w"], grads.get("grad_w2") if has_w2 else None,
                grads.get("grad_alpha") if has_a else None, grads.get("grad_beta") if has_b else None,
                g_gamma, g_bias, None, None)


def tropical_conv_bn(conv: "TropicalConv2d", bn: nn.BatchNorm2d, x):
    """conv followed by bn; in training mode with the layer's fused channel statistics."""
    if not (bn.training and x.is_cuda and conv.bias is None and bn.affine and bn.track_running_stats
            and conv.params in ("2p", "0p") and conv.checkpoint is None and type(conv) is TropicalConv2d):
        return bn(conv(x))
    geom = (conv.mode, conv.chan, conv.dtype, conv.stride, conv.padding, conv.dilation)
    out, mean, var = TropicalConvBNFn.apply(x, conv.weight, conv.weight2, conv.alpha, conv.beta, bn.weight, bn.bias,
                                            geom, bn.eps)
    with torch.no_grad():
        cnt = out.shape[0] * out.shape[2] * out.shape[3]
        m = bn.momentum if bn.momentum is not None else 0.1
        bn.running_mean.mul_(1 - m).add_(mean, alpha=m)
        bn.running_var.mul_(1 - m).add_(var * (cnt / max(cnt - 1, 1)), alpha=m)
        bn.num_batches_tracked += 1
    return out


class TropicalConv2d(nn.Module):
    """Tropical convolution layer with ``nn.Conv2d``'s constructor arguments.

    mode: "max_plus" | "min_plus" | "compound" | "parallel"; chan: "default" | "sum" | "max" | "min".
    params (compound / parallel; the paper's section "Specializations of compound/parallel tropical convolutions"): "2p" learnable alpha and beta
    per (c_out, c_in); "1p" complementary weights beta = 1 - alpha; "shared" beta = alpha;
    "opposite" beta = -alpha; "0p" alpha = beta = 1 (no scalars); "fixed" the constants
    ``fixed=(alpha, beta)``, e.g. (0.5, 0.5) or (1, -1), held as buffers.
    dtype: arithmetic type of the kernels ("f32" or "bf16"); parameters stay fp32.
    checkpoint="q8": the backward pass keeps the input in 8 bits (see Q8) in place of the tensor itself.  It is read for
    the gradients of alpha and beta alone, which are then those over the restored input; all others are the same.  Where
    neither learns (max_plus, min_plus, "0p", "fixed", frozen scalars) nothing of the input is kept.
    forward's `stored` is the input's Q8 where it is there already (rms_norm's second output)."""

    PARAMS = ("0p", "1p", "2p", "shared", "opposite", "fixed")
    ND = 2          # spatial dimensions
    KIND = "dense"
    checkpoint = None

    def __init__(self, in_channels, out_channels, kernel_size, stride=1, padding=0, dilation=1,
                 bias=True, mode="compound", chan="default", params="2p", dtype="f32", fixed=(0.5, 0.5), checkpoint=None):
        super().__init__()
        _kept(checkpoint)
        self.checkpoint = checkpoint
        two = lambda v: (v,) * self.ND if isinstance(v, int) else tuple(v)
        self.kernel_size, self.stride, self.padding, self.dilation = map(two, (kernel_size, stride, padding, dilation))
        self.in_channels, self.out_channels = in_channels, out_channels
        self.mode, self.chan, self.params, self.dtype = mode, chan, params, dtype
        self.weight = nn.Parameter(torch.empty(out_channels, in_channels, *self.kernel_size))
        self.weight2 = nn.Parameter(torch.empty(out_channels, in_channels, *self.kernel_size)) if mode == "parallel" else None
        two_branch = mode in ("compound", "parallel")
        if params not in self.PARAMS:
            raise ValueError(f"params must be one of {self.PARAMS}")
        learn_a = two_branch and params in ("1p", "2p", "shared", "opposite")
        self.alpha = nn.Parameter(torch.empty(out_channels, in_channels)) if learn_a else None
        self.beta = nn.Parameter(torch.empty(out_channels, in_channels)) if two_branch and params == "2p" else None
        if two_branch and params == "fixed":
            self.register_buffer("alpha_fixed", torch.full((out_channels, in_channels), float(fixed[0])))
            self.register_buffer("beta_fixed", torch.full((out_channels, in_channels), float(fixed[1])))
        self.bias = nn.Parameter(torch.zeros(out_channels)) if bias else None
        self.reset_parameters()

    def reset_parameters(self):
        fan_in = self.in_channels * math.prod(self.kernel_size)
        bound = 1.0 / math.sqrt(fan_in)
        for w in (self.weight, self.weight2):
            if w is not None:
                nn.init.uniform_(w, -bound, bound)
        # the paper gives no initial values for alpha / beta: start from the normalised average of
        # the two branches divided by the fan-in of the channel sum
        for a in (self.alpha, self.beta):
            if a is not None:
                nn.init.constant_(a, 0.5 / self.in_channels)

    def extra_repr(self):
        return (f"{self.in_channels}, {self.out_channels}, kernel_size={self.kernel_size}, stride={self.stride}, "
                f"padding={self.padding}, dilation={self.dilation}, mode={self.mode}, chan={self.chan}, "
                f"params={self.params}, dtype={self.dtype}" + (f", checkpoint={self.checkpoint}" if self.checkpoint else ""))

    def forward(self, x, stored=None):
        alpha, beta = self.alpha, self.beta
        if self.mode in ("compound", "parallel"):
            if self.params == "1p":
                beta = 1.0 - alpha
            elif self.params == "shared":
                beta = alpha
            elif self.params == "opposite":
                beta = -alpha
            elif self.params == "fixed":
                alpha, beta = self.alpha_fixed, self.beta_fixed
        if self.KIND == "dense" and (TropicalConvFn.events is not None or TropicalConvFn.fuse_cast):
            if self.checkpoint is not None:
                raise ValueError("checkpoint='q8' goes with neither TropicalConvFn.events nor TropicalConvFn.fuse_cast")
            geom = (self.mode, self.chan, self.dtype, self.stride, self.padding, self.dilation, torch.is_grad_enabled())
            return TropicalConvFn.apply(x, self.weight, self.weight2, alpha, beta, self.bias, geom)
        return _layer(self.KIND, self.mode, self.chan, self.dtype, self.stride, self.padding, self.dilation, x,
                      self.weight, self.weight2, alpha, beta, self.bias, self.checkpoint, stored)


class TropicalBasicBlock(nn.Module):
    """The paper's TCNN basic block 2: Tropical - BN - Tropical - BN, intermediate ReLU removed,
    identity (or 1x1 standard-convolution) shortcut, ReLU after the sum."""

    def __init__(self, cin, cout, stride, mode, dtype, fused_bn=False):
        super().__init__()
        self.fused_bn = fused_bn    # batch-normalisation statistics from the tropical kernels' epilogue
        self.conv1 = TropicalConv2d(cin, cout, 3, stride=stride, padding=1, bias=False, mode=mode, dtype=dtype)
        self.bn1 = nn.BatchNorm2d(cout)
        self.conv2 = TropicalConv2d(cout, cout, 3, stride=1, padding=1, bias=False, mode=mode, dtype=dtype)
        self.bn2 = nn.BatchNorm2d(cout)
        self.down = None
        if stride != 1 or cin != cout:
            self.down = nn.Sequential(nn.Conv2d(cin, cout, 1, stride=stride, bias=False), nn.BatchNorm2d(cout))

    def forward(self, x):
        if self.fused_bn:
            out = tropical_conv_bn(self.conv2, self.bn2, tropical_conv_bn(self.conv1, self.bn1, x))
        else:
            out = self.bn2(self.conv2(self.bn1(self.conv1(x))))
        return torch.relu(out + (x if self.down is None else self.down(x)))


class StandardBasicBlock(nn.Module):
    def __init__(self, cin, cout, stride):
        super().__init__()
        self.conv1 = nn.Conv2d(cin, cout, 3, stride=stride, padding=1, bias=False)
        self.bn1 = nn.BatchNorm2d(cout)
        self.conv2 = nn.Conv2d(cout, cout, 3, padding=1, bias=False)
        self.bn2 = nn.BatchNorm2d(cout)

    def forward(self, x):
        return torch.relu(self.bn2(self.conv2(torch.relu(self.bn1(self.conv1(x))))) + x)


class HybridResNet18(nn.Module):
    """ResNet-18 shape; every 3x3 convolution of stages 2-4 is a tropical layer of the given mode
    (stem, stage 1 and the 1x1 downsamples are standard convolutions)."""

    def __init__(self, mode="compound", dtype="bf16", num_classes=1000, fused_bn=False):
        super().__init__()
        self.stem = nn.Sequential(nn.Conv2d(3, 64, 7, stride=2, padding=3, bias=False), nn.BatchNorm2d(64),
                                  nn.ReLU(inplace=True), nn.MaxPool2d(3, stride=2, padding=1))
        self.layer1 = nn.Sequential(StandardBasicBlock(64, 64, 1), StandardBasicBlock(64, 64, 1))
        self.layer2 = nn.Sequential(TropicalBasicBlock(64, 128, 2, mode, dtype, fused_bn), TropicalBasicBlock(128, 128, 1, mode, dtype, fused_bn))
        self.layer3 = nn.Sequential(TropicalBasicBlock(128, 256, 2, mode, dtype, fused_bn), TropicalBasicBlock(256, 256, 1, mode, dtype, fused_bn))
        self.layer4 = nn.Sequential(TropicalBasicBlock(256, 512, 2, mode, dtype, fused_bn), TropicalBasicBlock(512, 512, 1, mode, dtype, fused_bn))
        self.head = nn.Sequential(nn.AdaptiveAvgPool2d(1), nn.Flatten(), nn.Linear(512, num_classes))

    def forward(self, x):
        x = self.layer1(self.stem(x))
        x = self.layer4(self.layer3(self.layer2(x)))
        return self.head(x)

    def tropical_layers(self):
        return [m for m in self.modules() if isinstance(m, TropicalConv2d)]


class TropicalDepthwiseFn(torch.autograd.Function):
    """Depthwise (groups = C) form over tconv_dw_forward / tconv_dw_backward; see TropicalConvFn."""

    @staticmethod
    def forward(ctx, x, w, w2, alpha, beta, bias, geom):
        mode, dtype, stride, pad, dil = geom
        dt = tconv.TORCH_DTYPE[dtype]
        N, C, H, W = x.shape
        _, R, S = w.shape
        d = dict(N=N, C=C, H=H, W=W, K=C, R=R, S=S, stride_h=stride[0], stride_w=stride[1],
                 pad_h=pad[0], pad_w=pad[1], dil_h=dil[0], dil_w=dil[1], mode=mode, chan="sum", dtype=dtype)
        xc, wc, w2c = _as(x, dt), _as(w, dt), _as(w2, dt)
        al, be, bi = _as(alpha, torch.float32), _as(beta, torch.float32), _as(bias, torch.float32)
        y, winners = tconv.dw_forward(d, xc, wc, w2c, al, be, bi,
                                      want_winners=_emit_winners(True, x, w, w2, alpha, beta, bias))
        ctx.d, ctx.in_dtype = d, x.dtype
        ctx.save_for_backward(xc, wc, w2c, al, be, winners)
        ctx.has = (w2 is not None, alpha is not None, beta is not None, bias is not None)
        return y.to(x.dtype) if x.dtype != dt else y

    @staticmethod
    def backward(ctx, gy):
        xc, wc, w2c, al, be, winners = ctx.saved_tensors
        grads = tconv.dw_backward(ctx.d, xc, wc, _as(gy, tconv.TORCH_DTYPE[ctx.d["dtype"]]), w2c, al, be, winners)
        has_w2, has_a, has_b, has_bias = ctx.has
        return (grads["grad_x"].to(ctx.in_dtype), grads["grad_w"], grads.get("grad_w2") if has_w2 else None,
                grads.get("grad_alpha") if has_a else None, grads.get("grad_beta") if has_b else None,
                grads["grad_bias"] if has_bias else None, None)


class TropicalDepthwiseConv2d(nn.Module):
    """Depthwise tropical convolution (``nn.Conv2d(channels, channels, k, groups=channels)``'s place in
    a MobileNetV2 block): per channel one window of weights, one alpha and one beta.

    mode, params and checkpoint as in TropicalConv2d ("2p", "1p", "shared", "opposite", "0p", "fixed")."""

    checkpoint = None

    def __init__(self, channels, kernel_size, stride=1, padding=0, dilation=1, bias=True,
                 mode="compound", params="2p", dtype="f32", fixed=(0.5, 0.5), checkpoint=None):
        super().__init__()
        _kept(checkpoint)
        self.checkpoint = checkpoint
        two = lambda v: (v, v) if isinstance(v, int) else tuple(v)
        self.kernel_size, self.stride, self.padding, self.dilation = map(two, (kernel_size, stride, padding, dilation))
        self.channels, self.mode, self.params, self.dtype = channels, mode, params, dtype
        if params not in TropicalConv2d.PARAMS:
            raise ValueError(f"params must be one of {TropicalConv2d.PARAMS}")
        R, S = self.kernel_size
        self.weight = nn.Parameter(torch.empty(channels, R, S))
        self.weight2 = nn.Parameter(torch.empty(channels, R, S)) if mode == "parallel" else None
        two_branch = mode in ("compound", "parallel")
        self.alpha = nn.Parameter(torch.empty(channels)) if two_branch and params in ("1p", "2p", "shared", "opposite") else None
        self.beta = nn.Parameter(torch.empty(channels)) if two_branch and params == "2p" else None
        if two_branch and params == "fixed":
            self.register_buffer("alpha_fixed", torch.full((channels,), float(fixed[0])))
            self.register_buffer("beta_fixed", torch.full((channels,), float(fixed[1])))
        self.bias = nn.Parameter(torch.zeros(channels)) if bias else None
        bound = 1.0 / math.sqrt(R * S)
        for w in (self.weight, self.weight2):
            if w is not None:
                nn.init.uniform_(w, -bound, bound)
        for a in (self.alpha, self.beta):
            if a is not None:
                nn.init.constant_(a, 0.5)

    def extra_repr(self):
        return (f"{self.channels}, kernel_size={self.kernel_size}, stride={self.stride}, padding={self.padding}, "
                f"dilation={self.dilation}, mode={self.mode}, params={self.params}, dtype={self.dtype}" +
                (f", checkpoint={self.checkpoint}" if self.checkpoint else ""))

    def forward(self, x, stored=None):
        alpha, beta = self.alpha, self.beta
        if self.mode in ("compound", "parallel"):
            if self.params == "1p":
                beta = 1.0 - alpha
            elif self.params == "shared":
                beta = alpha
            elif self.params == "opposite":
                beta = -alpha
            elif self.params == "fixed":
                alpha, beta = self.alpha_fixed, self.beta_fixed
        return _layer("depthwise", self.mode, "sum", self.dtype, self.stride, self.padding, self.dilation, x, self.weight,
                      self.weight2, alpha, beta, self.bias, self.checkpoint, stored)


class TropicalConv3dFn(torch.autograd.Function):
    """y = tconv3d_forward(...); backward = tconv3d_backward with the stored winners; see TropicalConvFn."""

    @staticmethod
    def forward(ctx, x, w, w2, alpha, beta, bias, geom):
        mode, chan, dtype, stride, pad, dil = geom
        dt = tconv.TORCH_DTYPE[dtype]
        N, C, D, H, W = x.shape
        K, _, T, R, S = w.shape
        d = dict(N=N, C=C, D=D, H=H, W=W, K=K, T=T, R=R, S=S, stride=tuple(stride), pad=tuple(pad),
                 dil=tuple(dil), mode=mode, chan=chan, dtype=dtype)
        xc, wc, w2c = _as(x, dt), _as(w, dt), _as(w2, dt)
        al, be, bi = _as(alpha, torch.float32), _as(beta, torch.float32), _as(bias, torch.float32)
        y, winners = tconv3d.forward(d, xc, wc, w2c, al, be, bi,
                                     want_winners=_emit_winners(True, x, w, w2, alpha, beta, bias))
        ctx.d, ctx.in_dtype = d, x.dtype
        ctx.save_for_backward(xc, wc, w2c, al, be, winners)
        ctx.has = (w2 is not None, alpha is not None, beta is not None, bias is not None)
        return y.to(x.dtype) if x.dtype != dt else y

    @staticmethod
    def backward(ctx, gy):
        xc, wc, w2c, al, be, winners = ctx.saved_tensors
        grads = tconv3d.backward(ctx.d, xc, wc, _as(gy, tconv.TORCH_DTYPE[ctx.d["dtype"]]), w2c, al, be, winners,
                                 need_grad_x=ctx.needs_input_grad[0])
        has_w2, has_a, has_b, has_bias = ctx.has
        gx = grads["grad_x"].to(ctx.in_dtype) if "grad_x" in grads else None
        return (gx, grads["grad_w"], grads.get("grad_w2") if has_w2 else None,
                grads.get("grad_alpha") if has_a else None, grads.get("grad_beta") if has_b else None,
                grads["grad_bias"] if has_bias else None, None)


class TropicalConv3d(TropicalConv2d):
    """Three-dimensional tropical convolution (Section 3.2 and the Conv3d forms of Sections 3.4 / 3.5)
    with ``nn.Conv3d``'s constructor arguments; input [N, C, D, H, W]; mode / chan / params / dtype
    as in TropicalConv2d.  Windows of up to 256 taps (the paper's 3-D LeNet uses 5 x 5 x 5)."""

    ND = 3
    KIND = "volume"


class TropicalConv1d(nn.Module):
    """1-D tropical convolution (Section 3.2) with ``nn.Conv1d``'s constructor arguments; mode / chan /
    params / dtype / checkpoint as in TropicalConv2d.  The length-3, stride-1 layers run as 1 x 3 windows on a signal
    of unit height through the tiled 2-D kernels; every other window (up to 256 taps; the paper's audio
    networks open with length 80 at stride 4) goes as a 1 x 1 x k window through the three-dimensional
    entry points, which run windows of four taps or more at stride 1, 2 or 4 (no dilation) on their
    one-dimensional kernels and the rest on the any-shape kernels."""

    def __init__(self, in_channels, out_channels, kernel_size, stride=1, padding=0, dilation=1,
                 bias=True, mode="compound", chan="default", params="2p", dtype="f32", fixed=(0.5, 0.5), checkpoint=None):
        super().__init__()
        self.tiled = (kernel_size == 3 and stride == 1 and dilation == 1)
        if self.tiled:
            self.conv = TropicalConv2d(in_channels, out_channels, (1, kernel_size), stride=(1, stride),
                                       padding=(0, padding), dilation=(1, dilation), bias=bias, mode=mode,
                                       chan=chan, params=params, dtype=dtype, fixed=fixed, checkpoint=checkpoint)
        else:
            self.conv = TropicalConv3d(in_channels, out_channels, (1, 1, kernel_size), stride=(1, 1, stride),
                                       padding=(0, 0, padding), dilation=(1, 1, dilation), bias=bias, mode=mode,
                                       chan=chan, params=params, dtype=dtype, fixed=fixed, checkpoint=checkpoint)

    def forward(self, x, stored=None):         # x: [N, C, L]
        if self.tiled:
            return self.conv(x.unsqueeze(2), stored).squeeze(2)
        # (reshapes, not slices: the gradient of a slice would be written into a zeroed copy)
        N, C, L = x.shape
        y = self.conv(x.reshape(N, C, 1, 1, L), stored)
        return y.reshape(N, y.shape[1], y.shape[4])


class Q8(NamedTuple):
    """A tensor kept in 8 bits: blocks of 32 values along a row (what lies behind the channel axis; the channels where
    nothing does) share a power of two, the smallest 2^e, e >= -126, with every magnitude below 127.5 * 2^e; a value is
    code * 2^e, finite for every finite value: e is 121 at most, and magnitudes from 127.5 * 2^121 on restore to
    127 * 2^121.  A block with a NaN or an infinity restores to NaN.  codes: int8 [rows, inner rounded up to 8]; scales:
    uint8 [rows, blocks], e + 127."""
    codes: torch.Tensor
    scales: torch.Tensor
    shape: tuple
    dtype: torch.dtype

    def restore(self, dtype=None):
        """The values, in the type of the tensor that was stored or in `dtype` (float32, bfloat16; exact in both)."""
        return _native.q8_restore(self.codes, self.scales, self.shape, _q8_type(dtype or self.dtype))

    @property
    def nbytes(self):
        return self.codes.nbytes + self.scales.nbytes


_Q8_TYPES = {t: tconv.DTYPES[name] for name, t in tconv.TORCH_DTYPE.items()}


def _q8_type(dtype):
    if dtype not in _Q8_TYPES:
        raise ValueError(f"dtype: need float32 or bfloat16, got {dtype}")
    return _Q8_TYPES[dtype]


def _kept(checkpoint):
    if checkpoint not in (None, "q8"):
        raise ValueError(f"checkpoint must be None or 'q8', got {checkpoint!r}")
    return checkpoint == "q8"


def q8_store(x) -> Q8:
    """x (float32 or bfloat16, on the GPU) in 8 bits; no gradients."""
    codes, scales = _native.q8_store(x)
    return Q8(codes, scales, x.shape, x.dtype)


def gated_scan(x, gate=None, h0=None, lengths=None, checkpoint=None):
    """Gated linear recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t, f = sigmoid(gate), along the last axis of x [N, C, L].

    gate: [N, C, L], x's type; without it x is [N, 2C, L] and its second half holds the gates (the two halves of one
    convolution's output, read and differentiated in place).  h0: float32 [N, C], zero if absent.  lengths: integers
    [N]; from a row's length on y is zero and the state stays.  checkpoint="q8": what the backward pass needs of x and
    gate is kept in 8 bits (see Q8) and its gradients are those of the recurrence over the restored values; the
    forward is unchanged.  Returns y [N, C, L] and the last state, float32 [N, C]."""
    return _native.gated_scan(x, gate, h0, lengths, _kept(checkpoint))


def gated_scan_step(h, x, gate=None, out=None):
    """One position of gated_scan for streaming: state h float32 [N, C], x and gate [N, C] (or x [N, 2C] alone).
    Returns y and the new state, written to `out` if given, which may be h and shares no memory with x or gate.  Records
    no gradients."""
    return _native.gated_scan_step(h, x, gate, out)


class NormOutput(NamedTuple):
    y: Optional[torch.Tensor]
    stream: torch.Tensor
    q8: Optional[Q8]


_OUTPUTS = {"same": 0, "q8": 1, "both": 2}


def rms_norm(x, weight, residual=None, eps=1e-6, output="same", checkpoint=None) -> NormOutput:
    """Root-mean-square norm over the channels of x [N, C, ...] with the residual's addition: stream = x + residual
    (rounded to x's type; x itself without a residual), y = stream / sqrt(mean_c(stream^2) + eps) * weight[c].

    output: "same" (y), "q8" (y in 8 bits alone; no gradients) or "both".  checkpoint="q8": the backward pass keeps
    the stream in 8 bits (see Q8) in place of the tensor itself."""
    if output not in _OUTPUTS:
        raise ValueError(f"output must be one of {tuple(_OUTPUTS)}, got {output!r}")
    y, s, codes, scales = _native.rms_norm(x, weight, residual, eps, _OUTPUTS[output], _kept(checkpoint))
    return NormOutput(y, x if s is None else s, None if codes is None else Q8(codes, scales, x.shape, x.dtype))


class RMSNorm(nn.Module):
    """rms_norm over the channels with a learned weight.  forward(x) gives y; forward(x, residual) gives y and the new
    stream."""

    def __init__(self, channels, eps=1e-6, checkpoint=None):
        super().__init__()
        _kept(checkpoint)
        self.channels, self.eps, self.checkpoint = channels, eps, checkpoint
        self.weight = nn.Parameter(torch.ones(channels))

    def extra_repr(self):
        return f"{self.channels}, eps={self.eps}, checkpoint={self.checkpoint}"

    def forward(self, x, residual=None):
        r = rms_norm(x, self.weight, residual, self.eps, checkpoint=self.checkpoint)
        return r.y if residual is None else (r.y, r.stream)


class TropicalRecurrent1d(nn.Module):
    """Gated recurrence whose candidates and gates one tropical convolution gives: [N, C_in, L] to 2 * channels signals,
    the first half candidates, the second half gates, then gated_scan over them in place.  Takes TropicalConv1d's arguments.

    gate_bias: initial bias of the gates (with bias=True): a new layer's states decay by sigmoid(gate_bias) a step.
    checkpoint="q8": convolution and recurrence keep their inputs in 8 bits for the backward pass.
    forward(x, h0, lengths, stored) gives y [N, channels, L'] and the last state, float32 [N, channels]; lengths counts
    output positions (the convolution itself sees all of x), stored is x's Q8 where it is there already."""

    def __init__(self, in_channels, channels, kernel_size=3, stride=1, padding=1, dilation=1, bias=True, mode="compound",
                 chan="default", params="2p", dtype="f32", gate_bias=2.0, checkpoint=None):
        super().__init__()
        self.channels, self.checkpoint = channels, checkpoint
        self.conv = TropicalConv1d(in_channels, 2 * channels, kernel_size, stride, padding, dilation, bias, mode, chan,
                                   params, dtype, checkpoint=checkpoint)
        if bias:
            nn.init.constant_(self.conv.conv.bias[channels:], gate_bias)

    def forward(self, x, h0=None, lengths=None, stored=None):
        return gated_scan(self.conv(x, stored), None, h0, lengths, self.checkpoint)


class TropicalRecurrentBlock1d(nn.Module):
    """Residual block of a network over long signals: RMS norm of the stream, tropical recurrence, and its output's addition
    left to the next block's norm.  forward(x, residual=None) gives the branch and the stream, which the next block
    (or a last RMSNorm) takes as its x and residual; the first block takes its input as x.  checkpoint="q8": the stream,
    the convolution's input (as the norm's own 8-bit output, of y before it is rounded to x's type or the layer's) and the
    recurrence's are kept in 8 bits."""

    def __init__(self, channels, kernel_size=3, padding=1, mode="compound", params="2p", dtype="f32", eps=1e-6,
                 checkpoint=None):
        super().__init__()
        self.norm = RMSNorm(channels, eps, checkpoint)
        self.rec = TropicalRecurrent1d(channels, channels, kernel_size, padding=padding, mode=mode, params=params, dtype=dtype,
                                       checkpoint=checkpoint)

    def forward(self, x, residual=None, lengths=None):
        keep = self.norm.checkpoint is not None and torch.is_grad_enabled()
        n = rms_norm(x, self.norm.weight, residual, self.norm.eps, "both" if keep else "same", self.norm.checkpoint)
        y, _ = self.rec(n.y, None, lengths, n.q8)
        return y, n.stream
