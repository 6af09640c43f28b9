"""The library's sequence and storage operators as cases that can be timed and compared: the gated linear
recurrence over [N, C, L] signals, the root-mean-square norm over channels with the residual's addition, and
activations kept in 8 bits for the backward pass.

`run` computes them in plain torch operations, or through the library's public functions
(`paper_2504_06881_b200.nn`) where `own` is true.  Sizes follow the networks of the library's benchmark
configurations: audio signals of 16000 samples at stride 4, the feature maps of the ResNet-18-shaped, the
MobileNetV2-shaped and the segmentation network.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_EPS = 1e-6


# ---- cases ---------------------------------------------------------------------------------------------------
def _scan(name, direction, dtype, N, C, L, packed=False, checkpoint="", ragged=False):
    c = dict(op="scan", direction=direction, dtype=dtype, N=N, C=C, L=L, packed=packed, checkpoint=checkpoint,
             ragged=ragged)
    return dict(c, name=name) if name else c


def _norm(name, direction, dtype, N, C, H, W, residual=True, output="same", checkpoint=""):
    c = dict(op="norm", direction=direction, dtype=dtype, N=N, C=C, H=H, W=W, residual=residual, output=output,
             checkpoint=checkpoint)
    return dict(c, name=name) if name else c


def _store(name, dtype, N, C, H, W):
    c = dict(op="store", direction="train", dtype=dtype, N=N, C=C, H=H, W=W)
    return dict(c, name=name) if name else c


def listed():
    return [
        # eight live audio streams, one new sample each: the latency of the smallest call
        _scan("scan_step_f32", "step", "f32", 8, 128, 1),
        # recurrent layer behind the opening layer of an audio network (80 samples at stride 4 on 16000): candidates
        # and gates of one convolution, odd length
        _scan("scan_audio_train_bf16", "train", "bf16", 32, 128, 3981, packed=True),
        # the same layer in fp32 with padding to whole vectors, its inputs kept in 8 bits for the backward pass
        _scan("scan_audio_q8_train_f32", "train", "f32", 32, 128, 4000, checkpoint="q8"),
        # one long recording in a single pass: few rows, a long axis
        _scan("scan_long_infer_bf16", "infer", "bf16", 1, 24, 400001),
        # a wide layer over a ragged batch: the largest training pass
        _scan("scan_wide_train_bf16", "train", "bf16", 64, 256, 8192, ragged=True),
        # features of one image before the classifier, in 8 bits for what follows
        _norm("norm_features_q8_infer_bf16", "infer", "bf16", 1, 512, 1, 1, residual=False, output="q8"),
        # residual stream of the audio network, odd length
        _norm("norm_audio_train_f32", "train", "f32", 32, 128, 1, 3981),
        # last stage of the ResNet-18-shaped network: 7x7 maps, the stream kept in 8 bits for the backward pass
        _norm("norm_last_stage_q8_train_bf16", "train", "bf16", 64, 512, 7, 7, checkpoint="q8"),
        # segmentation-scale maps: the normalised map and its 8-bit form for the next layer's backward pass
        _norm("norm_segmentation_train_bf16", "train", "bf16", 8, 256, 128, 256, output="both"),
        # two RGB images kept in 8 bits and restored: the smallest store
        _store("store_small_rgb_f32", "f32", 2, 3, 32, 32),
        # MobileNetV2's expanded 24-channel stage, a training batch
        _store("store_mobilenet_f32", "f32", 128, 144, 56, 56),
        # ImageNet-scale maps with odd rows: 7x7, the whole training batch of a wide last stage
        _store("store_last_stage_bf16", "bf16", 256, 512, 7, 7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges, odd and ragged sizes among them, no dearer than the largest listed."""
    op = rng.choices(["scan", "norm", "store"], [4, 3, 2])[0]
    dtype = rng.choice(["f32", "bf16"])
    cap = 6e7 if dtype == "f32" else 1.2e8
    if op == "scan":
        direction = rng.choices(["train", "infer", "step"], [5, 3, 1])[0]
        if direction == "step":
            return _scan(None, "step", dtype, _log_int(rng, 1, 512), _log_int(rng, 1, 512), 1, packed=rng.random() < 0.5)
        if rng.random() < 0.25:
            N, C, L = 1, _log_int(rng, 1, 32), _log_int(rng, 4000, 400000)
        else:
            N, C, L = _log_int(rng, 1, 64), _log_int(rng, 4, 256), _log_int(rng, 1, 16000)
        N = max(1, min(N, int(cap / (C * L))))
        return _scan(None, direction, dtype, N, C, L, packed=rng.random() < 0.5,
                     checkpoint="q8" if direction == "train" and rng.random() < 0.4 else "", ragged=rng.random() < 0.3)
    cap /= 2
    if op == "norm":
        direction = rng.choices(["train", "infer"], [3, 2])[0]
        N, C = _log_int(rng, 1, 128), _log_int(rng, 4, 1024)
        kind = rng.choice(["map", "signal", "features"])
        H, W = 1, 1
        if kind == "map":
            H = _log_int(rng, 4, 128)
            W = min(256, max(4, int(H * rng.uniform(0.7, 2.0))))
        elif kind == "signal":
            W = _log_int(rng, 16, 16000)
        N = max(1, min(N, int(cap / (C * H * W))))
        output = rng.choice(["same", "both"] if direction == "train" else ["same", "both", "q8"])
        return _norm(None, direction, dtype, N, C, H, W, residual=rng.random() < 0.7, output=output,
                     checkpoint="q8" if direction == "train" and rng.random() < 0.4 else "")
    N, C, H = _log_int(rng, 1, 256), _log_int(rng, 1, 512), _log_int(rng, 2, 128)
    W = min(256, max(2, int(H * rng.uniform(0.7, 2.0))))
    return _store(None, dtype, max(1, min(N, int(cap / (C * H * W)))), C, H, W)


# ---- inputs --------------------------------------------------------------------------------------------------
def prepare(case, seed):
    """Activations of a normalised network, gates whose channels remember from a few to some hundred steps, and
    upstream gradients."""
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _DT[c["dtype"]]
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    rand = lambda *s: torch.rand(*s, device="cuda", generator=gen)
    state = {"case": dict(c)}
    N, C = c["N"], c["C"]
    train = c["direction"] == "train"
    if c["op"] == "scan":
        L = c["L"]
        x = randn(N, C, L).to(dt)
        g = (randn(N, C, L) + 5 * rand(1, C, 1)).to(dt)
        if c["direction"] == "step":
            x, g = x[:, :, 0].contiguous(), g[:, :, 0].contiguous()
        state["inputs"] = [torch.cat([x, g], 1)] if c["packed"] else [x, g]
        state["h0"] = randn(N, C) * 0.5
        if c["ragged"]:
            lengths = (rand(N) * (L + 1)).to(torch.int32).clamp_(max=L)
            lengths[0] = L
            state["lengths"] = lengths
        if train:
            state["gy"], state["gh"] = randn(N, C, L).to(dt), randn(N, C)
            for t in state["inputs"] + [state["h0"]]:
                t.requires_grad_(True)
        return state
    shape = (N, C) if c["H"] * c["W"] == 1 else (N, C, c["W"]) if c["H"] == 1 else (N, C, c["H"], c["W"])
    x = randn(*shape)
    if c["op"] == "store":
        state["x"] = x.relu_().to(dt)
        return state
    state["x"] = x.to(dt)
    state["weight"] = 1 + 0.2 * randn(C)
    if c["residual"]:
        state["residual"] = (2 * randn(*shape)).to(dt)
    if train:
        state["gy"] = randn(*shape).to(dt)
        if c["residual"]:
            state["gs"] = randn(*shape).to(dt)
        for k in ("x", "weight", "residual"):
            if k in state:
                state[k].requires_grad_(True)
    return state


# ---- plain forms ---------------------------------------------------------------------------------------------
def _rows(t):
    """[rows, inner]: a row is what lies behind the channel axis, or the channels where nothing does."""
    inner = math.prod(t.shape[2:])
    return t.reshape(-1, inner) if inner > 1 else t.reshape(t.shape[0], -1)


def _q8(t):
    """The values that t's 8-bit form stands for, in 32 bits: blocks of 32 along a row share the smallest power of
    two 2^e, e >= -126, with every magnitude below 127.5 * 2^e."""
    r = _rows(t.float())
    rows, inner = r.shape
    nb = -(-inner // 32)
    b = torch.zeros(rows, nb * 32, dtype=torch.float32, device=r.device)
    b[:, :inner] = r
    b = b.view(rows, nb, 32)
    m, k = torch.frexp(b.abs().amax(-1, keepdim=True))        # amax = m 2^k, 0.5 <= m < 1
    e = (k - 7 + (m >= 127.5 / 128).int()).clamp(min=-126)
    e = torch.where(m == 0, -126, e)
    up, down = (((e + 127) << 23).view(torch.float32), ((127 - e) << 23).view(torch.float32))
    q = torch.round(b * down) * up
    return q.view(rows, -1)[:, :inner].reshape(t.shape)


def _linear_scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the last axis from zero, in log2(L) doublings."""
    k, L = 1, a.shape[-1]
    while k < L:
        b = torch.cat([b[..., :k], b[..., k:] + a[..., k:] * b[..., :-k]], -1)
        a = torch.cat([a[..., :k], a[..., k:] * a[..., :-k]], -1)
        k *= 2
    return b


def _before(h, h0):
    """h_{t-1} for every t."""
    return torch.cat([h0.unsqueeze(-1), h[..., :-1]], -1)


def _gates(x, g, live):
    f, u = torch.sigmoid(g), torch.sigmoid(-g)
    if live is not None:                                      # outside its length a row keeps its state
        f, u, x = (torch.where(live, t, v) for t, v in ((f, 1.0), (u, 0.0), (x, 0.0)))
    return x, f, u


def _recur(x, f, u, h0):
    b = u * x
    b = torch.cat([b[..., :1] + f[..., :1] * h0.unsqueeze(-1), b[..., 1:]], -1)
    return _linear_scan(f, b)


def _plain_scan(s):
    c = s["case"]
    N, C, L = c["N"], c["C"], c["L"]
    with torch.no_grad():
        x, g = (t.float() for t in (s["inputs"][0].split(C, 1) if c["packed"] else s["inputs"]))
        if c["direction"] == "step":
            f, u = torch.sigmoid(g), torch.sigmoid(-g)
            h = f * s["h0"] + u * x
            return h.to(_DT[c["dtype"]]), h
        h0 = s["h0"]
        live = None
        if c["ragged"]:
            live = (torch.arange(L, device=x.device) < s["lengths"].view(N, 1, 1))
        xm, f, u = _gates(x, g, live)
        h = _recur(xm, f, u, h0)
        y = (h if live is None else torch.where(live, h, 0.0)).to(_DT[c["dtype"]])
        last = h[..., -1].clone()
        if c["direction"] == "infer":
            return y, last
        del h
        if c["checkpoint"] == "q8":                           # the backward pass sees what was kept
            if live is not None:
                x, g = torch.where(live, x, 0.0), torch.where(live, g, 0.0)
            xm, f, u = _gates(_q8(x), _q8(g), live)
        del x, g
        d = s["gy"].float()
        if live is not None:
            d = torch.where(live, d, 0.0)
        d = torch.cat([d[..., :-1], d[..., -1:] + s["gh"].unsqueeze(-1)], -1)
        fn = torch.cat([f[..., 1:], torch.ones_like(f[..., :1])], -1)
        d = _linear_scan(fn.flip(-1), d.flip(-1)).flip(-1)
        gh0 = f[..., 0] * d[..., 0]
        prev = _before(_recur(xm, f, u, h0), h0)
        gx, gg = u * d, d * (prev - xm) * f * u
        if live is not None:
            gx, gg = torch.where(live, gx, 0.0), torch.where(live, gg, 0.0)
        gx, gg = gx.to(y.dtype), gg.to(y.dtype)
        return (y, last) + ((torch.cat([gx, gg], 1),) if c["packed"] else (gx, gg)) + (gh0,)


def _per_channel(w, t):
    return w.view((1, -1) + (1,) * (t.dim() - 2))


def _plain_norm(s):
    c = s["case"]
    dt = _DT[c["dtype"]]
    with torch.no_grad():
        x, w = s["x"].float(), s["weight"]
        stream = (x + s["residual"].float()).to(dt) if c["residual"] else s["x"].detach()
        v = stream.float()
        rstd = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + _EPS)
        y = v * rstd * _per_channel(w, v)
        out = {}
        if c["output"] != "q8":
            out["y"] = y.to(dt)
        if c["residual"]:
            out["stream"] = stream
        if c["output"] != "same":
            out["q8"] = _q8(y).to(torch.bfloat16)
        if c["direction"] == "infer":
            return out
        z = (_q8(v) if c["checkpoint"] == "q8" else v) * rstd
        gy = s["gy"].float()
        wd = _per_channel(w, v) * gy
        ds = rstd * (wd - z * (wd * z).mean(1, keepdim=True))
        if c["residual"]:
            ds = ds + s["gs"].float()
            out["grad_residual"] = ds.to(dt)
        out["grad_x"] = ds.to(dt)
        out["grad_weight"] = (gy * z).sum([d for d in range(v.dim()) if d != 1])
        return out


def _plain_store(s):
    return _q8(s["x"]).to(s["x"].dtype)


# ---- the library's calls -------------------------------------------------------------------------------------
def _own_scan(s):
    from paper_2504_06881_b200 import nn as tnn
    c = s["case"]
    if c["direction"] == "step":
        return tnn.gated_scan_step(s["h0"], *s["inputs"])
    if c["direction"] == "infer":
        with torch.no_grad():
            return tnn.gated_scan(*s["inputs"], h0=s["h0"], lengths=s.get("lengths"))
    y, last = tnn.gated_scan(*s["inputs"], h0=s["h0"], lengths=s.get("lengths"), checkpoint=c["checkpoint"] or None)
    grads = torch.autograd.grad((y, last), s["inputs"] + [s["h0"]], (s["gy"], s["gh"]))
    return (y.detach(), last.detach()) + grads


def _own_norm(s):
    from paper_2504_06881_b200 import nn as tnn
    c = s["case"]
    args = dict(residual=s.get("residual"), eps=_EPS, output=c["output"])
    out = {}
    if c["direction"] == "infer":
        with torch.no_grad():
            r = tnn.rms_norm(s["x"], s["weight"], **args)
    else:
        r = tnn.rms_norm(s["x"], s["weight"], checkpoint=c["checkpoint"] or None, **args)
    if r.y is not None:
        out["y"] = r.y.detach()
    if c["residual"]:
        out["stream"] = r.stream.detach()
    if r.q8 is not None:
        out["q8"] = r.q8.restore(torch.bfloat16)
    if c["direction"] == "train":
        if c["residual"]:
            out["grad_x"], out["grad_weight"], out["grad_residual"] = torch.autograd.grad(
                (r.y, r.stream), (s["x"], s["weight"], s["residual"]), (s["gy"], s["gs"]))
        else:
            out["grad_x"], out["grad_weight"] = torch.autograd.grad(r.y, (s["x"], s["weight"]), s["gy"])
    return out


def _own_store(s):
    from paper_2504_06881_b200 import nn as tnn
    return tnn.q8_store(s["x"]).restore()


def run(state):
    """Scan: y, the last state and, in training, the gradients of the inputs and of the first state.  Norm: y, the
    residual stream, the values of the 8-bit output and the gradients.  Store: the restored values."""
    op = state["case"]["op"]
    if own:
        return {"scan": _own_scan, "norm": _own_norm, "store": _own_store}[op](state)
    return {"scan": _plain_scan, "norm": _plain_norm, "store": _plain_store}[op](state)


# ---- work ----------------------------------------------------------------------------------------------------
def work(case):
    """Bytes: every input read once, every output written once; what is kept in 8 bits for the backward pass
    written once and read once.  Operations: counted from the formulas, a sigmoid as four."""
    c = case
    es = _BYTES[c["dtype"]]
    kept = lambda n: 2 * n * (1 + 1 / 32)
    if c["op"] == "scan":
        n, rows = c["N"] * c["C"] * c["L"], c["N"] * c["C"]
        nbytes, ops = 3 * n * es + 8 * rows, 8 * n
        if c["direction"] == "train":
            nbytes += 3 * n * es + 8 * rows + (kept(2 * n) if c["checkpoint"] else 0)
            ops += 18 * n
        return {"bytes": nbytes, "flops": ops}
    n = c["N"] * c["C"] * c["H"] * c["W"]
    if c["op"] == "store":
        return {"bytes": 2 * n * es + kept(n), "flops": 5 * n}
    res = c["residual"]
    nbytes = n * es * (1 + (2 if res else 0) + (c["output"] != "q8")) + 4 * c["C"]
    ops = n * (4 + res)
    if c["output"] != "same":
        nbytes += kept(n) + 2 * n
        ops += 5 * n
    if c["direction"] == "train":
        nbytes += n * es * (2 + (2 if res else 0)) + 4 * c["C"] + (kept(n) if c["checkpoint"] else 0)
        ops += n * (10 + res)
    return {"bytes": nbytes, "flops": ops}


# ---- 64-bit values -------------------------------------------------------------------------------------------
def _exact_q8(t):
    v = t.double()
    flat = v.reshape(v.shape[0], -1) if math.prod(v.shape[2:]) == 1 else v.reshape(v.shape[0] * v.shape[1], -1)
    rows, inner = flat.shape
    nb = (inner + 31) // 32
    b = torch.nn.functional.pad(flat, (0, nb * 32 - inner)).reshape(rows * nb, 32)
    top = b.abs().max(1).values.clamp(min=2.0 ** -300)
    two = lambda e: ((e.long() + 1023) << 52).view(torch.float64)      # 2^e itself: halves have to stay halves
    e = torch.ceil(torch.log2(top / 127.5)).clamp(min=-126)
    e = torch.where(top >= 127.5 * two(e), e + 1, e)
    e = torch.where((e > -126) & (top < 127.5 * two(e - 1)), e - 1, e)
    unit = two(e).unsqueeze(1)
    return (torch.round(b / unit) * unit).reshape(rows, nb * 32)[:, :inner].reshape(t.shape)


def _exact_recurrence(a, b, h0):
    """h_t = a_t h_{t-1} + b_t from h0, rows [R, L]: step by step inside blocks, all blocks of all rows at once, then
    block by block."""
    R, L = a.shape
    T = max(1, int(math.sqrt(L)))
    P = -(-L // T)
    pad = P * T - L
    A = torch.nn.functional.pad(a, (0, pad), value=1.0).view(R, P, T).permute(2, 0, 1).contiguous()
    B = torch.nn.functional.pad(b, (0, pad), value=0.0).view(R, P, T).permute(2, 0, 1).contiguous()
    for t in range(1, T):
        B[t].addcmul_(A[t], B[t - 1])
        A[t].mul_(A[t - 1])
    start, h = [], h0
    for p in range(P):
        start.append(h)
        h = A[-1, :, p] * h + B[-1, :, p]
    B += A * torch.stack(start, 1).unsqueeze(0)
    return B.permute(1, 2, 0).reshape(R, P * T)[:, :L]


def _exact_scan(s):
    c = s["case"]
    N, C, L = c["N"], c["C"], c["L"]
    x, g = (s["inputs"][0][:, :C], s["inputs"][0][:, C:]) if c["packed"] else s["inputs"]
    x, g, h0 = x.detach().reshape(N * C, L), g.detach().reshape(N * C, L), s["h0"].detach().double().reshape(N * C)
    n = s["lengths"].long().repeat_interleave(C) if c["ragged"] else torch.full((N * C,), L, device=x.device)
    inside = torch.arange(L, device=x.device).unsqueeze(0) < n.unsqueeze(1)

    def forward(x, g):
        e = torch.exp(-g.double().abs())
        small, large = e / (1 + e), 1 / (1 + e)
        f = torch.where(g >= 0, large, small).masked_fill_(~inside, 1.0)
        u = torch.where(g >= 0, small, large).masked_fill_(~inside, 0.0)
        x = x.double().masked_fill(~inside, 0.0)
        return x, f, u, _exact_recurrence(f, u * x, h0)

    xv, f, u, h = forward(x, g)
    shape = (N, C, L)
    last = h[:, -1].reshape(N, C).clone()
    if c["direction"] == "step":
        return last, last
    y = h.masked_fill(~inside, 0.0).reshape(shape)
    if c["direction"] == "infer":
        return y, last
    if c["checkpoint"] == "q8":
        kept = [_exact_q8(t.masked_fill(~inside, 0.0).reshape(shape)).reshape(N * C, L) for t in (x, g)]
        xv, f, u, h = forward(*kept)
    gy = s["gy"].double().reshape(N * C, L).masked_fill(~inside, 0.0)
    after = torch.cat([f[:, 1:], torch.ones_like(f[:, :1])], 1)
    d = _exact_recurrence(after.flip(1), gy.flip(1), s["gh"].double().reshape(N * C)).flip(1)
    gh0 = (f[:, 0] * d[:, 0]).reshape(N, C)
    h = torch.cat([h0.unsqueeze(1), h[:, :-1]], 1)
    gg = (d * (h - xv) * f * u).masked_fill_(~inside, 0.0).reshape(shape)
    gx = (u * d).masked_fill_(~inside, 0.0).reshape(shape)
    return (y, last) + ((torch.cat([gx, gg], 1),) if c["packed"] else (gx, gg)) + (gh0,)


def _exact_norm(s):
    c = s["case"]
    x = s["x"].detach()
    if c["residual"]:
        x = (x.double() + s["residual"].detach().double()).to(x.dtype)     # the stream in its own type
    N, C = x.shape[:2]
    v = x.double().reshape(N, C, -1)
    w = s["weight"].detach().double()
    r = torch.rsqrt(v.square().sum(1) / C + _EPS).unsqueeze(1)
    y = torch.einsum("ncp,c->ncp", v * r, w)
    out = {}
    if c["output"] != "q8":
        out["y"] = y.reshape(x.shape)
    if c["residual"]:
        out["stream"] = x.double()
    if c["output"] != "same":
        out["q8"] = _exact_q8(y.reshape(x.shape))
    if c["direction"] == "infer":
        return out
    if c["checkpoint"] == "q8":
        v = _exact_q8(x).reshape(N, C, -1)
    gy = s["gy"].double().reshape(N, C, -1)
    dot = torch.einsum("ncp,ncp,c->np", gy, v, w).unsqueeze(1)
    ds = gy * w.view(1, C, 1) * r - v * r.pow(3) * dot / C
    if c["residual"]:
        ds = ds + s["gs"].double().reshape(N, C, -1)
        out["grad_residual"] = ds.reshape(x.shape)
    out["grad_x"] = ds.reshape(x.shape)
    out["grad_weight"] = torch.einsum("ncp,ncp,np->c", gy, v, r.squeeze(1))
    return out


def exact(case, seed):
    """run()'s outputs from the definitions in 64 bits."""
    with torch.no_grad():
        s = prepare(case, seed)
        if case["op"] == "scan":
            return _exact_scan(s)
        if case["op"] == "norm":
            return _exact_norm(s)
        return _exact_q8(s["x"])
