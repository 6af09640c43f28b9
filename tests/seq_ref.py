"""Plain 64-bit forms of the sequence and storage operators, and how far a kernel in 32 bits may be from them.

Each reference returns values and, for every value, an absolute bound, from first-order error analysis:
EPS = 2^-24 is half a step of fp32.  __expf(g) is off by at most 2 + 1.173 |g| steps (its documented bound), a
division by __fdividef by 2 steps, every other operation by half a step."""
import numpy as np

EPS = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}     # half a step, relative: the rounding of an output


def q8(x, rows, inner):
    """(codes [rows, inner], scale bytes [rows, blocks], values) of a float array."""
    v = np.asarray(x, np.float64).reshape(rows, inner)
    nb = -(-inner // 32)
    codes, scales, vals = np.zeros((rows, inner), np.int64), np.zeros((rows, nb), np.int64), np.empty((rows, inner))
    for b in range(nb):
        blk = v[:, b * 32:(b + 1) * 32]
        top = np.abs(blk).max(1)
        ok = np.isfinite(top)
        e = np.full(rows, -126, np.int64)
        for r in np.nonzero(ok & (top > 0))[0]:
            k = int(np.floor(np.log2(top[r]))) - 8                      # a start below, then up to the smallest
            while top[r] >= 127.5 * 2.0 ** k:
                k += 1
            e[r] = max(k, -126)
        unit = 2.0 ** e.astype(np.float64)
        with np.errstate(invalid="ignore", over="ignore"):
            c = np.where(ok[:, None], np.rint(blk / unit[:, None]), 0.0)
        codes[:, b * 32:(b + 1) * 32] = c
        scales[:, b] = np.where(ok, e + 127, 255)
        vals[:, b * 32:(b + 1) * 32] = np.where(ok[:, None], c * unit[:, None], np.nan)
    return codes, scales, vals


def gates(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1, e) / (1 + e), np.where(g >= 0, e, 1) / (1 + e)


def _recur(f, b, h0):
    h = np.empty_like(b)
    cur = h0
    for t in range(b.shape[-1]):
        cur = f[..., t] * cur + b[..., t]
        h[..., t] = cur
    return h


def scan(x, g, h0=None, lengths=None, gy=None, gh=None, keep=None, dtype="f32"):
    """dict name -> (value, bound).  x, g [N, C, L]; keep: True = the backward sees the 8-bit forms of x and g."""
    x, g = np.asarray(x, np.float64), np.asarray(g, np.float64)
    N, C, L = x.shape
    h0 = np.zeros((N, C)) if h0 is None else np.asarray(h0, np.float64)
    n = np.full(N, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)
    live = np.broadcast_to(np.arange(L) < n[:, None, None], x.shape)

    def forward(x, g):
        xv, gv = np.where(live, x, 0.0), np.where(live, g, 0.0)
        f, u = gates(gv)
        f, u = np.where(live, f, 1.0), np.where(live, u, 0.0)
        h = _recur(f, u * xv, h0)
        habs = _recur(f, u * np.abs(xv), np.abs(h0))
        # relative error of e^-g, of which f has the share u and u the share f, and their own roundings
        de = (2 + 1.2 * np.abs(gv)) * 2 * EPS + EPS
        du = np.where(live, f * de + 8 * EPS, 0.0)
        df = np.where(live, u * de + 6 * EPS, 0.0)
        # error of h: first order, and 8 roundings a step in whatever order the products are joined
        before = np.concatenate([np.abs(h0)[..., None], habs[..., :-1]], -1)
        eh = _recur(f, u * np.abs(xv) * du + f * before * df + 8 * EPS * habs, np.zeros((N, C))) + 16 * EPS * habs
        return xv, f, u, h, eh, df, du

    xv, f, u, h, eh, df, du = forward(x, g)
    out = {"y": (np.where(live, h, 0.0), np.where(live, eh + HALF[dtype] * (np.abs(h) + eh), 0.0)),
           "h_last": (h[..., -1], eh[..., -1] + EPS * np.abs(h[..., -1]))}
    if gy is None:
        return out
    if keep:
        xv, gv = (q8(np.where(live, t, 0.0), N * C, L)[2].reshape(x.shape) for t in (x, g))
        xv, f, u, h, eh, df, du = forward(xv, gv)
    gy = np.where(live, np.asarray(gy, np.float64), 0.0)
    gh = np.zeros((N, C)) if gh is None else np.asarray(gh, np.float64)
    rev = lambda a: a[..., ::-1]
    fn = np.concatenate([f[..., 1:], np.ones((N, C, 1))], -1)
    dfn = np.concatenate([df[..., 1:], np.zeros((N, C, 1))], -1)
    last = lambda a, v: np.concatenate([a[..., :-1], a[..., -1:] + v[..., None]], -1)
    # (the share of D_t that comes from behind is f_{t+1} times what is there)
    D = rev(_recur(rev(fn), rev(last(gy, gh)), np.zeros((N, C))))
    Dabs = rev(_recur(rev(fn), rev(last(np.abs(gy), np.abs(gh))), np.zeros((N, C))))
    after = np.concatenate([Dabs[..., 1:], np.zeros((N, C, 1))], -1)
    eD = rev(_recur(rev(fn), rev(fn * after * dfn + 8 * EPS * Dabs), np.zeros((N, C)))) + 16 * EPS * Dabs
    prev = np.concatenate([h0[..., None], h[..., :-1]], -1)
    eprev = np.concatenate([np.zeros((N, C, 1)), eh[..., :-1]], -1) + EPS * np.abs(prev)
    gx = u * D
    ex = u * (eD + np.abs(D) * (du + 2 * EPS))
    gg = D * (prev - xv) * f * u
    k = f * u
    eg = k * (eD * np.abs(prev - xv) + np.abs(D) * (eprev + EPS * (np.abs(prev) + np.abs(xv)))) + np.abs(gg) * (df + du + 6 * EPS)
    out["grad_x"] = (np.where(live, gx, 0.0), np.where(live, ex + HALF[dtype] * (np.abs(gx) + ex), 0.0))
    out["grad_gate"] = (np.where(live, gg, 0.0), np.where(live, eg + HALF[dtype] * (np.abs(gg) + eg), 0.0))
    out["grad_h0"] = (f[..., 0] * D[..., 0], f[..., 0] * (eD[..., 0] + np.abs(D[..., 0]) * (df[..., 0] + 2 * EPS)))
    return out


def norm(s, w, eps=1e-6, gy=None, gs=None, keep=False, dtype="f32"):
    """s [N, C, P]: the stream as the kernels have it.  dict name -> (value, bound); "y32": y before it is rounded."""
    s, w = np.asarray(s, np.float64), np.asarray(w, np.float64)[None, :, None]
    N, C, P = s.shape
    r = 1 / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    er = (C + 8) * EPS                       # a sum of C non-negative terms in any order, halved by the root; its operations
    y = s * r * w
    ey = np.abs(y) * (er + 4 * EPS)
    out = {"y32": (y, ey), "y": (y, ey + HALF[dtype] * (np.abs(y) + ey)), "rstd": (r, r * er)}
    if gy is None:
        return out
    v = q8(s, *((N * C, P) if P > 1 else (N, C)))[2].reshape(s.shape) if keep else s
    gy = np.asarray(gy, np.float64)
    z = v * r
    wd = w * gy
    m = (wd * z).mean(1, keepdims=True)
    em = np.abs(wd * z).mean(1, keepdims=True) * ((C + 4) * EPS + er)
    d = r * (wd - z * m)
    ed = r * (np.abs(wd) * (er + 4 * EPS) + np.abs(z * m) * (2 * er + 6 * EPS) + np.abs(z) * em)
    if gs is not None:
        d = d + np.asarray(gs, np.float64)
        ed = ed + EPS * np.abs(d)
    out["grad_x"] = (d, ed + HALF[dtype] * (np.abs(d) + ed))
    out["grad_weight"] = ((gy * z).sum((0, 2)), np.abs(gy * z).sum((0, 2)) * ((N * P + 4) * EPS + er))
    return out


def check(got, ref, what):
    """got (an array) within ref = (value, bound); NaN and infinities where the value has them."""
    got = np.asarray(got, np.float64)
    val, bound = ref
    assert got.shape == val.shape, (what, got.shape, val.shape)
    fine = np.isfinite(val)
    assert np.array_equal(np.isnan(got), np.isnan(val)), what
    assert np.array_equal(got[~fine & ~np.isnan(val)], val[~fine & ~np.isnan(val)]), what
    err = np.abs(got - val)[fine]
    lim = (bound + 1e-30)[fine]
    assert (err <= lim).all(), (what, float((err / lim).max()), int((err > lim).sum()), err.size)
