"""Float64 oracle of the inner step's operators (test infrastructure only), written from their formulas.

Every function also returns, where asked, the sum of the magnitudes of the terms that make up each
result: a bound on what rounding the terms can do to it.
"""
from __future__ import annotations

import numpy as np


def _f8(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


# ------------------------------------------------------------------------------- attention
def attention(q, k, v, cu_seqlens, scale):
    """q [T, Hq, d], k and v [T, Hk, d] -> o [T, Hq, d], lse [Hq, T], and sum_j P_ij |v_j| [T, Hq, d]."""
    q, k, v = _f8(q), _f8(k), _f8(v)
    T, Hq, _ = q.shape
    Hk = k.shape[1]
    o, mag, lse = np.zeros(q.shape), np.zeros(q.shape), np.zeros((Hq, T))
    for a, b in zip(cu_seqlens[:-1], cu_seqlens[1:]):
        for h in range(Hq):
            g = h // (Hq // Hk)
            for i in range(a, b):
                s = scale * (k[a:i + 1, g] @ q[i, h])
                top = s.max()
                e = np.exp(s - top)
                p = e / e.sum()
                o[i, h], mag[i, h] = p @ v[a:i + 1, g], p @ np.abs(v[a:i + 1, g])
                lse[h, i] = top + np.log(e.sum())
    return o, lse, mag


def attention_grad(q, k, v, dout, cu_seqlens, scale):
    """Gradients of sum(dout * o): {"dq", "dk", "dv"} and the term magnitudes {"dq", "dk", "dv"}; those of dq and dk
    include what an error of 1 in units of sum_c |o||dout| in delta does."""
    q, k, v, dout = _f8(q), _f8(k), _f8(v), _f8(dout)
    Hq, Hk = q.shape[1], k.shape[1]
    g = {"dq": np.zeros(q.shape), "dk": np.zeros(k.shape), "dv": np.zeros(v.shape)}
    m = {n: np.zeros(x.shape) for n, x in g.items()}
    for a, b in zip(cu_seqlens[:-1], cu_seqlens[1:]):
        n = b - a
        if n == 0:
            continue
        keep = np.tril(np.ones((n, n), dtype=bool))
        for h in range(Hq):
            c = h // (Hq // Hk)
            Q, K, V, G = q[a:b, h], k[a:b, c], v[a:b, c], dout[a:b, h]
            s = np.where(keep, scale * (Q @ K.T), -np.inf)
            e = np.exp(s - s.max(1, keepdims=True))
            p = e / e.sum(1, keepdims=True)
            o = p @ V
            dp = G @ V.T
            delta, delta_mag = (G * o).sum(1, keepdims=True), (np.abs(G) * np.abs(o)).sum(1, keepdims=True)
            ds = scale * p * (dp - delta)
            ds_mag = abs(scale) * p * (np.abs(G) @ np.abs(V).T + delta_mag)
            g["dq"][a:b, h] = ds @ K
            g["dk"][a:b, c] += ds.T @ Q
            g["dv"][a:b, c] += p.T @ G
            m["dq"][a:b, h] = ds_mag @ np.abs(K)
            m["dk"][a:b, c] += ds_mag.T @ np.abs(Q)
            m["dv"][a:b, c] += p.T @ np.abs(G)
    return g, m


# ------------------------------------------------------------------------------- block norm
def _per_row(w, workers, rows):
    """[K, H] per-channel values as [K * rows, H]."""
    return np.repeat(_f8(w), rows, axis=0)


def block_norm(x, y, gate, gate_kind, w_post, w_pre, workers, eps, s):
    """-> x_new, n (n is None without w_pre)."""
    x, y = _f8(x), _f8(y)
    rows = x.shape[0] // workers
    xn = x
    if y is not None:
        u = y
        if w_post is not None:
            u = y / np.sqrt((y * y).mean(1, keepdims=True) + eps) * _per_row(w_post, workers, rows)
        if gate_kind == "channel":
            u = u * _per_row(gate, workers, rows)
        elif gate_kind == "element":
            u = u * _f8(gate)
        xn = x + s * u
    n = None
    if w_pre is not None:
        n = xn / np.sqrt((xn * xn).mean(1, keepdims=True) + eps) * _per_row(w_pre, workers, rows)
    return xn, n


def block_norm_grad(dn, dres, x_new, y, gate, gate_kind, w_post, w_pre, workers, eps, s):
    """-> gradients and term magnitudes, dicts with dx, dy, dgate, dw_post, dw_pre (None where absent)."""
    dn, dres, x, y = _f8(dn), _f8(dres), _f8(x_new), _f8(y)
    first = dn if dn is not None else dres
    T, H = first.shape
    rows = T // workers
    dX = np.zeros((T, H)) if dres is None else dres.copy()
    mX = np.abs(dX)
    g, m = {}, {}
    columns = lambda t: t.reshape(workers, rows, H).sum(1)  # noqa: E731
    if dn is not None:
        r = 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
        xh = x * r
        a = dn * _per_row(w_pre, workers, rows)
        dX = dX + r * (a - xh * (a * xh).mean(1, keepdims=True))
        mX = mX + r * (np.abs(a) + np.abs(xh) * np.abs(a * xh).mean(1, keepdims=True))
        g["dw_pre"], m["dw_pre"] = columns(dn * xh), columns(np.abs(dn * xh))
    g["dx"], m["dx"] = dX, mX
    if y is not None:
        gt = 1.0 if gate_kind is None else _per_row(gate, workers, rows) if gate_kind == "channel" else _f8(gate)
        t, mt = s * dX * gt, abs(s) * mX * np.abs(gt)
        if w_post is None:
            yh, wp = y, 1.0
            g["dy"], m["dy"] = t, mt
        else:
            r = 1.0 / np.sqrt((y * y).mean(1, keepdims=True) + eps)
            yh, wp = y * r, _per_row(w_post, workers, rows)
            b, mb = t * wp, mt * np.abs(wp)
            g["dy"] = r * (b - yh * (b * yh).mean(1, keepdims=True))
            m["dy"] = r * (mb + np.abs(yh) * (mb * np.abs(yh)).mean(1, keepdims=True))
            g["dw_post"], m["dw_post"] = columns(t * yh), columns(mt * np.abs(yh))
        dg, mg = s * dX * yh * wp, abs(s) * mX * np.abs(yh * wp)
        if gate_kind == "channel":
            g["dgate"], m["dgate"] = columns(dg), columns(mg)
        elif gate_kind == "element":
            g["dgate"], m["dgate"] = dg, mg
    return g, m


# ------------------------------------------------------------------------------- 8-bit checkpoints
def save8(x, group=32):
    """-> q8 [R, W] int8, e8 [R, ceil(W / group)] uint8."""
    x = np.asarray(x, dtype=np.float64)
    R, W = x.shape
    G = -(-W // group)
    q, e = np.zeros((R, W), dtype=np.int8), np.zeros((R, G), dtype=np.uint8)
    for r in range(R):
        for j in range(G):
            part = x[r, j * group:(j + 1) * group]
            if not np.isfinite(part).all():
                e[r, j] = 255
                continue
            top = np.abs(part).max()
            biased = int(np.frexp(top)[1]) + 126 if top > 0 else 0      # exponent field of the fp32 value (0: zero; fp32 subnormals are below 7 anyway)
            e[r, j] = max(biased - 6, 1)
            q[r, j * group:(j + 1) * group] = np.clip(np.rint(part * 2.0 ** (127 - int(e[r, j]))), -127, 127)
    return q, e


def load8(q, e, group=32):
    step = np.where(e == 255, np.nan, 2.0 ** (e.astype(np.int64) - 127.0))
    return q.astype(np.float64) * np.repeat(step, group, axis=1)[:, :q.shape[1]]


def swiglu(g, u):
    g, u = _f8(g), _f8(u)
    return g / (1.0 + np.exp(-g)) * u


def swiglu_grad(dh, g, u):
    """-> dg, du of sum(dh * swiglu(g, u))."""
    dh, g, u = _f8(dh), _f8(g), _f8(u)
    s = 1.0 / (1.0 + np.exp(-g))
    return dh * u * s * (1.0 + g * (1.0 - s)), dh * g * s
