"""CPU oracle of rows in 8-bit integers, of the products made of them and of the norms around a block: fp64, written from the
formulas.  TEST INFRASTRUCTURE ONLY, as `semmoe_oracle` is.

Inputs are taken as given (e.g. bf16-rounded values held in float32).
"""
from __future__ import annotations

import numpy as np


def quantize_rows(x):
    """(q int8, scale float32) in the sequence of fp32 operations that the definition names: 1 / amax, times 127, the product, rint;
    rows whose amax lies below 2^-64 times 2^64, above 2^64 times 2^-64"""
    x = np.asarray(x, dtype=np.float32)
    f = np.float32
    amax = np.abs(x).max(1) if x.shape[1] else np.zeros(x.shape[0], f)
    bad = ~np.isfinite(x).all(1)
    amax = np.where(bad, f(1), amax).astype(f)
    pre = np.where(amax < f(2.0 ** -64), f(2.0 ** 64), np.where(amax > f(2.0 ** 64), f(2.0 ** -64), f(1))).astype(f)
    with np.errstate(divide="ignore", invalid="ignore"):
        r = np.where(amax > 0, (f(1) / (amax * pre)).astype(f) * f(127), f(0)).astype(f)
        q = np.rint((x * pre[:, None]).astype(f) * r[:, None])
        scale = (amax * (f(1) / f(127))).astype(f)
    q[bad], scale[bad] = 0, np.nan
    return q.astype(np.int8), scale


def linear(q, x_scale, w, w_scale):
    sums = np.asarray(q, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T  # integers below 2^53: exact
    return sums * np.asarray(x_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)


def hidden(q, x_scale, w_gu, w_scale_gu):
    """(h, gate) of the FFN before h is rounded"""
    gu = linear(q, x_scale, w_gu, w_scale_gu)
    g, u = np.split(gu, 2, axis=1)
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * u, g


# ---- norms: n = Y / rms(Y) w_post, H = res_scale R + gate n, X = H / rms(H) w_pre
def _rms(x, eps):
    return np.sqrt((x * x).mean(1, keepdims=True) + eps)


def block_norm(R, Y, w_post, gate, w_pre, res_scale, eps_post, eps_pre):
    """(H, X); X is None without w_pre"""
    H = 0.0 if R is None else res_scale * np.asarray(R, np.float64)
    if Y is not None:
        n = np.asarray(Y, np.float64)
        if w_post is not None:
            n = n / _rms(n, eps_post) * np.asarray(w_post, np.float64)
        H = H + (n if gate is None else np.asarray(gate, np.float64) * n)
    return H, None if w_pre is None else H / _rms(H, eps_pre) * np.asarray(w_pre, np.float64)


def _norm_grad(x, eps, w, dn):
    """gradient of x / rms(x) w towards x and, row by row, towards w"""
    r = _rms(x, eps)
    xn, a = x / r, dn * w
    return (a - xn * (a * xn).mean(1, keepdims=True)) / r, dn * xn


def block_norm_grad(dH, dX, H, Y, w_post, gate, w_pre, res_scale, eps_post, eps_pre):
    """dict of dR, dY, dgate (row by row), dw_post, dw_pre (sums); those that have no meaning are None"""
    f = lambda t: None if t is None else np.asarray(t, np.float64)  # noqa: E731
    dH, dX, H, Y, w_post, gate, w_pre = map(f, (dH, dX, H, Y, w_post, gate, w_pre))
    out = dict.fromkeys(("dR", "dY", "dgate", "dw_post", "dw_pre"))
    total = 0.0 if dH is None else dH
    if dX is not None:
        through, dw = _norm_grad(H, eps_pre, w_pre, dX)
        total, out["dw_pre"] = total + through, dw.sum(0)
    out["dR"] = res_scale * total
    if Y is not None:
        n = Y if w_post is None else Y / _rms(Y, eps_post) * w_post
        out["dgate"] = total * n
        dn = total if gate is None else total * gate
        if w_post is None:
            out["dY"] = dn
        else:
            out["dY"], dw = _norm_grad(Y, eps_post, w_post, dn)
            out["dw_post"] = dw.sum(0)
    return out
