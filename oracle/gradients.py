"""CPU oracle of the low-rank adapters and of the gradients of the layer's steps: fp64, plain loops over experts and
requests, written from the formulas.  TEST INFRASTRUCTURE ONLY, as `semmoe_oracle` is.

Inputs are taken as given (e.g. bf16-rounded values held in float32).
"""
from __future__ import annotations

import numpy as np


def _f64(*arrays):
    return tuple(np.asarray(a, dtype=np.float64) for a in arrays)


# ---- combine: Out[i] = sum_j w[i,j] Y[slot(i,j)]
def combine_grad(dOut, Y, slot_of_pair, topk_w):
    """(dY, dw): dY rows that no pair names are zero"""
    dOut, Y, w = _f64(dOut, Y, topk_w)
    T, k = w.shape
    slots = np.asarray(slot_of_pair).reshape(T, k)
    dY, dw = np.zeros_like(Y), np.zeros_like(w)
    for i in range(T):
        for j in range(k):
            s = slots[i, j]
            if 0 <= s < T * k:
                dY[s] = w[i, j] * dOut[i]
                dw[i, j] = dOut[i] @ Y[s]
    return dY, dw


# ---- dispatch_rows: X_perm[slot(i,j)] = X[i]
def dispatch_grad(dX_perm, slot_of_pair, k, dX_add=None):
    (dX_perm,) = _f64(dX_perm)
    slots = np.asarray(slot_of_pair).reshape(-1, k)
    dX = np.zeros((slots.shape[0], dX_perm.shape[1])) if dX_add is None else _f64(dX_add)[0].copy()
    for i, row in enumerate(slots):
        for s in row:
            if 0 <= s < slots.size:
                dX[i] += dX_perm[s]
    return dX


# ---- expert FFN: y = W_down (silu(W_gate x) * (W_up x))
def swiglu_ffn_grad(x, dy, W_gu, W_down):
    """gradient towards x of rows x[n,d], for dy[n,d]"""
    x, dy, W_gu, W_down = _f64(x, dy, W_gu, W_down)
    F = W_down.shape[1]
    g, u = x @ W_gu[:F].T, x @ W_gu[F:].T
    sig = 1.0 / (1.0 + np.exp(-g))
    dh = dy @ W_down
    dg = dh * u * (sig + g * sig * (1.0 - sig))
    du = dh * g * sig
    return dg @ W_gu[:F] + du @ W_gu[F:]


# ---- adapters: Y[i] = Y_base[i] + s_a B_a (A_a X[i])
def adapter_of_token(req_offsets, adapter_of_req, n_adapters, T):
    """adapter of each of T tokens; -1: none, -2: behind the last request"""
    out = np.full(T, -2, dtype=np.int64)
    for q, a in enumerate(adapter_of_req):
        out[req_offsets[q]:req_offsets[q + 1]] = a if 0 <= a < n_adapters else -1
    return out


def adapter_index(req_offsets, adapter_of_req, n_adapters, T):
    """(order[T], adapter_offsets[n_adapters + 1])"""
    a = adapter_of_token(req_offsets, adapter_of_req, n_adapters, T)
    runs = [np.flatnonzero(a == v) for v in range(n_adapters)]
    offsets = np.concatenate([[0], np.cumsum([len(r) for r in runs])])
    order = np.concatenate(runs + [np.flatnonzero(a == -1), np.full(int((a == -2).sum()), -1)])
    return order.astype(np.int32), offsets.astype(np.int32)


def adapters(X, of_token, A, B, scale=None, Y_base=None, Y=None):
    """`Y`: what the rows behind the last request hold (zero)"""
    X, A, B = _f64(X, A, B)
    out = np.zeros((X.shape[0], B.shape[1])) if Y is None else _f64(Y)[0].copy()
    for i, a in enumerate(of_token):
        if a == -2:
            continue
        out[i] = 0.0 if Y_base is None else np.asarray(Y_base[i], dtype=np.float64)
        if a >= 0:
            out[i] += (1.0 if scale is None else float(scale[a])) * (B[a] @ (A[a] @ X[i]))
    return out


def adapters_grad(X, dY, of_token, A, B, scale=None, dX_base=None, dX=None):
    """(dX, dA, dB)"""
    X, dY, A, B = _f64(X, dY, A, B)
    out = np.zeros_like(X) if dX is None else _f64(dX)[0].copy()
    dA, dB = np.zeros_like(A), np.zeros_like(B)
    for i, a in enumerate(of_token):
        if a == -2:
            continue
        out[i] = 0.0 if dX_base is None else np.asarray(dX_base[i], dtype=np.float64)
        if a >= 0:
            s = 1.0 if scale is None else float(scale[a])
            v = s * (dY[i] @ B[a])
            out[i] += v @ A[a]
            dA[a] += np.outer(v, X[i])
            dB[a] += np.outer(dY[i], s * (A[a] @ X[i]))
    return out, dA, dB
