"""The gradient oracle pinned to its definitions: every gradient against central differences of the forward oracle, the index
against its properties."""
import numpy as np
import pytest

from oracle import gradients as G
from oracle import semmoe_oracle as O


def _differences(f, x, g, eps=1e-6):
    """central differences of <f(x), g> along every entry of x"""
    out = np.zeros_like(x)
    for at in np.ndindex(*x.shape):
        hi, lo = x.copy(), x.copy()
        hi[at] += eps
        lo[at] -= eps
        out[at] = ((f(hi) - f(lo)) * g).sum() / (2 * eps)
    return out


def _close(a, b):
    # differences of a smooth function: truncation eps^2, cancellation 2^-53 |f| / eps = 1e-10 |f|
    assert np.abs(a - b).max() <= 1e-7 * max(1.0, np.abs(b).max())


def test_combine_and_dispatch_gradients_are_those_of_the_forward_steps():
    r = np.random.default_rng(0)
    T, k, d = 5, 3, 6
    slots = r.permutation(T * k).astype(np.int32)
    Y, w, dOut = r.standard_normal((T * k, d)), r.random((T, k)), r.standard_normal((T, d))
    dY, dw = G.combine_grad(dOut, Y, slots, w)
    _close(dY, _differences(lambda y: O.combine(y, slots, w), Y, dOut))
    _close(dw, _differences(lambda v: O.combine(Y, slots, v), w, dOut))
    X, dXp, add = r.standard_normal((T, d)), r.standard_normal((T * k, d)), r.standard_normal((T, d))

    def rows(x):
        out = np.zeros((T * k, d))
        out[slots] = np.repeat(x, k, axis=0)
        return out
    _close(G.dispatch_grad(dXp, slots, k), _differences(rows, X, dXp))
    _close(G.dispatch_grad(dXp, slots, k, add), G.dispatch_grad(dXp, slots, k) + add)


def test_slots_outside_the_rows_have_no_gradient():
    r = np.random.default_rng(1)
    slots = np.array([0, -1, 4, 2], dtype=np.int32)  # 2 tokens, k = 2: rows 0..3
    Y, w, dOut = r.standard_normal((4, 3)), r.random((2, 2)), r.standard_normal((2, 3))
    dY, dw = G.combine_grad(dOut, Y, slots, w)
    assert (dY[[1, 3]] == 0).all() and dw[0, 1] == 0 and dw[1, 0] == 0 and dw[0, 0] != 0
    assert (G.dispatch_grad(Y, slots, 2)[0] == Y[0]).all()


def test_ffn_gradient():
    r = np.random.default_rng(2)
    n, d, F = 3, 5, 4
    x, dy = r.standard_normal((n, d)), r.standard_normal((n, d))
    W_gu, W_dn = r.standard_normal((2 * F, d)), r.standard_normal((d, F))
    _close(G.swiglu_ffn_grad(x, dy, W_gu, W_dn), _differences(lambda v: O.swiglu_ffn(v, W_gu, W_dn), x, dy))


@pytest.mark.parametrize("scaled", [False, True])
def test_adapter_gradients(scaled):
    r = np.random.default_rng(3)
    T, n, rank, d_in, d_out = 7, 3, 2, 4, 5
    of = np.array([2, -1, 0, 0, 2, -2, -2])  # adapter 1 has no token, the last two rows are padding
    X, dY, base = r.standard_normal((T, d_in)), r.standard_normal((T, d_out)), r.standard_normal((T, d_out))
    A, B = r.standard_normal((n, rank, d_in)), r.standard_normal((n, d_out, rank))
    s = r.random(n) + 0.5 if scaled else None
    dX, dA, dB = G.adapters_grad(X, dY, of, A, B, s)
    _close(dX, _differences(lambda v: G.adapters(v, of, A, B, s, base), X, dY))
    _close(dA, _differences(lambda v: G.adapters(X, of, v, B, s, base), A, dY))
    _close(dB, _differences(lambda v: G.adapters(X, of, A, v, s, base), B, dY))
    assert (dA[1] == 0).all() and (dX[[1, 5, 6]] == 0).all()
    add = r.standard_normal((T, d_in))
    with_base = G.adapters_grad(X, dY, of, A, B, s, dX_base=add, dX=np.full((T, d_in), 9.0))[0]
    _close(with_base[:5], dX[:5] + add[:5])
    assert (with_base[5:] == 9.0).all()


def test_adapter_index_sorts_tokens_by_adapter():
    off, ad = [0, 3, 3, 5, 9, 10], [1, 0, -1, 0, 7]
    order, starts = G.adapter_index(off, ad, 2, 12)
    assert order.tolist() == [5, 6, 7, 8, 0, 1, 2, 3, 4, 9, -1, -1] and starts.tolist() == [0, 4, 7]
    order, starts = G.adapter_index([0], [], 3, 2)
    assert order.tolist() == [-1, -1] and starts.tolist() == [0, 0, 0, 0]
