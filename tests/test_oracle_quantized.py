"""Pins of the oracle of 8-bit rows and of the norms around a block: closed forms and differences."""
import numpy as np
import pytest

from oracle import quantized as Q


def test_rows_in_8_bits_lie_within_half_a_step():
    r = np.random.default_rng(0)
    x = r.standard_normal((50, 64)).astype(np.float32)
    x[3] = 0
    q, scale = Q.quantize_rows(x)
    assert (np.abs(q).max(1)[np.arange(50) != 3] == 127).all() and (q[3] == 0).all() and scale[3] == 0
    # the reciprocal, the factor, the product and the scale's factor and product are rounded (2^-24 each, of at most 127)
    assert (np.abs(q * scale[:, None].astype(np.float64) - x) <= scale[:, None] * (0.5 + 5 * 127 * 2.0 ** -24)).all()


def test_ties_are_even_and_tiny_rows_keep_their_numbers():
    x = np.array([[128.0, 64.0, -64.0, 32.0, 1.0, -1.0, 0.5, 0.0]], np.float32)  # steps of 128 / 127: 64 is 63.5 of them
    q, scale = Q.quantize_rows(x)
    assert q.tolist() == [[127, 64, -64, 32, 1, -1, 0, 0]] and abs(scale[0] - 128 / 127) < 2.0 ** -23
    for e in (-140, -133, -100, 100, 120):
        q2, scale2 = Q.quantize_rows(x * np.float32(2.0) ** e)
        assert (q2 == q).all() and abs(scale2[0] / 2.0 ** e - 128 / 127) < (2.0 ** -23 if e > -120 else 2.0 ** -9)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_rows_that_are_no_numbers(bad):
    x = np.ones((2, 8), np.float32)
    x[1, 5] = bad
    q, scale = Q.quantize_rows(x)
    assert (q[1] == 0).all() and np.isnan(scale[1]) and (q[0] == 127).all()


def test_linear_is_the_product_of_what_the_integers_stand_for():
    r = np.random.default_rng(1)
    q, w = r.integers(-128, 128, (5, 48)), r.integers(-128, 128, (7, 48))
    xs, ws = r.random(5), r.random(7)
    assert np.allclose(Q.linear(q, xs, w, ws), (q * xs[:, None]) @ (w * ws[:, None]).T, rtol=1e-13, atol=1e-10)


CASES = [dict(), dict(gate_rows=False), dict(w_post=False), dict(R=False), dict(dX=False), dict(dH=False), dict(gate=False), dict(Y=False)]


@pytest.mark.parametrize("case", CASES)
def test_norm_gradient_against_differences(case):
    r = np.random.default_rng(2)
    T, d = 3, 16
    has = lambda n: case.get(n, True)  # noqa: E731
    p = dict(R=r.standard_normal((T, d)) if has("R") else None, Y=r.standard_normal((T, d)) if has("Y") else None)
    p["w_post"] = r.standard_normal(d) if has("w_post") and has("Y") else None
    p["gate"] = r.standard_normal((T, d) if has("gate_rows") else d) if has("gate") and has("Y") else None
    p["w_pre"] = r.standard_normal(d) if has("dX") else None
    par = (0.7, 1e-3, 1e-2)
    dH = r.standard_normal((T, d)) if has("dH") else None
    dX = r.standard_normal((T, d)) if has("dX") else None

    def loss():
        H, X = Q.block_norm(*p.values(), *par)
        return (0.0 if dH is None else (dH * H).sum()) + (0.0 if dX is None else (dX * X).sum())

    H, _ = Q.block_norm(*p.values(), *par)
    got = Q.block_norm_grad(dH, dX, H, p["Y"], p["w_post"], p["gate"], p["w_pre"], *par)
    if p["gate"] is not None and p["gate"].ndim == 1:
        got["dgate"] = got["dgate"].sum(0)
    names = dict(R="dR", Y="dY", w_post="dw_post", gate="dgate", w_pre="dw_pre")
    for name, t in p.items():
        if t is None:
            continue
        for at in list(np.ndindex(t.shape))[::5]:
            keep, step = t[at], 1e-5
            t[at] = keep + step
            up = loss()
            t[at] = keep - step
            down = loss()
            t[at] = keep
            # central differences: an error of step^2 times a third derivative of order 10, and of 1e-16 * |loss| / step
            assert abs((up - down) / (2 * step) - got[names[name]][at]) < 1e-7, (name, at)
