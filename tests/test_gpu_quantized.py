"""Rows in 8 bits, the products made of them and the norms around a block on the GPU against the fp64 oracle.

Bounds.  u = 2^-8 is the largest relative error of a rounding to bf16, e = 2^-24 that of fp32 (r: either, by the result's type).
  * quantize_rows: a named sequence of fp32 operations, bit for bit.
  * linear_i8: an exact integer sum, rounded to fp32, two products and the result's rounding: (u + 3e) |y|.
  * FFN: h of the kernel lies within eps = (12 + 4 |g|) 2^-23 of the oracle's (relative): g and u carry 3 e each and g's are times
    |d log silu / d log g| <= 1 + |g|; the exponential's argument is rounded, e |g|, and it and the reciprocal are 2^-23 off each; two
    products.  So its bf16 and 8-bit forms lie between those of h (1 - eps) and h (1 + eps): where the two differ the oracle's
    h may be off by their distance D, and y by sum |w| D.  Rows in which the largest magnitude may differ: their steps are
    at most 2^-7 apart (one bf16 step), so every number is off by 2^-7 |h| and two halves of a step at most.
  * norms, see _norm_bounds and _norm_grad_bounds."""
import numpy as np
import pytest
import torch

import paper_2503_04398_amd as S
from oracle import quantized as Q

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E32 = 2.0 ** -24
R = {"bf16": 2.0 ** -8, "fp32": E32}
TINY = 2.0 ** -126


def _act(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _np(t):
    return t.detach().cpu().double().numpy()


def _rand(r, shape, dtype, std=1.0, mean=0.0):
    return (mean + std * torch.from_numpy(r.standard_normal(shape, dtype=np.float32))).to(_act(dtype))


def _m(T=1, d=64, dtype="bf16", **kw):
    return S.SemMoE(S.Config(**{**dict(T=T, d=d, E=1, k=1, F=16, D=1, cap=max(T, 1), dtype=dtype), **kw}), device=DEV, allocate_workspace=False)


def _quantized(r, rows, cols, std=1.0):
    """(q, scale) on the GPU of random rows"""
    q, s = Q.quantize_rows(std * r.standard_normal((rows, cols), dtype=np.float32))
    return torch.from_numpy(q).to(DEV), torch.from_numpy(s).to(DEV)


def _within(got, want, bound, what):
    got, want = (_np(t) if torch.is_tensor(t) else t for t in (got, want))
    off = np.abs(got - want) - bound
    assert np.isfinite(got).all(), what
    at = np.unravel_index(int(off.argmax()), off.shape)
    assert off[at] <= 0, "%s at %s: %r for %r, bound %r" % (what, at, got[at], want[at], bound[at])


# ---- rows in 8 bits
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,cols", [(1, 8), (3, 64), (5, 504), (130, 512), (33, 520), (7, 2048), (9, 4096), (4, 4104), (3, 8200), (2, 16384),
                                    (2, 16392), (3, 40000), (5000, 24), (9, 3632), (3, 24584), (2, 32768), (2, 32776)])
def test_quantize_rows(n, cols, dtype):
    r = np.random.default_rng(n + cols)
    X = _rand(r, (n, cols), dtype) * torch.from_numpy(2.0 ** r.integers(-20, 20, (n, 1))).to(_act(dtype))
    if n > 2:
        X[1] = 0
        X[2, cols // 2] = 0.0
    q, s = torch.full((n + 1, cols), 77, dtype=torch.int8, device=DEV), torch.full((n + 1,), 77.0, device=DEV)
    _m(dtype=dtype).quantize_rows(X.to(DEV), q, s)
    want_q, want_s = Q.quantize_rows(X.float().numpy())
    assert (q[:n].cpu().numpy() == want_q).all() and (s[:n].cpu().numpy() == want_s).all()
    assert (q[n] == 77).all() and s[n] == 77.0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantize_rows_of_odd_numbers(dtype):
    X = torch.randn(12, 64, generator=torch.Generator().manual_seed(1)).to(_act(dtype))
    X[0, 3], X[1, 3], X[2, 3] = float("inf"), -float("inf"), float("nan")
    X[3] *= 2.0 ** -120
    X[4] *= 2.0 ** -128
    X[5] = 0
    X[5, 9] = 2.0 ** -133  # one number, below the normal ones
    X[6] *= 2.0 ** 120
    X[7] = -0.0
    X[8] = torch.tensor([254.0, 1, 3, 5, -1, -3, 2, 0] * 8)
    if dtype == "bf16":
        X.view(torch.int16)[9, 1] = -1       # NaN of other bits
    else:
        X.view(torch.int32)[9, 1] = -1
    q, s = torch.empty(12, 64, dtype=torch.int8, device=DEV), torch.empty(12, device=DEV)
    _m(dtype=dtype).quantize_rows(X.to(DEV), q, s)
    want_q, want_s = Q.quantize_rows(X.float().numpy())
    assert (q.cpu().numpy() == want_q).all()
    assert np.array_equal(s.cpu().numpy(), want_s, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantize_rows_of_a_wider_tensor(dtype):
    X = _rand(np.random.default_rng(0), (37, 304), dtype).to(DEV)
    q, s, q2, s2 = (torch.empty(37, 200, dtype=torch.int8, device=DEV), torch.empty(37, device=DEV),
                    torch.empty(37, 200, dtype=torch.int8, device=DEV), torch.empty(37, device=DEV))
    m = _m(dtype=dtype)
    m.quantize_rows(X[:, 64:264], q, s)
    m.quantize_rows(X[:, 64:264].contiguous(), q2, s2)
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("T,k,d", [(1, 1, 16), (7, 2, 64), (33, 3, 272), (64, 4, 512), (20, 8, 2880), (9, 13, 48), (5, 16, 7168), (3, 5, 8208)])
def test_dispatch_rows_i8(T, k, d):
    r = np.random.default_rng(T + k)
    m = _m(T=T, d=d, E=k, k=k)
    q, s = _quantized(r, T, d)
    slots = r.permutation(T * k).astype(np.int32)
    if T * k > 4:
        slots[1], slots[-1] = -1, T * k  # pairs without a row
    out, scale = torch.full((T * k, d), 77, dtype=torch.int8, device=DEV), torch.full((T * k,), 77.0, device=DEV)
    m.dispatch_rows_i8(q, s, torch.from_numpy(slots).to(DEV), out, scale)
    want, want_s = np.full((T * k, d), 77, np.int8), np.full(T * k, 77.0, np.float32)
    for p, slot in enumerate(slots):
        if 0 <= slot < T * k:
            want[slot], want_s[slot] = q[p // k].cpu().numpy(), s[p // k].item()
    assert (out.cpu().numpy() == want).all() and (scale.cpu().numpy() == want_s).all()


# ---- products
LINEAR = [(1, 16, 8), (1, 4096, 64), (5, 272, 200), (16, 512, 1032), (31, 2880, 304), (33, 1040, 128), (64, 4096, 512), (65, 192, 2056),
          (130, 1024, 264), (200, 7168, 136), (257, 48, 520), (300, 2064, 1040), (777, 640, 328), (1025, 384, 512), (2000, 2048, 264),
          (3001, 256, 1536), (4096, 512, 4096), (3000, 16, 3000), (3000, 48, 2048), (5000, 144, 4104), (2600, 256, 2600)]


@pytest.mark.parametrize("T,d_in,d_out", LINEAR)
def test_linear_i8(T, d_in, d_out):
    r = np.random.default_rng(T + d_in + d_out)
    (q, s), (w, ws) = _quantized(r, T, d_in), _quantized(r, d_out, d_in, d_in ** -0.5)
    Y = torch.full((T + 1, d_out), 7.0, dtype=torch.bfloat16, device=DEV)
    _m().linear_i8(q, s, w, ws, Y[:T])
    want = Q.linear(*(t.cpu().numpy() for t in (q, s, w, ws)))
    _within(Y[:T], want, (R["bf16"] + 3 * E32) * np.abs(want) + TINY, "Y")
    assert (Y[T] == 7.0).all()


@pytest.mark.parametrize("d_in", [400, 416, 464, 496, 528, 1168, 2880])
@pytest.mark.parametrize("T,d_out", [(150, 1024), (700, 2056), (1024, 2880), (2600, 5768)])
def test_linear_i8_of_partial_slices(T, d_out, d_in):
    """rows that end inside a slice of 128 bytes, through 128 x 128 pieces, 256 x 128 and 256 x 256 tiles; the rows behind the last
    one hold the largest numbers"""
    r = np.random.default_rng(T + d_in)
    (q, s), (w, ws) = _quantized(r, T + 1, d_in), _quantized(r, d_out + 1, d_in, d_in ** -0.5)
    q[T], w[d_out] = -128, -128
    Y = torch.empty(T, d_out, dtype=torch.bfloat16, device=DEV)
    _m().linear_i8(q[:T], s[:T], w[:d_out], ws[:d_out], Y)
    want = Q.linear(*(t.cpu().numpy() for t in (q[:T], s[:T], w[:d_out], ws[:d_out])))
    _within(Y, want, (R["bf16"] + 3 * E32) * np.abs(want) + TINY, "Y")


@pytest.mark.parametrize("d,F", [(400, 272), (528, 464), (720, 400)])
@pytest.mark.parametrize("rows", [[45] * 8, [130, 0, 257, 64, 1, 300], [700, 300, 900]])
def test_expert_ffn_i8_of_partial_slices(rows, d, F):
    _experts(rows, d, F, seed=5)


SHAPES = [0, 16, 22, 26, 28, 30, 31, 32, 33, 34, 35, 38, 39, 40, 7]  # the last one is none of theirs


@pytest.mark.parametrize("d,F", [(512, 384), (400, 272), (48, 32)])
@pytest.mark.parametrize("tile", SHAPES)
def test_every_tile_shape(tile, d, F):
    m = _m()
    try:
        m.set_tuning(0, tile)
        m.set_tuning(1, tile)
        _experts(RAGGED + [520, 129], d, F, seed=tile)
    finally:
        m.set_tuning(0, -1)
        m.set_tuning(1, -1)


@pytest.mark.parametrize("ring,grid,cut", [(-1, 16, -1), (1, 16, 16), (2, 24, 16), (3, 16, 16), (6, 16, 16), (-1, 8, 0), (-1, 40, 16)])
@pytest.mark.parametrize("tile", [22, 33, 16])
@pytest.mark.parametrize("d,F", [(512, 640), (720, 464)])
def test_tiles_and_pieces_in_every_form_of_launch(tile, ring, grid, cut, d, F):
    m = _m()
    knobs = {0: tile, 1: tile, 4: grid, 5: cut, 6: ring}
    try:
        for key, v in knobs.items():
            m.set_tuning(key, v)
        _experts([300, 0, 700, 33, 257, 1], d, F, seed=ring + 7)
    finally:
        for key in knobs:
            m.set_tuning(key, -1)


@pytest.mark.parametrize("d,F", [(256, 2048), (400, 272), (2048, 512)])
def test_every_tile_shape_gives_the_same_bits(d, F):
    """sums of integers do not depend on their order, and every tile makes h of them by the same operations; so many numbers that
    some lie within an fp32 rounding of a border between two of bf16"""
    r, rows = np.random.default_rng(d), [n * 4 for n in RAGGED] + [1520, 129]
    E, P = len(rows), sum(rows)
    m = _m(T=P, d=d, E=E, k=1, F=F)
    off = torch.tensor([0, *np.cumsum(rows)], dtype=torch.int32, device=DEV)
    of = torch.arange(E, dtype=torch.int32, device=DEV)
    (q, s), (w_gu, s_gu), (w_dn, s_dn) = _quantized(r, P, d), _quantized(r, E * 2 * F, d, 0.2), _quantized(r, E * d, F, 0.05)
    out = {}
    try:
        for tile in [-1, *SHAPES]:
            m.set_tuning(0, tile)
            m.set_tuning(1, tile)
            Y = torch.empty(P, d, dtype=torch.bfloat16, device=DEV)
            m.expert_ffn_i8(-1, q, s, off, of, w_gu, s_gu, w_dn, s_dn, Y)
            out[tile] = Y
    finally:
        m.set_tuning(0, -1)
        m.set_tuning(1, -1)
    assert [tile for tile, Y in out.items() if not torch.equal(Y, out[-1])] == []


def test_a_row_of_the_ffn_in_8_bits_is_the_same_in_any_batch():
    r = np.random.default_rng(11)
    n, d, F = 6000, 528, 3600
    (q, s), (w_gu, s_gu), (w_dn, s_dn) = _quantized(r, n, d), _quantized(r, 2 * F, d, 0.2), _quantized(r, d, F, 0.05)
    whole = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
    _m(T=n, d=d, F=F).shared_ffn_i8(q, s, n, w_gu, s_gu, w_dn, s_dn, whole)
    for lo, rows in ((0, 1), (7, 16), (100, 100), (250, 600), (2900, 100), (3000, 2000)):
        Y = torch.empty(rows, d, dtype=torch.bfloat16, device=DEV)
        _m(T=rows, d=d, F=F).shared_ffn_i8(q[lo:lo + rows], s[lo:lo + rows], rows, w_gu, s_gu, w_dn, s_dn, Y)
        assert torch.equal(Y, whole[lo:lo + rows]), (lo, rows)


@pytest.mark.parametrize("T,d_out", [(40, 512), (300, 2048), (700, 4096)])
def test_linear_i8_of_rows_far_apart(T, d_out):
    """rows of a tile that 32-bit offsets do not reach"""
    r = np.random.default_rng(T)
    (q, s), (w, ws) = _quantized(r, T, 512), _quantized(r, d_out, 512)
    wide = torch.zeros(T, 1 << 24, dtype=torch.int8, device=DEV)
    wide[:, 64:576] = q
    Y, Z = (torch.empty(T, d_out, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    m = _m()
    m.linear_i8(wide[:, 64:576], s, w, ws, Y)
    m.linear_i8(q, s, w, ws, Z)
    assert torch.equal(Y, Z)


def test_linear_i8_sums_are_exact():
    """the largest sums there are: rows of -128, as deep as a product may be, and sums that cancel but for one"""
    K = 131056
    q, w = torch.full((3, K), -128, dtype=torch.int8, device=DEV), torch.full((16, K), -128, dtype=torch.int8, device=DEV)
    w[1::2, ::2] = 127  # -128 * 127 beside 128 * 128
    w[2] = 127
    Y = torch.empty(3, 16, dtype=torch.bfloat16, device=DEV)
    _m().linear_i8(q, torch.ones(3, device=DEV), w, torch.ones(16, device=DEV), Y)
    want = q.cpu().double().numpy() @ w.cpu().double().numpy().T
    _within(Y, want, (R["bf16"] + 3 * E32) * np.abs(want), "Y")


def test_linear_i8_of_column_ranges():
    r = np.random.default_rng(5)
    (q, s), (w, ws) = _quantized(r, 70, 512), _quantized(r, 200, 256)
    Y = torch.full((70, 320), 7.0, dtype=torch.bfloat16, device=DEV)
    Z = torch.empty(70, 200, dtype=torch.bfloat16, device=DEV)
    m = _m()
    m.linear_i8(q[:, 128:384], s, w, ws, Y[:, 64:264])
    m.linear_i8(q[:, 128:384].contiguous(), s, w, ws, Z)
    assert torch.equal(Y[:, 64:264], Z) and (Y[:, :64] == 7.0).all() and (Y[:, 264:] == 7.0).all()


@pytest.mark.parametrize("bits", [0x7f800000, -8388608, 0x7fc00000, -1, 0x7f800001])
def test_scales_that_are_no_numbers_stay_in_their_rows(bits):
    r = np.random.default_rng(6)
    for T in (3, 200):
        (q, s), (w, ws) = _quantized(r, T, 256), _quantized(r, 320, 256)
        m, Y, Z = _m(), *(torch.empty(T, 320, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        m.linear_i8(q, s, w, ws, Y)
        s.view(torch.int32)[1] = bits
        m.linear_i8(q, s, w, ws, Z)
        assert not torch.isfinite(Z[1]).any()
        Z[1] = Y[1]
        assert torch.equal(Y, Z)
        ws.view(torch.int32)[5] = bits
        m.linear_i8(q, s, w, ws, Z)
        assert not torch.isfinite(Z[:, 5]).any() and torch.isfinite(Z[0, :5]).all()


def _bf16(x):
    return torch.from_numpy(x).to(torch.float32).to(torch.bfloat16).double().numpy()


def _ffn_check(got, q, s, w_gu, s_gu, w_dn, s_dn, what):
    """rows of one expert, numpy"""
    h, g = Q.hidden(q, s, w_gu, s_gu)
    eps = (12 + 4 * np.abs(g)) * 2.0 ** -23
    lo, hi, at = _bf16(h * (1 - eps)), _bf16(h * (1 + eps)), _bf16(h)
    hq, hs = Q.quantize_rows(at)
    (lq, ls), (uq, us) = Q.quantize_rows(lo), Q.quantize_rows(hi)
    step = hs.astype(np.float64)[:, None]
    D = step * np.maximum(np.abs(uq.astype(float) - hq), np.abs(lq.astype(float) - hq))
    loose = (ls != us)[:, None]
    D = np.where(loose, 2.0 ** -7 * np.abs(at) + 1.01 * step, D)
    want = Q.linear(hq, hs, w_dn, s_dn)
    W = np.abs(w_dn.astype(float)) * s_dn.astype(float)[:, None]
    _within(got, want, (R["bf16"] + 4 * E32) * np.abs(want) + (1 + R["bf16"]) * (D @ W.T) + TINY, what)
    return loose.mean()


def _experts(rows, d, F, D=1, rank=-1, seed=0, std=0.05):
    r = np.random.default_rng(seed)
    E, P = len(rows), int(sum(rows))
    k = next(k for k in (2, 1) if P % k == 0 and k <= E) if P else 1
    m = _m(T=P // k, d=d, E=E, k=k, F=F, D=D)
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    of = r.permutation(E).astype(np.int32)
    (q, s), (w_gu, s_gu), (w_dn, s_dn) = _quantized(r, P, d), _quantized(r, E * 2 * F, d, std), _quantized(r, E * d, F, std)
    w_gu, s_gu, w_dn, s_dn = w_gu.view(E, 2 * F, d), s_gu.view(E, 2 * F), w_dn.view(E, d, F), s_dn.view(E, d)
    Y = torch.full((P, d), 7.0, dtype=torch.bfloat16, device=DEV)
    m.expert_ffn_i8(rank, q, s, torch.from_numpy(off).to(DEV), torch.from_numpy(of).to(DEV), w_gu, s_gu, w_dn, s_dn, Y)
    per = E // D
    mine = range(E) if rank < 0 else range(rank * per, (rank + 1) * per)
    n = lambda t: t.cpu().numpy()  # noqa: E731
    for e in range(E):
        at = slice(off[e], off[e + 1])
        if e not in mine:
            assert (Y[at] == 7.0).all()
        elif rows[e]:
            o = of[e]
            _ffn_check(_np(Y[at]), n(q[at]), n(s[at]), n(w_gu[o]), n(s_gu[o]), n(w_dn[o]), n(s_dn[o]), "expert %d" % e)


RAGGED = [0, 1, 17, 0, 64, 65, 3, 130, 0, 40, 33, 7, 258, 2, 0, 20]


@pytest.mark.parametrize("d,F", [(256, 512), (272, 304), (80, 32), (512, 16), (16, 80), (1040, 384), (2048, 128)])
def test_expert_ffn_i8_of_ragged_groups(d, F):
    _experts(RAGGED, d, F)


@pytest.mark.parametrize("rows,d,F", [([8] * 16, 2048, 192), ([3] * 33, 1024, 400), ([30] * 24, 1536, 320), ([90] * 6, 640, 512),
                                      ([700, 520], 512, 640), ([1, 0, 0, 600], 768, 256), ([2000], 256, 384), ([260] * 10, 384, 256),
                                      ([0, 0, 0, 0], 64, 64), ([1], 16, 16)])
def test_expert_ffn_i8(rows, d, F):
    _experts(rows, d, F, seed=1)


@pytest.mark.parametrize("groups,rows,d,F", [(286, 100, 272, 272), (287, 100, 272, 272), (383, 100, 272, 80), (287, 200, 1280, 64), (512, 40, 400, 32)])
def test_expert_ffn_i8_of_many_groups(groups, rows, d, F):
    """as many groups as LDS holds beside a tile, and more"""
    _experts([rows] * groups, d, F, seed=3)


@pytest.mark.parametrize("rank", [0, 1, 3])
def test_expert_ffn_i8_of_one_rank(rank):
    _experts(RAGGED, 256, 320, D=4, rank=rank, seed=2)


@pytest.mark.parametrize("n,d,F", [(1, 64, 64), (31, 272, 80), (64, 2048, 512), (200, 512, 384), (777, 192, 640), (3000, 528, 1168)])
def test_shared_ffn_i8(n, d, F):
    r = np.random.default_rng(n)
    (q, s), (w_gu, s_gu), (w_dn, s_dn) = _quantized(r, n, d), _quantized(r, 2 * F, d, 0.05), _quantized(r, d, F, 0.05)
    Y = torch.full((n + 1, d), 7.0, dtype=torch.bfloat16, device=DEV)
    _m(T=n, d=d, F=F).shared_ffn_i8(q, s, n, w_gu, s_gu, w_dn, s_dn, Y)
    _ffn_check(_np(Y[:n]), *(t.cpu().numpy() for t in (q, s, w_gu, s_gu, w_dn, s_dn)), "Y")
    assert (Y[n] == 7.0).all()


def test_large_gate_values():
    """gates of hundreds either way: silu is 0 or the gate itself, never NaN"""
    r = np.random.default_rng(3)
    n, d, F = 70, 128, 192
    (q, s), (w_gu, s_gu), (w_dn, s_dn) = _quantized(r, n, d, 10.0), _quantized(r, 2 * F, d, 5.0), _quantized(r, d, F, 0.05)
    Y = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
    _m(T=n, d=d, F=F).shared_ffn_i8(q, s, n, w_gu, s_gu, w_dn, s_dn, Y)
    _ffn_check(_np(Y), *(t.cpu().numpy() for t in (q, s, w_gu, s_gu, w_dn, s_dn)), "Y")


@pytest.mark.parametrize("tile", [-1, 0, 16, 22, 26, 28, 32, 33, 35])
def test_gates_whose_sigmoid_lies_below_the_normal_numbers(tile):
    """sigmoid(g) between 2^-128 and 2^-126 beside large ups: small, and not nothing"""
    r = np.random.default_rng(13)
    n, d, F = 600, 384, 400
    m, q, w_gu = _m(T=n, d=d, F=F), np.zeros((n, d), np.int8), np.zeros((2 * F, d), np.int8)
    q[:, 0], w_gu[:F, 0], w_gu[F:, 0] = 127, -1, 1
    s = r.uniform(0.999, 1.001, n).astype(np.float32)
    s_gu = np.concatenate([np.linspace(87.45, 88.55, F) / 127, np.full(F, 2.0 ** 110 / 127)]).astype(np.float32)
    (w_dn, s_dn) = (t.cpu().numpy() for t in _quantized(r, d, F, 0.05))
    Y = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
    try:
        m.set_tuning(0, tile)
        m.shared_ffn_i8(*(torch.from_numpy(t).to(DEV) for t in (q, s)), n, *(torch.from_numpy(t).to(DEV) for t in (w_gu, s_gu, w_dn, s_dn)), Y)
    finally:
        m.set_tuning(0, -1)
    _ffn_check(_np(Y), q, s, w_gu, s_gu, w_dn, s_dn, "Y")
    assert (_np(Y) != 0).mean() > 0.9


def test_a_row_that_is_no_number_stays_alone_in_the_ffn():
    r = np.random.default_rng(4)
    n, d, F = 40, 256, 128
    X = torch.from_numpy(r.standard_normal((n, d), dtype=np.float32)).to(torch.bfloat16).to(DEV)
    (w_gu, s_gu), (w_dn, s_dn) = _quantized(r, 2 * F, d, 0.05), _quantized(r, d, F, 0.05)
    m, out = _m(T=n, d=d, F=F), []
    for bad in (False, True):
        if bad:
            X[11, 7], X[12, 0] = float("inf"), float("nan")
        q, s, Y = torch.empty(n, d, dtype=torch.int8, device=DEV), torch.empty(n, device=DEV), torch.empty_like(X)
        m.quantize_rows(X, q, s)
        m.shared_ffn_i8(q, s, n, w_gu, s_gu, w_dn, s_dn, Y)
        out.append(Y)
    assert torch.isnan(out[1][11:13]).all()
    out[1][11:13] = out[0][11:13]
    assert torch.equal(out[0], out[1])


# ---- norms
def _norm_case(r, T, d, dtype, gate="rows", without=()):
    g = None if gate is None else _rand(r, (T, d) if gate == "rows" else (d,), dtype, 0.7)
    c = dict(R=_rand(r, (T, d), dtype, 3.0), Y=_rand(r, (T, d), dtype, 0.5), w_post=_rand(r, (d,), dtype, 0.3, 1.0), gate=g,
             w_pre=_rand(r, (d,), dtype, 0.3, 1.0))
    return {n: None if n in without or t is None else t.to(DEV) for n, t in c.items()}


PAR = dict(res_scale=0.75, eps_post=1e-5, eps_pre=1e-6)


def _oracle_norm(c):
    v = {n: None if t is None else _np(t) for n, t in c.items()}
    return Q.block_norm(*v.values(), *PAR.values()), v


# additions that a number passes through in a row's sum: 4 pieces of 8 of a thread, 6 steps of a wave, 8 waves
ADDS = 4 * 8 + 6 + 8


def _norm_bounds(c, dtype):
    """H: n carries the sum's error halved by the root, ADDS / 2, and six more roundings (mean, eps, root, reciprocal, products); then
    a product and a sum.  X: the same for its own norm, and H's error as it goes through it: an error of H moves X by |w| rh times
    itself and, through the mean, by |X| times its share of the row."""
    (H, X), v = _oracle_norm(c)
    branch = 0.0 if v["Y"] is None else np.abs(Q.block_norm(None, v["Y"], v["w_post"], v["gate"], None, *PAR.values())[0])
    res = 0.0 if v["R"] is None else PAR["res_scale"] * np.abs(v["R"])
    dH = E32 * ((ADDS / 2 + 8) * branch + 2 * res + 2 * np.abs(H))
    out = {"H": (H, dH + R[dtype] * np.abs(H) + TINY)}
    if X is not None:
        rms = np.sqrt((H * H).mean(1, keepdims=True) + PAR["eps_pre"])
        share = np.sqrt((dH * dH).mean(1, keepdims=True)) / rms
        dX = np.abs(v["w_pre"]) * dH / rms + np.abs(X) * share + E32 * (ADDS / 2 + 8) * np.abs(X)
        out["X"], out["X32"] = (X, dX + R[dtype] * np.abs(X) + TINY), (X, dX)
    return out


NORMS = [(1, 8), (1, 64), (3, 512), (5, 520), (70, 256), (33, 1032), (9, 2048), (130, 2880), (7, 4096), (12, 4104), (5, 7168), (3, 8200), (2, 16384),
         (3000, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", NORMS)
def test_block_norm(T, d, dtype):
    r = np.random.default_rng(T + d)
    c = _norm_case(r, T, d, dtype, gate="rows" if T % 2 else "one")
    H, X = (torch.full((T + 1, d), 7.0, dtype=_act(dtype), device=DEV) for _ in range(2))
    Xq, s = torch.full((T + 1, d), 77, dtype=torch.int8, device=DEV), torch.full((T + 1,), 7.0, device=DEV)
    m = _m(T=T, d=d, dtype=dtype)
    m.block_norm(c["R"], H[:T], Y=c["Y"], X=X[:T], Xq=Xq, x_scale=s, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
    b = _norm_bounds(c, dtype)
    _within(H[:T], *b["H"], "H")
    _within(X[:T], *b["X"], "X")
    want, dX = b["X32"]
    step = _np(s[:T])[:, None]
    _within(_np(Xq[:T]) * step, want, step * 0.5 + dX + 6 * E32 * np.abs(want), "Xq")
    assert np.abs(_np(s[:T]) * 127 - np.abs(want).max(1)).max() <= (dX.max(1) + 3 * E32 * np.abs(want).max(1)).max()
    assert (np.abs(_np(Xq[:T])).max(1) == 127).all()
    assert (H[T] == 7.0).all() and (X[T] == 7.0).all() and (Xq[T] == 77).all() and s[T] == 7.0
    # the parts alone give the same bits
    X2, q2, s2 = torch.empty_like(X[:T]), torch.empty_like(Xq[:T]), torch.empty_like(s[:T])
    m.block_norm(c["R"], None, Y=c["Y"], X=X2, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
    m.block_norm(c["R"], None, Y=c["Y"], Xq=q2, x_scale=s2, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
    assert torch.equal(X2, X[:T]) and torch.equal(q2, Xq[:T]) and torch.equal(s2, s[:T])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("without", [("w_pre",), ("w_post",), ("gate",), ("R",), ("Y", "w_post", "gate"), ("w_post", "gate"),
                                     ("Y", "w_post", "gate", "w_pre"), ("R", "w_post", "gate")])
def test_block_norm_without(without, dtype):
    c = _norm_case(np.random.default_rng(1), 37, 264, dtype, without=without)
    H, X = (torch.empty(37, 264, dtype=_act(dtype), device=DEV) for _ in range(2))
    if c["w_pre"] is None:
        X = None
    _m(T=37, d=264, dtype=dtype).block_norm(c["R"], H, Y=c["Y"], X=X, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
    b = _norm_bounds(c, dtype)
    _within(H, *b["H"], "H")
    if X is not None:
        _within(X, *b["X"], "X")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_norms_of_wider_tensors_and_in_place(dtype):
    T, d = 45, 328
    c = _norm_case(np.random.default_rng(2), T, d, dtype)
    m, wide = _m(T=T, d=d, dtype=dtype), {}
    for n in ("R", "Y", "gate"):
        wide[n] = torch.full((T, d + 72), 7.0, dtype=_act(dtype), device=DEV)
        wide[n][:, 24:24 + d] = c[n]
    H, X, H2, X2 = (torch.full((T, d + 72), 7.0, dtype=_act(dtype), device=DEV) for _ in range(4))
    mid = slice(24, 24 + d)
    kw = dict(w_post=c["w_post"], w_pre=c["w_pre"], **PAR)
    m.block_norm(c["R"], (h := torch.empty_like(c["R"])), Y=c["Y"], X=(x := torch.empty_like(h)), gate=c["gate"], **kw)
    m.block_norm(wide["R"][:, mid], H[:, mid], Y=wide["Y"][:, mid], X=X[:, mid], gate=wide["gate"][:, mid], **kw)
    assert torch.equal(H[:, mid], h) and torch.equal(X[:, mid], x)
    for t in (H, X):
        assert (t[:, :24] == 7.0).all() and (t[:, 24 + d:] == 7.0).all()
    r, y = c["R"].clone(), c["Y"].clone()
    m.block_norm(r, r, Y=y, X=y, gate=c["gate"], **kw)
    assert torch.equal(r, h) and torch.equal(y, x)
    r, y = c["R"].clone(), c["Y"].clone()
    m.block_norm(r, y, Y=y, X=r, gate=c["gate"], **kw)
    assert torch.equal(y, h) and torch.equal(r, x)


def _norm_grad_bounds(c, g, gate_rows, dtype):
    """dH': the row's sums of ADDS + 2 roundings each, means of |terms|; its error through the rest as the formulas carry it; sums over
    rows pass T + 40 additions at most."""
    v = {n: None if t is None else _np(t) for n, t in {**c, **g}.items()}
    want = Q.block_norm_grad(v["dH"], v["dX"], v["H"], v["Y"], v["w_post"], v["gate"], v["w_pre"], *PAR.values())
    T = v["H"].shape[0]
    E, r = E32 * (ADDS + 12), R[dtype]
    mean = lambda t: t.mean(1, keepdims=True)  # noqa: E731
    total, tot_err = 0.0 if v["dH"] is None else v["dH"], 0.0
    if v["dX"] is not None:
        rh = 1 / np.sqrt(mean(v["H"] ** 2) + PAR["eps_pre"])
        a, xn = np.abs(v["dX"] * v["w_pre"]), np.abs(v["H"] * rh)
        tot_err = E * rh * (a + 2 * xn * mean(a * xn))
        total = total + rh * (v["dX"] * v["w_pre"] - v["H"] * rh * mean(v["dX"] * v["w_pre"] * v["H"] * rh))
    tot_err = tot_err + E32 * np.abs(total) * 2
    out = {"dR": (want["dR"], PAR["res_scale"] * tot_err + (r + E32) * np.abs(want["dR"]) + TINY)}
    if v["dX"] is not None:
        s = (np.abs(v["dX"]) * xn).sum(0)
        out["dw_pre"] = (want["dw_pre"], (E32 * (T + 40) + E) * s + r * np.abs(want["dw_pre"]) + TINY)
    if v["Y"] is not None:
        ry = 1.0 if v["w_post"] is None else 1 / np.sqrt(mean(v["Y"] ** 2) + PAR["eps_post"])
        w = 1.0 if v["w_post"] is None else np.abs(v["w_post"])
        yn, gate = np.abs(v["Y"] * ry), 1.0 if v["gate"] is None else np.abs(v["gate"])
        n_err = tot_err * yn * w + E * np.abs(want["dgate"])
        if v["gate"] is not None:
            if gate_rows:
                out["dgate"] = (want["dgate"], n_err + r * np.abs(want["dgate"]) + TINY)
            else:
                s, dg = (n_err + E32 * (T + 40) * np.abs(want["dgate"])).sum(0), want["dgate"].sum(0)
                out["dgate"] = (dg, s + r * np.abs(dg) + TINY)
        b, b_err = np.abs(total) * gate * w, tot_err * gate * w
        if v["w_post"] is None:
            err = b_err + 2 * E32 * b
        else:
            b_err = b_err + 3 * E32 * b
            err = ry * (b_err + yn * mean(b_err * yn) + E * (b + 2 * yn * mean(b * yn)))
            s = ((tot_err + (E + E32 * (T + 40)) * np.abs(total)) * gate * yn).sum(0)
            out["dw_post"] = (want["dw_post"], s + r * np.abs(want["dw_post"]) + TINY)
        out["dY"] = (want["dY"], err + r * np.abs(want["dY"]) + TINY)
    return out


def _grad_case(r, T, d, dtype, **kw):
    c = _norm_case(r, T, d, dtype, **kw)
    c.pop("R")
    return c, {n: _rand(r, (T, d), dtype, s).to(DEV) for n, s in (("dH", 0.1), ("dX", 0.1), ("H", 3.0))}


def _grad(m, c, g, **out):
    m.block_norm_grad(g["H"], out.get("dR"), Y=c["Y"], dH=g["dH"], dX=g["dX"], w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"],
                      **{n: t for n, t in out.items() if n != "dR"}, **PAR)


def _outs(c, T, d, dtype):
    new = lambda like: None if like is None else torch.empty_like(like)  # noqa: E731
    return {n: t for n, t in dict(dR=torch.empty(T, d, dtype=_act(dtype), device=DEV), dY=new(c["Y"]), dgate=new(c["gate"]),
                                  dw_post=new(c["w_post"]), dw_pre=new(c["w_pre"])).items() if t is not None}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gate", ["rows", "one"])
@pytest.mark.parametrize("T,d", NORMS + [(2100, 520), (1300, 136)])
def test_block_norm_grad(T, d, gate, dtype):
    c, g = _grad_case(np.random.default_rng(T + d), T, d, dtype, gate=gate)
    m, outs = _m(T=T, d=d, dtype=dtype), _outs(c, T, d, dtype)
    _grad(m, c, g, **outs)
    for n, (want, bound) in _norm_grad_bounds(c, g, gate == "rows", dtype).items():
        _within(outs[n], want, bound, n)
    again = _outs(c, T, d, dtype)
    _grad(m, c, g, **again)
    for n in outs:  # the same bits each time, and each result alone
        assert torch.equal(outs[n], again[n]), n
        alone = torch.empty_like(outs[n])
        _grad(m, c, g, **{n: alone})
        assert torch.equal(outs[n], alone), n


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("without", [("w_post",), ("gate",), ("w_post", "gate"), ("Y", "w_post", "gate"), ("dX", "H", "w_pre"), ("dH",)])
def test_block_norm_grad_without(without, dtype):
    T, d = 45, 264
    c, g = _grad_case(np.random.default_rng(3), T, d, dtype, gate="one", without=without)
    want = _norm_grad_bounds(c, {n: None if n in without and n != "H" else t for n, t in g.items()}, False, dtype)
    for n in without:
        if n in g:
            g[n] = None
    outs = _outs(c, T, d, dtype)
    _grad(_m(T=T, d=d, dtype=dtype), c, g, **outs)
    for n in outs:
        _within(outs[n], *want[n], n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_block_norm_grad_in_place_and_of_wider_tensors(dtype):
    T, d = 300, 200
    c, g = _grad_case(np.random.default_rng(4), T, d, dtype)
    m, outs = _m(T=T, d=d, dtype=dtype), _outs(c, T, d, dtype)
    _grad(m, c, g, **outs)
    for rows in (("dH", "Y"), ("H", "dX"), ("dX", "H"), ("Y", "dH")):
        c2, g2 = {**c, "Y": c["Y"].clone()}, {n: t.clone() for n, t in g.items()}
        got = {**_outs(c, T, d, dtype), "dR": {**c2, **g2}[rows[0]], "dY": {**c2, **g2}[rows[1]]}
        _grad(m, c2, g2, **got)
        for n in outs:
            assert torch.equal(outs[n], got[n]), (rows, n)
    widen = lambda t: torch.full((T, d + 16), 7.0, dtype=t.dtype, device=DEV)  # noqa: E731
    c2, g2, got = dict(c), dict(g), dict(_outs(c, T, d, dtype))
    for box, names in ((c2, ("Y", "gate")), (g2, ("dH", "dX", "H")), (got, ("dR", "dY", "dgate"))):
        for i, n in enumerate(names):
            t, at = widen(box[n]), 8 * (i % 3)
            t[:, at:at + d] = box[n]
            box[n] = t[:, at:at + d]
    _grad(m, c2, g2, **got)
    for n in outs:
        assert torch.equal(outs[n], got[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gate", ["rows", "one", None])
@pytest.mark.parametrize("T,d", [(1, 64), (7, 512), (777, 512), (5, 1000), (2, 1024), (301, 136), (3, 2048)])
def test_norms_without_eps(T, d, gate, dtype, monkeypatch):
    """eps 0, and fewer rows than the teams of the last workgroup: no row there is may be divided by zero, and none that isn't counts"""
    monkeypatch.setitem(PAR, "eps_post", 0.0)
    monkeypatch.setitem(PAR, "eps_pre", 0.0)
    r = np.random.default_rng(T + d)
    c, g = _grad_case(r, T, d, dtype, gate=gate)
    m, outs = _m(T=T, d=d, dtype=dtype), _outs(c, T, d, dtype)
    _grad(m, c, g, **outs)
    want = _norm_grad_bounds(c, g, gate == "rows", dtype)
    for n in outs:
        _within(outs[n], *want[n], n)
    c["R"] = _rand(r, (T, d), dtype, 3.0).to(DEV)
    H, X = torch.empty_like(c["R"]), torch.empty_like(c["R"])
    m.block_norm(c["R"], H, Y=c["Y"], X=X, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
    c = {n: c[n] for n in ("R", "Y", "w_post", "gate", "w_pre")}
    b = _norm_bounds(c, dtype)
    _within(H, *b["H"], "H")
    _within(X, *b["X"], "X")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", [(7, 512), (2, 1000), (301, 136)])
def test_infinite_weights_are_not_multiplied_with_rows_that_are_not_there(T, d, dtype):
    """a channel whose gate or weight is infinite and whose products are positive has an infinite gradient, as the formula says"""
    c, g = _grad_case(np.random.default_rng(T + d), T, d, dtype, gate="one", without=("w_pre",))
    g["dX"] = None
    for t in (g["dH"], c["Y"]):
        t[:, 5] = t[:, 5].abs() + 0.5
    m = _m(T=T, d=d, dtype=dtype)
    clean = _outs(c, T, d, dtype)
    _grad(m, c, g, **clean)
    for infinite, result in (("gate", "dw_post"), ("w_post", "dgate")):
        c2, out = {**c, infinite: c[infinite].clone()}, torch.empty_like(clean[result])
        c2[infinite][5] = float("inf")
        _grad(m, c2, g, **{result: out})
        assert out[5] == float("inf")
        out[5] = clean[result][5]
        assert torch.equal(out, clean[result])


def test_a_residual_scale_that_is_learned():
    """one tensor, another value in each step"""
    c, g = _grad_case(np.random.default_rng(8), 9, 64, "fp32")
    m, scale, H, dR = _m(T=9, d=64, dtype="fp32"), torch.tensor(1.0, device=DEV), torch.empty_like(g["H"]), torch.empty_like(g["H"])
    for v in (1.0, 0.5, -2.0):
        scale.fill_(v)
        m.block_norm(g["H"], H, res_scale=scale)
        m.block_norm_grad(g["H"], dR, dH=g["dH"], res_scale=scale)
        assert torch.equal(H, v * g["H"]) and torch.equal(dR, v * g["dH"])


def test_norms_of_rows_that_are_no_numbers():
    T, d = 40, 512
    r = np.random.default_rng(5)
    c, g = _grad_case(r, T, d, "bf16")
    m, clean, bad = _m(T=T, d=d), _outs(c, T, d, "bf16"), _outs(c, T, d, "bf16")
    _grad(m, c, g, **clean)
    g["dH"][7, 3], c["Y"][9, 4], g["H"][11, 5] = float("nan"), float("inf"), float("nan")
    _grad(m, c, g, **bad)
    rows = [i for i in range(T) if i not in (7, 9, 11)]
    for n in ("dR", "dY", "dgate"):
        assert torch.equal(clean[n][rows], bad[n][rows]), n
    assert torch.isnan(bad["dR"][11]).all() and torch.isnan(bad["dR"][7, 3]) and torch.equal(bad["dR"][9], clean["dR"][9])
    R0 = _rand(r, (T, d), "bf16").to(DEV)
    q, s, H = torch.empty(T, d, dtype=torch.int8, device=DEV), torch.empty(T, device=DEV), torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    R0[3, 3] = float("nan")
    m.block_norm(R0, H, Xq=q, x_scale=s, w_pre=c["w_pre"], **PAR)
    assert torch.isnan(s[3]) and (q[3] == 0).all() and torch.isfinite(s[rows[3] + 1:]).all()


def test_no_rows():
    for dtype in ("bf16", "fp32"):
        m, act = _m(T=0, d=64, dtype=dtype), _act(dtype)
        e, v = torch.empty(0, 64, dtype=act, device=DEV), torch.full((64,), 7.0, dtype=act, device=DEV)
        m.block_norm(e, e.clone(), Y=e.clone(), X=e.clone(), w_post=v, w_pre=v)
        dw, dv, dg = v.clone(), v.clone(), v.clone()
        m.block_norm_grad(e, e.clone(), Y=e, dH=e, dX=e, w_post=v, w_pre=v, gate=v, dw_post=dw, dw_pre=dv, dgate=dg)
        assert not dw.any() and not dv.any() and not dg.any()  # sums of nothing
        m.quantize_rows(e, torch.empty(0, 64, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV))
    q, s = torch.empty(0, 64, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV)
    w, ws = torch.zeros(32, 64, dtype=torch.int8, device=DEV), torch.zeros(32, device=DEV)
    _m().linear_i8(q, s, w, ws, torch.empty(0, 32, dtype=torch.bfloat16, device=DEV))


# ---- together
def test_a_layer_between_its_norms_in_8_bits():
    """norm -> router, 8-bit experts and shared expert -> norm, each step against the oracle on the step's own inputs"""
    r = np.random.default_rng(7)
    T, d, E, k, F = 150, 512, 8, 2, 256
    m = S.SemMoE(S.Config(T=T, d=d, E=E, k=k, F=F, D=2, cap=T // 2), device=DEV)
    c = _norm_case(r, T, d, "bf16")
    H, X = torch.empty_like(c["R"]), torch.empty_like(c["R"])
    q, s = torch.empty(T, d, dtype=torch.int8, device=DEV), torch.empty(T, device=DEV)
    m.block_norm(c["R"], H, Y=c["Y"], X=X, Xq=q, x_scale=s, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
    ids = torch.empty(T, k, dtype=torch.int32, device=DEV)
    tw = torch.empty(T, k, device=DEV)
    m.route(X, _rand(r, (E, d), "bf16", d ** -0.5).to(DEV), ids, tw)
    i32 = dict(dtype=torch.int32, device=DEV)
    e2r = torch.arange(E, **i32) // (E // 2)
    rank, shf, inv, count = (torch.empty(n, **i32) for n in (T, T, T, 2))
    m.reshuffle(ids, e2r, rank, shf, inv, count)
    slot, pair, off, roff = (torch.empty(n, **i32) for n in (T * k, T * k, E + 1, 3))
    phys = torch.arange(E, **i32)
    m.dispatch_index(ids, rank, shf, phys, slot, pair, off, roff, torch.empty(4, **i32), torch.empty(1, dtype=torch.int64, device=DEV))
    qp, sp = torch.empty(T * k, d, dtype=torch.int8, device=DEV), torch.empty(T * k, device=DEV)
    m.dispatch_rows_i8(q, s, slot, qp, sp)
    tok = pair.long() // k
    assert torch.equal(qp, q[tok]) and torch.equal(sp, s[tok])
    wts = [_quantized(r, E * 2 * F, d, 0.05), _quantized(r, E * d, F, 0.05), _quantized(r, 2 * F, d, 0.05), _quantized(r, d, F, 0.05)]
    Y, sh, out = torch.empty(T * k, d, dtype=torch.bfloat16, device=DEV), torch.empty_like(X), torch.empty_like(X)
    for rank_ in (0, 1):
        m.expert_ffn_i8(rank_, qp, sp, off, phys, *wts[0], *wts[1], Y)
    m.shared_ffn_i8(q, s, T, *wts[2], *wts[3], sh)
    m.combine(Y, slot, tw, out, Y_shared=sh)
    H2, X2 = torch.empty_like(X), torch.empty_like(X)
    m.block_norm(H, H2, Y=out, X=X2, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
    n = lambda t: t.cpu().numpy()  # noqa: E731
    offs = n(off)
    for e in range(E):
        at = slice(offs[e], offs[e + 1])
        if offs[e + 1] > offs[e]:
            w = [n(t.view(E, -1, t.shape[1])[e]) if t.dim() == 2 else n(t.view(E, -1)[e]) for pair_ in wts[:2] for t in pair_]
            _ffn_check(_np(Y[at]), n(qp[at]), n(sp[at]), *w, "expert %d" % e)
    _ffn_check(_np(sh), n(q), n(s), *(n(t) for pair_ in wts[2:] for t in pair_), "shared")
    want = (_np(tw)[:, :, None] * _np(Y)[n(slot)].reshape(T, k, d)).sum(1) + _np(sh)
    _within(out, want, (R["bf16"] + 4 * E32) * np.abs(want) + 4 * E32 * (np.abs(_np(Y)[n(slot)]).reshape(T, k, d).sum(1) + np.abs(_np(sh))), "out")
    b = _norm_bounds({**c, "R": H, "Y": out}, "bf16")
    _within(H2, *b["H"], "H")
    _within(X2, *b["X"], "X")


def _all_calls(r):
    """(calls, results): every entry point on one set of tensors"""
    T, d, E, k, F = 96, 512, 4, 2, 384
    m = S.SemMoE(S.Config(T=T, d=d, E=E, k=k, F=F, D=1, cap=T), device=DEV, allocate_workspace=False)
    c, g = _grad_case(r, T, d, "bf16", gate="one")
    c["R"] = _rand(r, (T, d), "bf16").to(DEV)
    H, X = torch.empty_like(c["R"]), torch.empty_like(c["R"])
    q, s = torch.empty(T, d, dtype=torch.int8, device=DEV), torch.empty(T, device=DEV)
    q2, s2 = torch.empty_like(q), torch.empty_like(s)
    slot = torch.from_numpy(r.permutation(T * k).astype(np.int32)).to(DEV)
    qp, sp = torch.empty(T * k, d, dtype=torch.int8, device=DEV), torch.empty(T * k, device=DEV)
    off = torch.tensor([0, 5, 70, 70, T * k], dtype=torch.int32, device=DEV)
    of = torch.arange(E, dtype=torch.int32, device=DEV)
    w = [*_quantized(r, E * 2 * F, d, 0.05), *_quantized(r, E * d, F, 0.05)]
    w[0], w[2] = w[0].view(E, 2 * F, d), w[2].view(E, d, F)
    Y, sh, lin = torch.empty(T * k, d, dtype=torch.bfloat16, device=DEV), torch.empty_like(X), torch.empty(T, 2 * F, dtype=torch.bfloat16, device=DEV)
    outs = _outs(c, T, d, "bf16")

    def calls():
        m.block_norm(c["R"], H, Y=c["Y"], X=X, Xq=q, x_scale=s, w_post=c["w_post"], w_pre=c["w_pre"], gate=c["gate"], **PAR)
        m.quantize_rows(X, q2, s2)
        m.dispatch_rows_i8(q, s, slot, qp, sp)
        m.expert_ffn_i8(-1, qp, sp, off, of, *w, Y)
        m.shared_ffn_i8(q2, s2, T, *w, sh)
        m.linear_i8(q2, s2, w[0][1], w[1].view(E, -1)[1], lin)
        _grad(m, c, g, **outs)

    return calls, [H, X, q, s, q2, s2, qp, sp, Y, sh, lin, *outs.values()], c["R"]


def test_same_bits_on_another_stream_and_in_a_replayed_graph():
    calls, results, R0 = _all_calls(np.random.default_rng(8))
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in results:
            t.zero_()
        calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(3):
        for t in results:
            t.zero_()
        if turn == 1:  # other inputs, between the replays
            R0.mul_(1.5)
            calls()
            want = [t.clone() for t in results]
            for t in results:
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), turn


def test_calls_on_two_streams_at_once():
    (a, ra, _), (b, rb, _) = _all_calls(np.random.default_rng(9)), _all_calls(np.random.default_rng(10))
    a(), b()
    torch.cuda.synchronize()
    want = [t.clone() for t in ra + rb]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(s1):
            a()
        with torch.cuda.stream(s2):
            b()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(ra + rb, want))


def test_offsets_past_32_bits():
    """rows whose numbers lie past 2^31 of the first one's: the last rows as a call of their own gives them"""
    T, d = 300007, 7168
    m, tail = _m(T=T, d=d), 5
    g = torch.Generator(device=DEV).manual_seed(0)
    X = torch.empty(T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    q, s = torch.empty(T, d, dtype=torch.int8, device=DEV), torch.empty(T, device=DEV)
    m.quantize_rows(X, q, s)
    q2, s2 = torch.empty(tail, d, dtype=torch.int8, device=DEV), torch.empty(tail, device=DEV)
    m.quantize_rows(X[-tail:], q2, s2)
    assert torch.equal(q[-tail:], q2) and torch.equal(s[-tail:], s2)
    w, ws = q[:64].contiguous(), s[:64].contiguous()
    Y, Y2 = torch.empty(T, 64, dtype=torch.bfloat16, device=DEV), torch.empty(tail, 64, dtype=torch.bfloat16, device=DEV)
    m.linear_i8(q, s, w, ws, Y)
    m.linear_i8(q2, s2, w, ws, Y2)
    assert torch.equal(Y[-tail:], Y2)
    H, v = torch.empty_like(X), torch.ones(d, dtype=torch.bfloat16, device=DEV)
    m.block_norm(X, H, Y=X, X=X, w_post=v, w_pre=v)
    H2, X2, x = torch.empty(tail, d, dtype=torch.bfloat16, device=DEV), torch.empty(tail, d, dtype=torch.bfloat16, device=DEV), None
    x = torch.empty(T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(0))[-tail:]
    m.block_norm(x, H2, Y=x, X=X2, w_post=v, w_pre=v)
    assert torch.equal(H[-tail:], H2) and torch.equal(X[-tail:], X2)
    dw = torch.empty_like(v)
    m.block_norm_grad(H, H, Y=X, dH=X, w_post=v, dw_post=dw)
    dR = torch.empty_like(H2)
    m.block_norm_grad(H2, dR, Y=X2, dH=X2, w_post=v)
    assert torch.equal(H[-tail:], dR)


def test_more_rows_than_one_launch_takes():
    """narrow rows whose teams have more threads together than a grid may have: as calls on parts of them, and by the values"""
    T, d = (1 << 26) + 77, 8
    g = torch.Generator(device=DEV).manual_seed(1)
    R = torch.empty(T, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    gate, w = torch.empty_like(R).normal_(generator=g), torch.full((d,), 1.5, dtype=torch.bfloat16, device=DEV)
    X, q, s = torch.full_like(R, 7.0), torch.full((T, d), 77, dtype=torch.int8, device=DEV), torch.full((T,), 7.0, device=DEV)
    m, part = _m(T=T, d=d), 1 << 24
    H = torch.full_like(R, 7.0)
    m.block_norm(R, H, Y=R, X=X, Xq=q, x_scale=s, w_pre=w, gate=gate, **PAR)
    for lo in range(0, T, part):
        a = slice(lo, min(lo + part, T))
        H2, X2, q2, s2 = torch.empty_like(R[a]), torch.empty_like(R[a]), torch.empty_like(q[a]), torch.empty_like(s[a])
        m.block_norm(R[a], H2, Y=R[a], X=X2, Xq=q2, x_scale=s2, w_pre=w, gate=gate[a], **PAR)
        assert torch.equal(H[a], H2) and torch.equal(X[a], X2) and torch.equal(q[a], q2) and torch.equal(s[a], s2), lo
    c = dict(R=R[-99:], Y=R[-99:], w_post=None, gate=gate[-99:], w_pre=w)
    b = _norm_bounds(c, "bf16")
    _within(H[-99:], *b["H"], "H")
    _within(X[-99:], *b["X"], "X")


def test_more_rows_to_move_than_one_launch_takes():
    T, d = (1 << 26) + 77, 16
    q = torch.randint(-128, 128, (T, d), dtype=torch.int8, device=DEV)
    s = torch.rand(T, device=DEV)
    slots = torch.arange(T - 1, -1, -1, dtype=torch.int32, device=DEV)
    out, scale = torch.zeros_like(q), torch.zeros_like(s)
    _m(T=T, d=d).dispatch_rows_i8(q, s, slots, out, scale)
    assert torch.equal(out, q.flip(0)) and torch.equal(scale, s.flip(0))


# Rows beyond what the workgroups of the gradient take at once, by the threads of a row: several rows a team, with the next one
# requested ahead or two and four pieces a thread, one team a workgroup and many
MANY_ROWS = [(2600, 1032), (1100, 2048), (1500, 3632), (1050, 4096), (700, 4104), (600, 7168), (600, 8200), (300, 12296), (300, 16384)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gate", ["rows", "one", None])
@pytest.mark.parametrize("T,d", MANY_ROWS)
def test_block_norm_grad_of_several_rows_a_team(T, d, gate, dtype):
    c, g = _grad_case(np.random.default_rng(T + d), T, d, dtype, gate=gate)
    m, outs = _m(T=T, d=d, dtype=dtype), _outs(c, T, d, dtype)
    _grad(m, c, g, **outs)
    for n, (want, bound) in _norm_grad_bounds(c, g, gate == "rows", dtype).items():
        if n in outs:
            _within(outs[n], want, bound, n)
    # in the place of the inputs: a team's next rows are read before its present ones are written, and no others are
    places = [("dH", "Y", "H"), ("H", "dX", "Y"), ("dX", "H", "dH"), ("Y", "dH", "dX")]
    for rows in places:
        c2, g2 = {**c, "Y": c["Y"].clone()}, {n: t.clone() for n, t in g.items()}
        at = {**c2, **g2}
        got = {**_outs(c, T, d, dtype), "dR": at[rows[0]], "dY": at[rows[1]]}
        if gate == "rows":
            got["dgate"] = at[rows[2]]
        _grad(m, c2, g2, **got)
        for n in outs:
            assert torch.equal(outs[n], got[n]), (rows, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("without", [("w_post",), ("w_post", "gate"), ("Y", "w_post", "gate"), ("dX", "H", "w_pre"), ("dH",)])
@pytest.mark.parametrize("T,d", [(2600, 1032), (1050, 4096), (600, 8200), (300, 16384)])
def test_block_norm_grad_of_several_rows_a_team_without(T, d, without, dtype):
    """without w_post a row's second sum, and the barrier that goes with it, falls away"""
    c, g = _grad_case(np.random.default_rng(T), T, d, dtype, gate="one", without=without)
    want = _norm_grad_bounds(c, {n: None if n in without and n != "H" else t for n, t in g.items()}, False, dtype)
    for n in without:
        if n in g:
            g[n] = None
    outs = _outs(c, T, d, dtype)
    _grad(_m(T=T, d=d, dtype=dtype), c, g, **outs)
    for n in outs:
        _within(outs[n], *want[n], n)


@pytest.mark.parametrize("gate", ["rows", "one"])
def test_norm_gradient_past_32_bits(gate):
    """numbers past 2^31 of the first one: the last rows as a call of their own gives them, sums over rows as those of parts"""
    T, d, tail = 300007, 7168, 5
    gen = torch.Generator(device=DEV).manual_seed(2)
    new = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)  # noqa: E731
    g, c = {n: new(T, d) for n in ("dH", "dX", "H")}, dict(Y=new(T, d), w_post=1 + new(d), w_pre=1 + new(d))
    c["gate"] = new(T, d) if gate == "rows" else new(d)
    outs = _outs(c, T, d, "bf16")
    _grad(_m(T=T, d=d), c, g, **outs)
    end = lambda t: t[-tail:].contiguous() if t.shape[0] == T else t  # noqa: E731
    c2, g2 = {n: end(t) for n, t in c.items()}, {n: end(t) for n, t in g.items()}
    last = _outs(c2, tail, d, "bf16")
    _grad(_m(T=tail, d=d), c2, g2, **last)
    rows = ("dR", "dY", "dgate") if gate == "rows" else ("dR", "dY")
    for n in rows:
        assert torch.equal(outs[n][-tail:], last[n]), n
    for n, (want, bound) in _norm_grad_bounds(c2, g2, gate == "rows", "bf16").items():
        _within(last[n], want, bound, n)
    # Sums over rows, in 64 bits by parts.  A term is off by ADDS + 12 roundings of the row's own sums and the products, as in
    # _norm_grad_bounds; its error through dH' is at most as much of |dX w_pre| rh (1 + 2 |xn| mean|xn|), which is taken below; a
    # column's sum passes T / 256 additions in a workgroup and 256 + 40 behind it.
    want = {n: torch.zeros(d, dtype=torch.float64, device=DEV) for n in outs if n not in rows}
    bound = {n: torch.zeros_like(t) for n, t in want.items()}
    E = E32 * (ADDS + 12 + T // 256 + 296)
    for lo in range(0, T, 20000):
        a = slice(lo, lo + 20000)
        dH, dX, H, Y = (t[a].double() for t in (g["dH"], g["dX"], g["H"], c["Y"]))
        gt, wp, wq = (c["gate"][a] if gate == "rows" else c["gate"]).double(), c["w_post"].double(), c["w_pre"].double()
        rh = 1 / (H.square().mean(1, keepdim=True) + PAR["eps_pre"]).sqrt()
        yn = Y / (Y.square().mean(1, keepdim=True) + PAR["eps_post"]).sqrt()
        xn, aw = H * rh, dX * wq
        u = dH + rh * (aw - xn * (aw * xn).mean(1, keepdim=True))
        size = u.abs() + dH.abs() + rh * (aw.abs() + 2 * xn.abs() * (aw * xn).abs().mean(1, keepdim=True))
        for n, term, most in (("dw_pre", dX * xn, (dX * xn).abs()), ("dw_post", u * gt * yn, size * (gt * yn).abs()),
                              ("dgate", u * yn * wp, size * (yn * wp).abs())):
            if n in want:
                want[n] += term.sum(0)
                bound[n] += E * most.sum(0)
    for n in want:
        _within(outs[n], want[n], _np(bound[n] + R["bf16"] * want[n].abs()), n)


@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("d_out", [33000, 66000])
def test_linear_i8_of_weights_past_32_bits(T, d_out):
    """weights beyond 2 and 4 GiB: the first and the last channels as a product of their own gives them"""
    d_in = 65552
    w = torch.randint(-128, 128, (d_out, d_in), dtype=torch.int8, device=DEV)
    q, s, ws = torch.randint(-128, 128, (T, d_in), dtype=torch.int8, device=DEV), torch.rand(T, device=DEV), torch.rand(d_out, device=DEV)
    m, Y = _m(), torch.full((T + 1, d_out), 7.0, dtype=torch.bfloat16, device=DEV)
    m.linear_i8(q, s, w, ws, Y[:T])
    for at in (slice(0, 64), slice(d_out // 2 - 40, d_out // 2 + 40), slice(d_out - 64, d_out)):
        part = w[at].contiguous()
        Z = torch.empty(T, part.shape[0], dtype=torch.bfloat16, device=DEV)
        m.linear_i8(q, s, part, ws[at].clone(), Z)
        assert torch.equal(Y[:T, at], Z)
        want = (q.double() @ part.double().t()) * s.double()[:, None] * ws[at].double()
        _within(Z, want, _np((R["bf16"] + 3 * E32) * want.abs() + TINY), "Z")
    assert (Y[T] == 7.0).all()


def test_expert_ffn_i8_of_an_expert_past_32_bits():
    """an expert's gate and up rows beyond 2 GiB, the second expert's past 4"""
    r = np.random.default_rng(12)
    d, F, rows = 65552, 16400, [0, 9, 3]
    P, E = sum(rows), 3
    m = _m(T=P, d=d, E=E, k=1, F=F)
    w_gu, w_dn = (torch.randint(-128, 128, s, dtype=torch.int8, device=DEV) for s in ((2, 2 * F, d), (2, d, F)))
    s_gu, s_dn = torch.rand(2, 2 * F, device=DEV) * 2e-7 + 1e-7, torch.rand(2, d, device=DEV) * 1e-5
    q, s = torch.randint(-128, 128, (P, d), dtype=torch.int8, device=DEV), torch.rand(P, device=DEV) + 0.5
    off, of = torch.tensor([0, *np.cumsum(rows)], dtype=torch.int32, device=DEV), torch.tensor([0, 1, 0], dtype=torch.int32, device=DEV)
    Y = torch.full((P, d), 7.0, dtype=torch.bfloat16, device=DEV)
    m.expert_ffn_i8(-1, q, s, off, of, w_gu, s_gu, w_dn, s_dn, Y)
    for e, lo, hi in ((1, 0, 9), (0, 9, 12)):
        gu = (q[lo:hi].double() @ w_gu[e].double().t()) * s[lo:hi].double()[:, None] * s_gu[e].double()
        gate = gu[:, :F]
        h = gate * torch.sigmoid(gate) * gu[:, F:]
        eps = (12 + 4 * gate.abs()) * 2.0 ** -23
        near, below, above = (t.to(torch.bfloat16).float().cpu().numpy() for t in (h, h * (1 - eps), h * (1 + eps)))
        (hq, hs), (lq, ls), (uq, us) = (Q.quantize_rows(t) for t in (near, below, above))
        step = hs.astype(np.float64)[:, None]
        D = step * np.maximum(np.abs(uq.astype(float) - hq), np.abs(lq.astype(float) - hq))
        D = np.where((ls != us)[:, None], 2.0 ** -7 * np.abs(near) + 1.01 * step, D)
        W = w_dn[e].double() * s_dn[e].double()[:, None]
        want = (torch.from_numpy(hq).to(DEV).double() @ W.t()) * torch.from_numpy(step).to(DEV)
        spread = torch.from_numpy(D).to(DEV) @ W.abs().t()
        _within(Y[lo:hi], want, _np((R["bf16"] + 4 * E32) * want.abs() + (1 + R["bf16"]) * spread + TINY), "expert %d" % e)
