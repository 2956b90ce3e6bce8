"""The gradients of the row moves and of the expert FFN on the GPU against the fp64 oracle, and a whole layer with adapters
forward and back.

Bounds.  u = 2^-8 is the largest relative error of a rounding to bf16, e = 2^-24 that of fp32.
  * dY = w g: a product in fp32 and a rounding, (r + e) |w g| with r = u or e.
  * dtopk_w: a sum of d products, off by at most e (n + 2) sum |g| |y|, n the most additions that one product passes through: the
    numbers of a thread's walk (8 or 4 a piece, d / (8 * 64) pieces or fewer) and the 6 + 8 steps that join threads.
  * dX of dispatch: k additions and a rounding, e k sum |x| + r |dX|.
  * FFN, a row against its own norm: g, u, dg, du and the result are rounded (r each).  A rounding of g moves dg by
    dh u silu''(g) g and du by dh silu'(g) g, one of u moves dg by dh u silu'(g); these norms over the norm of [dg | du], taken from
    the case's own numbers, times r, and r each for the roundings of [dg | du] and of the result, all pointing the same
    way.  The products with weights drawn at random carry a relative error over to within a few per cent: times 1.25.
    fp32 sums of up to 8192 terms add 2^-24 sqrt(8192) for each of three products, in quadrature below 2e-5."""
import numpy as np
import pytest
import torch

import paper_2503_04398_amd as S
from oracle import gradients as G
from oracle import semmoe_oracle as O
from tests import harness as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
R = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
E32 = 2.0 ** -24


def _act(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _rand(r, shape, dtype, std=1.0):
    return torch.from_numpy(std * r.standard_normal(shape, dtype=np.float32)).to(_act(dtype))


def _layer(T, k, d, dtype, **kw):
    E = kw.pop("E", max(k, 1))
    return S.SemMoE(S.Config(T=T, d=d, E=E, k=k, F=kw.pop("F", 8), D=kw.pop("D", 1), cap=T, dtype=dtype, **kw), device=DEV)


# ---- rows
SHAPES = [(1, 1, 8), (3, 2, 64), (7, 3, 136), (130, 4, 512), (33, 5, 520), (64, 8, 1032), (5, 16, 4104), (9, 13, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,k,d", SHAPES)
def test_combine_grad(T, k, d, dtype):
    r = np.random.default_rng(T + k + d)
    m = _layer(T, k, d, dtype)
    dOut, Y = _rand(r, (T, d), dtype), _rand(r, (T * k, d), dtype)
    w = torch.from_numpy(r.random((T, k), dtype=np.float32))
    slots = torch.from_numpy(r.permutation(T * k).astype(np.int32))
    if T * k > 4:
        slots[2], slots[-1] = -1, T * k  # pairs without a row
    dY = torch.full((T * k, d), 7.0, dtype=_act(dtype), device=DEV)
    dw = torch.full((T, k), 7.0, device=DEV)
    g, y, sl, wd = dOut.to(DEV), Y.to(DEV), slots.to(DEV), w.to(DEV)
    m.combine_grad(g, y, sl, wd, dY, dw)
    want_Y, want_w = G.combine_grad(_np(dOut), _np(Y), slots.numpy(), _np(w))
    named = np.zeros(T * k, dtype=bool)
    named[[s for s in slots.tolist() if 0 <= s < T * k]] = True
    assert (np.abs(_np(dY) - want_Y)[named] <= (R[dtype] + E32) * np.abs(want_Y)[named]).all()
    assert (_np(dY)[~named] == 7.0).all()  # rows that no pair names
    mag = G.combine_grad(np.abs(_np(dOut)), np.abs(_np(Y)), slots.numpy(), _np(w))[1]
    n = 8 * -(-d // 512) + 14 + 8
    assert (np.abs(_np(dw) - want_w) <= E32 * (n + 2) * mag).all()
    # one without the other, and rows over the rows they come from: the same bits
    only_Y, only_w = torch.full_like(dY, 7.0), torch.full_like(dw, 7.0)
    m.combine_grad(g, None, sl, wd, only_Y, None)
    m.combine_grad(g, y, sl, None, None, only_w)
    assert torch.equal(only_Y, dY) and torch.equal(only_w, dw)
    again = torch.full_like(dw, 7.0)
    m.combine_grad(g, y, sl, wd, y, again)
    assert torch.equal(y[torch.from_numpy(named).to(DEV)], dY[torch.from_numpy(named).to(DEV)]) and torch.equal(again, dw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,k,d", SHAPES)
def test_dispatch_grad(T, k, d, dtype):
    r = np.random.default_rng(T * k + d)
    m = _layer(T, k, d, dtype)
    dXp, add = _rand(r, (T * k, d), dtype), _rand(r, (T, d), dtype)
    slots = torch.from_numpy(r.permutation(T * k).astype(np.int32))
    if T * k > 4:
        slots[1], slots[-2] = -3, T * k + 5
    p, sl, ad = dXp.to(DEV), slots.to(DEV), add.to(DEV)
    for extra in (None, add):
        dX = torch.full((T, d), 7.0, dtype=_act(dtype), device=DEV)
        m.dispatch_grad(p, sl, dX, dX_add=None if extra is None else ad)
        want = G.dispatch_grad(_np(dXp), slots.numpy(), k, None if extra is None else _np(extra))
        mag = G.dispatch_grad(np.abs(_np(dXp)), slots.numpy(), k, None if extra is None else np.abs(_np(extra)))
        assert (np.abs(_np(dX) - want) <= R[dtype] * np.abs(want) + E32 * (k + 1) * mag).all()
    m.dispatch_grad(p, sl, ad, dX_add=ad)  # in place
    assert torch.equal(ad, dX)


def test_infinite_and_missing_numbers_stay_in_their_rows():
    r = np.random.default_rng(3)
    T, k, d = 6, 2, 72
    m = _layer(T, k, d, "bf16")
    dOut, Y = _rand(r, (T, d), "bf16").to(DEV), _rand(r, (T * k, d), "bf16").to(DEV)
    w = torch.rand(T, k, device=DEV)
    slots = torch.randperm(T * k, device=DEV).to(torch.int32)
    dY, dw, dX = torch.empty_like(Y), torch.empty_like(w), torch.empty_like(dOut)
    m.combine_grad(dOut, Y, slots, w, dY, dw)
    m.dispatch_grad(Y, slots, dX)
    bad_dY, bad_dw, bad_dX = torch.empty_like(Y), torch.empty_like(w), torch.empty_like(dOut)
    dOut[2, 5], Y[slots[7].long(), 3] = float("inf"), float("nan")  # pair 7: token 3, choice 1
    m.combine_grad(dOut, Y, slots, w, bad_dY, bad_dw)
    m.dispatch_grad(Y, slots, bad_dX)
    assert torch.isnan(bad_dw[3, 1]) and not torch.isfinite(bad_dw[2]).any() and torch.isnan(bad_dX[3, 3])
    keep = [0, 1, 4, 5]
    assert torch.equal(bad_dw[keep], dw[keep]) and torch.equal(bad_dX[keep], dX[keep]) and bad_dw[3, 0] == dw[3, 0]
    rows = slots.view(T, k)[keep].reshape(-1).long()
    assert torch.equal(bad_dY[rows], dY[rows])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_pair_without_a_row_has_no_gradient_whatever_its_token_holds(bad, dtype):
    """a slot outside [0,P) beside numbers of dOut that are not finite: dtopk_w is 0 there, as it is beside finite ones"""
    r = np.random.default_rng(5)
    T, k, d = 6, 3, 72
    m = _layer(T, k, d, dtype)
    dOut, Y = _rand(r, (T, d), dtype), _rand(r, (T * k, d), dtype).to(DEV)
    dOut[1, 7], dOut[4] = bad, bad
    slots = torch.from_numpy(r.permutation(T * k).astype(np.int32))
    gone = [1 * k + 2, 2 * k, 4 * k, 4 * k + 1]
    slots[gone] = torch.tensor([-1, T * k, T * k + 7, -2 ** 31], dtype=torch.int32)
    w = torch.from_numpy(r.random((T, k), dtype=np.float32)).to(DEV)
    for rows in (True, False):
        dY, dw = torch.full_like(Y, 7.0), torch.full((T, k), 7.0, device=DEV)
        m.combine_grad(dOut.to(DEV), Y, slots.to(DEV), w, dY if rows else None, dw)
        got = dw.view(-1).cpu()
        assert (got[gone] == 0.0).all(), got[gone]
        there = [p for p in (1 * k, 1 * k + 1, 4 * k + 2)]
        assert not torch.isfinite(got[there]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [-1, 0x7fffffff, 0x7fc00000, 0x7f800001])
def test_weights_that_are_no_numbers(bits, dtype):
    """NaN of any bits in topk_w (0xffffffff is what memory filled with ones holds) is NaN in that pair's row, and in no other"""
    r = np.random.default_rng(6)
    T, k, d = 5, 2, 72
    m = _layer(T, k, d, dtype)
    dOut, Y = _rand(r, (T, d), dtype).to(DEV), _rand(r, (T * k, d), dtype).to(DEV)
    w = torch.from_numpy(r.random((T, k), dtype=np.float32))
    w[3, 1] = torch.tensor([bits], dtype=torch.int32).view(torch.float32)[0]
    slots = torch.from_numpy(r.permutation(T * k).astype(np.int32))
    dY, dw = torch.full_like(Y, 7.0), torch.full((T, k), 7.0, device=DEV)
    m.combine_grad(dOut, Y, slots.to(DEV), w.to(DEV), dY, dw)
    bad = int(slots[3 * k + 1])
    assert torch.isnan(dY[bad]).all() and torch.isfinite(dY[[i for i in range(T * k) if i != bad]].float()).all()
    assert torch.isfinite(dw).all()


# ---- the expert FFN
def _ffn_tolerance(x, dy, w_gu, w_dn, dtype):
    """see above; of rows x, dy of one expert"""
    F = w_dn.shape[1]
    g, u = x @ w_gu[:F].T, x @ w_gu[F:].T
    dh, sig = dy @ w_dn, 1.0 / (1.0 + np.exp(-g))
    d1 = sig + g * sig * (1.0 - sig)
    d2 = sig * (1.0 - sig) * (2.0 + g * (1.0 - 2.0 * sig))
    norm = np.linalg.norm(np.concatenate([dh * u * d1, dh * g * sig], 1), axis=1)
    by_g = np.linalg.norm(np.concatenate([dh * u * d2 * g, dh * d1 * g], 1), axis=1)
    by_u = np.linalg.norm(dh * u * d1, axis=1)
    return 1.25 * R[dtype] * (2.0 + (by_g + by_u) / norm) + 2e-5


def _ffn(rows, d, F, dtype, D=1, rank=-1, seed=0, alias=None):
    r = np.random.default_rng(seed)
    E, P = len(rows), max(int(sum(rows)), 1)
    X, dY = _rand(r, (P, d), dtype), _rand(r, (P, d), dtype)
    W_gu, W_dn = _rand(r, (E, 2 * F, d), dtype, d ** -0.5), _rand(r, (E, d, F), dtype, F ** -0.5)
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    of_phys = r.permutation(E).astype(np.int32)
    m = _layer(P, 1, d, dtype, E=E, F=F, D=D)
    x, dy = X.to(DEV), dY.to(DEV)
    dX = torch.full((P, d), 512.0, dtype=_act(dtype), device=DEV)
    if alias:
        dX = x if alias == "X" else dy
    m._workspace("expert_ffn_grad", m._ffn_grad_bytes(P))
    for ws in m._own_ws.values():
        ws.fill_(0xff)  # NaN: what nobody writes does not pass for what another call left
    m.expert_ffn_grad(rank, x, dy, torch.from_numpy(off).to(DEV), torch.from_numpy(of_phys).to(DEV), W_gu.to(DEV), W_dn.to(DEV), dX)
    torch.cuda.synchronize()
    lo, hi = (0, E) if rank < 0 else (rank * (E // D), (rank + 1) * (E // D))
    got = _np(dX)
    mine = np.zeros(P, dtype=bool)
    mine[off[lo]:off[hi]] = True
    before = {"X": X, "dY": dY, None: None}[alias]
    assert (got[~mine] == (512.0 if before is None else _np(before)[~mine])).all()  # rows of other ranks stay as they were
    for q in range(lo, hi):
        at = slice(off[q], off[q + 1])
        if off[q] == off[q + 1]:
            continue
        args = [_np(t) for t in (X[at], dY[at], W_gu[of_phys[q]], W_dn[of_phys[q]])]
        want = G.swiglu_ffn_grad(*args)
        err = np.linalg.norm(got[at] - want, axis=1) / np.linalg.norm(want, axis=1)
        tol = _ffn_tolerance(*args, dtype)
        assert (err <= tol).all(), "expert %d: |a-b|/|b| = %.3e, %.3e allowed" % (q, err[(err - tol).argmax()], tol[(err - tol).argmax()])


RAGGED = (0, 1, 15, 16, 17, 33, 64, 65, 0, 130, 31, 48)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,F", [(256, 512), (264, 296), (72, 24), (512, 8), (8, 72), (192, 64)])
def test_ffn_grad_of_ragged_groups(d, F, dtype):
    _ffn(RAGGED, d, F, dtype, seed=d + F)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,d,F", [
    ((1,), 64, 32), ((1, 1, 1, 1), 128, 136), ((0, 0, 0, 5), 64, 64), ((700,), 256, 200), ((300, 290, 1, 513), 192, 320),
    ((600, 400, 520, 480, 700, 300, 510, 490), 256, 384), ((40,) * 16, 512, 1024), ((3,) * 8, 1024, 768)])
def test_ffn_grad(rows, d, F, dtype):
    _ffn(rows, d, F, dtype, seed=len(rows) + d)


# every tile shape with K in whole slices and with a last one that is half, barely or nearly full, columns that end inside a tile:
# few rows or few tiles (128 x 128), 80 rows and more (256 x 128), 192 and more with many tiles (256 x 256)
@pytest.mark.parametrize("rows,d,F", [
    ((70, 20, 5), 520, 264), ((3, 40) * 20, 776, 648), ((90, 130, 100) * 16, 1032, 328), ((250, 200, 300, 190) * 14, 520, 712),
    ((250, 200, 300, 190) * 8, 1016, 776), ((130,) * 40, 312, 1016), ((1100, 1400, 900, 1300) * 2, 568, 1160)])
def test_ffn_grad_with_partial_slices(rows, d, F):
    _ffn(rows, d, F, "bf16", seed=d + len(rows))


@pytest.mark.parametrize("d,F", [(72, 40), (136, 72), (200, 96), (8, 8)])
def test_short_products_give_the_same_bits_every_time(d, F):
    """K of one to three slices, the last with a few rows: nothing is read before its loads have landed"""
    r = np.random.default_rng(d)
    rows, E = (40, 100, 7, 129, 64, 300, 2, 31) * 8, 64
    P = sum(rows)
    m = _layer(P, 1, d, "bf16", E=E, F=F)
    x, dy = _rand(r, (P, d), "bf16").to(DEV), _rand(r, (P, d), "bf16").to(DEV)
    W_gu, W_dn = _rand(r, (E, 2 * F, d), "bf16", d ** -0.5).to(DEV), _rand(r, (E, d, F), "bf16", F ** -0.5).to(DEV)
    off = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device=DEV)
    of = torch.arange(E, dtype=torch.int32, device=DEV)
    other = torch.randn(64 << 20, device=DEV)
    want = None
    for _ in range(12):
        dX = torch.full((P, d), 512.0, dtype=torch.bfloat16, device=DEV)
        other.mul_(-1.0)  # what the caches held goes
        m.expert_ffn_grad(-1, x, dy, off, of, W_gu, W_dn, dX)
        want = dX if want is None else want
        assert torch.equal(dX, want)
    args = [_np(t) for t in (x[:40], dy[:40], W_gu[0], W_dn[0])]
    ref = G.swiglu_ffn_grad(*args)
    err = np.linalg.norm(_np(want)[:40] - ref, axis=1) / np.linalg.norm(ref, axis=1)
    assert (err <= _ffn_tolerance(*args, "bf16")).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rank", [0, 1, 3])
def test_ffn_grad_of_one_rank(rank, dtype):
    _ffn((5, 70, 0, 0, 33, 129, 0, 17), 136, 200, dtype, D=4, rank=rank, seed=rank)


@pytest.mark.parametrize("alias", ["X", "dY"])
def test_ffn_grad_in_place(alias):
    _ffn((5, 70, 0, 33), 136, 200, "bf16", D=2, rank=1, seed=4, alias=alias)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,d,F", [(1, 64, 64), (31, 264, 72), (200, 512, 384), (777, 192, 640), (9000, 520, 1160)])
def test_shared_ffn_grad(n, d, F, dtype):
    r = np.random.default_rng(n)
    m = _layer(n, 1, d, dtype, F=F)
    X, dY = _rand(r, (n, d), dtype), _rand(r, (n, d), dtype)
    W_gu, W_dn = _rand(r, (2 * F, d), dtype, d ** -0.5), _rand(r, (d, F), dtype, F ** -0.5)
    dX = torch.full((n + 1, d), 512.0, dtype=_act(dtype), device=DEV)
    m.shared_ffn_grad(X.to(DEV), dY.to(DEV), n, W_gu.to(DEV), W_dn.to(DEV), dX[:n])
    args = [_np(t) for t in (X, dY, W_gu, W_dn)]
    want = G.swiglu_ffn_grad(*args)
    err = np.linalg.norm(_np(dX)[:n] - want, axis=1) / np.linalg.norm(want, axis=1)
    assert (err <= _ffn_tolerance(*args, dtype)).all() and (dX[n] == 512.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_gate_values(dtype):
    """silu far out on both sides, where exp overflows: dg and du tend to dh u and dh g, or to nothing"""
    d, F = 64, 64
    m = _layer(4, 1, d, dtype, F=F)
    X = torch.zeros(4, d)
    X[0, 0], X[1, 0], X[2, 0], X[3, 0] = 120.0, -120.0, 3.0e4, -3.0e4
    X[:, 1] = 1.0
    W_gu = torch.zeros(2 * F, d)
    W_gu[:F, 0], W_gu[F:, 1] = 1.0, 1.0  # g = x0, u = 1
    dY, W_dn = torch.ones(4, d), torch.full((d, F), 1.0 / 64)  # dh = 1
    dX = torch.empty(4, d, dtype=_act(dtype), device=DEV)
    m.shared_ffn_grad(X.to(_act(dtype)).to(DEV), dY.to(_act(dtype)).to(DEV), 4, W_gu.to(_act(dtype)).to(DEV),
                      W_dn.to(_act(dtype)).to(DEV), dX)
    got = _np(dX)
    x0 = _np(X.to(_act(dtype)))[:, 0]
    assert np.allclose(got[:, 0], [F, 0, F, 0], rtol=2.0 ** -8, atol=1e-30)         # sum over F of dg
    assert np.allclose(got[:, 1], [F * x0[0], 0, F * x0[2], 0], rtol=2.0 ** -7, atol=1e-30)  # sum over F of du


# ---- the expert FFN, held to the roundings that the kernels make
def _rounding_var(x, dtype):
    """mean square of the error of rounding x to the act type: x lies in [2^e, 2^(e+1)), its error anywhere within half a step"""
    half = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}[dtype]
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -100)))
    return (half * 2.0 ** e) ** 2 / 3.0


def _ffn_check(got, x, dy, w_gu, w_dn, dtype):
    """Two roundings to the act type: [dg | du], an operand of the last product, and dX.  g, u and dh are fp32 sums.
    Whole: these roundings are independent, so the square of the error's norm is the sum of their mean squares, those of [dg | du]
        carried over by the squares of the weights, an eighth allowed for (each sum has thousands of terms).  fp32: its roundings are
        those of the sums too, sqrt(n) e for each of the three products of n terms.
    Entries: half a step of each, all pointing the same way, and e (n + 4) of what a sum of n terms adds up, through the
        derivatives of silu; the hardware's exp2 and reciprocal are within 4 e."""
    F, r = w_dn.shape[1], R[dtype]
    d = x.shape[1]
    g, u, dh = x @ w_gu[:F].T, x @ w_gu[F:].T, dy @ w_dn
    sig = 1.0 / (1.0 + np.exp(-g))
    d1 = sig + g * sig * (1.0 - sig)
    d2 = sig * (1.0 - sig) * (2.0 + g * (1.0 - 2.0 * sig))
    dgu = np.concatenate([dh * u * d1, dh * g * sig], 1)
    want = dgu @ w_gu
    e = E32 * (d + 4)
    mg, mu, mh = e * np.abs(x) @ np.abs(w_gu[:F]).T, e * np.abs(x) @ np.abs(w_gu[F:]).T, e * np.abs(dy) @ np.abs(w_dn)
    slack = 12 * E32
    off_g = mh * np.abs(u * d1) + mu * np.abs(dh * d1) + mg * np.abs(dh * u * d2) + slack * np.abs(dh * u) * sig * (1.0 + np.abs(g))
    off_u = mh * np.abs(g * sig) + mg * np.abs(dh * d1) + slack * np.abs(dh * g) * sig * (1.0 + np.abs(g))
    off = np.concatenate([off_g, off_u], 1)
    bound = (r * np.abs(dgu) + (1.0 + r) * off) @ np.abs(w_gu) + E32 * (2 * F + 4) * np.abs(dgu) @ np.abs(w_gu)
    bound = bound + r * (np.abs(want) + bound)
    err = np.abs(got - want)
    at = (err - bound).argmax()
    assert (err <= bound).all(), "an entry is off by %.3e, %.3e allowed" % (err.flat[at], bound.flat[at])
    if want.size >= 2048:
        square = (_rounding_var(dgu, dtype) @ (w_gu * w_gu)).sum() + _rounding_var(want, dtype).sum()
        sums = E32 * np.sqrt(2.0 * d + 2.0 * F) * 2.0
        rel = np.linalg.norm(err) / np.linalg.norm(want)
        allowed = 1.125 * np.sqrt(square) / np.linalg.norm(want) + sums
        assert rel <= allowed, "|a-b|/|b| = %.3e, %.3e allowed" % (rel, allowed)


# every family of tiles: streamed rows, 128 x 128, 256 x 128 and pieces, 256 x 256 and pieces, staged ones for widths that are no multiple
# of 64, short K
TIGHT = [
    ((1, 2, 15, 16, 17, 33), 256, 512), ((3,) * 8, 1024, 768), ((40,) * 16, 512, 1024), ((70, 20, 5), 520, 264), ((64, 65, 130), 72, 40),
    ((90, 130, 100) * 16, 1024, 320), ((250, 200, 300, 190) * 14, 512, 704), ((1100, 1400), 576, 1160), ((700,), 2048, 136)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,d,F", TIGHT)
def test_ffn_grad_rounds_what_it_says_and_nothing_else(rows, d, F, dtype):
    r = np.random.default_rng(d + F)
    E, P = len(rows), int(sum(rows))
    X, dY = _rand(r, (P, d), dtype), _rand(r, (P, d), dtype)
    W_gu, W_dn = _rand(r, (E, 2 * F, d), dtype, d ** -0.5), _rand(r, (E, d, F), dtype, F ** -0.5)
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    m = _layer(P, 1, d, dtype, E=E, F=F)
    dX = torch.full((P, d), 512.0, dtype=_act(dtype), device=DEV)
    m.expert_ffn_grad(-1, X.to(DEV), dY.to(DEV), torch.from_numpy(off).to(DEV), torch.arange(E, dtype=torch.int32, device=DEV),
                      W_gu.to(DEV), W_dn.to(DEV), dX)
    got = _np(dX)
    for q in list(range(E))[:6]:
        at = slice(off[q], off[q + 1])
        _ffn_check(got[at], *(_np(t) for t in (X[at], dY[at], W_gu[q], W_dn[q])), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,d,F", [(1, 64, 64), (256, 1032, 384), (777, 192, 640)])
def test_shared_ffn_grad_rounds_what_it_says_and_nothing_else(n, d, F, dtype):
    r = np.random.default_rng(n + d)
    m = _layer(n, 1, d, dtype, F=F)
    X, dY = _rand(r, (n, d), dtype), _rand(r, (n, d), dtype)
    W_gu, W_dn = _rand(r, (2 * F, d), dtype, d ** -0.5), _rand(r, (d, F), dtype, F ** -0.5)
    dX = torch.full((n, d), 512.0, dtype=_act(dtype), device=DEV)
    m.shared_ffn_grad(X.to(DEV), dY.to(DEV), n, W_gu.to(DEV), W_dn.to(DEV), dX)
    _ffn_check(_np(dX), *(_np(t) for t in (X, dY, W_gu, W_dn)), dtype)


# ---- a layer with adapters, forward and back
@pytest.mark.parametrize("dtype,score", [("fp32", "softmax"), ("bf16", "sigmoid")])
def test_layer_with_adapters_forward_and_back(dtype, score):
    """adapters beside a projection in front of the layer, the layer with its shared expert, and the way back to the adapters: each
    gradient against torch's own through the same graph in fp64, weights of the experts taken as given by the router.
    Tolerance: a chain of 8 rounded tensors forward and back (projection with adapter, X, gate and up, hidden, rows, sum; dY,
    dgate and dup, dX_perm, dX, v) and their sums, each within r of its norm or 2e-5: 12 r + 2e-4 of a gradient's norm."""
    T, d0, d, E, k, F, D, n, rank = 96, 48, 64, 8, 2, 40, 4, 3, 8
    act = _act(dtype)
    r = np.random.default_rng(21)
    cfg = S.Config(T=T, d=d, E=E, k=k, F=F, D=D, dtype=dtype, score=score, renorm=True, cap=-(-T // D))
    m = S.SemMoE(cfg, device=DEV)
    X0, W_p = _rand(r, (T, d0), dtype), _rand(r, (d, d0), dtype, d0 ** -0.5)
    A, B = _rand(r, (n, rank, d0), dtype, d0 ** -0.5), _rand(r, (n, d, rank), dtype, rank ** -0.5)
    scale = torch.from_numpy(r.random(n, dtype=np.float32) + 0.5)
    W_r = _rand(r, (E, d), dtype, 0.2)
    W_gu, W_dn = _rand(r, (E, 2 * F, d), dtype, d ** -0.5), _rand(r, (E, d, F), dtype, F ** -0.5)
    W_gus, W_dns = _rand(r, (2 * F, d), dtype, d ** -0.5), _rand(r, (d, F), dtype, F ** -0.5)
    dOut = _rand(r, (T, d), dtype)
    off, ads = np.array([0, 30, 31, 60, 90], dtype=np.int32), np.array([2, 0, -1, 2], dtype=np.int32)
    dev = lambda t: t.to(DEV)  # noqa: E731
    i32 = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)  # noqa: E731

    def buf(*s):
        return torch.empty(s, dtype=act, device=DEV)
    order, starts = i32(T), i32(n + 1)
    m.adapter_index(dev(torch.from_numpy(off)), dev(torch.from_numpy(ads)), n, order, starts)
    base = (X0.float() @ W_p.float().t()).to(act).to(DEV)  # the shared projection
    X = base.clone()
    m.adapters(dev(X0), order, starts, dev(A), dev(B), X, Y_base=X, scale=dev(scale))
    ids, w = i32(T, k), torch.empty(T, k, device=DEV)
    m.route(X, dev(W_r), ids, w)
    e2r = (torch.arange(E, dtype=torch.int32) // (E // D)).to(DEV)
    phys = torch.arange(E, dtype=torch.int32, device=DEV)
    tr, shf, inv, cnt = i32(T), i32(T), i32(T), i32(D)
    m.reshuffle(ids, e2r, tr, shf, inv, cnt)
    P = T * k
    Xp, slot, pair, eo, ro = buf(P, d), i32(P), i32(P), i32(E + 1), i32(D + 1)
    m.dispatch(X, ids, tr, shf, phys, Xp, slot, pair, eo, ro, i32(D, D), torch.empty(1, dtype=torch.int64, device=DEV))
    Y, Ys, Out = buf(P, d), buf(T, d), buf(T, d)
    Wg, Wd, Wgs, Wds = dev(W_gu), dev(W_dn), dev(W_gus), dev(W_dns)
    m.shared_ffn(X, T, Wgs, Wds, Ys)
    for rank_ in range(D):
        m.expert_ffn(rank_, Xp, eo, phys, Wg, Wd, Y)
    m.combine(Y, slot, w, Out, Y_shared=Ys)
    # back
    dYr, dw, dXp, dX = buf(P, d), torch.empty(T, k, device=DEV), buf(P, d), buf(T, d)
    m.combine_grad(dev(dOut), Y, slot, w, dYr, dw)
    for rank_ in range(D):
        m.expert_ffn_grad(rank_, Xp, dYr, eo, phys, Wg, Wd, dXp)
    m.shared_ffn_grad(X, dev(dOut), T, Wgs, Wds, dX)
    m.dispatch_grad(dXp, slot, dX, dX_add=dX)
    dA, dB, dX0 = torch.empty_like(A, device=DEV), torch.empty_like(B, device=DEV), buf(T, d0)
    m.adapters_grad(dev(X0), dX, order, starts, dev(A), dev(B), dX=dX0, dA=dA, dB=dB, scale=dev(scale))
    torch.cuda.synchronize()

    # the same graph in fp64
    a64, b64, x64 = (t.double().requires_grad_() for t in (A, B, X0))
    w64 = w.cpu().double().requires_grad_()
    of = G.adapter_of_token(off, ads, n, T)
    rows = []
    for i in range(T):
        y = base[i].cpu().double()
        if of[i] >= 0:
            y = y + scale[of[i]].double() * (b64[of[i]] @ (a64[of[i]] @ x64[i]))
        rows.append(y)
    h = torch.stack(rows)

    def ffn(x, gu, dn):
        gu, dn = gu.double(), dn.double()
        gate, up = x @ gu[:F].t(), x @ gu[F:].t()
        return (gate * torch.sigmoid(gate) * up) @ dn.t()
    out = ffn(h, W_gus, W_dns)
    idc = ids.cpu().long()
    every = torch.stack([ffn(h, W_gu[e], W_dn[e]) for e in range(E)])
    for j in range(k):
        out = out + w64[:, j, None] * every[idc[:, j], torch.arange(T)]
    out.backward(dOut.double())
    tol = 12 * R[dtype] + 2e-4
    for name, got, want in (("Out", Out, out.detach()), ("dw", dw, w64.grad), ("dA", dA, a64.grad), ("dB", dB, b64.grad),
                            ("dX0", dX0[:90], x64.grad[:90])):
        want = want.numpy()
        err = np.linalg.norm(_np(got) - want) / np.linalg.norm(want)
        assert err <= tol, "%s: |a-b|/|b| = %.3e" % (name, err)
    assert O.max_rel_err(_np(Out), out.detach().numpy()) <= H.TOL["bf16"]


def test_gradients_replay_in_a_graph():
    T, k, d, E, F = 50, 2, 72, 4, 40
    r = np.random.default_rng(30)
    m = _layer(T, k, d, "bf16", E=E, F=F)
    dOut, Y, X = (_rand(r, s, "bf16").to(DEV) for s in ((T, d), (T * k, d), (T * k, d)))
    w = torch.rand(T, k, device=DEV)
    slots = torch.from_numpy(r.permutation(T * k).astype(np.int32)).to(DEV)
    off = torch.tensor([0, 3, 40, 40, 100], dtype=torch.int32, device=DEV)
    of = torch.arange(4, dtype=torch.int32, device=DEV)
    W_gu, W_dn = _rand(r, (E, 2 * F, d), "bf16", 0.1).to(DEV), _rand(r, (E, d, F), "bf16", 0.1).to(DEV)
    dY, dw, dXp, dX = torch.empty_like(Y), torch.empty_like(w), torch.empty_like(Y), torch.empty_like(dOut)

    def step():
        m.combine_grad(dOut, Y, slots, w, dY, dw)
        m.expert_ffn_grad(-1, X, dY, off, of, W_gu, W_dn, dXp)
        m.shared_ffn_grad(X, dOut, T, W_gu[0], W_dn[0], dX)
        m.dispatch_grad(dXp, slots, dX, dX_add=dX)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (dY, dw, dXp, dX)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (dY, dw, dXp, dX):
            t.fill_(9.0)
        for ws in m._own_ws.values():
            ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        for got, x in zip((dY, dw, dXp, dX), want):
            assert torch.equal(got, x)
