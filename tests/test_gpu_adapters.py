"""Low-rank adapters on the GPU against the fp64 oracle: index, forward and gradient.

Bounds.  u = 2^-8 is the largest relative error of a rounding to bf16, e = 2^-24 that of fp32.  Every result is a chain of two
sums and a last rounding: with h = s A x, Y = base + B h is off by at most
    r |Y|  +  r |B| |h|  +  e (n_1 + n_2) |B| s |A| |x|,
r = u for bf16 rows (h is rounded once as an operand, Y once) and e for fp32, n_1 and n_2 the numbers of terms of the sums (the
worst case of any order of adding).  dX is the same chain.  dA = sum over t tokens of v x^T has |v| |x| summed over the tokens
in the place of |B| |h|, and so dB.  Each entry is held to that; and the whole, whose roundings do not all point the same
way, to 2^-8 (bf16) or 2e-6 (fp32: e times the square root of the terms, thrice) of its norm."""
import threading

import numpy as np
import pytest
import torch

import paper_2503_04398_amd as S
from oracle import gradients as G

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
R = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
E32 = 2.0 ** -24
NORM = {"bf16": 2.0 ** -8, "fp32": 2e-6}


def _act(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Batch:
    """requests of `lens` tokens, with adapters `ads`, then `pad` rows; everything on the CPU in the act type"""

    def __init__(self, lens, ads, n, rank, d_in, d_out, dtype, pad=0, scaled=True, seed=0):
        r = np.random.default_rng(seed)
        self.off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.ads = np.asarray(ads, dtype=np.int32)
        self.n, self.T, self.dtype = n, int(self.off[-1]) + pad, dtype
        act = _act(dtype)

        def make(*shape, std=1.0):
            return torch.from_numpy(std * r.standard_normal(shape, dtype=np.float32)).to(act)
        self.X, self.dY = make(self.T, d_in), make(self.T, d_out)
        self.Yb, self.dXb = make(self.T, d_out), make(self.T, d_in)
        self.A, self.B = make(n, rank, d_in, std=d_in ** -0.5), make(n, d_out, rank, std=rank ** -0.5)
        self.scale = torch.from_numpy(r.random(n, dtype=np.float32) + 0.5) if scaled else None
        self.of = G.adapter_of_token(self.off, self.ads, n, self.T)
        self.order, self.starts = (torch.from_numpy(v) for v in G.adapter_index(self.off, self.ads, n, self.T))
        self.m = S.SemMoE(S.Config(T=max(self.T, 1), d=d_in, E=1, k=1, F=8, D=1, cap=max(self.T, 1), dtype=dtype), device=DEV)

    def dev(self, *names):
        return tuple(None if getattr(self, n) is None else getattr(self, n).to(DEV) for n in names)


def _check(got, want, bound, dtype, what):
    got = _np(got)
    assert np.isfinite(got).all(), what
    off = np.abs(got - want)
    worst = (off - bound).max() if off.size else 0.0
    assert worst <= 0, "%s: off by %.3e where %.3e is allowed" % (what, off.flat[(off - bound).argmax()], bound.flat[(off - bound).argmax()])
    if off.size and np.linalg.norm(want) > 0:
        rel = np.linalg.norm(got - want) / np.linalg.norm(want)
        assert rel <= NORM[dtype], "%s: |a-b|/|b| = %.3e" % (what, rel)


def _bounds(b, Y=None, grads=None):
    """entrywise bounds of the module's header"""
    r, T = R[b.dtype], b.T
    X, dY, A, B = _np(b.X), _np(b.dY), _np(b.A), _np(b.B)
    s = np.ones(b.n) if b.scale is None else _np(b.scale)
    rank, d_in, d_out = A.shape[1], A.shape[2], B.shape[1]
    mine = [np.flatnonzero(b.of == a) for a in range(b.n)]
    if Y is not None:
        out = r * np.abs(Y)
        for a, t in enumerate(mine):
            h = s[a] * np.abs(X[t] @ A[a].T)
            mag = s[a] * np.abs(X[t]) @ np.abs(A[a]).T @ np.abs(B[a]).T
            out[t] += r * h @ np.abs(B[a]).T + E32 * (d_in + rank + 4) * mag
        return out
    dX, dA, dB = grads
    bX, bA, bB = r * np.abs(dX), r * np.abs(dA), r * np.abs(dB)
    for a, t in enumerate(mine):
        v, u = s[a] * np.abs(dY[t] @ B[a]), s[a] * np.abs(X[t] @ A[a].T)
        vm, um = s[a] * np.abs(dY[t]) @ np.abs(B[a]), s[a] * np.abs(X[t]) @ np.abs(A[a]).T
        bX[t] += r * v @ np.abs(A[a]) + E32 * (d_out + rank + 4) * vm @ np.abs(A[a])
        bA[a] += r * v.T @ np.abs(X[t]) + E32 * (d_out + len(t) + 4) * vm.T @ np.abs(X[t])
        bB[a] += r * np.abs(dY[t]).T @ u + E32 * (d_in + len(t) + 4) * np.abs(dY[t]).T @ um
    return bX, bA, bB


def _forward(b, in_place=False, base=True):
    X, order, starts, A, B, scale, Yb = b.dev("X", "order", "starts", "A", "B", "scale", "Yb")
    Y = Yb if in_place else torch.full_like(Yb, 7.0)
    if b.T:
        b.m.adapters(X, order, starts, A, B, Y, Y_base=Yb if base else None, scale=scale)
    torch.cuda.synchronize()
    return Y


def _gradient(b, base=True):
    X, dY, order, starts, A, B, scale, dXb = b.dev("X", "dY", "order", "starts", "A", "B", "scale", "dXb")
    dX, dA, dB = torch.full_like(X, 7.0), torch.full_like(A, 7.0), torch.full_like(B, 7.0)
    b.m.adapters_grad(X, dY, order, starts, A, B, dX=dX, dA=dA, dB=dB, dX_base=dXb if base else None, scale=scale)
    torch.cuda.synchronize()
    return dX, dA, dB


def _both(b, base=True):
    Yb, dXb = (_np(b.Yb), _np(b.dXb)) if base else (None, None)
    s = None if b.scale is None else _np(b.scale)
    X, dY, A, B = _np(b.X), _np(b.dY), _np(b.A), _np(b.B)
    want = G.adapters(X, b.of, A, B, s, Yb, Y=np.full((b.T, B.shape[1]), 7.0))
    _check(_forward(b, base=base), want, _bounds(b, Y=want), b.dtype, "Y")
    wants = G.adapters_grad(X, dY, b.of, A, B, s, dXb, dX=np.full(X.shape, 7.0))
    for got, w, bound, name in zip(_gradient(b, base), wants, _bounds(b, grads=wants), ("dX", "dA", "dB")):
        _check(got, w, bound, b.dtype, name)


# ---- index
INDEX_CASES = [
    ([1], [0], 1, 0), ([5], [-1], 3, 0), ([], [], 2, 3), ([0, 0, 4, 0], [1, 0, 1, 0], 2, 1),
    ([1] * 7, [2, 0, 2, 1, 0, 9, 2], 3, 0), ([3, 1, 64, 65, 0, 2], [0, 4, 2, 2, 1, 4], 5, 5),
    ([1] * 300, [i * 7 % 65 - 1 for i in range(300)], 64, 0), ([700, 1, 1300, 40], [3, 3, 0, 1], 1024, 11),
    ([9] * 1500, [i * i % 37 for i in range(1500)], 30, 0), ([20000], [0], 2, 77), ([0] * 200 + [1], [0] * 201, 1, 0),
]


@pytest.mark.parametrize("case", range(len(INDEX_CASES)))
def test_index(case):
    lens, ads, n, pad = INDEX_CASES[case]
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(off[-1]) + pad
    m = S.SemMoE(S.Config(T=T, d=8, E=1, k=1, F=8, D=1, cap=T), device=DEV)
    order = torch.full((T + 4,), -9, dtype=torch.int32, device=DEV)
    starts = torch.full((n + 5,), -9, dtype=torch.int32, device=DEV)
    m.adapter_index(torch.from_numpy(off).to(DEV), torch.tensor(ads, dtype=torch.int32, device=DEV), n, order[:T], starts[:n + 1])
    torch.cuda.synchronize()
    want_order, want_starts = G.adapter_index(off, ads, n, T)
    assert (order[:T].cpu().numpy() == want_order).all() and (starts[:n + 1].cpu().numpy() == want_starts).all()
    assert (order[T:] == -9).all() and (starts[n + 1:] == -9).all()  # nothing behind them


def test_index_of_offsets_that_say_nonsense_stays_in_bounds():
    """offsets beyond the batch and descending ones: the result is not defined, but every store is inside the arrays"""
    m = S.SemMoE(S.Config(T=40, d=8, E=1, k=1, F=8, D=1, cap=40), device=DEV)
    for off in ([0, 900, 3, -5, 40], [50, 60, 70, 80, 90], [0, -1, -2, -3, -4]):
        order = torch.full((60,), -9, dtype=torch.int32, device=DEV)
        starts = torch.full((8,), -9, dtype=torch.int32, device=DEV)
        m.adapter_index(torch.tensor(off, dtype=torch.int32, device=DEV),
                        torch.tensor([0, 1, 1, 2], dtype=torch.int32, device=DEV), 3, order[10:50], starts[2:6])
        torch.cuda.synchronize()
        assert (order[:10] == -9).all() and (order[50:] == -9).all() and (starts[:2] == -9).all() and (starts[6:] == -9).all()


# ---- forward and gradient: sizes around the tiles (16, 32, 64 tokens; 128 columns; 64, 32 and 16 deep), all ranks' widths
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,ads,n,rank,d_in,d_out,pad", [
    ([1], [0], 1, 8, 8, 8, 0),                                    # one token, the narrowest
    ([1], [0], 3, 16, 72, 40, 0),
    ([2], [-1], 2, 16, 64, 64, 1),                                # nobody has an adapter
    ([3, 0, 2], [0, 0, 5], 4, 24, 136, 264, 2),                   # odd widths, an adapter out of range is none
    ([15, 16, 17, 33], [0, 1, 2, 0], 4, 16, 256, 128, 0),
    ([64, 65, 1, 130], [1, 0, -1, 2], 3, 32, 512, 520, 7),
    ([40] * 3, [0, 0, 0], 1, 48, 248, 72, 0),                     # one adapter, requests of it side by side
    ([5, 9, 4, 70, 3], [1, 0, 1, 1, 0], 2, 64, 328, 640, 0),      # and apart
    ([90, 100], [0, 1], 2, 128, 1032, 392, 3),                    # the widest rank
    ([1] * 50, [i % 17 - 1 for i in range(50)], 16, 8, 2048, 136, 0),  # decode: K in parts
    ([1] * 9, [0, 1, 2, 3, 4, 5, 6, 7, 8], 9, 16, 4096, 4096, 0),
])
def test_adapters_and_gradient(lens, ads, n, rank, d_in, d_out, pad, dtype):
    _both(Batch(lens, ads, n, rank, d_in, d_out, dtype, pad=pad, seed=rank + d_in))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_segments_are_joined(dtype):
    """an adapter with more tokens than one segment of the sums over tokens, beside one with few and one with none"""
    _both(Batch([700, 30, 800], [0, 2, 0], 3, 16, 264, 72, dtype, seed=5))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_without_base_and_scale(dtype):
    _both(Batch([3, 20, 40], [1, -1, 0], 2, 16, 96, 160, dtype, pad=2, scaled=False, seed=6), base=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place_gives_the_same_bits(dtype):
    b = Batch([3, 20, 40], [1, -1, 0], 2, 16, 96, 160, dtype, pad=2, seed=7)
    apart, there = _forward(b), _forward(b, in_place=True)
    assert torch.equal(apart[:63], there[:63]) and torch.equal(there[63:], b.Yb[63:].to(DEV)) and (apart[63:] == 7.0).all()
    X, dY, order, starts, A, B, scale, dXb = b.dev("X", "dY", "order", "starts", "A", "B", "scale", "dXb")
    dX = _gradient(b)[0]
    b.m.adapters_grad(X, dY, order, starts, A, B, dX=dXb, dX_base=dXb, scale=scale)
    assert torch.equal(dX[:63], dXb[:63])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_parts_of_the_gradient_alone(dtype):
    b = Batch([5, 9, 300], [1, 0, 1], 3, 24, 136, 264, dtype, seed=8)
    dX, dA, dB = _gradient(b)
    X, dY, order, starts, A, B, scale, dXb = b.dev("X", "dY", "order", "starts", "A", "B", "scale", "dXb")
    for name, want in (("dX", dX), ("dA", dA), ("dB", dB)):
        got = torch.full_like(want, 3.0)
        b.m.adapters_grad(X, dY, order, starts, A, B, dX_base=dXb, scale=scale, **{name: got})
        assert torch.equal(got, want), name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_column_ranges_of_wider_tensors(dtype):
    """one projection of a fused one: rows further apart than they are wide; what lies beside them is not touched"""
    b = Batch([4, 33, 1], [0, 1, -1], 2, 16, 72, 136, dtype, pad=3, seed=9)
    X, dY, order, starts, A, B, scale, Yb, dXb = b.dev("X", "dY", "order", "starts", "A", "B", "scale", "Yb", "dXb")

    def wide(t, left, right):
        w = torch.full((t.shape[0], left + t.shape[1] + right), 5.0, dtype=t.dtype, device=DEV)
        w[:, left:left + t.shape[1]] = t
        return w, w[:, left:left + t.shape[1]]
    (_, x), (_, dy), (_, yb), (_, dxb) = wide(X, 8, 16), wide(dY, 16, 0), wide(Yb, 0, 8), wide(dXb, 8, 8)
    y_all, y = wide(torch.full_like(Yb, 7.0), 24, 8)
    b.m.adapters(x, order, starts, A, B, y, Y_base=yb, scale=scale)
    assert torch.equal(y, _forward(b)) and (y_all[:, :24] == 5.0).all() and (y_all[:, -8:] == 5.0).all()
    dx_all, dx = wide(torch.full_like(dXb, 7.0), 8, 24)
    dA, dB = torch.empty_like(A), torch.empty_like(B)
    b.m.adapters_grad(x, dy, order, starts, A, B, dX=dx, dA=dA, dB=dB, dX_base=dxb, scale=scale)
    for got, want in zip((dx, dA, dB), _gradient(b)):
        assert torch.equal(got, want)
    assert (dx_all[:, :8] == 5.0).all() and (dx_all[:, -24:] == 5.0).all()


def test_one_row_of_a_wider_tensor():
    b = Batch([1], [0], 1, 8, 16, 24, "bf16", seed=10)
    X, order, starts, A, B, scale, Yb = b.dev("X", "order", "starts", "A", "B", "scale", "Yb")
    X_all = torch.randn(1, 40, device=DEV).bfloat16()
    X_all[:, 8:24] = X
    Y = torch.empty_like(Yb)
    b.m.adapters(X_all[:, 8:24], order, starts, A, B, Y, Y_base=Yb, scale=scale)
    assert torch.equal(Y, _forward(b))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_token_is_touched_by_its_own_adapter_alone(dtype):
    """infinities and NaN in one request's rows and in one adapter stay there"""
    b = Batch([20, 20, 5, 30], [0, 1, -1, 2], 3, 16, 136, 72, dtype, pad=4, seed=11)
    clean, clean_grad = _forward(b), _gradient(b)
    for t in (b.X, b.dY):
        t[20:40] = float("nan")
        t[45:75, ::2] = float("inf")
        t[75:] = float("nan")  # padding
    b.A[1], b.B[2, :, 3] = float("nan"), float("inf")
    Y, (dX, dA, dB) = _forward(b), _gradient(b)
    for got, want in ((Y, clean), (dX, clean_grad[0])):
        assert torch.equal(got[:20], want[:20]) and torch.equal(got[40:45], want[40:45]) and torch.equal(got[75:], want[75:])
        assert not torch.isfinite(got[20:40].float()).any()
    assert torch.equal(dA[0], clean_grad[1][0]) and torch.equal(dB[0], clean_grad[2][0])


def test_an_order_that_says_nonsense_stays_in_bounds():
    """tokens outside the batch and offsets that overlap or descend: nothing outside the tensors is read or written"""
    b = Batch([20, 300, 30], [0, 1, 2], 3, 16, 72, 136, "bf16", pad=2, seed=12)
    X, dY, A, B = b.dev("X", "dY", "A", "B")
    bad = b.order.clone()
    bad[::7], bad[3::11] = 10 ** 9, -5
    for starts in ([0, 20, 320, 350], [0, 400, 0, 400], [-7, 10 ** 9, -10 ** 9, 5], [352, 3, 2, 1]):
        off = torch.tensor(starts, dtype=torch.int32, device=DEV)
        Y = torch.full((b.T + 8, 136), 7.0, dtype=torch.bfloat16, device=DEV)
        b.m.adapters(X, bad.to(DEV), off, A, B, Y[4:-4])
        dX = torch.full((b.T + 8, 72), 7.0, dtype=torch.bfloat16, device=DEV)
        dA = torch.full((5, 16, 72), 7.0, dtype=torch.bfloat16, device=DEV)
        dB = torch.full((5, 136, 16), 7.0, dtype=torch.bfloat16, device=DEV)
        b.m.adapters_grad(X, dY, bad.to(DEV), off, A, B, dX=dX[4:-4], dA=dA[1:4], dB=dB[1:4])
        torch.cuda.synchronize()
        for t, n in ((Y, 4), (dX, 4), (dA, 1), (dB, 1)):
            assert (t[:n] == 7.0).all() and (t[-n:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,n,rank,d_in,d_out", [
    ([7] * 100, 130, 16, 72, 136),      # more adapters than a wave has lanes
    ([2] * 40, 1000, 8, 64, 40),        # far more than tokens
    ([700, 3, 900, 5, 640], 200, 24, 136, 72),  # long segments behind many empty adapters
])
def test_many_adapters(lens, n, rank, d_in, d_out, dtype):
    _both(Batch(lens, [i * 37 % n for i in range(len(lens))][::-1], n, rank, d_in, d_out, dtype, pad=3, seed=n))


@pytest.mark.parametrize("T", [2048, 8200])
def test_larger_tiles(T):
    """the token tiles of long batches: 32 in the first kernel, 32 and 64 in the second; 64 in both at rank 64"""
    b = Batch([T // 3, T // 3, T - 2 * (T // 3)], [0, 1, 0], 2, 64 if T < 8192 else 16, 72, 136, "bf16", seed=T)
    _both(b)


def test_largest_tiles():
    T = 16384
    _both(Batch([9000, T - 9000 - 5], [0, 1], 2, 64, 136, 72, "bf16", pad=5, seed=3))


@pytest.mark.parametrize("T,rank", [(65600, 16), (32800, 32), (40000, 40), (16400, 128), (131100, 8)])
def test_long_batches_of_every_rank(T, rank):
    """T * rank past every line of the tiles' choice, where only some ranks have the largest tiles"""
    _both(Batch([T // 2 + 11, 3, T - T // 2 - 30], [1, 2, 0], 3, rank, 40, 72, "bf16", pad=16, seed=rank))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gradient_in_the_place_of_its_inputs(dtype):
    b = Batch([40, 300, 7], [0, 1, -1], 2, 16, 136, 136, dtype, pad=2, seed=16)
    want = _gradient(b)
    for place in ("X", "dY"):
        X, dY, order, starts, A, B, scale, dXb = b.dev("X", "dY", "order", "starts", "A", "B", "scale", "dXb")
        dX, dA, dB = (X if place == "X" else dY), torch.empty_like(A), torch.empty_like(B)
        b.m.adapters_grad(X, dY, order, starts, A, B, dX=dX, dA=dA, dB=dB, dX_base=dXb, scale=scale)
        for got, w in zip((dX[:347], dA, dB), (want[0][:347], want[1], want[2])):
            assert torch.equal(got, w), place


def test_calls_on_two_streams_at_once():
    """each stream has a workspace of its own"""
    a, c = Batch([500, 700], [0, 1], 2, 32, 1032, 1032, "bf16", seed=17), Batch([900, 300], [1, 0], 2, 32, 1032, 1032, "bf16", seed=18)
    c.m = a.m
    want = [_forward(a), _forward(c), *_gradient(a), *_gradient(c)]
    ins = [x.dev("X", "dY", "order", "starts", "A", "B", "scale", "Yb", "dXb") for x in (a, c)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [None, None]
        for i, s in enumerate(streams):
            X, dY, order, starts, A, B, scale, Yb, dXb = ins[i]
            with torch.cuda.stream(s):
                out = [torch.empty_like(Yb), torch.empty_like(X), torch.empty_like(A), torch.empty_like(B)]
                for _ in range(4):
                    a.m.adapters(X, order, starts, A, B, out[0], Y_base=Yb, scale=scale)
                    a.m.adapters_grad(X, dY, order, starts, A, B, dX=out[1], dA=out[2], dB=out[3], dX_base=dXb, scale=scale)
                got[i] = out
        torch.cuda.synchronize()
        assert torch.equal(got[0][0], want[0]) and torch.equal(got[1][0], want[1])
        for x, y in zip(got[0][1:] + got[1][1:], want[2:]):
            assert torch.equal(x, y)


def test_no_tokens_through_the_binding():
    b = Batch([], [], 2, 8, 16, 24, "bf16")
    X, dY, order, starts, A, B = b.dev("X", "dY", "order", "starts", "A", "B")
    starts.fill_(9)
    b.m.adapter_index(torch.zeros(1, dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), 2, order, starts)
    assert (starts == 0).all()
    b.m.adapters(X, order, starts, A, B, dY)
    dA, dB = torch.ones_like(A), torch.ones_like(B)
    b.m.adapters_grad(X, dY, order, starts, A, B, dX=X, dA=dA, dB=dB)
    assert (dA == 0).all() and (dB == 0).all()


def test_no_tokens():
    b = Batch([], [], 2, 8, 16, 24, "bf16")
    m, lib = b.m, b.m.lib
    dA, dB = torch.full((2, 8, 16), 7.0, device=DEV).bfloat16(), torch.full((2, 24, 8), 7.0, device=DEV).bfloat16()
    one = torch.zeros(8, 24, dtype=torch.bfloat16, device=DEV)  # a tensor without rows has no address
    import ctypes as C
    from paper_2503_04398_amd import binding as Bn
    c, s = m._cfg(T=0), Bn._CAdapterShape(2, 8, 16, 24, 0, 0, 0, 0)
    A, B, starts = b.A.to(DEV), b.B.to(DEV), b.starts.to(DEV)
    ws = torch.empty(1024, dtype=torch.uint8, device=DEV)
    p = one.data_ptr()
    assert lib.semmoe_adapters(C.byref(c), None, C.byref(s), p, p, starts.data_ptr(), A.data_ptr(), B.data_ptr(), None, None, p,
                               ws.data_ptr(), 1024) == 0
    assert lib.semmoe_adapters_grad(C.byref(c), None, C.byref(s), p, p, p, starts.data_ptr(), A.data_ptr(), B.data_ptr(), None,
                                    None, p, dA.data_ptr(), dB.data_ptr(), ws.data_ptr(), 1024) == 0
    torch.cuda.synchronize()
    assert (dA == 0).all() and (dB == 0).all() and (one == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_same_bits_on_another_stream_and_in_a_replayed_graph(dtype):
    b = Batch([5, 80, 300, 1], [1, 0, 1, -1], 3, 16, 264, 136, dtype, pad=2, seed=13)
    eager_Y, eager = _forward(b), _gradient(b)
    X, dY, A, B, scale, Yb, dXb = b.dev("X", "dY", "A", "B", "scale", "Yb", "dXb")
    off, ads = torch.from_numpy(b.off).to(DEV), torch.from_numpy(b.ads).to(DEV)
    order, starts = torch.empty(b.T, dtype=torch.int32, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV)
    Y, dX, dA, dB = torch.empty_like(Yb), torch.empty_like(X), torch.empty_like(A), torch.empty_like(B)

    def step():
        b.m.adapter_index(off, ads, 3, order, starts)
        b.m.adapters(X, order, starts, A, B, Y, Y_base=Yb, scale=scale)
        b.m.adapters_grad(X, dY, order, starts, A, B, dX=dX, dA=dA, dB=dB, dX_base=dXb, scale=scale)

    def same():
        n = int(b.off[-1])
        assert torch.equal(Y[:n], eager_Y[:n]) and torch.equal(dX[:n], eager[0][:n])
        assert torch.equal(dA, eager[1]) and torch.equal(dB, eager[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (Y, dX, dA, dB):
            t.fill_(9.0)
        order.zero_()
        _forward(b)  # the program's own work between replays, on the same workspace
        graph.replay()
        torch.cuda.synchronize()
        same()


def test_a_larger_call_leaves_the_workspace_of_a_captured_graph_alone():
    small, large = (Batch([n], [0], 1, 16, 64, 64, "bf16", seed=14) for n in (40, 900))
    X, order, starts, A, B, scale, Yb = small.dev("X", "order", "starts", "A", "B", "scale", "Yb")
    want = _forward(small)
    Y = torch.empty_like(Yb)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        small.m.adapters(X, order, starts, A, B, Y, Y_base=Yb, scale=scale)
    held = large.dev("X", "order", "starts", "A", "B", "scale", "Yb")
    for _ in range(3):
        small.m.adapters(held[0], held[1], held[2], held[3], held[4], torch.empty_like(held[6]), Y_base=held[6], scale=held[5])
        other = torch.full((1 << 20,), 77, dtype=torch.uint8, device=DEV)  # would take a freed workspace's place
        Y.fill_(0.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want) and (other == 77).all()


def test_graphs_beside_each_other():
    """a captured graph has a workspace of its own, whatever stream it was captured on and whatever runs beside it"""
    a, c = Batch([500, 700], [0, 1], 2, 32, 1032, 1032, "bf16", seed=19), Batch([900, 300], [1, 0], 2, 32, 1032, 1032, "bf16", seed=20)
    c.m = a.m
    want = [[_forward(x), *_gradient(x)] for x in (a, c)]
    capture, streams, graphs, outs = torch.cuda.Stream(), [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    kept, held = dict(a.m._own_ws), []
    for x in (a, c):
        X, dY, order, starts, A, B, scale, Yb, dXb = ins = x.dev("X", "dY", "order", "starts", "A", "B", "scale", "Yb", "dXb")
        out = [torch.empty_like(Yb), torch.empty_like(X), torch.empty_like(A), torch.empty_like(B)]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=capture):
            a.m.adapters(X, order, starts, A, B, out[0], Y_base=Yb, scale=scale)
            a.m.adapters_grad(X, dY, order, starts, A, B, dX=out[1], dA=out[2], dB=out[3], dX_base=dXb, scale=scale)
        held.append(ins)
        graphs.append(graph)
        outs.append(out)
    assert a.m._own_ws.keys() == kept.keys() and all(a.m._own_ws[k] is kept[k] for k in kept)
    for _ in range(3):
        for out in outs:
            for t in out:
                t.fill_(9.0)
        torch.cuda.synchronize()
        for _ in range(4):
            for s, graph in zip(streams, graphs):
                with torch.cuda.stream(s):
                    graph.replay()
        eager = _forward(a)
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0][0])
        for out, w in zip(outs, want):
            for got, x in zip(out, w):
                assert torch.equal(got, x)


def test_offsets_past_32_bits():
    """rows of a wide tensor whose last ones lie more than 2^31 elements behind the first"""
    T, d, r, wide = 66000, 64, 8, 36864
    if torch.cuda.mem_get_info()[0] < 3 * T * wide * 2:
        pytest.skip("not enough memory")
    g = torch.Generator(device=DEV).manual_seed(15)
    X_all = torch.empty(T, wide, dtype=torch.bfloat16, device=DEV)
    Y_all = torch.empty(T, wide, dtype=torch.bfloat16, device=DEV)
    X, Y = X_all[:, wide - d:], Y_all[:, wide - d:]
    X.copy_(torch.randn(T, d, device=DEV, generator=g))
    Y.zero_()
    A = torch.randn(2, r, d, device=DEV, generator=g).mul_(0.125).bfloat16()
    B = torch.randn(2, d, r, device=DEV, generator=g).mul_(0.25).bfloat16()
    m = S.SemMoE(S.Config(T=T, d=d, E=1, k=1, F=8, D=1, cap=T), device=DEV)
    off = torch.tensor([0, 30000, T], dtype=torch.int32, device=DEV)
    ads = torch.tensor([1, 0], dtype=torch.int32, device=DEV)
    order, starts = torch.empty(T, dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    m.adapter_index(off, ads, 2, order, starts)
    m.adapters(X, order, starts, A, B, Y)
    packed = torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    m.adapters(X.contiguous(), order, starts, A, B, packed)
    assert torch.equal(Y.contiguous(), packed)
    for t in (0, 29999, 30000, T - 1):
        a = 1 if t < 30000 else 0
        want = _np(B[a]) @ (_np(A[a]) @ _np(X[t]))
        # one rounding of h as an operand, one of the result
        assert np.linalg.norm(_np(Y[t]) - want) <= 2.0 ** -7 * np.linalg.norm(want)


def test_calls_of_two_threads_on_one_stream():
    """the launches of two threads' calls may come in turns: each thread has sums of its own"""
    a, c = Batch([500, 700], [0, 1], 2, 32, 1032, 1032, "bf16", seed=21), Batch([900, 300], [1, 0], 2, 32, 1032, 1032, "bf16", seed=22)
    want = [[_forward(x), *_gradient(x)] for x in (a, c)]
    ins = [x.dev("X", "dY", "order", "starts", "A", "B", "scale", "Yb", "dXb") for x in (a, c)]
    outs = [[torch.empty_like(t) for t in (i[7], i[0], i[4], i[5])] for i in ins]
    torch.cuda.synchronize()
    start, failed = threading.Barrier(2), []

    def work(i):
        X, dY, order, starts, A, B, scale, Yb, dXb = ins[i]
        Y, dX, dA, dB = outs[i]
        start.wait()
        try:
            for _ in range(100):
                a.m.adapters(X, order, starts, A, B, Y, Y_base=Yb, scale=scale)
                a.m.adapters_grad(X, dY, order, starts, A, B, dX=dX, dA=dA, dB=dB, dX_base=dXb, scale=scale)
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for out, w in zip(outs, want):
        for got, x in zip(out, w):
            assert torch.equal(got, x)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,n", [
    ([129, 257, 1, 300, 128, 2, 385], 7),   # adapters of one and of several segments of 128 tokens side by side
    ([130] * 20, 20),                       # each just longer than a segment
    ([1300, 1, 1100, 5, 2500, 1025, 7], 300)])
def test_adapters_of_several_segments_side_by_side(lens, n, dtype):
    _both(Batch(lens, list(range(len(lens))), n, 16, 72, 136, dtype, pad=3, seed=n))


def test_the_sums_of_segments_stay_in_their_places():
    """what lies behind the workspace that the library asks for is not written, whatever the lengths"""
    import ctypes as C
    from paper_2503_04398_amd import binding as Bn
    for lens, n in (([129, 257, 1, 300, 128, 2, 385], 7), ([2600], 1), ([1000, 1040], 2), ([1] * 40 + [1500], 41)):
        b = Batch(lens, list(range(n)), n, 16, 72, 136, "bf16", seed=n)
        want, want_Y = _gradient(b), _forward(b)
        X, dY, order, starts, A, B, scale, Yb, dXb = b.dev("X", "dY", "order", "starts", "A", "B", "scale", "Yb", "dXb")
        c, s, size = b.m._cfg(T=b.T), Bn._CAdapterShape(n, 16, 72, 136, 0, 0, 0, 0), C.c_size_t(0)
        dX, dA, dB, Y = torch.empty_like(X), torch.empty_like(A), torch.empty_like(B), torch.empty_like(Yb)
        p = lambda *ts: [t.data_ptr() for t in ts]  # noqa: E731
        assert b.m.lib.semmoe_adapter_workspace_bytes(C.byref(c), C.byref(s), C.byref(size)) == 0
        ws = torch.full((size.value + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
        assert b.m.lib.semmoe_adapters_grad(C.byref(c), None, C.byref(s), *p(X, dY, order, starts, A, B, scale, dXb, dX, dA, dB, ws),
                                            size.value) == 0
        torch.cuda.synchronize()
        assert (ws[size.value:] == 0xa5).all()
        for got, w in zip((dX, dA, dB), want):
            assert torch.equal(got, w)
        assert b.m.lib.semmoe_adapter_forward_workspace_bytes(C.byref(c), C.byref(s), C.byref(size)) == 0
        ws.fill_(0xa5)
        assert b.m.lib.semmoe_adapters(C.byref(c), None, C.byref(s), *p(X, order, starts, A, B, scale, Yb, Y, ws), size.value) == 0
        torch.cuda.synchronize()
        assert (ws[size.value:] == 0xa5).all() and torch.equal(Y, want_Y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [-1, 0x7fffffff, 0x7fc00000, 0x7f800001, -4194304])
def test_a_scale_that_is_no_number(bits, dtype):
    """NaN of any bits (0xffffffff is what memory filled with ones holds) reaches all that the adapter adds to, and nothing else"""
    b = Batch([20, 3, 300], [0, 1, 0], 2, 16, 64, 40, dtype, seed=31)
    clean, clean_grad = _forward(b), _gradient(b)
    b.scale[0] = torch.tensor([bits], dtype=torch.int32).view(torch.float32)[0]
    Y, (dX, dA, dB) = _forward(b), _gradient(b)
    for got, want in ((Y, clean), (dX, clean_grad[0])):
        assert torch.isnan(got[:20]).all() and torch.isnan(got[23:]).all() and torch.equal(got[20:23], want[20:23])
    for got, want in ((dA, clean_grad[1]), (dB, clean_grad[2])):
        assert torch.isnan(got[0]).all() and torch.equal(got[1], want[1])


def test_infinite_products_stay_infinite():
    """an infinity in a row is one in what its token gets, and no NaN"""
    b = Batch([20, 3], [0, 1], 2, 16, 64, 40, "bf16", seed=31)
    b.A[0], b.B[0], b.X[:20] = 1.0, 1.0, 1.0
    b.X[4, 9] = float("inf")
    Y = _forward(b)
    assert (Y[4] == float("inf")).all() and torch.isfinite(Y[:4].float()).all() and torch.isfinite(Y[5:].float()).all()


# ---- one rounding: u and v are operands in two parts that hold 16 bits between them, the results are rounded once
def _once(got, want, parts, dtype, what):
    """parts: |B| |h| and the like, what a relative error of h is carried over by.  Entries: half a step of the result, 2^-16 of the
    parts (the second half of h is within 2^-8 of what the first leaves, which is 2^-8 of h) and the sums' fp32.  Whole: the
    errors of the rounding lie anywhere within half a step, so their mean square is a third of its square; an eighth allowed for."""
    got, (h, mag, n) = _np(got), parts
    assert np.isfinite(got).all(), what
    off, u = np.abs(got - want), R[dtype]
    bound = u * np.abs(want) + (1.0 + u) * ((2.0 ** -16 if dtype == "bf16" else 0.0) * h + E32 * n * mag)
    at = (off - bound).argmax()
    assert (off <= bound).all(), "%s: off by %.3e where %.3e is allowed" % (what, off.flat[at], bound.flat[at])
    if want.size >= 2048 and dtype == "bf16":
        e = np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -100)))
        allowed = 1.125 * np.sqrt(((u * 2.0 ** e) ** 2 / 3.0).sum()) / np.linalg.norm(want)
        rel = np.linalg.norm(off) / np.linalg.norm(want)
        assert rel <= allowed, "%s: |a-b|/|b| = %.3e, %.3e allowed" % (what, rel, allowed)


def _both_once(b):
    X, dY, A, B = _np(b.X), _np(b.dY), _np(b.A), _np(b.B)
    s = np.ones(b.n) if b.scale is None else _np(b.scale)
    rank, d_in, d_out = A.shape[1], A.shape[2], B.shape[1]
    zero = lambda t: np.zeros(t.shape)  # noqa: E731
    Y, Yh, Ym = (np.zeros((b.T, d_out)) for _ in range(3))
    (dX, Xh, Xm), (dA, Ah, Am), (dB, Bh, Bm) = ([zero(t) for _ in range(3)] for t in (X, A, B))
    for a in range(b.n):
        t = np.flatnonzero(b.of == a)
        u, v, um, vm = s[a] * X[t] @ A[a].T, s[a] * dY[t] @ B[a], s[a] * np.abs(X[t]) @ np.abs(A[a]).T, s[a] * np.abs(dY[t]) @ np.abs(B[a])
        for out, h, m_, left, hi, mag in ((Y, Yh, Ym, B[a].T, u, um), (dX, Xh, Xm, A[a], v, vm)):
            out[t], h[t], m_[t] = hi @ left, np.abs(hi) @ np.abs(left), mag @ np.abs(left)
        dA[a], Ah[a], Am[a] = v.T @ X[t], np.abs(v).T @ np.abs(X[t]), vm.T @ np.abs(X[t])
        dB[a], Bh[a], Bm[a] = dY[t].T @ u, np.abs(dY[t]).T @ np.abs(u), np.abs(dY[t]).T @ um
    longest = max([int((b.of == a).sum()) for a in range(b.n)] + [rank])
    got = _forward(b, base=False)
    own = b.of >= 0
    _once(got[torch.from_numpy(own).to(DEV)], Y[own], (Yh[own], Ym[own], d_in + rank + 4), b.dtype, "Y")
    g = _gradient(b, base=False)
    _once(g[0][torch.from_numpy(own).to(DEV)], dX[own], (Xh[own], Xm[own], d_out + rank + 4), b.dtype, "dX")
    _once(g[1], dA, (Ah, Am, d_out + longest + 4), b.dtype, "dA")
    _once(g[2], dB, (Bh, Bm, d_in + longest + 4), b.dtype, "dB")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,ads,n,rank,d_in,d_out", [
    ([1], [0], 1, 8, 64, 40), ([3, 0, 2], [0, 0, 5], 4, 24, 136, 264), ([64, 65, 1, 130], [1, 0, -1, 2], 3, 32, 512, 520),
    ([700, 30, 800], [0, 2, 0], 3, 16, 264, 72), ([5, 9, 4, 70, 3], [1, 0, 1, 1, 0], 2, 64, 328, 640),
    ([90, 100], [0, 1], 2, 128, 1032, 392), ([1] * 50, [i % 17 - 1 for i in range(50)], 16, 8, 2048, 136),
    ([1300, 1200], [0, 1], 2, 72, 136, 72), ([5000, 3300], [0, 1], 2, 64, 72, 40)])
def test_results_are_rounded_once(lens, ads, n, rank, d_in, d_out, dtype):
    _both_once(Batch(lens, ads, n, rank, d_in, d_out, dtype, seed=rank + 3))


# ---- the token tiles of long batches in fp32, and results in the place of X
@pytest.mark.parametrize("T,n,rank,d_in,d_out", [
    (2048, 2, 16, 72, 136), (2100, 3, 64, 136, 72), (4200, 2, 128, 136, 264), (8200, 2, 16, 72, 40), (8250, 3, 32, 40, 136),
    (8192, 2, 64, 264, 72), (8300, 2, 128, 72, 136), (16400, 2, 64, 136, 72), (16500, 1, 40, 40, 72), (16400, 2, 128, 40, 72), (131100, 2, 8, 40, 24)])
def test_wide_tiles_in_fp32(T, n, rank, d_in, d_out):
    """32 and 64 tokens in `expand`, 32 and (ranks 33 to 64) 64 in `shrink`, with tiles that end inside a request"""
    lens = [T // 2 + 11, 3, T - T // 2 - 30]
    _both(Batch(lens, [(i + 1) % n if n > 1 else 0 for i in range(3)] if n > 2 else [0, n - 1, 0], n, rank, d_in, d_out, "fp32", pad=16, seed=rank + T))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,rank", [(40, 16), (2100, 64), (8300, 128)])
def test_result_in_the_place_of_x(T, rank, dtype):
    b = Batch([T // 2, T - T // 2 - 5, 3], [0, 1, -1], 2, rank, 136, 136, dtype, pad=2, seed=T)
    want, none = _forward(b), _forward(b, base=False)
    for base, w in ((True, want), (False, none)):
        X, order, starts, A, B, scale, Yb = b.dev("X", "order", "starts", "A", "B", "scale", "Yb")
        b.m.adapters(X, order, starts, A, B, X, Y_base=Yb if base else None, scale=scale)
        assert torch.equal(X[:T - 2], w[:T - 2]) and torch.equal(X[T - 2:], b.X[T - 2:].to(DEV))
    # X as base, too: Y = X + scale B (A X)
    X, order, starts, A, B, scale = b.dev("X", "order", "starts", "A", "B", "scale")
    apart = torch.full_like(X, 7.0)
    b.m.adapters(X, order, starts, A, B, apart, Y_base=X, scale=scale)
    b.m.adapters(X, order, starts, A, B, X, Y_base=X, scale=scale)
    assert torch.equal(X[:T - 2], apart[:T - 2])


# ---- the index at the ends of its range
@pytest.mark.parametrize("n_req,n,longest", [(65536, 1024, 1), (65536, 1, 3), (4097, 1024, 40), (20000, 77, 2)])
def test_index_of_the_most_requests(n_req, n, longest):
    r = np.random.default_rng(n)
    lens = r.integers(0, longest + 1, n_req)
    ads = r.integers(-1, n + 1, n_req).astype(np.int32)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(off[-1]) + 3
    key = np.repeat(np.where((ads < 0) | (ads >= n), n, ads), lens)
    want = np.concatenate([np.argsort(key, kind="stable"), np.full(3, -1)]).astype(np.int32)
    m = S.SemMoE(S.Config(T=T, d=8, E=1, k=1, F=8, D=1, cap=T), device=DEV)
    order, starts = torch.empty(T, dtype=torch.int32, device=DEV), torch.empty(n + 1, dtype=torch.int32, device=DEV)
    m.adapter_index(torch.from_numpy(off).to(DEV), torch.from_numpy(ads).to(DEV), n, order, starts)
    assert (order.cpu().numpy() == want).all()
    assert (starts.cpu().numpy() == np.searchsorted(np.sort(key), np.arange(n + 1))).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,rank", [
    (2047, 16), (2048, 72), (3999, 24), (4000, 32), (4999, 40), (5000, 64), (4095, 128), (4096, 128), (8191, 96), (8192, 104), (13999, 64),
    (14000, 64), (20000, 48), (18600, 48)])
def test_both_sides_of_the_lines_of_the_token_tiles(T, rank, dtype):
    _both(Batch([T // 2 + 5, 9, T - T // 2 - 21], [1, 0, 1], 2, rank, 40, 24, dtype, pad=7, seed=T))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_an_adapter_are_the_base_bit_for_bit(dtype):
    """zeros of both signs, infinities and NaN of any bits among them, as in place"""
    b = Batch([3, 40, 2], [-1, 5, 0], 2, 16, 72, 136, dtype, seed=41)
    as_int, odd = (torch.int16, [-32768, 0, 0x7f80, 0x7f81, -1, 1]) if dtype == "bf16" else (torch.int32, [-2 ** 31, 0, 0x7f800000, 0x7f800001, -1, 1])
    for t in (b.Yb, b.dXb):
        bits = t.view(as_int)
        bits[:43, ::2] = torch.tensor(odd, dtype=as_int).repeat(43 * bits.shape[1] // 2 // 6 + 1)[:43 * (bits.shape[1] // 2)].view(43, -1)
    Y, dX = _forward(b), _gradient(b)[0]
    assert torch.equal(Y[:43].view(as_int).cpu(), b.Yb[:43].view(as_int))
    assert torch.equal(dX[:43].view(as_int).cpu(), b.dXb[:43].view(as_int))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("where", ["X", "dY", "A", "B", "large"])
def test_infinities_keep_their_signs(where, dtype):
    """one infinity in a row or a factor: what it meets is infinite with the sign of the product, all else is as exact as ever; u
    and v near the end of the range stay finite"""
    b = Batch([1, 40], [0, 1], 2, 16, 136, 72, dtype, seed=43)
    if where == "large":
        b.A[0], b.X[0] = 0.0, 0.0
        b.A[0, :, 0], b.X[0, 0] = 1.0, 3.3895e38  # u = s times that, s below 1
        b.scale[0], b.B[0] = 1.0 - 2.0 ** -20, b.B[0] * 2.0 ** -10
    else:
        t = getattr(b, where)
        t[(0, 9) if t.dim() == 2 else (0, 2, 9) if where == "A" else (0, 9, 2)] = float("inf") if where in "XA" else -float("inf")
    with np.errstate(invalid="ignore"):
        of, s = b.of, _np(b.scale)
        X, dY, A, B = _np(b.X), _np(b.dY), _np(b.A), _np(b.B)
        wants = [G.adapters(X, of, A, B, s, _np(b.Yb)), *G.adapters_grad(X, dY, of, A, B, s, _np(b.dXb))]
    for name, got, want in zip(("Y", "dX", "dA", "dB"), [_forward(b), *_gradient(b)], wants):
        got = _np(got)
        odd = ~np.isfinite(want)
        if where == "large":
            assert not odd.any()
            odd = np.abs(want) > 3e38  # within a step of the end of the range
        else:
            inf = np.isinf(want)
            assert (got[inf] == want[inf]).all() and not np.isfinite(got[np.isnan(want)]).any(), name  # NaN: infinities of both signs meet
        assert np.isfinite(got[~odd]).all(), name
        assert np.linalg.norm((got - want)[~odd] / 1e20) <= 2.0 ** -8 * np.linalg.norm(want[~odd] / 1e20), name
