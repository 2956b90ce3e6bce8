"""CPU-only: the calls on rows in 8 bits and the norms around a block check their arguments before they touch a GPU."""
import ctypes as C

import numpy as np
import pytest

import paper_2503_04398_amd as S
from paper_2503_04398_amd import binding as B

EINVAL, ESHAPE, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -5


def _lib(**kw):
    m = S.SemMoE(S.Config(**{**dict(T=64, d=64, E=16, k=2, F=32, D=4, cap=16), **kw}), allocate_workspace=False)
    buf = np.zeros(4096 + 16, dtype=np.int32)
    p = buf.ctypes.data + (-buf.ctypes.data) % 16
    return m.lib, m.cfg.c(), p, buf


def test_quantize_rows_refuses():
    lib, c, p, _keep = _lib()
    r = C.byref(c)

    def call(X=p, n=4, cols=64, ldx=0, Xq=p, scale=p):
        return lib.semmoe_quantize_rows(r, None, X, n, cols, ldx, Xq, scale)

    assert call(X=None) == call(Xq=None) == call(scale=None) == EINVAL
    assert call(n=-1) == call(cols=0) == call(ldx=-8) == EINVAL
    assert call(X=p + 4) == call(Xq=p + 8) == EINVAL
    assert call(cols=60) == call(ldx=68) == call(ldx=56) == ESHAPE
    assert lib.semmoe_quantize_rows(None, None, p, 4, 64, 0, p, p) == EINVAL
    assert call(n=0) == 0
    assert call(n=0x40000000) == EUNSUPPORTED
    c.dtype = 7
    assert call() == EUNSUPPORTED


def test_dispatch_rows_i8_refuses():
    lib, c, p, _keep = _lib()
    r = C.byref(c)
    for i in range(5):
        args = [p] * 5
        args[i] = None
        assert lib.semmoe_dispatch_rows_i8(r, None, *args) == EINVAL
    assert lib.semmoe_dispatch_rows_i8(r, None, p + 8, p, p, p, p) == EINVAL
    assert lib.semmoe_dispatch_rows_i8(r, None, p, p, p, p + 8, p) == EINVAL
    c.d = 72  # rows of 8-bit numbers lie on 16 bytes
    assert lib.semmoe_dispatch_rows_i8(r, None, p, p, p, p, p) == ESHAPE
    c.d, c.T = 64, 0
    assert lib.semmoe_dispatch_rows_i8(r, None, p, p, p, p, p) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(n_rows=-1), EINVAL), (dict(d_in=0), EINVAL), (dict(d_out=-8), EINVAL), (dict(ldx=-16), EINVAL), (dict(ldy=-8), EINVAL),
    (dict(d_in=72), ESHAPE), (dict(d_out=36), ESHAPE), (dict(ldx=72), ESHAPE), (dict(ldx=48), ESHAPE), (dict(ldy=36), ESHAPE),
    (dict(ldy=24), ESHAPE), (dict(d_in=131072), EUNSUPPORTED), (dict(n_rows=0x40000000), EUNSUPPORTED),
    (dict(ldy=1 << 26), EUNSUPPORTED), (dict(d_out=1 << 26), EUNSUPPORTED), (dict(ldx=1 << 31), EUNSUPPORTED), (dict(n_rows=0), 0),
])
def test_linear_i8_refuses_shapes(kw, status):
    lib, c, p, _keep = _lib()
    s = B._CLinearShape(*{**dict(n_rows=4, d_in=64, d_out=32, ldx=0, ldy=0), **kw}.values())
    assert lib.semmoe_linear_i8(C.byref(c), None, C.byref(s), p, p, p, p, p) == status


def test_linear_i8_refuses():
    lib, c, p, _keep = _lib()
    s = C.byref(B._CLinearShape(4, 64, 32, 0, 0))
    for i in range(5):
        args = [p] * 5
        args[i] = None
        assert lib.semmoe_linear_i8(C.byref(c), None, s, *args) == EINVAL
    for i in (0, 2, 3, 4):
        args = [p] * 5
        args[i] = p + 4
        assert lib.semmoe_linear_i8(C.byref(c), None, s, *args) == EINVAL
    assert lib.semmoe_linear_i8(C.byref(c), None, None, p, p, p, p, p) == EINVAL
    c.dtype = B.FP32
    assert lib.semmoe_linear_i8(C.byref(c), None, s, p, p, p, p, p) == EUNSUPPORTED


def test_ffn_i8_refuses():
    lib, c, p, _keep = _lib()
    r, big = C.byref(c), 1 << 30
    assert lib.semmoe_expert_ffn_i8(r, None, 4, *[p] * 9, p, big) == EINVAL   # rank >= D
    assert lib.semmoe_expert_ffn_i8(r, None, -2, *[p] * 9, p, big) == EINVAL
    for i in range(9):
        args = [p] * 9
        args[i] = None
        assert lib.semmoe_expert_ffn_i8(r, None, 0, *args, p, big) == EINVAL
    for i in range(7):
        args = [p] * 7
        args[i] = None
        assert lib.semmoe_shared_ffn_i8(r, None, *args[:2], 4, *args[2:], p, big) == EINVAL
    need = 128 * 32 * 3 + 128 * 4
    assert lib.semmoe_expert_ffn_i8(r, None, 0, *[p] * 9, None, big) == EWORKSPACE
    assert lib.semmoe_expert_ffn_i8(r, None, 0, *[p] * 9, p, need - 1) == EWORKSPACE
    assert lib.semmoe_shared_ffn_i8(r, None, p, p, 129, p, p, p, p, p, p, big) == ESHAPE  # more tokens than pairs
    assert lib.semmoe_shared_ffn_i8(r, None, p, p, -1, p, p, p, p, p, p, big) == EINVAL
    assert lib.semmoe_shared_ffn_i8(r, None, p, p, 4, p, p, p, p, p, p, 4 * 100 - 1) == EWORKSPACE
    assert lib.semmoe_shared_ffn_i8(r, None, p, p, 0, p, p, p, p, p, p, 1024) == 0
    for field, value, status in (("d", 72, ESHAPE), ("F", 40, ESHAPE), ("F", 131072, EUNSUPPORTED), ("dtype", B.FP32, EUNSUPPORTED)):
        lib, c, p, _keep = _lib()
        setattr(c, field, value)
        assert lib.semmoe_expert_ffn_i8(C.byref(c), None, 0, *[p] * 9, p, big) == status
        assert lib.semmoe_shared_ffn_i8(C.byref(c), None, p, p, 4, p, p, p, p, p, p, big) == status


def _norm(**kw):
    s = B._CNormShape(1.0, 1e-6, 1e-6, 0)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


FORWARD = ("R", "Y", "w_post", "gate", "w_pre", "H", "X", "Xq", "x_scale")
BACKWARD = ("dH", "dX", "H", "Y", "w_post", "gate", "w_pre", "dR", "dY", "dgate", "dw_post", "dw_pre")


@pytest.mark.parametrize("without,status", [
    (("R", "Y"), EINVAL), (("Y",), EINVAL), (("H", "X", "Xq", "x_scale", "w_pre"), EINVAL), (("w_pre",), EINVAL), (("X", "Xq", "x_scale"), EINVAL),
    (("Xq",), EINVAL), (("x_scale",), EINVAL)])
def test_block_norm_refuses(without, status):
    lib, c, p, _keep = _lib()
    s = _norm()
    args = [None if n in without else p for n in FORWARD]
    assert lib.semmoe_block_norm(C.byref(c), None, C.byref(s), *args) == status


@pytest.mark.parametrize("without,status", [
    (("dH", "dX", "w_pre", "dw_pre"), EINVAL), (("w_pre",), EINVAL), (("dX",), EINVAL), (("H",), EINVAL), (("Y",), EINVAL), (("gate",), EINVAL),
    (("w_post",), EINVAL), (("dR", "dY", "dgate", "dw_post", "dw_pre"), EINVAL)])
def test_block_norm_grad_refuses(without, status):
    lib, c, p, _keep = _lib()
    s = _norm()
    args = [None if n in without else p for n in BACKWARD]
    assert lib.semmoe_block_norm_grad(C.byref(c), None, C.byref(s), *args, p, 1 << 30) == status


def test_norms_refuse_sizes():
    lib, c, p, _keep = _lib()
    forward, backward, s, need = [p] * 9, [p] * 12, _norm(), C.c_size_t(0)
    assert lib.semmoe_block_norm(C.byref(c), None, None, *forward) == EINVAL
    assert lib.semmoe_block_norm_grad(C.byref(c), None, None, *backward, p, 1 << 30) == EINVAL
    assert lib.semmoe_block_norm_grad_workspace_bytes(C.byref(c), None) == EINVAL
    assert lib.semmoe_block_norm_grad_workspace_bytes(C.byref(c), C.byref(need)) == 0
    assert lib.semmoe_block_norm_grad(C.byref(c), None, C.byref(s), *backward, p, need.value - 257) == EWORKSPACE
    assert lib.semmoe_block_norm_grad(C.byref(c), None, C.byref(s), *backward, None, 1 << 30) == EWORKSPACE
    for i in range(8):
        args = list(forward)
        args[i] = p + 4
        assert lib.semmoe_block_norm(C.byref(c), None, C.byref(s), *args) == EINVAL
    for i in range(12):
        args = list(backward)
        args[i] = p + 4
        assert lib.semmoe_block_norm_grad(C.byref(c), None, C.byref(s), *args, p, 1 << 30) == EINVAL
    for kw, status in ((dict(ld_r=-8), EINVAL), (dict(ld_x=68), ESHAPE), (dict(ld_gate=56), ESHAPE), (dict(eps_pre=-1.0), EINVAL),
                       (dict(eps_post=float("nan")), EINVAL)):
        assert lib.semmoe_block_norm(C.byref(c), None, C.byref(_norm(**kw)), *forward) == status
    for kw, status in ((dict(ld_dh=-8), EINVAL), (dict(ld_dgate=68), ESHAPE), (dict(ld_dy=56), ESHAPE)):
        assert lib.semmoe_block_norm_grad(C.byref(c), None, C.byref(_norm(**kw)), *backward, p, 1 << 30) == status
    for field, value, status in (("d", 60, ESHAPE), ("d", 16392, EUNSUPPORTED), ("d", 0, EINVAL), ("T", -1, EINVAL), ("T", 0x40000000, EUNSUPPORTED), ("dtype", 3, EUNSUPPORTED)):
        lib, c, p, _keep = _lib()
        setattr(c, field, value)
        assert lib.semmoe_block_norm(C.byref(c), None, C.byref(s), *forward) == status
        assert lib.semmoe_block_norm_grad(C.byref(c), None, C.byref(s), *backward, p, 1 << 30) == status
        assert lib.semmoe_block_norm_grad_workspace_bytes(C.byref(c), C.byref(need)) == status
    lib, c, p, _keep = _lib(T=0)
    assert lib.semmoe_block_norm(C.byref(c), None, C.byref(s), *forward) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    m = S.SemMoE(S.Config(T=4, d=64, E=4, k=2, F=32, D=1, cap=4), allocate_workspace=False)
    rows, vec = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    q, scale = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)

    def refused(status, f, *a, **kw):
        with pytest.raises(S.SemMoEError) as e:
            f(*a, **kw)
        assert e.value.status == status

    # host tensors, wherever they stand
    refused(-1, m.quantize_rows, rows, q, scale)
    refused(-1, m.dispatch_rows_i8, q, scale, torch.zeros(8, dtype=torch.int32), torch.zeros(8, 64, dtype=torch.int8), torch.zeros(8))
    refused(-1, m.linear_i8, q, scale, torch.zeros(32, 64, dtype=torch.int8), torch.zeros(32), torch.zeros(4, 32, dtype=torch.bfloat16))
    refused(-1, m.block_norm, rows, rows.clone(), Y=rows)
    refused(-1, m.block_norm_grad, rows, rows.clone(), Y=rows, dH=rows)
    refused(-1, m.shared_ffn_i8, q, scale, 4, torch.zeros(64, 64, dtype=torch.int8), torch.zeros(64), torch.zeros(64, 32, dtype=torch.int8),
            torch.zeros(64), rows)
    # shapes
    refused(-2, m.linear_i8, q, scale, torch.zeros(32, 48, dtype=torch.int8), torch.zeros(32), torch.zeros(4, 32, dtype=torch.bfloat16))
    refused(-2, m.block_norm, rows, rows.clone(), Y=rows[:3])
    refused(-2, m.block_norm, rows, rows.clone(), Y=rows, w_post=vec[:56])
    refused(-2, m.block_norm_grad, rows, rows.clone(), Y=rows, dH=rows, gate=vec, dgate=rows.clone())
    # two results in one place
    refused(-1, m.block_norm, rows, rows, X=rows, w_pre=vec)
    refused(-1, m.block_norm_grad, rows, rows, Y=rows, dH=rows, dY=rows)
    with pytest.raises(ValueError):
        m.block_norm(rows, rows.clone(), Y=vec.expand(4, 64))  # rows on one another


def test_the_binding_refuses_vectors_that_are_not_packed():
    """a column, every second number, one number for all: each would be read or written as if its numbers lay behind one another"""
    import torch
    m = S.SemMoE(S.Config(T=4, d=64, E=4, k=2, F=32, D=1, cap=4), allocate_workspace=False)
    new = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16)  # noqa: E731
    rows, vec = new(4, 64), new(64)
    for odd in (new(64, 64)[:, 0], new(128)[::2], new(1).expand(64)):
        assert odd.shape == vec.shape
        for name in ("w_post", "w_pre", "gate"):
            with pytest.raises(S.SemMoEError, match="behind one another") as e:
                m.block_norm(rows, new(4, 64), Y=rows, X=new(4, 64), **{"w_pre": vec, name: odd})
            assert e.value.status == ESHAPE
        for name in ("w_post", "w_pre", "gate", "dw_post", "dw_pre", "dgate"):
            kw = {**dict(w_post=vec, w_pre=vec, gate=vec, dw_post=new(64), dw_pre=new(64), dgate=new(64)), name: odd}
            with pytest.raises(S.SemMoEError, match="behind one another") as e:
                m.block_norm_grad(rows, new(4, 64), Y=rows, dH=rows, dX=rows, **kw)
            assert e.value.status == ESHAPE
    assert not m._norm_calls  # what has been refused is not taken for checked


def test_the_binding_keeps_values_and_not_what_held_them():
    """a residual scale that is learned is one tensor with another value in each step; -0 is another scale than 0"""
    import torch
    m = S.SemMoE(S.Config(T=4, d=64, E=4, k=2, F=32, D=1, cap=4), allocate_workspace=False)
    rows, scale, eps = torch.zeros(4, 64, dtype=torch.bfloat16), torch.tensor(0.0), torch.tensor(0.5)
    for s, e in ((0.0, 0.5), (0.75, 0.5), (-0.0, 0.5), (0.75, 0.25)):
        scale.fill_(s), eps.fill_(e)
        for call, kw in ((m.block_norm, {}), (m.block_norm_grad, dict(dH=rows))):
            with pytest.raises(S.SemMoEError):  # the rows lie on the host; what the library would be given has been made before
                call(rows, rows.clone(), Y=rows, res_scale=scale, eps_post=eps, eps_pre=eps, **kw)
            made = list(m._norm_calls.values())[-1][1]
            assert (str(made.res_scale), made.eps_post, made.eps_pre) == (str(s), e, e)
