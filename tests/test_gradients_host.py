"""CPU-only: the adapter and gradient calls check their arguments before they touch a GPU."""
import ctypes as C
import gc
import os
import re
import subprocess
import sys
import threading
import weakref

import numpy as np
import pytest
import torch

import paper_2503_04398_amd as S
from paper_2503_04398_amd import binding as B
from paper_2503_04398_amd import build as BLD

EINVAL, ESHAPE, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -5


def _lib():
    m = S.SemMoE(S.Config(T=64, d=64, E=16, k=2, F=32, D=4, cap=16), allocate_workspace=False)
    buf = np.zeros(4096 + 16, dtype=np.int32)
    p = buf.ctypes.data + (-buf.ctypes.data) % 16
    return m.lib, m.cfg.c(), p, buf


def test_row_gradients_refuse():
    lib, c, p, _keep = _lib()
    r = C.byref(c)
    assert lib.semmoe_combine_grad(r, None, None, p, p, p, p, p) == EINVAL   # no dOut
    assert lib.semmoe_combine_grad(r, None, p, p, None, p, p, p) == EINVAL   # no slots
    assert lib.semmoe_combine_grad(r, None, p, p, p, p, None, None) == EINVAL  # nothing asked for
    assert lib.semmoe_combine_grad(r, None, p, None, p, p, p, p) == EINVAL   # dtopk_w needs Y
    assert lib.semmoe_combine_grad(r, None, p, p, p, None, p, p) == EINVAL   # dY needs topk_w
    assert lib.semmoe_combine_grad(r, None, p + 4, p, p, p, p, p) == EINVAL  # rows on 16 bytes
    assert lib.semmoe_combine_grad(r, None, p, p, p, p, p + 8, p) == EINVAL
    assert lib.semmoe_dispatch_grad(r, None, None, p, None, p) == EINVAL
    assert lib.semmoe_dispatch_grad(r, None, p, p, None, None) == EINVAL
    assert lib.semmoe_dispatch_grad(r, None, p, p, p + 4, p) == EINVAL
    c.d = 60
    assert lib.semmoe_combine_grad(r, None, p, p, p, p, p, p) == ESHAPE
    assert lib.semmoe_dispatch_grad(r, None, p, p, None, p) == ESHAPE
    c.d, c.T = 64, 0
    assert lib.semmoe_combine_grad(r, None, p, p, p, p, p, p) == 0  # nothing to do
    assert lib.semmoe_dispatch_grad(r, None, p, p, None, p) == 0


def test_ffn_gradients_refuse():
    lib, c, p, _keep = _lib()
    r, big = C.byref(c), 1 << 30
    args = [p] * 7
    assert lib.semmoe_expert_ffn_grad(r, None, 4, *args, p, big) == EINVAL  # rank >= D
    assert lib.semmoe_expert_ffn_grad(r, None, -2, *args, p, big) == EINVAL
    for i in range(7):
        bad = list(args)
        bad[i] = None
        assert lib.semmoe_expert_ffn_grad(r, None, 0, *bad, p, big) == EINVAL
    assert lib.semmoe_expert_ffn_grad(r, None, 0, p, p + 4, p, p, p, p, p, p, big) == EINVAL
    need = 64 * 2 * 2 * 32 * 2
    assert lib.semmoe_expert_ffn_grad(r, None, 0, *args, None, big) == EWORKSPACE
    assert lib.semmoe_expert_ffn_grad(r, None, 0, *args, p, need - 1) == EWORKSPACE
    assert lib.semmoe_shared_ffn_grad(r, None, p, p, 129, p, p, p, p, big) == ESHAPE  # more tokens than pairs
    assert lib.semmoe_shared_ffn_grad(r, None, p, p, -1, p, p, p, p, big) == EINVAL
    assert lib.semmoe_shared_ffn_grad(r, None, p, None, 4, p, p, p, p, big) == EINVAL
    assert lib.semmoe_shared_ffn_grad(r, None, p, p, 4, p, p, p, p, 4 * 2 * 32 * 2 - 1) == EWORKSPACE
    assert lib.semmoe_shared_ffn_grad(r, None, p, p, 0, p, p, p, p, 256) == 0


def _shape(**kw):
    v = dict(n_adapters=4, rank=8, d_in=64, d_out=32, ldx=0, ldy=0, ld_base=0, ld_out=0)
    v.update(kw)
    return B._CAdapterShape(*v.values())


@pytest.mark.parametrize("kw,status", [
    (dict(n_adapters=0), EINVAL), (dict(rank=0), EINVAL), (dict(d_in=-8), EINVAL), (dict(ldx=-8), EINVAL),
    (dict(rank=12), ESHAPE), (dict(d_in=60), ESHAPE), (dict(d_out=12), ESHAPE), (dict(ld_out=36), ESHAPE),
    (dict(rank=136), EUNSUPPORTED), (dict(n_adapters=1025), EUNSUPPORTED), (dict(d_in=(1 << 20) + 8), EUNSUPPORTED),
])
def test_adapter_shapes_are_refused(kw, status):
    lib, c, p, _keep = _lib()
    s, n = _shape(**kw), C.c_size_t(0)
    assert lib.semmoe_adapter_workspace_bytes(C.byref(c), C.byref(s), C.byref(n)) == status
    big = 1 << 30
    assert lib.semmoe_adapters(C.byref(c), None, C.byref(s), p, p, p, p, p, None, None, p, p, big) == status
    assert lib.semmoe_adapters_grad(C.byref(c), None, C.byref(s), p, p, p, p, p, p, None, None, p, None, None, p, big) == status


def test_adapter_calls_refuse():
    lib, c, p, _keep = _lib()
    r, s, big = C.byref(c), _shape(), 1 << 30
    sr = C.byref(s)
    n = C.c_size_t(0)
    assert lib.semmoe_adapter_workspace_bytes(r, sr, None) == EINVAL
    assert lib.semmoe_adapter_workspace_bytes(r, None, C.byref(n)) == EINVAL
    assert lib.semmoe_adapter_workspace_bytes(r, sr, C.byref(n)) == 0 and n.value >= 64 * 8 * 4
    # X, order, offsets, A, B, (scale), (Y_base), Y
    full = [p, p, p, p, p, None, None, p]
    for i in (0, 1, 2, 3, 4, 7):
        bad = list(full)
        bad[i] = None
        assert lib.semmoe_adapters(r, None, sr, *bad, p, big) == EINVAL, i
    for i in (0, 3, 4, 6, 7):
        bad = list(full)
        bad[i] = p + 4
        assert lib.semmoe_adapters(r, None, sr, *bad, p, big) == EINVAL, i
    assert lib.semmoe_adapters(r, None, sr, *full, None, 0) == EWORKSPACE
    assert lib.semmoe_adapters(r, None, sr, *full, p, 64 * 8 * 4 - 1) == EWORKSPACE
    for kw in (dict(ldx=56), dict(ld_base=24), dict(ld_out=24)):
        assert lib.semmoe_adapters(r, None, C.byref(_shape(**kw)), *full, p, big) == ESHAPE, kw
    # in place needs one distance of rows
    assert lib.semmoe_adapters(r, None, C.byref(_shape(ld_out=40)), p, p, p, p, p, None, p, p, p, big) == ESHAPE
    # X, dY, order, offsets, A, B, (scale), (dX_base), dX, dA, dB
    grad = [p, p, p, p, p, p, None, None, p, p, p]
    for i in range(6):
        bad = list(grad)
        bad[i] = None
        assert lib.semmoe_adapters_grad(r, None, sr, *bad, p, big) == EINVAL, i
    assert lib.semmoe_adapters_grad(r, None, sr, *grad[:8], None, None, None, p, big) == EINVAL  # nothing asked for
    assert lib.semmoe_adapters_grad(r, None, sr, *grad, p, 64) == EWORKSPACE
    for kw in (dict(ldx=56), dict(ldy=24), dict(ld_base=56), dict(ld_out=56)):
        assert lib.semmoe_adapters_grad(r, None, C.byref(_shape(**kw)), *grad, p, big) == ESHAPE, kw
    assert lib.semmoe_adapter_index(r, None, p, 4, p, 0, p, p) == EINVAL
    assert lib.semmoe_adapter_index(r, None, p, -1, p, 4, p, p) == EINVAL
    assert lib.semmoe_adapter_index(r, None, None, 4, p, 4, p, p) == EINVAL
    assert lib.semmoe_adapter_index(r, None, p, 4, p, 4, None, p) == EINVAL
    assert lib.semmoe_adapter_index(r, None, p, 4, p, 1025, p, p) == EUNSUPPORTED
    assert lib.semmoe_adapter_index(r, None, p, 65537, p, 4, p, p) == EUNSUPPORTED


def test_binding_refuses_shapes_that_do_not_fit():
    m = S.SemMoE(S.Config(T=8, d=16, E=1, k=1, F=8, D=1, cap=8, dtype="fp32"), allocate_workspace=False)
    m.device = "cpu"
    T, X, Y = 8, torch.zeros(8, 16), torch.zeros(8, 24)
    A, Bm = torch.zeros(2, 8, 16), torch.zeros(2, 24, 8)
    order, off = torch.zeros(T, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(S.SemMoEError):
        m.adapters(X, order[:7], off, A, Bm, Y)
    with pytest.raises(S.SemMoEError):
        m.adapters(X, order, off[:2], A, Bm, Y)
    with pytest.raises(S.SemMoEError):
        m.adapters(X, order, off, A, Bm.transpose(1, 2), Y)
    with pytest.raises(S.SemMoEError):
        m.adapters(X, order, off, A, Bm, torch.zeros(7, 24))
    with pytest.raises(ValueError):
        m.adapters(X, order, off, A, Bm, torch.zeros(8, 25))
    with pytest.raises(ValueError):
        m.adapters(torch.zeros(16, 8).t(), order, off, A, Bm, Y)           # columns and not rows in one run
    with pytest.raises(ValueError):
        m.adapters_grad(X, torch.zeros(1, 24).expand(8, 24), order, off, A, Bm, dX=X.clone())  # a broadcast row
    with pytest.raises(S.SemMoEError):
        m.adapters_grad(X, Y, order, off, A, Bm, dA=torch.zeros(2, 8, 8))
    with pytest.raises(S.SemMoEError):
        m.adapter_index(torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 2, order, off)


def test_binding_refuses_tensors_of_other_types_and_places():
    """host tensors and numbers of another type are refused before they reach a kernel"""
    m = S.SemMoE(S.Config(T=8, d=16, E=4, k=2, F=8, D=2, cap=4, dtype="bf16"), allocate_workspace=False)
    bf, i32 = dict(dtype=torch.bfloat16), dict(dtype=torch.int32)
    X, P = torch.zeros(8, 16, **bf), torch.zeros(16, 16, **bf)
    slots, w = torch.zeros(16, **i32), torch.zeros(8, 2)
    for bad in (dict(Y=P.float()), dict(Y=P[:15]), dict(slots=slots.long()), dict(w=w.double()), dict(dOut=X[:7])):
        a = dict(dOut=X, Y=P, slots=slots, w=w)
        a.update(bad)
        with pytest.raises(S.SemMoEError):
            m.combine_grad(a["dOut"], a["Y"], a["slots"], a["w"], P.clone(), w.clone())
    with pytest.raises(S.SemMoEError, match="device"):
        m.combine_grad(X, P, slots, w, P.clone(), w.clone())
    with pytest.raises(S.SemMoEError, match="device"):
        m.dispatch_grad(P, slots, X)
    off, of = torch.zeros(5, **i32), torch.zeros(4, **i32)
    gu, dn = torch.zeros(4, 16, 16, **bf), torch.zeros(4, 16, 8, **bf)
    with pytest.raises(S.SemMoEError, match="needed"):
        m.expert_ffn_grad(0, P, P, off[:4], of, gu, dn, P)
    with pytest.raises(S.SemMoEError, match="device"):
        m.expert_ffn_grad(0, P, P, off, of, gu, dn, P)
    with pytest.raises(S.SemMoEError, match="device"):
        m.shared_ffn_grad(X, X, 8, gu[0], dn[0], X)
    with pytest.raises(S.SemMoEError, match="needed"):
        m.shared_ffn_grad(X, X, 9, gu[0], dn[0], X)
    A, Bm = torch.zeros(2, 8, 16, **bf), torch.zeros(2, 24, 8, **bf)
    order, starts, Y = torch.zeros(8, **i32), torch.zeros(3, **i32), torch.zeros(8, 24, **bf)
    with pytest.raises(S.SemMoEError, match="device"):
        m.adapters(X, order, starts, A, Bm, Y)
    with pytest.raises(S.SemMoEError, match="needed"):
        m.adapters(X, order, starts, A, Bm, Y.float())
    with pytest.raises(S.SemMoEError, match="needed"):
        m.adapters_grad(X, Y, order.long(), starts, A, Bm, dA=A.clone())
    with pytest.raises(S.SemMoEError, match="device"):
        m.adapter_index(torch.zeros(3, **i32), torch.zeros(2, **i32), 2, order, starts)


def test_nothing_to_do_is_no_call():
    """batches without a token: no address to hand over and no kernel to run"""
    m = S.SemMoE(S.Config(T=0, d=16, E=4, k=2, F=8, D=2, cap=1, dtype="fp32"), allocate_workspace=False)
    e = torch.empty(0, 16)
    m.combine_grad(e, e, e, e, e, e)
    m.dispatch_grad(e, e, e)
    m.expert_ffn_grad(0, e, e, e, e, e, e, e)
    m.shared_ffn_grad(e, e, 0, e, e, e)


def test_workspaces_of_devices_streams_and_graphs_are_apart(monkeypatch):
    """a default stream has the same handle on every device, and a graph's workspace is no other's"""
    m = S.SemMoE(S.Config(T=64, d=64, E=16, k=2, F=32, D=4, cap=16), allocate_workspace=False)
    now, made = {"dev": 0, "stream": 0, "capturing": False}, []

    class Torch:
        uint8 = torch.uint8

        @staticmethod
        def empty(n, dtype, device):
            made.append(device)
            return torch.empty(n, dtype=dtype)
    m._torch, m._capturing, m._types = Torch, lambda: now["capturing"], (lambda: now["dev"],) + m._types[1:]
    monkeypatch.setattr(B, "_stream", lambda: now["stream"])

    def get(call="adapters", need=1000, **at):
        now.update({"dev": 0, "stream": 0, "capturing": False, **at})
        p, n, owner = m._workspace(call, need)
        assert n >= need and p == owner.data_ptr()
        return owner
    first = get()
    others = [get(dev=1), get(stream=7), get("shared_ffn_grad"), get(capturing=True), get(capturing=True)]
    assert made == [0, 1, 0, 0, 0, 0]
    assert len({t.data_ptr() for t in [first] + others}) == 6
    assert get(need=900) is first and get(dev=1) is others[0] and get(stream=7) is others[1]
    larger = get(need=5000)
    assert larger is not first and get() is larger and get(dev=1) is others[0]


@pytest.mark.skipif(not os.path.exists(BLD.HIPCC), reason="needs the compiler")
@pytest.mark.parametrize("source,kernel,may_coincide", [
    ("combine.hip", "combine_kernel", (6, 7)),         # dispatch_grad: dX may be dX_add
    ("rows_grad.hip", "combine_grad_kernel", (4, 7)),  # combine_grad: dY may be Y
])
def test_kernels_do_not_deny_that_a_result_lies_in_the_place_of_an_input(source, kernel, may_coincide):
    """what the compiler was told of pointers that the header lets coincide: none of them is `noalias`"""
    cmd = [BLD.HIPCC] + [f for f in BLD.HIP_FLAGS if f != "-fPIC"] + ["-O1", "--cuda-device-only", "-S", "-emit-llvm", "-o", "-",
                                                                        os.path.join(BLD.CSRC, source)]
    text = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, check=True, timeout=120).stdout
    heads = re.findall(r"^define [^\n]*amdgpu_kernel void @_ZN6semmoe\d+%sI\w+\((.*)\) \S*unnamed_addr" % kernel, text, re.M)
    assert heads
    for head in heads:
        args = re.split(r", (?=ptr |i32 )", head)
        for i in may_coincide:
            assert args[i].startswith("ptr") and "noalias" not in args[i], args[i]
        assert any("noalias" in a for a in args)  # the word means what the test takes it for


def test_workspaces_of_threads_are_apart(monkeypatch):
    """a call enqueues several launches, and those of two threads on one stream may come in turns: neither finds the other's sums"""
    m = S.SemMoE(S.Config(T=64, d=64, E=16, k=2, F=32, D=4, cap=16), allocate_workspace=False)

    class Torch:
        uint8 = torch.uint8

        @staticmethod
        def empty(n, dtype, device):
            return torch.empty(n, dtype=dtype)
    m._torch, m._capturing, m._types = Torch, lambda: False, (lambda: 0,) + m._types[1:]
    monkeypatch.setattr(B, "_stream", lambda: 0)
    mine = m._workspace("adapters", 1000)[2]
    both, theirs, gone = threading.Barrier(2), [], []

    def work():
        first = m._workspace("adapters", 1000)[2]
        both.wait()
        theirs.append(first.data_ptr())
        assert m._workspace("adapters", 900)[2] is first
        both.wait()  # neither has ended before the other's is seen
        gone.append(weakref.ref(first))
    threads = [threading.Thread(target=work) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len({mine.data_ptr(), *theirs}) == 3 and m._workspace("adapters", 1000)[2] is mine
    gc.collect()
    assert [r() for r in gone] == [None, None]  # a thread's workspaces go with it


HOST_ONLY = """
import sys
%s
import numpy as np
import paper_2503_04398_amd as S
m = S.SemMoE(S.Config(T=8, d=8, E=4, k=2, F=8, D=2, cap=4), allocate_workspace=False)
assert m.workspace_bytes() > 0
e2r, phys, inv = m.place(np.array([4, 1, 1, 4]), np.zeros((4, 4)))
assert sorted(phys.tolist()) == [0, 1, 2, 3]
try:
    m._no_such_name
except AttributeError:
    print("done")
"""


@pytest.mark.parametrize("torch_is", [
    "sys.modules['torch'] = None  # not there",
    "import torch; del torch._C._cuda_getDevice, torch._C._cuda_isCurrentStreamCapturing  # built without a GPU's support"])
def test_host_calls_need_no_torch_that_knows_a_gpu(torch_is):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", HOST_ONLY % torch_is], cwd=root, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True,
                       timeout=120)
    assert p.returncode == 0 and p.stdout.strip().endswith("done"), p.stdout


def _sizes(T, dtype="bf16", **kw):
    lib = S.load_library()
    c, s, n, f = S.Config(T=T, d=8, E=1, k=1, F=8, D=1, cap=max(T, 1), dtype=dtype).c(), _shape(**kw), C.c_size_t(0), C.c_size_t(0)
    assert lib.semmoe_adapter_workspace_bytes(C.byref(c), C.byref(s), C.byref(n)) == 0
    assert lib.semmoe_adapter_forward_workspace_bytes(C.byref(c), C.byref(s), C.byref(f)) == 0
    return n.value, f.value


@pytest.mark.parametrize("n_adapters", [1, 4, 64, 1024])
def test_adapter_workspaces_follow_the_tokens_and_not_the_adapters(n_adapters):
    """u and v: at most four planes of T x rank each; the sums over tokens: two places of rank x width for every segment (of no fewer than
    `seg` tokens for these widths), however many adapters there are"""
    for T, rank, d_in, d_out, seg in ((32768, 128, 4096, 4096, 4096), (9000, 64, 8192, 256, 1024), (500, 16, 64, 64, 128), (0, 8, 64, 64, 1)):
        both, forward = _sizes(T, n_adapters=n_adapters, rank=rank, d_in=d_in, d_out=d_out)
        planes, places = 4 * T * rank * 4, 2 * -(-T // seg)
        assert forward <= planes + 256
        assert both <= 2 * planes + places * rank * (d_in + d_out) * 4 + 1024
        assert forward <= both


def test_the_forward_call_asks_for_its_own_part():
    m = S.SemMoE(S.Config(T=3000, d=16, E=1, k=1, F=8, D=1, cap=3000, dtype="fp32"), allocate_workspace=False)
    X, Y, A, Bm = torch.zeros(3000, 16), torch.zeros(3000, 24), torch.zeros(2, 8, 16), torch.zeros(2, 24, 8)
    order, off = torch.zeros(3000, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    both, forward = _sizes(3000, "fp32", n_adapters=2, rank=8, d_in=16, d_out=24)
    assert m._adapter_call("adapters", X, order, off, A, Bm, None, None, None, Y)[2] == forward < both
    assert m._adapter_call("adapters_grad", X, order, off, A, Bm, None, Y, None, X)[2] == both
    assert m.lib.semmoe_adapter_forward_workspace_bytes(None, None, None) == EINVAL


def test_gradients_in_the_place_of_the_factors_are_refused():
    """dX reads the factors after dA and dB have been written"""
    m = S.SemMoE(S.Config(T=8, d=16, E=1, k=1, F=8, D=1, cap=8, dtype="fp32"), allocate_workspace=False)
    X, dY = torch.zeros(8, 16), torch.zeros(8, 16)
    A, Bm = torch.zeros(2, 8, 16), torch.zeros(2, 16, 8)
    order, off = torch.zeros(8, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    same = torch.zeros(2, 8, 16)
    for kw in (dict(dA=A), dict(dB=Bm), dict(dA=A, dB=Bm, dX=X), dict(dA=Bm.view(2, 8, 16)), dict(dA=same, dB=same.view(2, 16, 8))):
        with pytest.raises(S.SemMoEError, match="place"):
            m.adapters_grad(X, dY, order, off, A, Bm, **kw)
    with pytest.raises(S.SemMoEError, match="device"):  # apart: the next thing that is wrong with them
        m.adapters_grad(X, dY, order, off, A, Bm, dA=A.clone(), dB=Bm.clone())
