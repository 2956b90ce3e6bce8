"""ctypes binding of libsemmoe.so: argument marshalling only.

Every step of the path runs inside the library's HIP kernels; this module turns torch tensors into
raw pointers, passes torch's current stream, and raises on a non-zero status.  torch is used for
device memory and streams, nothing else.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
import struct
import threading
from dataclasses import dataclass
from typing import Optional

HERE = os.path.dirname(os.path.abspath(__file__))

STATUS_NAMES = {0: "OK", -1: "EINVAL", -2: "ESHAPE", -3: "EWORKSPACE", -4: "EHIP", -5: "EUNSUPPORTED"}
FP32, BF16 = 0, 1
SOFTMAX, SIGMOID = 0, 1


class SemMoEError(RuntimeError):
    def __init__(self, call: str, status: int, hip_error: int = 0):
        self.call, self.status, self.hip_error = call, status, hip_error
        msg = "%s failed: %s (%d)" % (call, STATUS_NAMES.get(status, "?"), status)
        if status == -4:
            msg += ", hipError_t %d" % hip_error
        super().__init__(msg)


class _CConfig(C.Structure):
    _fields_ = [("T", C.c_int32), ("d", C.c_int32), ("E", C.c_int32), ("k", C.c_int32), ("F", C.c_int32),
                ("D", C.c_int32), ("dtype", C.c_int32), ("score", C.c_int32), ("renorm", C.c_int32),
                ("n_group", C.c_int32), ("topk_group", C.c_int32), ("routed_scale", C.c_float),
                ("cap", C.c_int32), ("num_classes", C.c_int32)]


_three_numbers = struct.Struct("3d")
_config_values = operator.attrgetter(*(name for name, _ in _CConfig._fields_))


class CoschedParams(C.Structure):
    """semmoe_cosched_params of the C header, field for field"""
    _fields_ = [("alpha_e", C.c_int64), ("beta_e", C.c_int64), ("gamma_e", C.c_int64), ("alpha_r", C.c_int64),
                ("beta_r", C.c_int64), ("w_load", C.c_int64), ("w_comm", C.c_int64), ("ft_passes", C.c_int32),
                ("n_steps", C.c_int32)]


class _CAdapterShape(C.Structure):
    """semmoe_adapter_shape of the C header, field for field"""
    _fields_ = [("n_adapters", C.c_int32), ("rank", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32),
                ("ldx", C.c_int64), ("ldy", C.c_int64), ("ld_base", C.c_int64), ("ld_out", C.c_int64)]


class _CLinearShape(C.Structure):
    """semmoe_linear_shape of the C header, field for field"""
    _fields_ = [("n_rows", C.c_int32), ("d_in", C.c_int32), ("d_out", C.c_int32), ("ldx", C.c_int64), ("ldy", C.c_int64)]


class _CNormShape(C.Structure):
    """semmoe_norm_shape of the C header, field for field"""
    _fields_ = [("res_scale", C.c_float), ("eps_post", C.c_float), ("eps_pre", C.c_float), ("gate_rows", C.c_int32)] + [
        (n, C.c_int64) for n in ("ld_r", "ld_y", "ld_h", "ld_x", "ld_gate", "ld_dh", "ld_dx", "ld_dr", "ld_dy", "ld_dgate")]


@dataclass
class Config:
    T: int
    d: int
    E: int
    k: int
    F: int
    D: int
    dtype: int = BF16
    score: int = SOFTMAX
    renorm: bool = True
    n_group: int = 1
    topk_group: int = 1
    routed_scale: float = 1.0
    cap: int = 0
    num_classes: int = 0

    def __post_init__(self):
        # the names of the workload descriptions are accepted for the two enumerations
        if isinstance(self.dtype, str):
            if self.dtype not in ("bf16", "fp32"):
                raise ValueError("dtype must be 'bf16' or 'fp32' (or the BF16 / FP32 constants)")
            self.dtype = BF16 if self.dtype == "bf16" else FP32
        if isinstance(self.score, str):
            if self.score not in ("softmax", "sigmoid"):
                raise ValueError("score must be 'softmax' or 'sigmoid' (or the SOFTMAX / SIGMOID constants)")
            self.score = SIGMOID if self.score == "sigmoid" else SOFTMAX

    def c(self) -> _CConfig:
        return _CConfig(self.T, self.d, self.E, self.k, self.F, self.D, self.dtype, self.score, int(self.renorm),
                        self.n_group, self.topk_group, self.routed_scale, self.cap, self.num_classes)

    @staticmethod
    def from_workload(w, cap: Optional[int] = None, T: Optional[int] = None) -> "Config":
        return Config(T=w.T if T is None else T, d=w.d, E=w.E, k=w.k, F=w.F, D=w.D,
                      dtype=BF16 if w.dtype == "bf16" else FP32,
                      score=SIGMOID if w.score == "sigmoid" else SOFTMAX, renorm=bool(w.renorm),
                      n_group=w.n_group, topk_group=w.topk_group, routed_scale=w.routed_scale,
                      cap=w.cap if cap is None else cap, num_classes=w.C)


def lib_path() -> str:
    return os.environ.get("SEMMOE_LIB", os.path.join(HERE, "lib", "libsemmoe.so"))


_LIB = None
_P = C.c_void_p
_SIGS = {
    "semmoe_version": ([], C.c_int32),
    "semmoe_last_hip_error": ([], C.c_int32),
    "semmoe_workspace_bytes": ([_P, C.POINTER(C.c_size_t)], C.c_int32),
    "semmoe_set_tuning": ([C.c_int32, C.c_int32], C.c_int32),
    "semmoe_get_tuning": ([C.c_int32, _P], C.c_int32),
    "semmoe_route": ([_P] * 12 + [C.c_size_t], C.c_int32),
    "semmoe_route_from_logits": ([_P] * 6, C.c_int32),
    "semmoe_coact_hist": ([_P, _P, _P, C.c_int32, _P, _P], C.c_int32),
    "semmoe_token_expert_hist": ([_P, _P, _P, _P, C.c_int32, C.c_int32, _P], C.c_int32),
    "semmoe_lookup_tables": ([_P, _P, _P, C.c_int32, _P, _P, _P], C.c_int32),
    "semmoe_place": ([_P, _P, _P, C.c_int64, C.c_int64, C.c_int32, _P, _P, _P], C.c_int32),
    "semmoe_coschedule": ([_P, _P, _P, _P, _P, C.c_int32, _P, _P, _P, _P, _P, _P, _P], C.c_int32),
    "semmoe_token_labels": ([_P, _P, C.c_int32, _P, _P, C.c_int32, _P, _P, _P], C.c_int32),
    "semmoe_reshuffle": ([_P] * 9 + [C.c_size_t], C.c_int32),
    "semmoe_reshuffle_static": ([_P] * 8, C.c_int32),
    "semmoe_reshuffle_rounds": ([_P] * 4 + [C.c_int32] + [_P] * 5 + [C.c_size_t], C.c_int32),
    "semmoe_reshuffle_refine": ([_P] * 4 + [C.c_int32, C.c_int32] + [_P] * 6 + [C.c_size_t], C.c_int32),
    "semmoe_reshuffle_lookup": ([_P, _P, _P, C.c_int32, _P, _P, _P, C.c_int32] + [_P] * 5 + [C.c_size_t], C.c_int32),
    "semmoe_reshuffle_cond": ([_P, _P, _P, C.c_int32, _P, _P, _P, _P, C.c_int32, _P, _P, _P, C.c_int32] + [_P] * 5
                              + [C.c_size_t], C.c_int32),
    "semmoe_device_sequence": ([_P, _P, _P, _P, C.c_int32, _P, _P], C.c_int32),
    "semmoe_request_schedule": ([_P, _P, _P, C.c_int32, _P, C.c_int32] + [_P] * 7 + [C.c_size_t], C.c_int32),
    "semmoe_dispatch": ([_P] * 15 + [C.c_size_t], C.c_int32),
    "semmoe_dispatch_index": ([_P] * 13 + [C.c_size_t], C.c_int32),
    "semmoe_dispatch_rows": ([_P] * 5, C.c_int32),
    "semmoe_expert_ffn": ([_P, _P, C.c_int32] + [_P] * 7 + [C.c_size_t], C.c_int32),
    "semmoe_shared_ffn": ([_P, _P, _P, C.c_int32, _P, _P, _P, _P, C.c_size_t], C.c_int32),
    "semmoe_combine": ([_P] * 7, C.c_int32),
    "semmoe_combine_grad": ([_P] * 8, C.c_int32),
    "semmoe_dispatch_grad": ([_P] * 6, C.c_int32),
    "semmoe_expert_ffn_grad": ([_P, _P, C.c_int32] + [_P] * 8 + [C.c_size_t], C.c_int32),
    "semmoe_shared_ffn_grad": ([_P] * 4 + [C.c_int32] + [_P] * 4 + [C.c_size_t], C.c_int32),
    "semmoe_adapter_index": ([_P, _P, _P, C.c_int32, _P, C.c_int32, _P, _P], C.c_int32),
    "semmoe_adapter_workspace_bytes": ([_P, _P, C.POINTER(C.c_size_t)], C.c_int32),
    "semmoe_adapter_forward_workspace_bytes": ([_P, _P, C.POINTER(C.c_size_t)], C.c_int32),
    "semmoe_adapters": ([_P] * 12 + [C.c_size_t], C.c_int32),
    "semmoe_adapters_grad": ([_P] * 15 + [C.c_size_t], C.c_int32),
    "semmoe_quantize_rows": ([_P, _P, _P, C.c_int32, C.c_int32, C.c_int64, _P, _P], C.c_int32),
    "semmoe_dispatch_rows_i8": ([_P] * 7, C.c_int32),
    "semmoe_linear_i8": ([_P] * 8, C.c_int32),
    "semmoe_expert_ffn_i8": ([_P, _P, C.c_int32] + [_P] * 10 + [C.c_size_t], C.c_int32),
    "semmoe_shared_ffn_i8": ([_P] * 4 + [C.c_int32] + [_P] * 6 + [C.c_size_t], C.c_int32),
    "semmoe_block_norm": ([_P] * 12, C.c_int32),
    "semmoe_block_norm_grad_workspace_bytes": ([_P, C.POINTER(C.c_size_t)], C.c_int32),
    "semmoe_block_norm_grad": ([_P] * 16 + [C.c_size_t], C.c_int32),
    "semmoe_probe_copy": ([_P, _P, _P, C.c_size_t], C.c_int32),
    "semmoe_probe_stream": ([_P, _P, C.c_size_t, C.c_int32, _P], C.c_int32),
    "semmoe_probe_mfma": ([_P, _P, C.c_int32, _P, C.POINTER(C.c_double)], C.c_int32),
    "semmoe_probe_tile_loop": ([_P, _P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P, C.POINTER(C.c_double)], C.c_int32),
}
EXPORTS = tuple(_SIGS)


def load_library():
    """Load libsemmoe.so (built by `python -m paper_2503_04398_amd.build`).  No fallback."""
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise SemMoEError("load_library: %s is missing; build it with "
                              "`python -m paper_2503_04398_amd.build`" % path, -1)
        lib = C.CDLL(path)
        for name, (args, res) in _SIGS.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, res
        _LIB = lib
    return _LIB


def _ptr(t):
    """device (or host) pointer of a torch tensor / numpy array / None / int"""
    if t is None:
        return None
    get = getattr(t, "data_ptr", None)
    if get is not None:
        assert t.is_contiguous(), "tensors must be contiguous"
        return get()
    if isinstance(t, int):
        return t
    return t.ctypes.data


def _row_distance(t, n_cols: int, name: str) -> int:
    """distance of rows, in elements, of a matrix whose rows are runs of n_cols numbers, however far apart"""
    if t.dim() != 2 or t.shape[1] != n_cols or (t.shape[0] and t.stride(1) != 1):
        raise ValueError("%s must be a matrix of rows of %d numbers, each row one run of memory" % (name, n_cols))
    if t.shape[0] <= 1:
        return n_cols
    if t.stride(0) < n_cols:  # a broadcast row, too: the library takes a distance of 0 as packed
        raise ValueError("rows of %s overlap" % name)
    return t.stride(0)


def _stream():
    """handle of torch's current stream on the current device.  A call costs the host a few microseconds, as much as a
    small kernel; once torch has initialised the GPU the handle comes without the availability check and the stream
    object around it (2.4 us of a call that took 9.7)."""
    import torch
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None


class _OfThread(threading.local):
    """what a thread keeps for itself; it goes when the thread ends"""

    def __init__(self):
        self.workspaces = {}


class SemMoE:
    """One config + one workspace; methods mirror the C entry points one to one.

    Calls that use the workspace of the config (`ws`, `ws_shared`) take their turns on one stream.  Those that name a size of their own
    (the gradients of FFN and norms, the adapters, the FFN in 8 bits) may be made from several threads and on several streams at once."""

    def __init__(self, cfg: Config, device="cuda:0", allocate_workspace: bool = True):
        self.lib = load_library()
        self.cfg = cfg
        self.device = device
        self.ws = None
        self.ws_bytes = 0
        self.ws_shared = None
        self._mine = _OfThread()
        self._adapter_calls = {}  # config, shape and workspace bytes of the adapter calls seen, by their shapes
        self._norm_calls = {}  # the same of the calls on the norms
        self._linear_shapes = {}  # semmoe_linear_shape by its fields
        self._c_config = None  # (values, C struct of them)
        if allocate_workspace:
            import torch
            self.ws_bytes = self.workspace_bytes()
            self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)

    # -- helpers
    def __getattr__(self, name):
        """What the calls on the GPU ask of torch, looked up by the first of them and kept: the host's calls need neither torch nor
        one that knows a GPU."""
        if name not in ("_torch", "_types", "_capturing"):
            raise AttributeError("%s has no %s" % (type(self).__name__, name))
        import torch
        for n, v in (("_torch", torch), ("_capturing", torch._C._cuda_isCurrentStreamCapturing),
                     ("_types", (torch._C._cuda_getDevice, torch.int32, torch.float32, (torch.float32, torch.bfloat16)))):
            self.__dict__.setdefault(n, v)
        return self.__dict__[name]

    def _check(self, name: str, st: int):
        if st != 0:
            raise SemMoEError(name, st, self.lib.semmoe_last_hip_error())

    def _cfg(self, **over):
        # the C struct of the config's present values: built again when any of them has changed, read by the library and
        # written by nobody, so that a call does not fill fourteen fields through ctypes
        values = _config_values(self.cfg)
        kept = self._c_config
        if kept is None or kept[0] != values:
            self._c_config = kept = (values, self.cfg.c())
        if not over:
            return kept[1]
        c = self.cfg.c()
        for k_, v in over.items():
            setattr(c, k_, v)
        return c

    @property
    def _own_ws(self):
        """this thread's workspaces of the calls that name a size of their own, by call, device and stream"""
        return self._mine.workspaces

    def _workspace(self, call: str, need: int):
        """(pointer, bytes, owner) of a workspace that only `call` of this thread on the present stream uses, of at least `need`
        bytes: kept from call to call, so that calls on two streams may overlap, and calls of two threads on one, whose launches may
        come in turns.  It lies on the current device, where the call's tensors have been found.  While a graph is captured it is of the graph's own memory and goes back there when the owner does, so that
        graphs may run beside each other and beside calls on any stream."""
        dev = self._types[0]()
        if self._capturing():
            t = self._torch.empty(max(need, 256), dtype=self._torch.uint8, device=dev)
            return t.data_ptr(), t.numel(), t
        key = (call, dev, _stream())  # a default stream's handle is the same on every device
        t = self._own_ws.get(key)
        if t is None or t.numel() < need:
            self._own_ws[key] = t = self._torch.empty(max(need, 256), dtype=self._torch.uint8, device=dev)
        return t.data_ptr(), t.numel(), t

    def _fit(self, call: str, args):
        """Refuses tensors that the library would read or write past their end, or as numbers of another type, or that lie on
        another device than the current one.  args: (tensor or None, type, least numbers); the type None is the config's
        activation type.  The calls of a few microseconds ask the same of their tensors in one expression first (a tuple and
        a loop cost them 2 us more) and come here for what is wrong."""
        torch = self._torch
        dev = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else 0
        act = torch.bfloat16 if self.cfg.dtype == BF16 else torch.float32
        for t, dtype, least in args:
            if t is not None and (t.dtype is not (dtype or act) or t.numel() < least or t.get_device() != dev):
                size = t.numel() < least
                raise SemMoEError("%s: %d numbers of %s on %s where %s%s on the current device (%d) are needed" % (
                    call, t.numel(), t.dtype, t.device, "at least %d of " % least if least else "", dtype or act, dev),
                    -2 if size else -1)

    def workspace_bytes(self) -> int:
        n = C.c_size_t(0)
        c = self._cfg()
        self._check("semmoe_workspace_bytes", self.lib.semmoe_workspace_bytes(C.byref(c), C.byref(n)))
        return int(n.value)

    def set_tuning(self, key: int, value: int):
        self._check("semmoe_set_tuning", self.lib.semmoe_set_tuning(int(key), int(value)))

    def get_tuning(self, key: int) -> int:
        v = C.c_int32(0)
        self._check("semmoe_get_tuning", self.lib.semmoe_get_tuning(int(key), C.byref(v)))
        return int(v.value)

    # -- entry points
    def route(self, X, W_r, topk_ids, topk_w, b_g=None, token_class=None, class_bias=None, sel_bias=None,
              logits_out=None, T=None):
        c = self._cfg(**({"T": T} if T is not None else {}))
        self._check("semmoe_route", self.lib.semmoe_route(
            C.byref(c), _stream(), _ptr(X), _ptr(W_r), _ptr(b_g), _ptr(token_class), _ptr(class_bias),
            _ptr(sel_bias), _ptr(logits_out), _ptr(topk_ids), _ptr(topk_w), _ptr(self.ws), self.ws_bytes))

    def route_from_logits(self, logits, topk_ids, topk_w, sel_bias=None, T=None):
        c = self._cfg(**({"T": T} if T is not None else {}))
        self._check("semmoe_route_from_logits", self.lib.semmoe_route_from_logits(
            C.byref(c), _stream(), _ptr(logits), _ptr(sel_bias), _ptr(topk_ids), _ptr(topk_w)))

    def coact_hist(self, topk_ids, T_batch, load, coact):
        c = self._cfg()
        self._check("semmoe_coact_hist", self.lib.semmoe_coact_hist(
            C.byref(c), _stream(), _ptr(topk_ids), int(T_batch), _ptr(load), _ptr(coact)))

    def token_expert_hist(self, token_key, topk_ids, T_batch, V, table):
        c = self._cfg()
        self._check("semmoe_token_expert_hist", self.lib.semmoe_token_expert_hist(
            C.byref(c), _stream(), _ptr(token_key), _ptr(topk_ids), int(T_batch), int(V), _ptr(table)))

    def lookup_tables(self, table_u32, expert_to_rank):
        """host call: numpy uint32 [V,E] and int32 [E] in, three numpy int32 [V] arrays out"""
        import numpy as np
        table_u32 = np.ascontiguousarray(table_u32, dtype=np.uint32)
        e2r = np.ascontiguousarray(expert_to_rank, dtype=np.int32)
        V = table_u32.shape[0]
        dev, conf, level = (np.zeros(V, dtype=np.int32) for _ in range(3))
        c = self._cfg()
        self._check("semmoe_lookup_tables", self.lib.semmoe_lookup_tables(
            C.byref(c), _ptr(table_u32), _ptr(e2r), int(V), _ptr(dev), _ptr(conf), _ptr(level)))
        return dev, conf, level

    def place(self, load_u64, coact_u64, alpha=1, gamma=0, ft_passes=8):
        """host call: numpy uint64 in, three numpy int32 arrays out"""
        import numpy as np
        load_u64 = np.ascontiguousarray(load_u64, dtype=np.uint64)
        coact_u64 = np.ascontiguousarray(coact_u64, dtype=np.uint64)
        E = self.cfg.E
        e2r, phys, inv = (np.zeros(E, dtype=np.int32) for _ in range(3))
        c = self._cfg()
        self._check("semmoe_place", self.lib.semmoe_place(
            C.byref(c), _ptr(load_u64), _ptr(coact_u64), int(alpha), int(gamma), int(ft_passes), _ptr(e2r),
            _ptr(phys), _ptr(inv)))
        return e2r, phys, inv

    def coschedule(self, load_u64, coact_u64, unit_act_u64, unit_len_u64, alpha_e=1, beta_e=1, gamma_e=0, alpha_r=0,
                   beta_r=1, ft_passes=8, n_steps=4, w_load=1, w_comm=1):
        """host call: numpy uint64 in; (expert_to_rank, phys_of_expert, expert_of_phys, unit_rank, step_score,
        best_step) out"""
        import numpy as np
        load_u64 = np.ascontiguousarray(load_u64, dtype=np.uint64)
        coact_u64 = np.ascontiguousarray(coact_u64, dtype=np.uint64)
        unit_act_u64 = np.ascontiguousarray(unit_act_u64, dtype=np.uint64)
        unit_len_u64 = np.ascontiguousarray(unit_len_u64, dtype=np.uint64)
        E = self.cfg.E
        U = unit_len_u64.shape[0]
        if unit_act_u64.shape != (U, E) or load_u64.shape != (E,) or coact_u64.shape != (E, E):
            raise SemMoEError("coschedule: shapes must be load[E], coact[E,E], unit_act[U,E], unit_len[U]", -2)
        e2r, phys, inv = (np.zeros(E, dtype=np.int32) for _ in range(3))
        unit_rank = np.zeros(max(U, 1), dtype=np.int32)
        step_score = np.zeros(max(int(n_steps), 1), dtype=np.int64)
        best = C.c_int32(-1)
        prm = CoschedParams(int(alpha_e), int(beta_e), int(gamma_e), int(alpha_r), int(beta_r), int(w_load),
                            int(w_comm), int(ft_passes), int(n_steps))
        c = self._cfg()
        self._check("semmoe_coschedule", self.lib.semmoe_coschedule(
            C.byref(c), _ptr(load_u64), _ptr(coact_u64), _ptr(unit_act_u64), _ptr(unit_len_u64), int(U),
            C.cast(C.byref(prm), C.c_void_p), _ptr(e2r), _ptr(phys), _ptr(inv), _ptr(unit_rank), _ptr(step_score),
            C.cast(C.byref(best), C.c_void_p)))
        return e2r, phys, inv, unit_rank[:U], step_score, int(best.value)

    def token_labels(self, req_offsets, token_key, req_rank, V):
        """host call: numpy int32 in, three numpy int32 [V] arrays out"""
        import numpy as np
        req_offsets = np.ascontiguousarray(req_offsets, dtype=np.int32)
        token_key = np.ascontiguousarray(token_key, dtype=np.int32)
        req_rank = np.ascontiguousarray(req_rank, dtype=np.int32)
        n_req = req_offsets.shape[0] - 1
        if n_req < 0 or req_rank.shape[0] != n_req or token_key.shape[0] < int(req_offsets[-1]):
            raise SemMoEError("token_labels: req_offsets[n_req+1], req_rank[n_req], token_key[req_offsets[-1]]", -2)
        dev, conf, level = (np.zeros(max(int(V), 1), dtype=np.int32) for _ in range(3))
        c = self._cfg()
        self._check("semmoe_token_labels", self.lib.semmoe_token_labels(
            C.byref(c), _ptr(req_offsets), int(n_req), _ptr(token_key), _ptr(req_rank), int(V), _ptr(dev), _ptr(conf),
            _ptr(level)))
        return dev, conf, level

    def reshuffle(self, topk_ids, expert_to_rank, token_rank, shf, inv_shf, rank_count, cap=None):
        c = self._cfg(**({"cap": cap} if cap is not None else {}))
        self._check("semmoe_reshuffle", self.lib.semmoe_reshuffle(
            C.byref(c), _stream(), _ptr(topk_ids), _ptr(expert_to_rank), _ptr(token_rank), _ptr(shf),
            _ptr(inv_shf), _ptr(rank_count), _ptr(self.ws), self.ws_bytes))

    def reshuffle_static(self, topk_ids, expert_to_rank, token_rank, shf, inv_shf, rank_count, cap=None):
        """the reshuffle on the library's own fixed scratch array: no workspace argument, no allocation"""
        c = self._cfg(**({"cap": cap} if cap is not None else {}))
        self._check("semmoe_reshuffle_static", self.lib.semmoe_reshuffle_static(
            C.byref(c), _stream(), _ptr(topk_ids), _ptr(expert_to_rank), _ptr(token_rank), _ptr(shf),
            _ptr(inv_shf), _ptr(rank_count)))

    def reshuffle_rounds(self, topk_ids, expert_to_rank, rounds, token_rank, shf, inv_shf, rank_count, cap=None):
        c = self._cfg(**({"cap": cap} if cap is not None else {}))
        self._check("semmoe_reshuffle_rounds", self.lib.semmoe_reshuffle_rounds(
            C.byref(c), _stream(), _ptr(topk_ids), _ptr(expert_to_rank), int(rounds), _ptr(token_rank), _ptr(shf),
            _ptr(inv_shf), _ptr(rank_count), _ptr(self.ws), self.ws_bytes))

    def reshuffle_refine(self, topk_ids, expert_to_rank, rounds, max_cycles, token_rank, shf, inv_shf, rank_count,
                         info, cap=None):
        c = self._cfg(**({"cap": cap} if cap is not None else {}))
        self._check("semmoe_reshuffle_refine", self.lib.semmoe_reshuffle_refine(
            C.byref(c), _stream(), _ptr(topk_ids), _ptr(expert_to_rank), int(rounds), int(max_cycles),
            _ptr(token_rank), _ptr(shf), _ptr(inv_shf), _ptr(rank_count), _ptr(info), _ptr(self.ws), self.ws_bytes))

    def reshuffle_lookup(self, token_key, V, dev, conf_q16, level, thr_q16, token_rank, shf, inv_shf, rank_count,
                         cap=None):
        c = self._cfg(**({"cap": cap} if cap is not None else {}))
        self._check("semmoe_reshuffle_lookup", self.lib.semmoe_reshuffle_lookup(
            C.byref(c), _stream(), _ptr(token_key), int(V), _ptr(dev), _ptr(conf_q16), _ptr(level), int(thr_q16),
            _ptr(token_rank), _ptr(shf), _ptr(inv_shf), _ptr(rank_count), _ptr(self.ws), self.ws_bytes))

    def reshuffle_cond(self, token_key, V, dev, conf_q16, level, seq_key, VA, dev_a, conf_a_q16, level_a, thr_q16,
                       token_rank, shf, inv_shf, rank_count, cap=None):
        c = self._cfg(**({"cap": cap} if cap is not None else {}))
        self._check("semmoe_reshuffle_cond", self.lib.semmoe_reshuffle_cond(
            C.byref(c), _stream(), _ptr(token_key), int(V), _ptr(dev), _ptr(conf_q16), _ptr(level), _ptr(seq_key),
            int(VA), _ptr(dev_a), _ptr(conf_a_q16), _ptr(level_a), int(thr_q16), _ptr(token_rank), _ptr(shf),
            _ptr(inv_shf), _ptr(rank_count), _ptr(self.ws), self.ws_bytes))

    def device_sequence(self, topk_ids, expert_to_rank, T_batch, seq_in, seq_out):
        c = self._cfg()
        self._check("semmoe_device_sequence", self.lib.semmoe_device_sequence(
            C.byref(c), _stream(), _ptr(topk_ids), _ptr(expert_to_rank), int(T_batch), _ptr(seq_in), _ptr(seq_out)))

    def request_schedule(self, req_offsets, n_req, token_key, V, dev, req_rank, token_rank, shf, inv_shf, rank_count):
        c = self._cfg()
        self._check("semmoe_request_schedule", self.lib.semmoe_request_schedule(
            C.byref(c), _stream(), _ptr(req_offsets), int(n_req), _ptr(token_key), int(V), _ptr(dev), _ptr(req_rank),
            _ptr(token_rank), _ptr(shf), _ptr(inv_shf), _ptr(rank_count), _ptr(self.ws), self.ws_bytes))

    def dispatch(self, X, topk_ids, token_rank, shf, phys_of_expert, X_perm, slot_of_pair, pair_of_slot,
                 expert_offsets, rank_offsets, send_matrix, remote_pairs):
        c = self._cfg()
        self._check("semmoe_dispatch", self.lib.semmoe_dispatch(
            C.byref(c), _stream(), _ptr(X), _ptr(topk_ids), _ptr(token_rank), _ptr(shf), _ptr(phys_of_expert),
            _ptr(X_perm), _ptr(slot_of_pair), _ptr(pair_of_slot), _ptr(expert_offsets), _ptr(rank_offsets),
            _ptr(send_matrix), _ptr(remote_pairs), _ptr(self.ws), self.ws_bytes))

    def dispatch_index(self, topk_ids, token_rank, shf, phys_of_expert, slot_of_pair, pair_of_slot, expert_offsets,
                       rank_offsets, send_matrix, remote_pairs):
        c = self._cfg()
        self._check("semmoe_dispatch_index", self.lib.semmoe_dispatch_index(
            C.byref(c), _stream(), _ptr(topk_ids), _ptr(token_rank), _ptr(shf), _ptr(phys_of_expert),
            _ptr(slot_of_pair), _ptr(pair_of_slot), _ptr(expert_offsets), _ptr(rank_offsets), _ptr(send_matrix),
            _ptr(remote_pairs), _ptr(self.ws), self.ws_bytes))

    def dispatch_rows(self, X, slot_of_pair, X_perm):
        c = self._cfg()
        self._check("semmoe_dispatch_rows", self.lib.semmoe_dispatch_rows(
            C.byref(c), _stream(), _ptr(X), _ptr(slot_of_pair), _ptr(X_perm)))

    def expert_ffn(self, rank, X_perm, expert_offsets, expert_of_phys, W_gu, W_down, Y):
        c = self._cfg()
        self._check("semmoe_expert_ffn", self.lib.semmoe_expert_ffn(
            C.byref(c), _stream(), int(rank), _ptr(X_perm), _ptr(expert_offsets), _ptr(expert_of_phys),
            _ptr(W_gu), _ptr(W_down), _ptr(Y), _ptr(self.ws), self.ws_bytes))

    def shared_ffn(self, X, n_tokens, W_gu_sh, W_down_sh, Y_shared):
        """the shared expert has a workspace of its own (n_tokens x F activations), so that it may run on another
        stream beside the routed path's calls, which share `self.ws`"""
        c = self._cfg()
        need = int(n_tokens) * self.cfg.F * (2 if self.cfg.dtype == BF16 else 4) + 512
        if self.ws_shared is None or self.ws_shared.numel() < need:
            import torch
            self.ws_shared = torch.empty(need, dtype=torch.uint8, device=X.device)
        self._check("semmoe_shared_ffn", self.lib.semmoe_shared_ffn(
            C.byref(c), _stream(), _ptr(X), int(n_tokens), _ptr(W_gu_sh), _ptr(W_down_sh), _ptr(Y_shared),
            _ptr(self.ws_shared), self.ws_shared.numel()))

    def probe_copy(self, dst, src, nbytes):
        self._check("semmoe_probe_copy", self.lib.semmoe_probe_copy(_stream(), _ptr(dst), _ptr(src), int(nbytes)))

    def probe_stream(self, buf, nbytes, write, sink):
        self._check("semmoe_probe_stream", self.lib.semmoe_probe_stream(_stream(), _ptr(buf), int(nbytes), int(bool(write)),
                                                                        _ptr(sink)))

    def probe_mfma(self, operands, iters, sink):
        """returns the flops of the launch"""
        fl = C.c_double(0.0)
        self._check("semmoe_probe_mfma", self.lib.semmoe_probe_mfma(_stream(), _ptr(operands), int(iters), _ptr(sink),
                                                                    C.byref(fl)))
        return fl.value

    def probe_tile_loop(self, panels, n_panels, row_bytes, variant, n_slices, sink):
        """returns the flops of the launch"""
        fl = C.c_double(0.0)
        self._check("semmoe_probe_tile_loop", self.lib.semmoe_probe_tile_loop(
            _stream(), _ptr(panels), int(n_panels), int(row_bytes), int(variant), int(n_slices), _ptr(sink), C.byref(fl)))
        return fl.value

    def combine(self, Y, slot_of_pair, topk_w, Out, Y_shared=None):
        c = self._cfg()
        self._check("semmoe_combine", self.lib.semmoe_combine(
            C.byref(c), _stream(), _ptr(Y), _ptr(slot_of_pair), _ptr(topk_w), _ptr(Y_shared), _ptr(Out)))

    # -- gradients of the layer's steps
    def combine_grad(self, dOut, Y, slot_of_pair, topk_w, dY, dtopk_w):
        """dY or dtopk_w may be None (then topk_w or Y may be, too); dY may be Y itself"""
        T, d, P = self.cfg.T, self.cfg.d, self.cfg.T * self.cfg.k
        if T == 0:
            return
        here, i32, f32, acts = self._types
        dev, act = dOut.get_device(), acts[self.cfg.dtype == BF16]
        if dev < 0 or dev != here() or not (
                act is dOut.dtype and i32 is slot_of_pair.dtype and dev == slot_of_pair.get_device() and dOut.numel() >= T * d
                and slot_of_pair.numel() >= P
                and (Y is None or (act is Y.dtype and dev == Y.get_device() and Y.numel() >= P * d))
                and (dY is None or (act is dY.dtype and dev == dY.get_device() and dY.numel() >= P * d))
                and (topk_w is None or (f32 is topk_w.dtype and dev == topk_w.get_device() and topk_w.numel() >= P))
                and (dtopk_w is None or (f32 is dtopk_w.dtype and dev == dtopk_w.get_device() and dtopk_w.numel() >= P))):
            self._fit("combine_grad", ((dOut, None, T * d), (Y, None, P * d), (slot_of_pair, i32, P),
                    (topk_w, f32, P), (dY, None, P * d), (dtopk_w, f32, P)))
        c = self._cfg()
        self._check("semmoe_combine_grad", self.lib.semmoe_combine_grad(
            C.byref(c), _stream(), _ptr(dOut), _ptr(Y), _ptr(slot_of_pair), _ptr(topk_w), _ptr(dY), _ptr(dtopk_w)))

    def dispatch_grad(self, dX_perm, slot_of_pair, dX, dX_add=None):
        """dX_add may be dX itself"""
        T, d, P = self.cfg.T, self.cfg.d, self.cfg.T * self.cfg.k
        if T == 0:
            return
        here, i32, _, acts = self._types
        dev, act = dX.get_device(), acts[self.cfg.dtype == BF16]
        if dev < 0 or dev != here() or not (
                act is dX.dtype is dX_perm.dtype and i32 is slot_of_pair.dtype
                and dev == dX_perm.get_device() == slot_of_pair.get_device() and dX.numel() >= T * d
                and dX_perm.numel() >= P * d and slot_of_pair.numel() >= P
                and (dX_add is None or (act is dX_add.dtype and dev == dX_add.get_device() and dX_add.numel() >= T * d))):
            self._fit("dispatch_grad", ((dX_perm, None, P * d), (slot_of_pair, i32, P),
                    (dX, None, T * d), (dX_add, None, T * d)))
        c = self._cfg()
        self._check("semmoe_dispatch_grad", self.lib.semmoe_dispatch_grad(
            C.byref(c), _stream(), _ptr(dX_perm), _ptr(slot_of_pair), _ptr(dX_add), _ptr(dX)))

    def _ffn_grad_bytes(self, rows: int) -> int:
        return self.cfg.F * ((rows + 31) // 32 * 128 + rows * (4 if self.cfg.dtype == BF16 else 8)) + 768

    def expert_ffn_grad(self, rank, X_perm, dY, expert_offsets, expert_of_phys, W_gu, W_down, dX_perm):
        """dX_perm may be X_perm or dY itself.  W_gu and W_down hold every expert that expert_of_phys names for the rank."""
        torch = self._torch
        d, F, E, P = self.cfg.d, self.cfg.F, self.cfg.E, self.cfg.T * self.cfg.k
        if P == 0:
            return
        self._fit("expert_ffn_grad", ((X_perm, None, P * d), (dY, None, P * d),
                  (expert_offsets, torch.int32, E + 1), (expert_of_phys, torch.int32, E),
                  (W_gu, None, 2 * F * d), (W_down, None, F * d), (dX_perm, None, P * d)))
        c = self._cfg()
        ws, n, owner = self._workspace("expert_ffn_grad", self._ffn_grad_bytes(P))
        self._check("semmoe_expert_ffn_grad", self.lib.semmoe_expert_ffn_grad(
            C.byref(c), _stream(), int(rank), _ptr(X_perm), _ptr(dY), _ptr(expert_offsets), _ptr(expert_of_phys),
            _ptr(W_gu), _ptr(W_down), _ptr(dX_perm), ws, n))

    def shared_ffn_grad(self, X, dY, n_tokens, W_gu_sh, W_down_sh, dX):
        """dX may be X or dY itself"""
        d, F, n = self.cfg.d, self.cfg.F, int(n_tokens)
        if n == 0:
            return
        self._fit("shared_ffn_grad", ((X, None, n * d), (dY, None, n * d), (W_gu_sh, None, 2 * F * d),
                  (W_down_sh, None, F * d), (dX, None, n * d)))
        c = self._cfg()
        ws, size, owner = self._workspace("shared_ffn_grad", self._ffn_grad_bytes(max(n, 0)))
        self._check("semmoe_shared_ffn_grad", self.lib.semmoe_shared_ffn_grad(
            C.byref(c), _stream(), _ptr(X), _ptr(dY), n, _ptr(W_gu_sh), _ptr(W_down_sh), _ptr(dX), ws, size))

    # -- low-rank adapters
    def adapter_index(self, req_offsets, adapter_of_req, n_adapters, order, adapter_offsets):
        """the batch is order's length; requests are adapter_of_req's"""
        n_req, T = adapter_of_req.shape[0], order.shape[0]
        if req_offsets.shape[0] != n_req + 1 or adapter_offsets.shape[0] != int(n_adapters) + 1:
            raise SemMoEError("adapter_index: shapes must be req_offsets[n_req+1], adapter_of_req[n_req], "
                              "adapter_offsets[n_adapters+1]", -2)
        here, i32, _, _ = self._types
        dev = order.get_device()
        if dev < 0 or dev != here() or not (
                i32 is req_offsets.dtype is adapter_of_req.dtype is order.dtype is adapter_offsets.dtype
                and dev == req_offsets.get_device() == adapter_of_req.get_device() == adapter_offsets.get_device()):
            self._fit("adapter_index", ((req_offsets, i32, 1), (adapter_of_req, i32, 0),
                    (order, i32, 0), (adapter_offsets, i32, 1)))
        if T == 0:
            adapter_offsets.zero_()
            return
        c = self._cfg() if T == self.cfg.T else self._cfg(T=T)
        self._check("semmoe_adapter_index", self.lib.semmoe_adapter_index(
            C.byref(c), _stream(), _ptr(req_offsets), int(n_req), _ptr(adapter_of_req), int(n_adapters), _ptr(order),
            _ptr(adapter_offsets)))

    def _adapter_call(self, call, X, order, adapter_offsets, A, B, scale, dY, base, out):
        """(config, shape, workspace bytes) of an adapter call: made and checked once for shapes and distances of rows, which a
        serving step repeats for every layer; the call itself then costs the host as much as its kernels take.
        dY: None in the forward call, whose base and out have d_out columns; with it they have d_in."""
        key = (call, _config_values(self.cfg), X.shape, X.stride(), order.shape, adapter_offsets.shape, A.shape, B.shape,
               None if scale is None else scale.shape, None if dY is None else (dY.shape, dY.stride()),
               None if base is None else (base.shape, base.stride()), None if out is None else (out.shape, out.stride()))
        made = self._adapter_calls.get(key)
        if made is not None:
            return made
        if A.dim() != 3:
            raise SemMoEError("%s: A is [n_adapters, rank, d_in]" % call, -2)
        n_ad, rank, d_in = A.shape
        if B.dim() != 3 or B.shape[0] != n_ad or B.shape[2] != rank or tuple(adapter_offsets.shape) != (n_ad + 1,) \
                or tuple(order.shape) != (X.shape[0],) or (scale is not None and tuple(scale.shape) != (n_ad,)):
            raise SemMoEError("%s: shapes must be A[n,r,d_in], B[n,d_out,r], adapter_offsets[n+1], order[T], scale[n]" % call, -2)
        c, s = self._cfg(T=X.shape[0]), _CAdapterShape(n_ad, rank, d_in, B.shape[1], 0, 0, 0, 0)
        n_out = s.d_out if dY is None else d_in
        for t, field, n_cols, name in ((X, "ldx", d_in, "X"), (dY, "ldy", s.d_out, "dY"), (base, "ld_base", n_out, "the base"),
                                       (out, "ld_out", n_out, "the result")):
            if t is not None:
                setattr(s, field, _row_distance(t, n_cols, name))
                if t.shape[0] != X.shape[0]:
                    raise SemMoEError("%s: all row tensors have X's rows" % call, -2)
        n = C.c_size_t(0)
        size = "semmoe_adapter_forward_workspace_bytes" if dY is None else "semmoe_adapter_workspace_bytes"
        self._check(size, getattr(self.lib, size)(C.byref(c), C.byref(s), C.byref(n)))
        if len(self._adapter_calls) >= 256:
            self._adapter_calls.clear()
        self._adapter_calls[key] = made = (c, s, int(n.value))
        return made

    def adapters(self, X, order, adapter_offsets, A, B, Y, Y_base=None, scale=None):
        """Y = Y_base + scale * B (A x) by each token's adapter; Y_base=None adds to nothing, Y_base=Y adds in place"""
        c, s, need = self._adapter_call("adapters", X, order, adapter_offsets, A, B, scale, None, Y_base, Y)
        here, i32, f32, acts = self._types
        dev, act = X.get_device(), acts[self.cfg.dtype == BF16]
        if dev < 0 or dev != here() or not (
                act is X.dtype is A.dtype is B.dtype is Y.dtype and i32 is order.dtype is adapter_offsets.dtype
                and dev == order.get_device() == adapter_offsets.get_device() == A.get_device() == B.get_device() == Y.get_device()
                and (scale is None or (f32 is scale.dtype and dev == scale.get_device()))
                and (Y_base is None or (act is Y_base.dtype and dev == Y_base.get_device()))):
            self._fit("adapters", ((X, None, 0), (order, i32, 0), (adapter_offsets, i32, 1),
                    (A, None, 0), (B, None, 0), (scale, f32, 0), (Y_base, None, 0),
                    (Y, None, 0)))
        if X.shape[0] == 0:
            return
        ws, n, owner = self._workspace("adapters", need)
        self._check("semmoe_adapters", self.lib.semmoe_adapters(
            C.byref(c), _stream(), C.byref(s), X.data_ptr(), _ptr(order), _ptr(adapter_offsets), _ptr(A), _ptr(B), _ptr(scale),
            None if Y_base is None else Y_base.data_ptr(), Y.data_ptr(), ws, n))

    def adapters_grad(self, X, dY, order, adapter_offsets, A, B, dX=None, dA=None, dB=None, dX_base=None, scale=None):
        """each of dX, dA, dB may be left out; dX_base=dX adds in place; dX may be X or dY itself"""
        torch = self._torch
        c, s, need = self._adapter_call("adapters_grad", X, order, adapter_offsets, A, B, scale, dY, dX_base, dX)
        if (dA is not None and dA.shape != A.shape) or (dB is not None and dB.shape != B.shape):
            raise SemMoEError("adapters_grad: dA and dB have the shapes of A and B", -2)
        taken = [A.data_ptr(), B.data_ptr()]  # dX is made from A after dA has been written
        for t in (dA, dB):
            if t is not None:
                if t.data_ptr() in taken:
                    raise SemMoEError("adapters_grad: dA and dB may not lie in the place of A, B or one another", -1)
                taken.append(t.data_ptr())
        self._fit("adapters_grad", ((X, None, 0), (dY, None, 0), (order, torch.int32, 0),
                  (adapter_offsets, torch.int32, 1), (A, None, 0), (B, None, 0),
                  (scale, torch.float32, 0), (dX_base, None, 0), (dX, None, 0), (dA, None, 0),
                  (dB, None, 0)))
        if X.shape[0] == 0:
            for t in (dA, dB):
                if t is not None:
                    t.zero_()
            return
        ws, n, owner = self._workspace("adapters", need)
        self._check("semmoe_adapters_grad", self.lib.semmoe_adapters_grad(
            C.byref(c), _stream(), C.byref(s), X.data_ptr(), dY.data_ptr(), _ptr(order), _ptr(adapter_offsets), _ptr(A), _ptr(B),
            _ptr(scale), None if dX_base is None else dX_base.data_ptr(), None if dX is None else dX.data_ptr(), _ptr(dA),
            _ptr(dB), ws, n))

    # -- rows and weights in 8-bit integers
    def quantize_rows(self, X, Xq, x_scale):
        """X's rows may lie further apart than they are wide; Xq is packed.  Serves activations and weights alike."""
        n, cols = X.shape
        here, _, f32, acts = self._types
        dev, act = X.get_device(), acts[self.cfg.dtype == BF16]
        if dev < 0 or dev != here() or not (
                act is X.dtype and self._torch.int8 is Xq.dtype and f32 is x_scale.dtype
                and dev == Xq.get_device() == x_scale.get_device() and Xq.numel() >= n * cols and x_scale.numel() >= n):
            self._fit("quantize_rows", ((X, None, 0), (Xq, self._torch.int8, n * cols), (x_scale, f32, n)))
        if n == 0:
            return
        c = self._cfg()
        self._check("semmoe_quantize_rows", self.lib.semmoe_quantize_rows(
            C.byref(c), _stream(), X.data_ptr(), n, cols, cols if X.is_contiguous() else _row_distance(X, cols, "X"), _ptr(Xq),
            _ptr(x_scale)))

    def dispatch_rows_i8(self, Xq, x_scale, slot_of_pair, Xq_perm, x_scale_perm):
        T, d, P = self.cfg.T, self.cfg.d, self.cfg.T * self.cfg.k
        if T == 0:
            return
        here, i32, f32, _ = self._types
        dev, i8 = Xq.get_device(), self._torch.int8
        if dev < 0 or dev != here() or not (
                i8 is Xq.dtype is Xq_perm.dtype and f32 is x_scale.dtype is x_scale_perm.dtype and i32 is slot_of_pair.dtype
                and dev == x_scale.get_device() == slot_of_pair.get_device() == Xq_perm.get_device() == x_scale_perm.get_device()
                and Xq.numel() >= T * d and x_scale.numel() >= T and slot_of_pair.numel() >= P and Xq_perm.numel() >= P * d
                and x_scale_perm.numel() >= P):
            self._fit("dispatch_rows_i8", ((Xq, i8, T * d), (x_scale, f32, T), (slot_of_pair, i32, P), (Xq_perm, i8, P * d),
                                           (x_scale_perm, f32, P)))
        c = self._cfg()
        self._check("semmoe_dispatch_rows_i8", self.lib.semmoe_dispatch_rows_i8(
            C.byref(c), _stream(), _ptr(Xq), _ptr(x_scale), _ptr(slot_of_pair), _ptr(Xq_perm), _ptr(x_scale_perm)))

    def linear_i8(self, Xq, x_scale, Wq, w_scale, Y):
        """Y[T,d_out] of Xq[T,d_in], Wq[d_out,d_in]; Xq and Y may be column ranges of wider tensors"""
        (n, d_in), d_out = Xq.shape, Wq.shape[0]
        if Wq.shape != (d_out, d_in) or Y.shape != (n, d_out):
            raise SemMoEError("linear_i8: shapes must be Xq[T,d_in], Wq[d_out,d_in], Y[T,d_out]", -2)
        here, _, f32, acts = self._types
        dev, i8 = Xq.get_device(), self._torch.int8
        if dev < 0 or dev != here() or not (
                i8 is Xq.dtype is Wq.dtype and f32 is x_scale.dtype is w_scale.dtype and acts[1] is Y.dtype
                and dev == x_scale.get_device() == Wq.get_device() == w_scale.get_device() == Y.get_device()
                and x_scale.numel() >= n and w_scale.numel() >= d_out):
            self._fit("linear_i8", ((Xq, i8, 0), (x_scale, f32, n), (Wq, i8, 0), (w_scale, f32, d_out), (Y, acts[1], 0)))
        if n == 0:
            return
        key = (n, d_in, d_out, d_in if Xq.is_contiguous() else _row_distance(Xq, d_in, "Xq"),
               d_out if Y.is_contiguous() else _row_distance(Y, d_out, "Y"))
        s = self._linear_shapes.get(key)
        if s is None:
            if len(self._linear_shapes) >= 256:
                self._linear_shapes.clear()
            self._linear_shapes[key] = s = _CLinearShape(*key)
        c = self._cfg()
        self._check("semmoe_linear_i8", self.lib.semmoe_linear_i8(
            C.byref(c), _stream(), C.byref(s), Xq.data_ptr(), _ptr(x_scale), _ptr(Wq), _ptr(w_scale), Y.data_ptr()))

    def expert_ffn_i8(self, rank, Xq_perm, x_scale_perm, expert_offsets, expert_of_phys, Wq_gu, w_scale_gu, Wq_down, w_scale_down, Y):
        """the weights and their scales hold every expert that expert_of_phys names for the rank"""
        d, F, E, P = self.cfg.d, self.cfg.F, self.cfg.E, self.cfg.T * self.cfg.k
        if P == 0:
            return
        here, i32, f32, acts = self._types
        dev, i8 = Y.get_device(), self._torch.int8
        if dev < 0 or dev != here() or not (
                i8 is Xq_perm.dtype is Wq_gu.dtype is Wq_down.dtype and acts[1] is Y.dtype and i32 is expert_offsets.dtype is expert_of_phys.dtype
                and f32 is x_scale_perm.dtype is w_scale_gu.dtype is w_scale_down.dtype
                and dev == Xq_perm.get_device() == x_scale_perm.get_device() == expert_offsets.get_device() == expert_of_phys.get_device()
                and dev == Wq_gu.get_device() == w_scale_gu.get_device() == Wq_down.get_device() == w_scale_down.get_device()
                and Xq_perm.numel() >= P * d and x_scale_perm.numel() >= P and expert_offsets.numel() > E and expert_of_phys.numel() >= E
                and Wq_gu.numel() >= 2 * F * d and w_scale_gu.numel() >= 2 * F and Wq_down.numel() >= F * d and w_scale_down.numel() >= d
                and Y.numel() >= P * d):
            self._fit("expert_ffn_i8", ((Xq_perm, i8, P * d), (x_scale_perm, f32, P), (expert_offsets, i32, E + 1),
                                        (expert_of_phys, i32, E), (Wq_gu, i8, 2 * F * d), (w_scale_gu, f32, 2 * F), (Wq_down, i8, F * d),
                                        (w_scale_down, f32, d), (Y, acts[1], P * d)))
        c = self._cfg()
        ws, n, owner = self._workspace("expert_ffn_i8", P * (3 * F + 4) + 1024)
        self._check("semmoe_expert_ffn_i8", self.lib.semmoe_expert_ffn_i8(
            C.byref(c), _stream(), int(rank), _ptr(Xq_perm), _ptr(x_scale_perm), _ptr(expert_offsets), _ptr(expert_of_phys),
            _ptr(Wq_gu), _ptr(w_scale_gu), _ptr(Wq_down), _ptr(w_scale_down), _ptr(Y), ws, n))

    def shared_ffn_i8(self, Xq, x_scale, n_tokens, Wq_gu_sh, w_scale_gu_sh, Wq_down_sh, w_scale_down_sh, Y_shared):
        d, F, n = self.cfg.d, self.cfg.F, int(n_tokens)
        if n == 0:
            return
        here, _, f32, acts = self._types
        dev, i8 = Y_shared.get_device(), self._torch.int8
        if dev < 0 or dev != here() or not (
                i8 is Xq.dtype is Wq_gu_sh.dtype is Wq_down_sh.dtype and acts[1] is Y_shared.dtype
                and f32 is x_scale.dtype is w_scale_gu_sh.dtype is w_scale_down_sh.dtype
                and dev == Xq.get_device() == x_scale.get_device() == Wq_gu_sh.get_device() == w_scale_gu_sh.get_device()
                and dev == Wq_down_sh.get_device() == w_scale_down_sh.get_device() and Xq.numel() >= n * d and x_scale.numel() >= n
                and Wq_gu_sh.numel() >= 2 * F * d and w_scale_gu_sh.numel() >= 2 * F and Wq_down_sh.numel() >= F * d
                and w_scale_down_sh.numel() >= d and Y_shared.numel() >= n * d):
            self._fit("shared_ffn_i8", ((Xq, i8, n * d), (x_scale, f32, n), (Wq_gu_sh, i8, 2 * F * d), (w_scale_gu_sh, f32, 2 * F),
                                        (Wq_down_sh, i8, F * d), (w_scale_down_sh, f32, d), (Y_shared, acts[1], n * d)))
        c = self._cfg()
        ws, size, owner = self._workspace("shared_ffn_i8", max(n, 0) * (3 * F + 4) + 1024)
        self._check("semmoe_shared_ffn_i8", self.lib.semmoe_shared_ffn_i8(
            C.byref(c), _stream(), _ptr(Xq), _ptr(x_scale), n, _ptr(Wq_gu_sh), _ptr(w_scale_gu_sh), _ptr(Wq_down_sh),
            _ptr(w_scale_down_sh), _ptr(Y_shared), ws, size))

    # -- the norms around a block
    def _norm_call(self, call, T, d, par, gate, vectors, rows):
        """(config, shape) of a call on the norms: made and checked once for shapes, distances of rows and par (the bytes of
        res_scale, eps_post, eps_pre), which every layer of a step repeats.  vectors are w_post and w_pre with the gradients of such, and a gate of one
        dimension with its gradient, which are all rows'; rows the tensors [T,d] by the name of their distance."""
        s = _CNormShape(*_three_numbers.unpack(par), int(gate is not None and gate.dim() == 2))
        for t in vectors:
            if t is not None and (tuple(t.shape) != (d,) or not t.is_contiguous()):
                raise SemMoEError("%s: a norm's weights, a gate of all rows and their gradients are %d numbers behind one another" % (call, d), -2)
        for name, t in rows:
            if t is not None:
                if tuple(t.shape) != (T, d):
                    raise SemMoEError("%s: rows must be [%d, %d]" % (call, T, d), -2)
                setattr(s, name, _row_distance(t, d, name))
        return (self._cfg() if (self.cfg.T, self.cfg.d) == (T, d) else self._cfg(T=T, d=d)), s

    def _kept_norm_call(self, key, make):
        kept = self._norm_calls.get(key)
        if kept is None:
            if len(self._norm_calls) >= 256:
                self._norm_calls.clear()
            self._norm_calls[key] = kept = make()
        return kept

    def block_norm(self, R, H, Y=None, X=None, Xq=None, x_scale=None, w_post=None, w_pre=None, gate=None, res_scale=1.0,
                   eps_post=1e-6, eps_pre=1e-6):
        """H = res_scale R + gate norm(Y) w_post, X = norm(H) w_pre, and X in 8 bits as Xq and x_scale; what is None is left out.
        gate: [d] or [T,d].  H and X may lie in the place of R or Y."""
        T, d = (Y if R is None else R).shape
        tensors = (R, Y, w_post, gate, w_pre, H, X)
        par = _three_numbers.pack(res_scale, eps_post, eps_pre)  # their values now, and their signs
        key = (_config_values(self.cfg), par, *[None if t is None else (t.shape, t.stride()) for t in tensors])

        def make():
            of_all = gate is not None and gate.dim() == 1
            return self._norm_call("block_norm", T, d, par, gate, (w_post, w_pre, gate if of_all else None), (
                ("ld_r", R), ("ld_y", Y), ("ld_h", H), ("ld_x", X), ("ld_gate", None if of_all else gate)))

        c, s = self._kept_norm_call(key, make)
        here, _, f32, acts = self._types
        dev, act, i8 = (Y if R is None else R).get_device(), acts[self.cfg.dtype == BF16], self._torch.int8
        if dev < 0 or dev != here():
            self._fit("block_norm", ((Y if R is None else R, None, 0),))
        for t in tensors:
            if t is not None and (t.dtype is not act or t.get_device() != dev):
                self._fit("block_norm", ((t, None, 0),))
        if not (Xq is None is x_scale) and not (
                Xq is not None and x_scale is not None and i8 is Xq.dtype and f32 is x_scale.dtype
                and dev == Xq.get_device() == x_scale.get_device() and Xq.numel() >= T * d and x_scale.numel() >= T):
            self._fit("block_norm", ((Xq, i8, T * d), (x_scale, f32, T)))
        if T == 0:
            return
        R, Y, w_post, gate, w_pre, H, X = [None if t is None else t.data_ptr() for t in tensors]
        if H == X is not None:
            raise SemMoEError("block_norm: H and X lie in the same place", -1)
        self._check("semmoe_block_norm", self.lib.semmoe_block_norm(
            C.byref(c), _stream(), C.byref(s), R, Y, w_post, gate, w_pre, H, X, _ptr(Xq), _ptr(x_scale)))

    def block_norm_grad(self, H, dR, Y=None, dH=None, dX=None, w_post=None, w_pre=None, gate=None, dY=None, dgate=None, dw_post=None,
                        dw_pre=None, res_scale=1.0, eps_post=1e-6, eps_pre=1e-6):
        """each of dR, dY, dgate, dw_post and dw_pre may be None; dH or dX may, and H without dX.  dR, dY and a dgate of rows may lie in
        the place of one of dH, dX, H and Y, not in each other's."""
        T, d = (dX if dH is None else dH).shape
        tensors = (dH, dX, H, Y, w_post, gate, w_pre, dR, dY, dgate, dw_post, dw_pre)
        par = _three_numbers.pack(res_scale, eps_post, eps_pre)  # their values now, and their signs
        key = (_config_values(self.cfg), par, *[None if t is None else (t.shape, t.stride()) for t in tensors])
        of_all = gate is not None and gate.dim() == 1

        def make():
            if dgate is not None and (gate is None or dgate.shape != gate.shape):
                raise SemMoEError("block_norm_grad: dgate has gate's shape", -2)
            c, s = self._norm_call("block_norm_grad", T, d, par, gate, (w_post, w_pre, dw_post, dw_pre, *((gate, dgate) if of_all else ())), (
                ("ld_dh", dH), ("ld_dx", dX), ("ld_h", H), ("ld_y", Y), ("ld_dr", dR), ("ld_dy", dY),
                ("ld_gate", None if of_all else gate), ("ld_dgate", None if of_all else dgate)))
            need = C.c_size_t(0)
            self._check("semmoe_block_norm_grad_workspace_bytes",
                        self.lib.semmoe_block_norm_grad_workspace_bytes(C.byref(c), C.byref(need)))
            return c, s, int(need.value)

        c, s, need = self._kept_norm_call(key, make)
        dev, act = (dX if dH is None else dH).get_device(), self._types[3][self.cfg.dtype == BF16]
        if dev < 0 or dev != self._types[0]():
            self._fit("block_norm_grad", ((dX if dH is None else dH, None, 0),))
        for t in tensors:
            if t is not None and (t.dtype is not act or t.get_device() != dev):
                self._fit("block_norm_grad", ((t, None, 0),))
        if T == 0:
            for t in (dgate, dw_post, dw_pre):
                if t is not None:
                    t.zero_()
            return
        at = [None if t is None else t.data_ptr() for t in tensors]
        outs = [p for p in at[7:] if p is not None]
        if len(set(outs)) != len(outs):
            raise SemMoEError("block_norm_grad: two results lie in the same place", -1)
        ws, n, owner = None, 0, None
        if dw_post is not None or dw_pre is not None or (of_all and dgate is not None):
            ws, n, owner = self._workspace("block_norm_grad", need)
        self._check("semmoe_block_norm_grad", self.lib.semmoe_block_norm_grad(
            C.byref(c), _stream(), C.byref(s), *at, ws, n))
