"""Operators that stand around and inside an MoE layer served in 8 bits and trained: what is measured of them.

  norm       block_norm: H = res_scale R + gate * norm(Y) w_post behind a block, X = norm(H) w_pre before the next, in one pass
  norm_grad  the gradient of that towards the residual, the block's rows, the gate and both norms' weights
  linear     quantize_rows, linear_i8: a projection of rows and weights in 8-bit integers with a scale for each token and channel;
             with norm, the rows come out of block_norm in 8 bits
  experts    quantize_rows, dispatch_rows_i8, expert_ffn_i8: the grouped SwiGLU FFN of one rank's experts in 8 bits
  shared     quantize_rows, shared_ffn_i8: the same FFN with one set of weights

Widths, experts and token counts are those of `workloads.CONFIGS` and `perf/cases.py`.  With `own` the calls go through `SemMoE`;
without, the same is computed by elementary torch operations in 32 bits.
"""
import math

import torch

DEV = "cuda:0"
own = False
EPS = 1e-6

SHAPES = {
    "qwen3_30b": dict(d=2048, E=128, k=8, F=768, D=8),
    "qwen3_235b": dict(d=4096, E=128, k=8, F=1536, D=8),
    "gpt_oss_120b": dict(d=2880, E=128, k=4, F=2880, D=16),
    "deepseek_v3": dict(d=7168, E=256, k=8, F=2048, D=32),
}


def listed():
    def norm(name, op, T, d, gate="channel", dtype="bf16"):
        return dict(name=name, op=op, T=T, d=d, gate=gate, dtype=dtype)

    def linear(name, T, d_in, d_out, norm=False):
        return dict(name=name, op="linear", T=T, d_in=d_in, d_out=d_out, norm=norm, gate="channel", dtype="bf16")

    def experts(name, shape, **kw):
        return dict(name=name, op="experts", **SHAPES[shape], **kw)

    return [
        # between two blocks of a decode step: the smallest call, where latency counts
        norm("norm_decode", "norm", T=64, d=4096),
        # a prefill batch
        norm("norm_prefill", "norm", T=16384, d=7168),
        # a training step's batch, one gate for each channel
        norm("norm_grad_train", "norm_grad", T=8192, d=4096),
        # a small fp32 model, ragged, with a gate computed for each token
        norm("norm_grad_tiny_fp32", "norm_grad", T=777, d=512, gate="token", dtype="fp32"),
        # a projection in a decode step of few requests: the weights are read for a handful of rows
        linear("linear_decode", T=16, d_in=4096, d_out=4096),
        # the norm before a projection hands over its rows in 8 bits; an odd token count
        linear("norm_linear_chunk", T=1001, d_in=2880, d_out=5760, norm=True),
        # a prefill batch through a wide projection
        linear("linear_prefill", T=8192, d_in=7168, d_out=4096),
        # a decode step with all experts on one GPU: every expert is read for eight rows
        experts("experts_decode", "qwen3_30b", T=128, rank=-1, rows=1024, skew=0.5),
        # a chunk of a prompt on one of sixteen ranks, ragged
        experts("experts_chunk", "gpt_oss_120b", T=2500, rank=3, rows=1210, skew=0.6),
        # experts of the most loaded rank under an affinity placement, prefill
        experts("experts_prefill", "qwen3_30b", T=8192, rank=0, rows=20865, skew=0.3),
        # the shared expert in a decode step
        dict(name="shared_decode", op="shared", T=64, d=7168, F=2048),
        # the shared expert on a prefill batch
        dict(name="shared_prefill", op="shared", T=4096, d=7168, F=2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "norm_grad", "linear", "linear", "experts", "experts", "shared"])
    if op in ("norm", "norm_grad"):
        d = 8 * _log_int(rng, 8, 896)
        return dict(op=op, T=_log_int(rng, 1, min(32768, int((1.1e8 if op == "norm" else 3.3e7) / d))), d=d,
                    gate=rng.choice(["channel", "token", "none"]), dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if op == "linear":
        d_in, d_out = 16 * _log_int(rng, 16, 448), 8 * _log_int(rng, 32, 896)
        return dict(op=op, T=_log_int(rng, 1, min(16384, int(2.3e11 / (d_in * d_out)))), d_in=d_in, d_out=d_out,
                    norm=rng.random() < 0.3, gate=rng.choice(["channel", "token", "none"]), dtype="bf16")
    if op == "shared":
        d, F = 16 * _log_int(rng, 16, 448), 16 * _log_int(rng, 8, 180)
        return dict(op=op, T=_log_int(rng, 1, min(16384, int(6e10 / (d * F)))), d=d, F=F)
    c = dict(op=op, **SHAPES[rng.choice(list(SHAPES))])
    if rng.random() < 0.3:  # widths that are no multiples of the tiles
        c["d"], c["F"] = 16 * rng.randrange(64, 180), 16 * rng.randrange(32, 120)
    m = c["E"] // c["D"]
    c["rank"] = rng.choice([0, c["D"] - 1]) if c["E"] * c["F"] * c["d"] > 3e8 else rng.choice([-1, 0, c["D"] - 1])
    groups = m if c["rank"] >= 0 else c["E"]
    most = min(1200 if c["rank"] >= 0 else 200, int(3.2e10 / (groups * c["d"] * c["F"])))
    c["rows"] = groups * _log_int(rng, 2, most) + rng.randrange(groups)
    c["skew"] = rng.choice([0.1, 0.3, 0.6])
    c["T"] = -(-c["rows"] // c["k"]) * (rng.choice([2, c["D"] // 2]) if c["rank"] >= 0 else 1)
    return c


# ------------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(g, shape, std, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _weights(g, n, rows, cols, std):
    """(8-bit weights [n, rows, cols], scales [n, rows]): a scale for each output channel, as a checkpoint holds them"""
    q, s = torch.empty(n, rows, cols, dtype=torch.int8, device=DEV), torch.empty(n, rows, device=DEV)
    for e in range(n):
        q[e], s[e] = _quantize(_randn(g, (rows, cols), std).float())
    return q, s


def _norm_inputs(s, case, g, d):
    T, act = case["T"], torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s["R"], s["Y"] = _randn(g, (T, d), 3.0, act), _randn(g, (T, d), 0.5, act)
    s["w_post"], s["w_pre"] = 1.0 + _randn(g, (d,), 0.2, act), 1.0 + _randn(g, (d,), 0.2, act)
    shape = {"channel": (d,), "token": (T, d), "none": None}[case["gate"]]
    s["gate"] = None if shape is None else _randn(g, shape, 0.7, act)
    s["res_scale"] = 0.9
    return act


def prepare(case, seed):
    g = _gen(seed)
    op, T = case["op"], case["T"]
    s = {"op": op}
    config = dict(T=T, d=case.get("d") or case["d_in"], E=1, k=1, F=16, D=1, cap=T, dtype=case.get("dtype", "bf16"))
    if op in ("norm", "norm_grad"):
        d = case["d"]
        act = _norm_inputs(s, case, g, d)
        new = lambda *shape: torch.empty(*shape, dtype=act, device=DEV)  # noqa: E731
        if op == "norm":
            s["H"], s["X"] = new(T, d), new(T, d)
        else:
            s["H"] = _randn(g, (T, d), 3.0, act)  # what the forward call stored
            s["dH"], s["dX"] = _randn(g, (T, d), 0.1, act), _randn(g, (T, d), 0.1, act)
            s["dR"], s["dY"], s["dw_post"], s["dw_pre"] = new(T, d), new(T, d), new(d), new(d)
            s["dgate"] = None if s["gate"] is None else torch.empty_like(s["gate"])
    elif op == "linear":
        d_in, d_out = case["d_in"], case["d_out"]
        s["norm"] = case["norm"]
        if case["norm"]:
            _norm_inputs(s, case, g, d_in)
            s["H"] = torch.empty(T, d_in, dtype=torch.bfloat16, device=DEV)
        else:
            s["X"] = _randn(g, (T, d_in), 1.0)
        W, w_scale = _weights(g, 1, d_out, d_in, d_in ** -0.5)
        s["W"], s["w_scale"] = W[0], w_scale[0]
        s["out"] = torch.empty(T, d_out, dtype=torch.bfloat16, device=DEV)
        s["Xq"], s["x_scale"] = torch.empty(T, d_in, dtype=torch.int8, device=DEV), torch.empty(T, device=DEV)
    else:
        d, F = case["d"], case["F"]
        s["X"] = _randn(g, (T, d), 1.0)
        s["Xq"], s["x_scale"] = torch.empty(T, d, dtype=torch.int8, device=DEV), torch.empty(T, device=DEV)
        n = 1
        if op == "experts":
            E, k, D, rank, rows = (case[x] for x in ("E", "k", "D", "rank", "rows"))
            P, m = T * k, E // D
            config.update(E=E, k=k, D=D, cap=-(-T // D))
            lo, n = (rank * m, m) if rank >= 0 else (0, E)
            counts = torch.zeros(E, dtype=torch.int64, device=DEV)
            p = _randn(g, (E,), case["skew"], torch.float32).exp()
            counts[lo:lo + n] = torch.bincount(torch.multinomial(p[lo:lo + n], rows, replacement=True, generator=g), minlength=n)
            if n < E and P > rows:  # the pairs of the other ranks lie before and after this rank's
                p[lo:lo + n] = 0
                counts += torch.bincount(torch.multinomial(p, P - rows, replacement=True, generator=g), minlength=E)
            elif P > rows:  # all experts here: what the token count rounds up to
                counts[E - 1] += P - rows
            s["expert_offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
            s["of_phys"] = torch.randperm(n, device=DEV, generator=g).to(torch.int32).repeat(E // n).contiguous()
            s["slot_of_pair"] = torch.randperm(P, device=DEV, generator=g).to(torch.int32)
            s["Xq_perm"] = torch.empty(P, d, dtype=torch.int8, device=DEV)
            s["x_scale_perm"] = torch.empty(P, device=DEV)
            s["out"] = torch.zeros(P, d, dtype=torch.bfloat16, device=DEV)
            s["rank"], s["lo"], s["n"], s["most"] = rank, lo, n, int(counts[lo:lo + n].max())
        else:
            s["out"] = torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
        config.update(F=F)
        # a rank's program holds the weights of its own experts
        s["W_gu"], s["w_scale_gu"] = _weights(g, n, 2 * F, d, 0.02)
        s["W_down"], s["w_scale_down"] = _weights(g, n, d, F, 0.02)
    if own:
        import paper_2503_04398_amd as S
        s["m"] = S.SemMoE(S.Config(**config), device=DEV)
    return s


# --------------------------------------------------------------------------------------------- the plain forms
def _quantize(x):
    """(x in 8 bits, scale of each row): the largest magnitude of a row is 127; ties go to the even number"""
    amax = x.abs().amax(1, keepdim=True)
    r = torch.where(amax > 0, 127.0 / amax, 0.0)
    return (x * r).round().to(torch.int8), (amax / 127.0)[:, 0]


def _normed(x, w):
    return x * (1.0 / (x.square().mean(1, keepdim=True) + EPS).sqrt()) * w


def _plain_norm(s):
    """(H, X) in 32 bits"""
    n = _normed(s["Y"].float(), s["w_post"].float())
    if s["gate"] is not None:
        n = s["gate"].float() * n
    H = s["res_scale"] * s["R"].float() + n
    return H, _normed(H, s["w_pre"].float())


def _plain_norm_grad(s):
    act = s["R"].dtype
    H, Y, dX, w_post, w_pre = (s[n].float() for n in ("H", "Y", "dX", "w_post", "w_pre"))

    def back(x, g, w):  # x, the gradient of norm(x) w: (the gradient towards x, towards w)
        r = 1.0 / (x.square().mean(1, keepdim=True) + EPS).sqrt()
        xn, gw = x * r, g * w
        return r * (gw - xn * (gw * xn).mean(1, keepdim=True)), (g * xn).sum(0)

    through, dw_pre = back(H, dX, w_pre)
    dH = s["dH"].float() + through
    n = _normed(Y, w_post)
    out = {"dR": (s["res_scale"] * dH).to(act), "dw_pre": dw_pre.to(act)}
    dn = dH
    if s["gate"] is not None:
        dgate, dn = dH * n, dH * s["gate"].float()
        out["dgate"] = (dgate.sum(0) if s["gate"].dim() == 1 else dgate).to(act)
    dY, dw_post = back(Y, dn, w_post)
    return {**out, "dY": dY.to(act), "dw_post": dw_post.to(act)}


def _plain_linear(s):
    out = {}
    if s["norm"]:
        H, x = _plain_norm(s)
        out["H"] = H.to(torch.bfloat16)
    else:
        x = s["X"].float()
    q, scale = _quantize(x)
    y = (q.float() @ s["W"].float().t()) * scale[:, None] * s["w_scale"]
    return {**out, "Y": y.to(torch.bfloat16)}


def _swiglu(gu, F):
    """the hidden row, rounded to the activations' type as expert_ffn's is"""
    gate, up = gu[..., :F], gu[..., F:]
    return (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16).float()


def _plain_shared(s):
    F = s["W_down"].shape[2]
    q, scale = _quantize(s["X"].float())
    h = _swiglu((q.float() @ s["W_gu"][0].float().t()) * scale[:, None] * s["w_scale_gu"][0], F)
    q, scale = _quantize(h)
    y = (q.float() @ s["W_down"][0].float().t()) * scale[:, None] * s["w_scale_down"][0]
    return {"Y": y.to(torch.bfloat16)}


def _plain_experts(s):
    """every expert's rows padded to the longest of them, and a batch of products"""
    lo, n, most, F = s["lo"], s["n"], s["most"], s["W_down"].shape[2]
    P, T = s["slot_of_pair"].shape[0], s["X"].shape[0]
    off = s["expert_offsets"].long()[lo:lo + n + 1]
    row = torch.arange(P, device=DEV)
    of = (torch.searchsorted(off, row, right=True) - 1).clamp(0, n - 1)
    mine = (row >= off[0]) & (row < off[-1])
    place = torch.where(mine, of * most + (row - off[of]), n * most)  # the last one: rows of other ranks
    token_of_slot = torch.empty_like(row)
    token_of_slot[s["slot_of_pair"].long()] = row // (P // T)
    e = s["of_phys"].long()[lo:lo + n]
    q, scale = _quantize(s["X"].float())

    def padded(x):
        return torch.zeros(n * most + 1, x.shape[1], device=DEV).index_copy(0, place, x)[:-1].view(n, most, -1)

    x, x_scale = padded(q[token_of_slot].float()), padded(scale[token_of_slot][:, None])
    gu = torch.bmm(x, s["W_gu"][e].float().transpose(1, 2).contiguous()) * x_scale * s["w_scale_gu"][e][:, None]
    q, scale = _quantize(_swiglu(gu, F).view(n * most, F))
    y = torch.bmm(q.float().view(n, most, F), s["W_down"][e].float().transpose(1, 2).contiguous())
    y = (y * scale.view(n, most, 1) * s["w_scale_down"][e][:, None]).view(n * most, -1)
    return {"Y": torch.where(mine[:, None], y[place.clamp(max=n * most - 1)], 0.0).to(torch.bfloat16)}


# --------------------------------------------------------------------------------------------------- the calls
def run(s):
    op = s["op"]
    if not own:
        if op == "norm":
            H, X = _plain_norm(s)
            return {"H": H.to(s["R"].dtype), "X": X.to(s["R"].dtype)}
        return {"norm_grad": _plain_norm_grad, "linear": _plain_linear, "experts": _plain_experts, "shared": _plain_shared}[op](s)
    m = s["m"]
    if op == "norm":
        m.block_norm(s["R"], s["H"], Y=s["Y"], X=s["X"], w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate"],
                     res_scale=s["res_scale"], eps_post=EPS, eps_pre=EPS)
        return {"H": s["H"], "X": s["X"]}
    if op == "norm_grad":
        m.block_norm_grad(s["H"], s["dR"], Y=s["Y"], dH=s["dH"], dX=s["dX"], w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate"],
                          dY=s["dY"], dgate=s["dgate"], dw_post=s["dw_post"], dw_pre=s["dw_pre"], res_scale=s["res_scale"],
                          eps_post=EPS, eps_pre=EPS)
        grads = {n: s[n] for n in ("dR", "dw_pre", "dgate", "dY", "dw_post")}
        return {n: t for n, t in grads.items() if t is not None}
    if op == "linear":
        out = {}
        if s["norm"]:
            m.block_norm(s["R"], s["H"], Y=s["Y"], Xq=s["Xq"], x_scale=s["x_scale"], w_post=s["w_post"], w_pre=s["w_pre"],
                         gate=s["gate"], res_scale=s["res_scale"], eps_post=EPS, eps_pre=EPS)
            out["H"] = s["H"]
        else:
            m.quantize_rows(s["X"], s["Xq"], s["x_scale"])
        m.linear_i8(s["Xq"], s["x_scale"], s["W"], s["w_scale"], s["out"])
        return {**out, "Y": s["out"]}
    m.quantize_rows(s["X"], s["Xq"], s["x_scale"])
    if op == "shared":
        m.shared_ffn_i8(s["Xq"], s["x_scale"], s["X"].shape[0], s["W_gu"], s["w_scale_gu"], s["W_down"], s["w_scale_down"], s["out"])
        return {"Y": s["out"]}
    m.dispatch_rows_i8(s["Xq"], s["x_scale"], s["slot_of_pair"], s["Xq_perm"], s["x_scale_perm"])
    m.expert_ffn_i8(s["rank"], s["Xq_perm"], s["x_scale_perm"], s["expert_offsets"], s["of_phys"], s["W_gu"], s["w_scale_gu"],
                    s["W_down"], s["w_scale_down"], s["out"])
    return {"Y": s["out"]}


def work(case):
    op, T = case["op"], case["T"]
    b = 4 if case.get("dtype") == "fp32" else 2
    if op in ("norm", "norm_grad"):
        d = case["d"]
        g = {"channel": 1, "token": T, "none": 0}[case["gate"]]
        if op == "norm":
            return {"bytes": (4 * T + g + 2) * d * b, "flops": 12 * T * d}
        return {"bytes": (6 * T + 2 * g + 4) * d * b, "flops": 30 * T * d}
    if op == "linear":
        d_in, d_out = case["d_in"], case["d_out"]
        rows = (3 * T + {"channel": 1, "token": T, "none": 0}[case["gate"]] + 2) * d_in * 2 if case["norm"] else T * d_in * 2
        return {"bytes": rows + d_in * d_out + 4 * d_out + 2 * T * d_out, "flops": 2 * T * d_in * d_out}
    d, F = case["d"], case["F"]
    if op == "shared":
        return {"bytes": 4 * T * d + 3 * F * d + 4 * (2 * F + d), "flops": 6 * T * F * d}
    rows, n = case["rows"], case["E"] // case["D"] if case["rank"] >= 0 else case["E"]
    used = n * (1.0 - (1.0 - 1.0 / n) ** rows)  # experts that get a row
    return {"bytes": 2 * T * d + 2 * rows * d + 4 * T * case["k"] + used * (3 * F * d + 4 * (2 * F + d)), "flops": 6 * rows * F * d}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _rows8(x):
    """rows in 8 bits as what they stand for"""
    step = x.abs().max(1, keepdim=True).values / 127
    return torch.where(step > 0, (x / step).round() * step, x)


def _channels8(q, scale):
    return q.double() * scale.double()[:, None]


def _hidden8(x, W_gu, F):
    gu = _rows8(x) @ W_gu.t()
    h = gu[:, :F] * torch.sigmoid(gu[:, :F]) * gu[:, F:]
    return _rows8(h.to(torch.bfloat16).double())


def _rms(x):
    return (x.pow(2).sum(1, keepdim=True) / x.shape[1] + EPS).pow(-0.5)


def exact(case, seed):
    op, s = case["op"], prepare(case, seed)
    if op in ("norm", "norm_grad") or s.get("norm"):
        Y, w_post, w_pre = (s[n].double() for n in ("Y", "w_post", "w_pre"))
        gate = torch.ones_like(w_post) if s["gate"] is None else s["gate"].double()
    if op == "norm" or s.get("norm"):
        H = s["res_scale"] * s["R"].double() + gate * w_post * Y * _rms(Y)
        X = H * _rms(H) * w_pre
        if op == "norm":
            return {"H": H, "X": X}
        return {"H": H, "Y": _rows8(X) @ _channels8(s["W"], s["w_scale"]).t()}
    if op == "norm_grad":
        H, d = s["H"].double(), case["d"]
        rh, ry = _rms(H), _rms(Y)
        a = s["dX"].double() * w_pre
        dH = s["dH"].double() + rh * a - rh.pow(3) / d * (a * H).sum(1, keepdim=True) * H
        b = dH * gate * w_post
        out = {"dR": s["res_scale"] * dH, "dw_pre": (s["dX"].double() * H * rh).sum(0)}
        if s["gate"] is not None:
            dgate = dH * Y * ry * w_post
            out["dgate"] = dgate if s["gate"].dim() == 2 else dgate.sum(0)
        out["dY"] = ry * b - ry.pow(3) / d * (b * Y).sum(1, keepdim=True) * Y
        out["dw_post"] = (dH * gate * Y * ry).sum(0)
        return out
    if op == "linear":
        return {"Y": _rows8(s["X"].double()) @ _channels8(s["W"], s["w_scale"]).t()}
    F = case["F"]
    if op == "shared":
        h = _hidden8(s["X"].double(), _channels8(s["W_gu"][0], s["w_scale_gu"][0]), F)
        return {"Y": h @ _channels8(s["W_down"][0], s["w_scale_down"][0]).t()}
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    off, pair = s["expert_offsets"].tolist(), torch.argsort(s["slot_of_pair"])
    for q in range(s["lo"], s["lo"] + s["n"]):
        at, e = slice(off[q], off[q + 1]), int(s["of_phys"][q])
        if off[q + 1] == off[q]:
            continue
        h = _hidden8(s["X"][pair[at] // case["k"]].double(), _channels8(s["W_gu"][e], s["w_scale_gu"][e]), F)
        out[at] = h @ _channels8(s["W_down"][e], s["w_scale_down"][e]).t()
    return {"Y": out}
