"""Operators that serve and train low-rank adapters on a semantic-parallel MoE layer: what is measured of them.

  index          adapter_index: tokens of a batch of requests, ordered by the adapter that their request asks for
  adapters       Y = Y_base + scale B (A x), every token with its request's adapter, beside a shared projection
  adapters_grad  the gradient of that towards x, A and B
  rows_grad      combine_grad and dispatch_grad: the gradient of the row moves of a layer (rows to experts and back, weighted)
  ffn_grad       expert_ffn_grad: the gradient of the grouped SwiGLU FFN towards its rows, experts frozen

Widths, experts and token counts are those of `workloads.CONFIGS` and `perf/cases.py`.  With `own` the calls go through `SemMoE`;
without, the same is computed by elementary torch operations in 32 bits.
"""
import math

import torch

DEV = "cuda:0"
own = False

SHAPES = {
    "tiny": dict(d=512, E=16, k=2, F=1024, D=4, dtype="fp32"),
    "qwen3_30b": dict(d=2048, E=128, k=8, F=768, D=8, dtype="bf16"),
    "qwen3_235b": dict(d=4096, E=128, k=8, F=1536, D=8, dtype="bf16"),
    "gpt_oss_120b": dict(d=2880, E=128, k=4, F=2880, D=16, dtype="bf16"),
    "deepseek_v3": dict(d=7168, E=256, k=8, F=2048, D=32, dtype="bf16"),
}


def listed():
    def lora(name, op, T, n_req, n_ad, r, d_in, d_out, pad=0, dtype="bf16"):
        return dict(name=name, op=op, T=T, n_req=n_req, n_ad=n_ad, r=r, d_in=d_in, d_out=d_out, pad=pad, dtype=dtype)

    def layer(name, op, shape, **kw):
        return dict(name=name, op=op, **SHAPES[shape], **kw)

    return [
        # a decode step of 256 requests (one token each), a quarter of an adapter each: once a step, before the first layer
        lora("index_decode", "index", T=256, n_req=256, n_ad=64, r=16, d_in=4096, d_out=4096),
        # a prefill batch of a few long requests, padded at its end
        lora("index_prefill", "index", T=32768, n_req=96, n_ad=32, r=16, d_in=4096, d_out=4096, pad=768),
        # the smallest call: four requests, a token each, on a narrow projection: latency
        lora("adapters_decode_few", "adapters", T=4, n_req=4, n_ad=4, r=16, d_in=2048, d_out=2048),
        # a decode step with many adapters: every adapter is read for a handful of tokens
        lora("adapters_decode", "adapters", T=256, n_req=256, n_ad=64, r=16, d_in=4096, d_out=4096),
        # a prefill batch of long requests with wide adapters, padded
        lora("adapters_prefill", "adapters", T=16384, n_req=40, n_ad=16, r=64, d_in=7168, d_out=7168, pad=100),
        # a training step's batch: few adapters with many tokens each
        lora("adapters_grad_train", "adapters_grad", T=8192, n_req=64, n_ad=8, r=16, d_in=4096, d_out=4096),
        # a small fp32 model: ragged requests, more features out than in
        lora("adapters_grad_tiny_fp32", "adapters_grad", T=777, n_req=29, n_ad=12, r=24, d_in=512, d_out=1024, dtype="fp32"),
        # rows of a training or prefill batch: back from the experts and to the tokens
        layer("rows_grad_prefill", "rows_grad", "deepseek_v3", T=16384),
        # the same where every launch is short
        layer("rows_grad_tiny_fp32", "rows_grad", "tiny", T=256),
        # experts of the most loaded rank under an affinity placement
        layer("ffn_grad_prefill", "ffn_grad", "qwen3_30b", T=8192, rank=0, rows=20865, skew=0.3),
        # all experts on one GPU, a ragged token count: some sixty rows an expert
        layer("ffn_grad_chunk", "ffn_grad", "qwen3_30b", T=1000, rank=-1, rows=8000, skew=0.5),
        # a small fp32 model
        layer("ffn_grad_tiny_fp32", "ffn_grad", "tiny", T=256, rank=-1, rows=512, skew=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["index", "adapters", "adapters", "adapters_grad", "adapters_grad", "rows_grad", "ffn_grad", "ffn_grad"])
    if op in ("index", "adapters", "adapters_grad"):
        c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp32"]))
        if rng.random() < 0.4:  # decode: a token a request
            c["T"] = c["n_req"] = _log_int(rng, 1, 512)
            c["pad"] = 0
        else:
            c["T"] = _log_int(rng, 2, 32768 if op == "index" else 8192)
            c["n_req"] = _log_int(rng, 1, min(c["T"], 256))
            c["pad"] = rng.choice([0, rng.randrange(64)])
        c["r"] = rng.choice([8, 16, 24, 32, 48, 64, 128])
        most = 1024 if c["T"] > 2048 else 4096
        c["n_ad"] = _log_int(rng, 1, min(128, most // c["r"]))
        c["d_in"], c["d_out"] = 8 * _log_int(rng, 32, 896), 8 * _log_int(rng, 32, 896)
        return c
    if op == "rows_grad":
        c = dict(op=op, **SHAPES[rng.choice(list(SHAPES))])
        c["T"] = _log_int(rng, 1, 12000 if c["d"] > 2048 else 16384)
        return c
    c = dict(op=op, **SHAPES[rng.choice(list(SHAPES))])
    if c["dtype"] == "fp32":
        c["d"], c["F"] = 8 * _log_int(rng, 32, 128), 8 * _log_int(rng, 32, 160)
    elif rng.random() < 0.25:  # a width that is no multiple of the tiles
        c["d"], c["F"] = 8 * rng.randrange(128, 360), 8 * rng.randrange(64, 240)
    m = c["E"] // c["D"]
    c["rank"] = rng.choice([0, c["D"] - 1]) if c["E"] * c["F"] * c["d"] > 3e8 else rng.choice([-1, 0, c["D"] - 1])
    groups = m if c["rank"] >= 0 else c["E"]
    most = min(1200 if c["rank"] >= 0 else 200, int((3e9 if c["dtype"] == "fp32" else 3.2e10) / (groups * c["d"] * c["F"])))
    c["rows"] = groups * _log_int(rng, 2, most) + rng.randrange(groups)
    c["skew"] = rng.choice([0.1, 0.3, 0.6])
    c["T"] = -(-c["rows"] // c["k"]) * (rng.choice([2, c["D"] // 2]) if c["rank"] >= 0 else 1)
    return c


# ------------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _act(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(g, shape, std, dtype):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _requests(case, g):
    """Ragged requests over the batch's first T - pad tokens, each with an adapter (some asked for more often) or, one in
    eight, with none: req_offsets[n_req + 1], adapter_of_req[n_req]."""
    n, n_req, n_ad = case["T"] - case["pad"] if case["T"] > case["pad"] else case["T"], case["n_req"], case["n_ad"]
    n_req = min(n_req, n)
    cut = torch.randperm(max(n - 1, 1), device=DEV, generator=g)[:n_req - 1].sort().values + 1
    off = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), n)]).to(torch.int32)
    p = torch.arange(1, n_ad + 1, device=DEV, dtype=torch.float32).pow(-0.5)
    ad = torch.multinomial(p, n_req, replacement=True, generator=g)
    none = torch.rand(n_req, device=DEV, generator=g) < (0.125 if n_req > 1 else 0.0)
    return off, torch.where(none, -1, ad).to(torch.int32)


def _order(T, off, ad, n_ad):
    """(order[T], adapter_offsets[n_ad + 1]): tokens by adapter, the order of the batch inside one, then those without an
    adapter, then -1 for the rows behind the last request."""
    tok = torch.arange(T, device=DEV, dtype=torch.int32)
    req = torch.searchsorted(off, tok, right=True) - 1
    inside = tok < off[-1]
    a = ad[req.clamp(0, ad.shape[0] - 1)].long()
    key = torch.where(inside, torch.where(a < 0, n_ad, a), n_ad + 1)
    order = torch.argsort(key, stable=True)
    starts = torch.searchsorted(key[order], torch.arange(n_ad + 1, device=DEV))
    return torch.where(inside[order], order, -1).to(torch.int32), starts.to(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    op, act = case["op"], _act(case)
    s = {"op": op}
    if op in ("index", "adapters", "adapters_grad"):
        T, n_ad, r, d_in, d_out = (case[n] for n in ("T", "n_ad", "r", "d_in", "d_out"))
        s["req_offsets"], s["adapter_of_req"] = _requests(case, g)
        s["n_ad"], s["T"] = n_ad, T
        if op == "index":
            s["order"] = torch.empty(T, dtype=torch.int32, device=DEV)
            s["adapter_offsets"] = torch.empty(n_ad + 1, dtype=torch.int32, device=DEV)
        else:  # the order is made once a step and serves every projection of every layer
            s["order"], s["adapter_offsets"] = _order(T, s["req_offsets"], s["adapter_of_req"], n_ad)
            s["X"] = _randn(g, (T, d_in), 1.0, act)
            s["A"] = _randn(g, (n_ad, r, d_in), d_in ** -0.5, act)
            s["B"] = _randn(g, (n_ad, d_out, r), 0.5 * r ** -0.5, act)
            s["scale"] = 0.5 + 1.5 * torch.rand(n_ad, device=DEV, generator=g)
        if op == "adapters":
            s["Y_base"], s["Y"] = _randn(g, (T, d_out), 1.0, act), torch.zeros(T, d_out, dtype=act, device=DEV)
        if op == "adapters_grad":
            s["dY"], s["dX_base"] = _randn(g, (T, d_out), 0.1, act), _randn(g, (T, d_in), 0.1, act)
            s["dX"] = torch.zeros(T, d_in, dtype=act, device=DEV)
            s["dA"], s["dB"] = torch.empty_like(s["A"]), torch.empty_like(s["B"])
        config = dict(T=T, d=d_in, E=1, k=1, F=8, D=1, cap=T, dtype=case["dtype"])
    else:
        T, d, E, k, F, D = (case[n] for n in ("T", "d", "E", "k", "F", "D"))
        P, m = T * k, E // D
        config = dict(T=T, d=d, E=E, k=k, F=F, D=D, cap=-(-T // D), dtype=case["dtype"])
        if op == "rows_grad":
            s["dOut"], s["Y"] = _randn(g, (T, d), 0.1, act), _randn(g, (P, d), 0.2, act)
            s["dX_perm"], s["dX_add"] = _randn(g, (P, d), 0.1, act), _randn(g, (T, d), 0.1, act)
            s["slot_of_pair"] = torch.randperm(P, device=DEV, generator=g).to(torch.int32)
            s["w"] = torch.rand(T, k, device=DEV, generator=g).softmax(1).contiguous()
            s["dY"], s["dw"] = torch.empty(P, d, dtype=act, device=DEV), torch.empty(T, k, device=DEV)
            s["dX"] = torch.empty(T, d, dtype=act, device=DEV)
        else:
            rank, rows = case["rank"], case["rows"]
            lo, n = (rank * m, m) if rank >= 0 else (0, E)
            counts = torch.zeros(E, dtype=torch.int64, device=DEV)
            p = _randn(g, (E,), case["skew"], torch.float32).exp()
            counts[lo:lo + n] = torch.bincount(torch.multinomial(p[lo:lo + n], rows, replacement=True, generator=g), minlength=n)
            if n < E and P > rows:  # the pairs of the other ranks lie before and after this rank's
                p[lo:lo + n] = 0
                counts += torch.bincount(torch.multinomial(p, P - rows, replacement=True, generator=g), minlength=E)
            off = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
            s["expert_offsets"], s["rank"] = off.to(torch.int32), rank
            # a rank's program holds the weights of its own experts
            s["of_phys"] = torch.randperm(n, device=DEV, generator=g).to(torch.int32).repeat(E // n).contiguous()
            s["W_gu"], s["W_down"] = _randn(g, (n, 2 * F, d), 0.02, act), _randn(g, (n, d, F), 0.02, act)
            s["X_perm"], s["dY"] = _randn(g, (P, d), 1.0, act), _randn(g, (P, d), 0.1, act)
            s["dX_perm"] = torch.zeros(P, d, dtype=act, device=DEV)
            s["lo"], s["n"], s["most"] = lo, n, int(counts[lo:lo + n].max())
    if own:
        import paper_2503_04398_amd as S
        s["m"] = S.SemMoE(S.Config(**config), device=DEV)
    return s


# --------------------------------------------------------------------------------------------- the plain forms
def _shared_adapters(s):
    """Adapters side by side, and for every token which of their columns are its own."""
    n_ad, r = s["A"].shape[:2]
    T = s["X"].shape[0]
    place = torch.arange(T, device=DEV)
    a_at = torch.searchsorted(s["adapter_offsets"].long(), place, right=True) - 1
    a_at = torch.where(place < s["adapter_offsets"][-1], a_at, -1)
    order = s["order"].long()
    to = torch.where(order >= 0, order, T)
    a = torch.full((T + 1,), -1, dtype=torch.int64, device=DEV).scatter(0, to, a_at)[:T]
    there = torch.zeros(T + 1, dtype=torch.bool, device=DEV).scatter(0, to, True)[:T, None]
    mine = (a[:, None] == torch.arange(n_ad, device=DEV)).repeat_interleave(r, 1)
    A = s["A"].float().reshape(n_ad * r, -1)
    B = s["B"].float().transpose(1, 2).reshape(n_ad * r, -1)
    return mine, there, A, B, s["scale"].repeat_interleave(r)


def _plain_adapters(s):
    mine, there, A, B, scale = _shared_adapters(s)
    u = torch.where(mine, s["X"].float() @ A.t() * scale, 0.0)
    return {"Y": torch.where(there, s["Y_base"].float() + u @ B, s["Y"].float()).to(s["Y"].dtype)}


def _plain_adapters_grad(s):
    mine, there, A, B, scale = _shared_adapters(s)
    x, g, act = s["X"].float(), s["dY"].float(), s["X"].dtype
    n_ad, r = s["A"].shape[:2]
    u = torch.where(mine, x @ A.t() * scale, 0.0)
    v = torch.where(mine, g @ B.t() * scale, 0.0)
    return {"dX": torch.where(there, s["dX_base"].float() + v @ A, s["dX"].float()).to(act),
            "dA": (v.t() @ x).view(n_ad, r, -1).to(act),
            "dB": (u.t() @ g).view(n_ad, r, -1).transpose(1, 2).to(act).contiguous()}


def _plain_rows_grad(s):
    k, act = s["w"].shape[1], s["dOut"].dtype
    slots = s["slot_of_pair"].long()
    g = s["dOut"].float()
    dY = torch.empty_like(s["Y"])
    dY[slots] = (s["w"][:, :, None] * g[:, None]).to(act).view(dY.shape)
    dw = (g[:, None] * s["Y"][slots].float().view(-1, k, g.shape[1])).sum(2)
    dX = s["dX_perm"][slots].float().view(-1, k, g.shape[1]).sum(1) + s["dX_add"].float()
    return {"dY": dY, "dw": dw, "dX": dX.to(act)}


def _plain_ffn_grad(s):
    """every expert's rows padded to the longest of them, and a batch of products"""
    lo, n, most, F = s["lo"], s["n"], s["most"], s["W_down"].shape[2]
    off = s["expert_offsets"].long()[lo:lo + n + 1]
    row = torch.arange(s["X_perm"].shape[0], device=DEV)
    q = (torch.searchsorted(off, row, right=True) - 1).clamp(0, n - 1)
    mine = (row >= off[0]) & (row < off[-1])
    place = torch.where(mine, q * most + (row - off[q]), n * most)  # the last one: rows of other ranks
    e = s["of_phys"].long()[lo:lo + n]
    w_gu, w_down = s["W_gu"][e].float(), s["W_down"][e].float()

    def padded(x):
        d = x.shape[1]
        return torch.zeros(n * most + 1, d, device=DEV).index_copy(0, place, x.float())[:-1].view(n, most, d)

    gu = torch.bmm(padded(s["X_perm"]), w_gu.transpose(1, 2).contiguous())
    gate, up = gu[:, :, :F], gu[:, :, F:]
    dh = torch.bmm(padded(s["dY"]), w_down)
    sig = 1.0 / (1.0 + torch.exp(-gate))
    dgu = torch.cat([dh * up * sig * (1.0 + gate * (1.0 - sig)), dh * gate * sig], 2)
    dx = torch.bmm(dgu, w_gu).view(n * most, -1)
    return {"dX_perm": torch.where(mine[:, None], dx[place.clamp(max=n * most - 1)], 0.0).to(s["X_perm"].dtype)}


# --------------------------------------------------------------------------------------------------- the calls
def run(s):
    op = s["op"]
    if not own:
        if op == "index":
            order, offsets = _order(s["T"], s["req_offsets"], s["adapter_of_req"], s["n_ad"])
            return {"order": order, "adapter_offsets": offsets}
        return {"adapters": _plain_adapters, "adapters_grad": _plain_adapters_grad, "rows_grad": _plain_rows_grad,
                "ffn_grad": _plain_ffn_grad}[op](s)
    m = s["m"]
    if op == "index":
        m.adapter_index(s["req_offsets"], s["adapter_of_req"], s["n_ad"], s["order"], s["adapter_offsets"])
        return {"order": s["order"], "adapter_offsets": s["adapter_offsets"]}
    if op == "adapters":
        m.adapters(s["X"], s["order"], s["adapter_offsets"], s["A"], s["B"], s["Y"], Y_base=s["Y_base"], scale=s["scale"])
        return {"Y": s["Y"]}
    if op == "adapters_grad":
        m.adapters_grad(s["X"], s["dY"], s["order"], s["adapter_offsets"], s["A"], s["B"], dX=s["dX"], dA=s["dA"], dB=s["dB"],
                        dX_base=s["dX_base"], scale=s["scale"])
        return {"dX": s["dX"], "dA": s["dA"], "dB": s["dB"]}
    if op == "rows_grad":
        m.combine_grad(s["dOut"], s["Y"], s["slot_of_pair"], s["w"], s["dY"], s["dw"])
        m.dispatch_grad(s["dX_perm"], s["slot_of_pair"], s["dX"], dX_add=s["dX_add"])
        return {"dY": s["dY"], "dw": s["dw"], "dX": s["dX"]}
    m.expert_ffn_grad(s["rank"], s["X_perm"], s["dY"], s["expert_offsets"], s["of_phys"], s["W_gu"], s["W_down"], s["dX_perm"])
    return {"dX_perm": s["dX_perm"]}


def work(case):
    b = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("index", "adapters", "adapters_grad"):
        T, n_req, n_ad, r, d_in, d_out = (case[n] for n in ("T", "n_req", "n_ad", "r", "d_in", "d_out"))
        n = max(T - case["pad"], 1)
        used = n_ad * (1.0 - (1.0 - 1.0 / n_ad) ** n_req)  # adapters that some request asks for
        if case["op"] == "index":
            return {"bytes": 4 * (2 * n_req + T + n_ad), "flops": 0}
        plan, panels = 4 * (T + n_ad), used * r * (d_in + d_out) * b
        if case["op"] == "adapters":
            return {"bytes": plan + panels + n * (d_in + 2 * d_out) * b, "flops": 2 * n * r * (d_in + d_out)}
        return {"bytes": plan + panels + n_ad * r * (d_in + d_out) * b + n * (3 * d_in + d_out) * b,
                "flops": 2 * n * r * (3 * d_in + 2 * d_out)}
    T, d, E, k, F, D = (case[n] for n in ("T", "d", "E", "k", "F", "D"))
    P = T * k
    if case["op"] == "rows_grad":
        return {"bytes": (3 * T + 3 * P) * d * b + 16 * P, "flops": 4 * P * d}
    rows, groups = case["rows"], E // D if case["rank"] >= 0 else E
    used = groups * (1.0 - (1.0 - 1.0 / groups) ** rows)  # experts that get a row
    return {"bytes": 3 * rows * d * b + used * 3 * F * d * b, "flops": 10 * rows * d * F}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    op = case["op"]
    if op == "index":
        return None
    s = prepare(case, seed)
    if op in ("adapters", "adapters_grad"):
        off, ads = s["req_offsets"].tolist(), s["adapter_of_req"].tolist()
        X, A, B, scale = (s[n].double() for n in ("X", "A", "B", "scale"))
        if op == "adapters":
            out = {"Y": torch.zeros(s["Y"].shape, dtype=torch.float64, device=DEV)}
            out["Y"][:off[-1]] = s["Y_base"][:off[-1]].double()
        else:
            out = {n: torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in ("dX", "dA", "dB")}
            out["dX"][:off[-1]] = s["dX_base"][:off[-1]].double()
            G = s["dY"].double()
        for q, a in enumerate(ads):
            if a < 0:
                continue
            at = slice(off[q], off[q + 1])
            if op == "adapters":
                out["Y"][at] += (X[at] @ A[a].t()) @ B[a].t() * scale[a]
                continue
            v = G[at] @ B[a] * scale[a]
            out["dX"][at] += v @ A[a]
            out["dA"][a] += v.t() @ X[at]
            out["dB"][a] += G[at].t() @ (X[at] @ A[a].t()) * scale[a]
        return out
    if op == "rows_grad":
        T, k = s["w"].shape
        slots, G = s["slot_of_pair"].view(T, k).long(), s["dOut"].double()
        dX, dw = s["dX_add"].double(), torch.zeros(T, k, dtype=torch.float64, device=DEV)
        dY = torch.zeros(s["Y"].shape, dtype=torch.float64, device=DEV)
        for j in range(k):
            dY[slots[:, j]] = s["w"][:, j, None].double() * G
            dw[:, j] = (s["Y"][slots[:, j]].double() * G).sum(1)
            dX = dX + s["dX_perm"][slots[:, j]].double()
        return {"dY": dY, "dw": dw, "dX": dX}
    out = torch.zeros(s["dX_perm"].shape, dtype=torch.float64, device=DEV)
    off, F = s["expert_offsets"].tolist(), case["F"]
    for q in range(s["lo"], s["lo"] + s["n"]):
        at, e = slice(off[q], off[q + 1]), int(s["of_phys"][q])
        if off[q + 1] == off[q]:
            continue
        w = s["W_gu"][e].double()
        gate, up = s["X_perm"][at].double() @ w[:F].t(), s["X_perm"][at].double() @ w[F:].t()
        dh, sig = s["dY"][at].double() @ s["W_down"][e].double(), torch.sigmoid(gate)
        out[at] = (dh * up * (sig + gate * sig * (1 - sig))) @ w[:F] + (dh * gate * sig) @ w[F:]
    return {"dX_perm": out}
