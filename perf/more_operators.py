"""Products in 8-bit integers and the norms around a block, as measurable cases.

Operators of the C ABI: rows and weights in 8-bit integers with a scale for each row
(``reflex_quantize_int8``, ``reflex_quantize_int8_weight``), the product of two such matrices
(``reflex_matmul_int8``), the SwiGLU experts on them (``reflex_grouped_swiglu_int8``), and what stands
between a block's output and the next block's input (``reflex_block_norm``): the norm after the block, its
gate, the scaled residual stream, the norm before the next block and that one's 8-bit rows; the block's output
comes as rows or as the experts' rows with their weights.

Shapes are the repository's own layers (hidden size 2048, 64 experts of width 1024 or 256 of width 512,
sequences of 1024, 32 tokens a block) and generic vocabularies.
"""
from __future__ import annotations

import math

import torch

own = False

KINDS = ("quantize", "product", "experts", "norm", "join")
EPS = 2.0 ** -20


def listed():
    return [
        # the open positions of one active block, picked out of a sequence's hidden states
        dict(name="quantize_rows_t1024", kind="quantize", what="rows", T=1024, M=32, K=2048, pick=True),
        # the layer input of sixteen sequences
        dict(name="quantize_t16384", kind="quantize", what="rows", T=16384, M=16384, K=2048, pick=False),
        # the head over the open positions of two blocks: bound by its weights
        dict(name="head_m64_n131072", kind="product", M=64, N=131072, K=2048, out="float32"),
        # the head over all positions of a sequence, an odd vocabulary
        dict(name="head_m1024_n50257", kind="product", M=1024, N=50257, K=2048, out="bfloat16"),
        # a projection of eight sequences
        dict(name="project_m8192_n8192", kind="product", M=8192, N=8192, K=2048, out="bfloat16"),
        # the experts of a block's last open positions
        dict(name="experts_t4_e64", kind="experts", T=4, d=2048, E=64, f=1024, k=8, skew=0.0),
        # one sequence, 256 experts: bound by their weights
        dict(name="experts_t1024_e256", kind="experts", T=1024, d=2048, E=256, f=512, k=12, skew=0.0),
        # eight sequences, unevenly loaded experts
        dict(name="experts_t8192_e64", kind="experts", T=8192, d=2048, E=64, f=1024, k=12, skew=0.5),
        # one active block: the stream in 32 bits, a norm, 8-bit rows; a launch's latency
        dict(name="norm_t32", kind="norm", T=32, d=2048, stream="float32", gate="none", post=False, q=True),
        # sixteen sequences: norm after, a gate for each sequence, norm before, 8-bit rows
        dict(name="norm_t16384", kind="norm", T=16384, d=2048, stream="bfloat16", gate="sequence", post=True, q=True),
        # one sequence: its experts' rows to the stream and the next block's input
        dict(name="join_t1024", kind="join", T=1024, d=2048, k=12, shared=False, stream="bfloat16", gate="none",
             post=False),
        # eight sequences with a shared expert, a gate a channel and the norm after
        dict(name="join_t8192", kind="join", T=8192, d=2048, k=12, shared=True, stream="bfloat16", gate="one", post=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))))


def draw(rng):
    kind = rng.choice(KINDS)
    if kind == "quantize":
        K = 128 * _log(rng, 1, 32)
        if rng.random() < 0.4:
            return dict(kind=kind, what="weight", E=_log(rng, 1, 8), N=_log(rng, 1, 4096), K=K)
        T = _log(rng, 1, 8192)
        pick = rng.random() < 0.5
        return dict(kind=kind, what="rows", T=T, M=_log(rng, 1, T) if pick else T, K=K, pick=pick)
    if kind == "product":
        M, K = _log(rng, 1, 8192), 128 * _log(rng, 1, 32)
        N = _log(rng, 1, 131072)
        while M * N * K > 8192 * 8192 * 2048 or M * N > 1 << 27:
            N = (N + 1) // 2
        return dict(kind=kind, M=M, N=N, K=K, out=rng.choice(["float32", "bfloat16"]))
    if kind == "experts":
        E, f = rng.choice([(8, 512), (64, 1024), (256, 512), (33, 640)])
        return dict(kind=kind, T=_log(rng, 1, 4096), d=rng.choice([256, 1152, 2048]), E=E, f=f,
                    k=rng.choice([1, 4, 8]), skew=rng.choice([0.0, 0.0, 0.5, 1.2]))
    T, d = _log(rng, 1, 8192), 128 * _log(rng, 1, 32)
    more = dict(stream=rng.choice(["bfloat16", "float32"]), gate=rng.choice(["none", "one", "sequence", "token"]),
                post=rng.random() < 0.5)
    if kind == "norm":
        return dict(kind=kind, T=T, d=d, q=rng.random() < 0.5, **more)
    return dict(kind=kind, T=T, d=min(d, 2048), k=rng.choice([1, 4, 8, 12]), shared=rng.random() < 0.5, **more)


# ---- 8-bit integers --------------------------------------------------------------------------
def _quantize(x):
    """x [.., K] -> codes int8, scales float32 [..]; a row that is not finite: codes 0, scale NaN."""
    v = x.float()
    amax = v.abs().amax(-1).clamp_min(2.0 ** -100)
    fine = torch.isfinite(v).all(-1)
    most = torch.full_like(amax, 127.0)      # (a quotient of two tensors is rounded once)
    q = torch.round(v * (most / amax)[..., None])
    return torch.where(fine[..., None], q, 0.0).to(torch.int8), torch.where(fine, amax / most, torch.nan)


# ---- inputs ----------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = dict(device="cuda")

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, dtype=dtype, **dev) * std

    def hidden(T, d):
        """Hidden states: a spread of row norms, a few large channels."""
        x = normal(T, d) * torch.exp(0.5 * normal(T, 1))
        x *= torch.where(torch.rand(1, d, generator=g, **dev) < 0.01, 10.0, 1.0).bfloat16()
        return x

    def weights(E, N, K):
        q = torch.empty(E, N, K, dtype=torch.int8, **dev)
        s = torch.empty(E, N, dtype=torch.float32, **dev)
        for i in range(E):
            q[i], s[i] = _quantize(normal(N, K, std=0.02))
        return q, s

    def counts(T, kmax):
        return torch.randint(1, kmax + 1, (T, 1), generator=g, **dev)

    c, s = case, {"case": case}
    if c["kind"] == "quantize" and c["what"] == "weight":
        s["x"] = normal(c["E"], c["N"], c["K"], std=0.02)
        s["q"] = torch.zeros(c["E"], c["N"], c["K"], dtype=torch.int8, **dev)
        s["s"] = torch.zeros(c["E"], c["N"], dtype=torch.float32, **dev)
    elif c["kind"] == "quantize":
        s["x"] = hidden(c["T"], c["K"])
        s["rows"] = s["n"] = None
        if c["pick"]:      # three quarters of the room in use
            s["rows"] = torch.randperm(c["T"], generator=g, **dev)[:c["M"]].sort().values.int()
            s["n"] = torch.tensor([(3 * c["M"] + 3) // 4], dtype=torch.int32, **dev)
        s["q"] = torch.zeros(c["M"], c["K"], dtype=torch.int8, **dev)
        s["s"] = torch.zeros(c["M"], dtype=torch.float32, **dev)
    elif c["kind"] == "product":
        s["x"], s["xs"] = _quantize(hidden(c["M"], c["K"]))
        w, ws = weights(1, c["N"], c["K"])
        s["w"], s["ws"] = w[0], ws[0]
        s["y"] = torch.zeros(c["M"], c["N"], dtype=getattr(torch, c["out"]), **dev)
    elif c["kind"] == "experts":
        T, d, E, f = c["T"], c["d"], c["E"], c["f"]
        kmax = min(c["k"], E)
        s["h"], s["hs"] = _quantize(normal(T, d))
        for name, n, k in (("gate", f, d), ("up", f, d), ("down", d, f)):
            s["w_" + name], s["s_" + name] = weights(E, n, k)
        # every token's own number of experts, some experts more often than others
        score = torch.randn(T, E, generator=g, **dev) - c["skew"] * torch.log(torch.arange(1, E + 1, **dev))
        on = score.argsort(1, descending=True).argsort(1) < counts(T, kmax)
        pairs = on.t().nonzero()                      # (expert, token), in that order
        s["P"] = pairs.shape[0]
        s["most"] = int(on.sum(0).max())
        s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, **dev)
        s["offsets"][1:] = on.sum(0).cumsum(0)
        s["token"] = torch.zeros(T * kmax, dtype=torch.int32, **dev)
        s["token"][:s["P"]] = pairs[:, 1]
        s["y"] = torch.zeros(T * kmax, d, dtype=torch.bfloat16, **dev)
    else:
        T, d = c["T"], c["d"]
        kind = getattr(torch, c["stream"])
        s["x"] = hidden(T, d).to(kind)
        s["gate"] = s["seq"] = None
        if c["gate"] == "sequence":      # ragged sequences, one of them empty
            B = (T + 1023) // 1024 + 1
            cuts = torch.randint(0, T + 1, (B - 1,), generator=g, **dev).sort().values
            s["seq"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), T)]).int()
            s["gate"] = normal(B, d, std=0.5)
        elif c["gate"] != "none":
            s["gate"] = normal(T if c["gate"] == "token" else 1, d, std=0.5)
        s["scale"] = 1.0 if c["gate"] == "none" else 0.875
        s["w_pre"] = 1.0 + normal(d, std=0.2, dtype=torch.float32)
        s["w_post"] = 1.0 + normal(d, std=0.2, dtype=torch.float32) if c["post"] else None
        s["x_out"] = torch.zeros(T, d, dtype=kind, **dev)
        s["n_out"] = torch.zeros(T, d, dtype=torch.bfloat16, **dev)
        if c["kind"] == "norm":
            s["y"] = normal(T, d, std=0.3)
            if c["q"]:
                s["q"] = torch.zeros(T, d, dtype=torch.int8, **dev)
                s["s"] = torch.zeros(T, dtype=torch.float32, **dev)
        else:
            n = counts(T, c["k"])[:, 0]
            s["offsets"] = torch.cat([n.new_zeros(1), n.cumsum(0)]).int()
            P, cap = int(s["offsets"][-1]), T * c["k"]
            s["y"] = normal(cap, d, std=0.3)
            s["at"] = torch.zeros(cap, dtype=torch.int32, **dev)
            s["at"][:P] = torch.randperm(P, generator=g, **dev)
            # a token's weights sum to one
            owner = torch.repeat_interleave(torch.arange(T, **dev), n)
            w = 0.05 + torch.rand(P, generator=g, **dev)
            s["alpha"] = torch.zeros(cap, dtype=torch.float32, **dev)
            s["alpha"][:P] = w / torch.zeros(T, **dev).index_add_(0, owner, w)[owner]
            s["shared"] = normal(T, d, std=0.3) if c["shared"] else None
    return s


# ---- one pass --------------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    from paper_2608_01784_amd import _lib as lib
    c = s["case"]
    if c["kind"] == "quantize":
        if c["what"] == "weight":
            lib.reflex_quantize_int8_weight(s["x"], s["q"], s["s"])
        else:
            lib.reflex_quantize_int8(s["x"], s["q"], s["s"], s["rows"], s["n"])
        return {"q": s["q"], "scale": s["s"]}
    if c["kind"] == "product":
        lib.reflex_matmul_int8(s["x"], s["xs"], s["w"], s["ws"], s["y"])
        return s["y"]
    if c["kind"] == "experts":
        if "work" not in s:
            n = lib.reflex_swiglu_int8_workspace_size(s["y"].shape[0], c["E"], c["f"])
            s["work"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        lib.reflex_grouped_swiglu_int8(s["h"], s["hs"], s["token"], s["offsets"], s["w_gate"], s["w_up"], s["w_down"],
                                       s["s_gate"], s["s_up"], s["s_down"], s["y"], s["work"])
        return s["y"]
    if c["kind"] == "norm":
        lib.reflex_block_norm(x=s["x"], y=s["y"], w_post=s["w_post"], gate=s["gate"], seq_offsets=s["seq"],
                              w_pre=s["w_pre"], x_out=s["x_out"], n_out=s["n_out"], q_out=s.get("q"),
                              q_scale=s.get("s"), eps=EPS, residual_scale=s["scale"])
        out = {"x": s["x_out"], "n": s["n_out"]}
        return {**out, "q": s["q"], "scale": s["s"]} if c["q"] else out
    lib.reflex_block_norm(x=s["x"], y_sorted=s["y"], pair_offsets=s["offsets"], pair_to_sorted=s["at"],
                          pair_weight=s["alpha"], shared_y=s["shared"], w_post=s["w_post"], gate=s["gate"],
                          seq_offsets=s["seq"], w_pre=s["w_pre"], x_out=s["x_out"], n_out=s["n_out"], eps=EPS,
                          residual_scale=s["scale"])
    return {"x": s["x_out"], "n": s["n_out"]}


def _plain(s):
    c = s["case"]
    if c["kind"] == "quantize" and c["what"] == "weight":
        q, e = _quantize(s["x"])
        return {"q": q, "scale": e}
    if c["kind"] == "quantize":
        q, e = _quantize(s["x"] if s["rows"] is None else s["x"][s["rows"]])
        if s["n"] is not None:
            on = torch.arange(c["M"], device="cuda") < s["n"]
            q, e = torch.where(on[:, None], q, 0), torch.where(on, e, 0.0)
        return {"q": q, "scale": e}
    if c["kind"] == "product":
        sums = torch.mm(s["x"].float(), s["w"].float().t())
        return (sums * (s["xs"][:, None] * s["ws"][None, :])).to(s["y"].dtype)
    if c["kind"] == "experts":
        return _experts(s)
    y = s["y"].float() if c["kind"] == "norm" else _joined(s)
    if s["w_post"] is not None:
        y = y * _inverse_rms(y) * s["w_post"]
    if s["gate"] is not None:
        y = _gate_rows(s) * y
    u = (s["scale"] * s["x"].float() + y).to(s["x"].dtype)
    v = u.float()
    n = (v * _inverse_rms(v) * s["w_pre"]).bfloat16()
    if not c.get("q"):
        return {"x": u, "n": n}
    q, e = _quantize(n)
    return {"x": u, "n": n, "q": q, "scale": e}


def _inverse_rms(v):
    """One over the root of the mean square (summed in 64 bits) of each row, in 32 bits."""
    return (1.0 / torch.sqrt(v.double().square().mean(1, keepdim=True) + EPS)).float()


def _gate_rows(s):
    gate = s["gate"].float()
    if s["seq"] is None:
        return gate
    i = torch.arange(s["case"]["T"], device="cuda", dtype=torch.int32)
    return gate[torch.searchsorted(s["seq"][1:-1].contiguous(), i, right=True)]


def _joined(s):
    """Each token's experts' rows by their weights, and the shared expert's."""
    c = s["case"]
    first, last = s["offsets"][:-1, None], s["offsets"][1:, None]
    at = first + torch.arange(c["k"], device="cuda", dtype=torch.int32)
    on = at < last
    at = torch.where(on, at, 0).long()
    y = (s["y"].float()[s["at"].long()[at]] * torch.where(on, s["alpha"][at], 0.0)[:, :, None]).sum(1)
    return y if s["shared"] is None else y + s["shared"].float()


def _experts(s):
    """Each expert's rows, filled up to the longest expert's, in one batched product a projection."""
    off, cap = s["offsets"].long(), s["y"].shape[0]
    most = max(s["most"], 1)
    at = off[:-1, None] + torch.arange(most, device="cuda")          # [E, most]: rows in sorted order
    on = at < off[1:, None]
    at = torch.where(on, at, cap)
    token = torch.cat([s["token"], s["token"][:1]]).long()[at]
    x, xs = s["h"].float()[token], s["hs"][token]

    def times(q, qs, name):
        w = s["w_" + name].float().transpose(1, 2).contiguous()
        return torch.bmm(q, w) * (qs[:, :, None] * s["s_" + name][:, None, :])
    g, u = times(x, xs, "gate"), times(x, xs, "up")
    q, e = _quantize((g / (1.0 + torch.exp(-g)) * u).bfloat16())
    y = times(q.float(), e, "down")
    out = torch.zeros(cap + 1, y.shape[2], dtype=torch.float32, device="cuda")
    out[at.view(-1)] = torch.where(on[:, :, None], y, 0.0).view(-1, y.shape[2])
    return out[:cap].to(torch.bfloat16)


# ---- what a pass cannot do without -----------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "quantize" and c["what"] == "weight":
        n = c["E"] * c["N"]
        return {"bytes": 3 * n * c["K"] + 4 * n, "flops": 3 * n * c["K"]}
    if c["kind"] == "quantize":
        n = (3 * c["M"] + 3) // 4 if c["pick"] else c["M"]
        return {"bytes": 3 * n * c["K"] + 4 * n, "flops": 3 * n * c["K"]}
    if c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": (M + N) * (K + 4) + M * N * (4 if c["out"] == "float32" else 2), "flops": 2 * M * N * K}
    if c["kind"] == "experts":
        pairs = c["T"] * (1 + min(c["k"], c["E"])) / 2
        touched = c["E"] * (1 - (1 - pairs / c["T"] / c["E"]) ** c["T"])
        return {"bytes": touched * (3 * c["d"] * c["f"] + 8 * c["f"] + 4 * c["d"]) + c["T"] * (c["d"] + 4)
                + 2 * pairs * c["d"], "flops": 6 * c["d"] * c["f"] * pairs}
    wide = 4 if c["stream"] == "float32" else 2
    gates = {"none": 0, "one": 1, "sequence": (c["T"] + 1023) // 1024 + 1, "token": c["T"]}[c["gate"]]
    row = 2 * wide + 2                                                # the stream in and out, the next input
    if c["kind"] == "norm":
        row += 2 + (1 if c["q"] else 0)
    else:
        row += (1 + c["k"]) + (2 if c["shared"] else 0)               # (1 + k) / 2 expert rows a token
    return {"bytes": c["d"] * (c["T"] * row + 2 * gates + 8), "flops": c["T"] * c["d"] * 12}


# ---- the definitions in 64 bits --------------------------------------------------------------
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "quantize":      # (codes are whole numbers)
        x = s["x"].double()
        if c["what"] == "rows" and c["pick"]:
            x = x[s["rows"].long()]
        e = x.abs().max(dim=-1).values / 127.0
        if c["what"] == "rows" and c["pick"]:
            e[int(s["n"]):] = 0.0
        return {"q": None, "scale": e}
    if c["kind"] == "product":
        y = torch.empty(c["M"], c["N"], dtype=torch.float64, device="cuda")
        x = s["xs"].double()[:, None] * s["x"].double()
        for n in range(0, c["N"], 16384):
            y[:, n:n + 16384] = x @ (s["ws"][n:n + 16384].double()[:, None] * s["w"][n:n + 16384].double()).t()
        return y
    if c["kind"] == "experts":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        x = s["hs"].double()[:, None] * s["h"].double()
        off = s["offsets"].tolist()
        for i in range(c["E"]):
            lo, hi = off[i], off[i + 1]
            if lo == hi:
                continue
            gate, up, down = (s["s_" + n][i].double()[:, None] * s["w_" + n][i].double() for n in ("gate", "up", "down"))
            xi = x[s["token"][lo:hi].long()]
            g = xi @ gate.t()
            a = (g * torch.sigmoid(g) * (xi @ up.t())).bfloat16().double()
            step = a.abs().max(dim=1, keepdim=True).values.clamp_min(2.0 ** -100) / 127.0
            y[lo:hi] = (torch.round(a / step) * step) @ down.t()
        return y
    T, x, stream = c["T"], s["x"].double(), getattr(torch, c["stream"])
    if c["kind"] == "norm":
        y = s["y"].double()
    else:
        P = int(s["offsets"][-1])
        owner = torch.repeat_interleave(torch.arange(T, device="cuda"), s["offsets"].diff().long())
        y = torch.zeros(T, c["d"], dtype=torch.float64, device="cuda")
        for lo in range(0, P, 16384):
            at = s["at"][lo:min(lo + 16384, P)].long()
            y.index_add_(0, owner[lo:lo + 16384], s["alpha"][lo:lo + len(at)].double()[:, None] * s["y"][at].double())
        if s["shared"] is not None:
            y += s["shared"].double()
    if s["w_post"] is not None:
        y = y / (y.pow(2).mean(1, keepdim=True) + EPS).sqrt() * s["w_post"].double()
    if s["gate"] is not None:
        gate = s["gate"].double()
        y = y * (gate if s["seq"] is None else gate.repeat_interleave(s["seq"].diff().long(), 0))
    u = s["scale"] * x + y
    v = u.to(stream).double()
    out = {"x": u, "n": v / (v.pow(2).mean(1, keepdim=True) + EPS).sqrt() * s["w_pre"].double()}
    return {**out, "q": None, "scale": None} if c.get("q") else out
