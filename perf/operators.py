"""The 8-bit products of a denoising forward and the step from hidden states to tokens, as measurable cases.

Five operators of the C ABI: the rows of the masked positions (``reflex_select_rows``), rows and
weights in 8 bits with a power-of-two scale for each block of 128 (``reflex_quantize_fp8``,
``reflex_quantize_fp8_weight``), the product of two such matrices (``reflex_matmul_fp8``), the
SwiGLU experts on them (``reflex_grouped_swiglu_fp8``), and tokens with their confidence from
logits and given uniform numbers (``reflex_sample_tokens``).

Layouts: codes are e4m3 [rows, K].  A row's scales are bytes e (2^(e - 127)), block b of row r at
[b // 4, r, b % 4]; a weight's, for 128 x 128 blocks, at [r // 128, b] with the columns padded to
a multiple of four.  Shapes are the repository's own layers (hidden size 2048, 64 experts of width
1024 or 256 of width 512, sequences of 1024, 32 tokens a block) and generic vocabularies.
"""
from __future__ import annotations

import math

import torch

own = False

KINDS = ("select", "quantize", "product", "experts", "sample")


def listed():
    return [
        # masked positions of one sequence: a launch's latency
        dict(name="select_t1024", kind="select", T=1024, open=0.4),
        # the batch of the largest decoding run: 4096 sequences of 1021 positions
        dict(name="select_t4182016", kind="select", T=4182016, open=0.2),
        # the open positions of one active block, picked out of a sequence's hidden states
        dict(name="quantize_rows_t1024", kind="quantize", what="rows", T=1024, M=32, K=2048, pick=True),
        # the layer input of eight sequences
        dict(name="quantize_t8192", kind="quantize", what="rows", T=8192, M=8192, K=2048, pick=False),
        # the head over the open positions of three blocks: bound by its weights
        dict(name="head_m48_n131072", kind="product", M=48, N=131072, K=2048, out="float32"),
        # the head over all positions of a sequence, an odd vocabulary
        dict(name="head_m1024_n100003", kind="product", M=1024, N=100003, K=2048, out="bfloat16"),
        # the experts of a block's last open positions
        dict(name="experts_t8_e64", kind="experts", T=8, d=2048, E=64, f=1024, k=8, skew=0.0),
        # one sequence, 64 experts: bound by their weights
        dict(name="experts_t1024_e64", kind="experts", T=1024, d=2048, E=64, f=1024, k=12, skew=0.0),
        # eight sequences, unevenly loaded experts
        dict(name="experts_t8192_e64", kind="experts", T=8192, d=2048, E=64, f=1024, k=12, skew=0.5),
        # one open position, the most probable token
        dict(name="sample_m1_v32000", kind="sample", M=1, V=32000, dtype="bfloat16", temperature=0.0,
             top_k=0, top_p=1.0, min_p=0.0),
        # one active block with every filter
        dict(name="sample_m32_v131072", kind="sample", M=32, V=131072, dtype="float32", temperature=0.7,
             top_k=50, top_p=0.9, min_p=0.02),
        # all positions of a sequence, an odd vocabulary, nucleus sampling
        dict(name="sample_m1024_v100003", kind="sample", M=1024, V=100003, dtype="bfloat16", temperature=1.0,
             top_k=0, top_p=0.95, min_p=0.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))))


def draw(rng):
    kind = rng.choice(KINDS)
    if kind == "select":
        return dict(kind=kind, T=_log(rng, 1, 4 << 20), open=round(rng.uniform(0.0, 1.0), 3))
    if kind == "quantize":
        K = 128 * _log(rng, 1, 32)
        if rng.random() < 0.4:
            return dict(kind=kind, what="weight", E=_log(rng, 1, 8), N=_log(rng, 1, 4096), K=K)
        T = _log(rng, 1, 8192)
        pick = rng.random() < 0.5
        return dict(kind=kind, what="rows", T=T, M=_log(rng, 1, T) if pick else T, K=K, pick=pick)
    if kind == "product":
        M, K = _log(rng, 1, 1024), 128 * _log(rng, 1, 32)
        N = _log(rng, 1, 100000)
        while M * N * K > 1024 * 100003 * 2048:
            N = (N + 1) // 2
        return dict(kind=kind, M=M, N=N, K=K, out=rng.choice(["float32", "bfloat16"]))
    if kind == "experts":
        E, f = rng.choice([(8, 512), (64, 1024), (256, 512), (33, 640)])
        return dict(kind=kind, T=_log(rng, 1, 4096), d=rng.choice([256, 1152, 2048]), E=E, f=f,
                    k=rng.choice([1, 4, 8]), skew=rng.choice([0.0, 0.0, 0.5, 1.2]))
    filters = [dict(top_k=0, top_p=1.0, min_p=0.0), dict(top_k=rng.randint(1, 200), top_p=1.0, min_p=0.0),
               dict(top_k=0, top_p=round(rng.uniform(0.1, 0.99), 3), min_p=0.0),
               dict(top_k=0, top_p=1.0, min_p=round(rng.uniform(0.001, 0.3), 4)),
               dict(top_k=rng.randint(1, 5000), top_p=round(rng.uniform(0.5, 0.99), 3), min_p=0.01)]
    return dict(kind=kind, M=_log(rng, 1, 512), V=_log(rng, 500, 131072), dtype=rng.choice(["float32", "bfloat16"]),
                temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 1.0, 1.5]), **rng.choice(filters))


# ---- 8-bit rows and weights ------------------------------------------------------------------
def _pow2(e):
    """2^(e - 127) in float32, exactly."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def _scale_of(amax):
    """The byte of the smallest power of two s with amax <= 448 s, from 1 to 254; 127 for zero."""
    m, n = torch.frexp(amax)
    return torch.where(amax > 0, (n - 9 + (m > 0.875).int() + 127).clamp(1, 254), 127)


def _codes(v, e):
    return (v * _pow2(254 - e)).to(torch.float8_e4m3fn)


def _quantize(x):
    """x [M, K] -> codes [M, K], scale bytes [M, K / 128] (int32)."""
    M, K = x.shape
    v = x.float()
    fine = torch.isfinite(v)
    v = torch.where(fine, v, torch.nan).view(M, K // 128, 128)
    e = _scale_of(torch.where(fine, x.float().abs(), 0.0).view(M, K // 128, 128).amax(2))
    return _codes(v, e[:, :, None]).view(M, K), e


def _quantize_weight(w):
    """w [N, K] -> codes [N, K], scale bytes [ceil(N / 128), K / 128] (int32)."""
    N, K = w.shape
    nb = (N + 127) // 128
    p = torch.zeros(nb * 128, K, dtype=torch.float32, device=w.device)
    p[:N] = w
    p = p.view(nb, 128, K // 128, 128)
    e = _scale_of(p.abs().amax((1, 3)))
    return _codes(p, e[:, None, :, None]).view(nb * 128, K)[:N].contiguous(), e


def _pack(e):
    """Row scale bytes [M, B] in the rows' layout [ceil(B / 4), M, 4]."""
    M, B = e.shape
    s = torch.zeros(M, (B + 3) // 4 * 4, dtype=torch.uint8, device=e.device)
    s[:, :B] = e
    return s.view(M, -1, 4).transpose(0, 1).contiguous()


def _pad4(e):
    s = torch.zeros(*e.shape[:-1], (e.shape[-1] + 3) // 4 * 4, dtype=torch.uint8, device=e.device)
    s[..., :e.shape[-1]] = e
    return s


def _rows_value(q, s, dtype=torch.float32):
    """The numbers that rows stand for."""
    M, K = q.shape
    e = s.transpose(0, 1).reshape(M, -1)[:, :K // 128]
    return (q.to(dtype).view(M, K // 128, 128) * _pow2(e).to(dtype)[:, :, None]).view(M, K)


def _weight_value(q, s, dtype=torch.float32):
    """The numbers that weights [.., N, K] stand for."""
    N, K = q.shape[-2:]
    e = _pow2(s[..., :K // 128]).to(dtype).repeat_interleave(128, -2)[..., :N, :]
    return (q.to(dtype).view(*q.shape[:-1], K // 128, 128) * e[..., None]).view(q.shape)


# ---- inputs ----------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = dict(device="cuda")

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, dtype=torch.bfloat16, **dev) * std

    def weights(E, N, K):
        q = torch.empty(E, N, K, dtype=torch.float8_e4m3fn, **dev)
        s = torch.empty(E, (N + 127) // 128, (K // 128 + 3) // 4 * 4, dtype=torch.uint8, **dev)
        for i in range(E):
            qi, e = _quantize_weight(normal(N, K, std=0.02))
            q[i], s[i] = qi, _pad4(e)
        return q, s

    c, s = case, {"case": case}
    if c["kind"] == "select":
        s["masked"] = (torch.rand(c["T"], generator=g, **dev) < c["open"]).to(torch.uint8)
        s["rows"] = torch.zeros(c["T"], dtype=torch.int32, **dev)
        s["n"] = torch.zeros(1, dtype=torch.int32, **dev)
    elif c["kind"] == "quantize" and c["what"] == "weight":
        s["x"] = normal(c["E"], c["N"], c["K"], std=0.02)
        s["q"] = torch.zeros(c["E"], c["N"], c["K"], dtype=torch.float8_e4m3fn, **dev)
        s["s"] = torch.zeros(c["E"], (c["N"] + 127) // 128, (c["K"] // 128 + 3) // 4 * 4, dtype=torch.uint8, **dev)
    elif c["kind"] == "quantize":
        # hidden states: a spread of row norms, a few large channels
        x = normal(c["T"], c["K"]) * torch.exp(torch.randn(c["T"], 1, generator=g, **dev)).bfloat16()
        x *= torch.where(torch.rand(1, c["K"], generator=g, **dev) < 0.01, 20.0, 1.0).bfloat16()
        s["x"] = x
        s["rows"] = s["n"] = None
        if c["pick"]:      # three quarters of the room in use
            s["rows"] = torch.randperm(c["T"], generator=g, **dev)[:c["M"]].sort().values.int()
            s["n"] = torch.tensor([(3 * c["M"] + 3) // 4], dtype=torch.int32, **dev)
        s["q"] = torch.zeros(c["M"], c["K"], dtype=torch.float8_e4m3fn, **dev)
        s["s"] = torch.zeros((c["K"] // 128 + 3) // 4, c["M"], 4, dtype=torch.uint8, **dev)
    elif c["kind"] == "product":
        q, e = _quantize(normal(c["M"], c["K"]))
        s["x"], s["xs"] = q, _pack(e)
        w, ws = weights(1, c["N"], c["K"])
        s["w"], s["ws"] = w[0], ws[0]
        s["y"] = torch.zeros(c["M"], c["N"], dtype=getattr(torch, c["out"]), **dev)
    elif c["kind"] == "experts":
        T, d, E, f = c["T"], c["d"], c["E"], c["f"]
        kmax = min(c["k"], E)
        q, e = _quantize(normal(T, d))
        s["h"], s["hs"] = q, _pack(e)
        for name, n, k in (("gate", f, d), ("up", f, d), ("down", d, f)):
            s["w_" + name], s["s_" + name] = weights(E, n, k)
        # every token's own number of experts, some experts more often than others
        score = torch.randn(T, E, generator=g, **dev) - c["skew"] * torch.log(torch.arange(1, E + 1, **dev))
        count = torch.randint(1, kmax + 1, (T, 1), generator=g, **dev)
        rank = score.argsort(1, descending=True).argsort(1)
        pairs = (rank < count).t().nonzero()                      # (expert, token), in that order
        s["P"] = pairs.shape[0]
        s["most"] = int((rank < count).sum(0).max())
        s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, **dev)
        s["offsets"][1:] = (rank < count).sum(0).cumsum(0)
        s["token"] = torch.zeros(T * kmax, dtype=torch.int32, **dev)
        s["token"][:s["P"]] = pairs[:, 1]
        s["y"] = torch.zeros(T * kmax, d, dtype=torch.bfloat16, **dev)
    else:
        M, V = c["M"], c["V"]
        # from flat rows to sure ones: a few tokens raised, some never allowed
        x = torch.randn(M, V, generator=g, **dev) * 2.0
        top = torch.randint(0, V, (M, 8), generator=g, **dev)
        x.scatter_add_(1, top, 24.0 * torch.rand(M, 1, generator=g, **dev) * torch.rand(M, 8, generator=g, **dev))
        x[:, V - 1 - V // 50:] = -torch.inf
        s["x"] = x.to(getattr(torch, c["dtype"]))
        s["u"] = torch.rand(M, generator=g, **dev)
        s["token"] = torch.zeros(M, dtype=torch.int32, **dev)
        s["conf"] = torch.zeros(M, dtype=torch.float32, **dev)
    return s


# ---- one pass --------------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    from paper_2608_01784_amd import _lib as lib
    c = s["case"]
    if c["kind"] == "select":
        if "work" not in s:
            s["work"] = torch.empty(lib.reflex_select_rows_workspace_size(c["T"]), dtype=torch.uint8, device="cuda")
        lib.reflex_select_rows(s["masked"], s["rows"], s["n"], s["work"])
        return {"rows": s["rows"], "n": s["n"]}
    if c["kind"] == "quantize" and c["what"] == "weight":
        lib.reflex_quantize_fp8_weight(s["x"], s["q"], s["s"])
        return {"q": s["q"], "scale": s["s"]}
    if c["kind"] == "quantize":
        lib.reflex_quantize_fp8(s["x"], s["q"], s["s"], s["rows"], s["n"])
        return {"q": s["q"], "scale": s["s"]}
    if c["kind"] == "product":
        lib.reflex_matmul_fp8(s["x"], s["xs"], s["w"], s["ws"], s["y"])
        return s["y"]
    if c["kind"] == "experts":
        if "work" not in s:
            n = lib.reflex_swiglu_fp8_workspace_size(s["y"].shape[0], c["E"], c["f"])
            s["work"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        lib.reflex_grouped_swiglu_fp8(s["h"], s["hs"], s["token"], s["offsets"], s["w_gate"], s["w_up"], s["w_down"],
                                      s["s_gate"], s["s_up"], s["s_down"], s["y"], s["work"])
        return s["y"]
    if "params" not in s:
        s["params"] = lib.SampleParamsC(c["temperature"], c["top_k"], c["top_p"], c["min_p"])
        n = lib.reflex_sample_workspace_size(c["M"], c["V"])
        s["work"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    lib.reflex_sample_tokens(s["x"], s["u"], s["params"], s["token"], s["conf"], ws=s["work"])
    return {"token": s["token"], "conf": s["conf"]}


def _plain(s):
    c = s["case"]
    if c["kind"] == "select":
        on = s["masked"] != 0
        place = torch.cumsum(on, 0)
        rows = torch.zeros(c["T"] + 1, dtype=torch.int32, device="cuda")
        # closed positions all go to the entry behind the last one
        rows.scatter_(0, torch.where(on, place - 1, c["T"]), torch.arange(c["T"], dtype=torch.int32, device="cuda"))
        return {"rows": rows[:c["T"]], "n": place[-1:].int()}
    if c["kind"] == "quantize" and c["what"] == "weight":
        E, N, K = s["x"].shape
        nb = (N + 127) // 128
        p = torch.zeros(E, nb * 128, K, dtype=torch.bfloat16, device="cuda")
        p[:, :N] = s["x"]
        q, e = _quantize_weight(p.view(E * nb * 128, K))
        return {"q": q.view(E, nb * 128, K)[:, :N].contiguous(), "scale": _pad4(e.view(E, nb, -1))}
    if c["kind"] == "quantize":
        x = s["x"] if s["rows"] is None else s["x"][s["rows"]]
        q, e = _quantize(x)
        scale = _pack(e)
        if s["n"] is not None:
            on = torch.arange(c["M"], device="cuda") < s["n"]
            q = torch.where(on[:, None], q.view(torch.uint8), 0).view(torch.float8_e4m3fn)
            scale = torch.where(on[None, :, None], scale, 0)
        return {"q": q, "scale": scale}
    if c["kind"] == "product":
        y = torch.mm(_rows_value(s["x"], s["xs"]), _weight_value(s["w"], s["ws"]).t())
        return y.to(s["y"].dtype)
    if c["kind"] == "experts":
        return _experts(s, torch.float32)
    return _sample(s)


def _experts(s, dtype):
    """Each expert's rows, filled up to the longest expert's, in one batched product a projection."""
    off, cap = s["offsets"].long(), s["y"].shape[0]
    most = max(s["most"], 1)
    at = off[:-1, None] + torch.arange(most, device="cuda")          # [E, most]: rows in sorted order
    on = at < off[1:, None]
    at = torch.where(on, at, cap)
    token = torch.cat([s["token"], s["token"][:1]]).long()[at]
    x = _rows_value(s["h"], s["hs"], dtype)[token]
    g = torch.bmm(x, _weight_value(s["w_gate"], s["s_gate"], dtype).transpose(1, 2).contiguous())
    u = torch.bmm(x, _weight_value(s["w_up"], s["s_up"], dtype).transpose(1, 2).contiguous())
    a = (g / (1.0 + torch.exp(-g)) * u).float()
    q, e = _quantize(a.view(-1, a.shape[2]))
    a = _rows_value(q, _pack(e), dtype).view(a.shape)
    y = torch.bmm(a, _weight_value(s["w_down"], s["s_down"], dtype).transpose(1, 2).contiguous())
    out = torch.zeros(cap + 1, y.shape[2], dtype=dtype, device="cuda")
    out[at.view(-1)] = torch.where(on[:, :, None], y, 0.0).view(-1, y.shape[2])
    return out[:cap].to(torch.bfloat16)


def _sample(s):
    c = s["case"]
    x = s["x"].double()
    top = x.amax(1, keepdim=True)
    flat = torch.exp(x - top)
    if c["temperature"] > 0:
        # the tokens in order of rank: value descending, the lower index first
        v, order = s["x"].sort(dim=1, descending=True, stable=True)
        w = torch.exp((v.double() - top) / _f32(c["temperature"]))
        if c["top_k"] > 0:
            w[:, c["top_k"]:] = 0.0
        mass = torch.cumsum(w, 1)
        before = torch.cat([torch.zeros_like(mass[:, :1]), mass[:, :-1]], 1)
        keep = w >= _f32(c["min_p"])
        if c["top_p"] < 1.0:
            keep &= before < _f32(c["top_p"]) * mass[:, -1:]
        # the draw goes over the kept tokens by index
        cum = torch.cumsum(torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0)), 1)
        token = torch.searchsorted(cum, s["u"].double()[:, None] * cum[:, -1:], right=True)
    else:
        token = (x == top).int().argmax(1, keepdim=True)
    conf = flat.gather(1, token) / flat.sum(1, keepdim=True)
    return {"token": token[:, 0].int(), "conf": conf[:, 0].float()}


def _f32(v):
    """A parameter as the call holds it, in 32 bits."""
    return float(torch.tensor(v, dtype=torch.float32))


# ---- what a pass cannot do without -----------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "select":
        return {"bytes": c["T"] * (1 + 4 * c["open"]) + 4, "flops": c["T"]}
    if c["kind"] == "quantize" and c["what"] == "weight":
        n = c["E"] * c["N"] * c["K"]
        return {"bytes": 3 * n + n / 16384, "flops": 3 * n}
    if c["kind"] == "quantize":
        n = c["K"] * ((3 * c["M"] + 3) // 4 if c["pick"] else c["M"])
        return {"bytes": 3 * n + n / 128, "flops": 3 * n}
    if c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": (M + N) * K + M * K / 128 + N * K / 16384 + M * N * (4 if c["out"] == "float32" else 2),
                "flops": 2 * M * N * K}
    if c["kind"] == "experts":
        pairs = c["T"] * (1 + min(c["k"], c["E"])) / 2
        touched = c["E"] * (1 - (1 - pairs / c["T"] / c["E"]) ** c["T"])
        return {"bytes": 3 * touched * c["d"] * c["f"] + c["T"] * c["d"] + 2 * pairs * c["d"],
                "flops": 6 * c["d"] * c["f"] * pairs}
    return {"bytes": c["M"] * c["V"] * (4 if c["dtype"] == "float32" else 2) + 12 * c["M"],
            "flops": 4 * c["M"] * c["V"]}


# ---- the definitions in 64 bits --------------------------------------------------------------
def _e4m3(v):
    """float64 to the nearest number with three fraction bits, exponents from -6, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -20))).clamp_min(-6) - 3)
    return torch.round(v / step) * step


def _exact_codes(v, over):
    """float64 v [R, K / 128, 128] in 8 bits, one scale for all values along the dimensions `over`."""
    amax = v.abs().amax(over, keepdim=True)
    e = torch.ceil(torch.log2(amax.clamp_min(2.0 ** -200) / 448.0))
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)       # the logarithm's own rounding
    e = torch.where(amax <= 448.0 * torch.exp2(e - 1), e - 1, e)
    e = torch.where(amax > 0, e.clamp_min(-126), 0.0)
    return _e4m3(v / torch.exp2(e)), e


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "select":
        return None       # whole numbers only
    if c["kind"] == "quantize":
        if c["what"] == "weight":
            q = torch.empty(c["E"], c["N"], c["K"], dtype=torch.float64, device="cuda")
            for i in range(c["E"]):
                for n in range(0, c["N"], 128):
                    v = s["x"][i, n:n + 128].double().view(-1, c["K"] // 128, 128)
                    q[i, n:n + 128] = _exact_codes(v, (0, 2))[0].view(-1, c["K"])
            return {"q": q, "scale": None}
        x = s["x"].double()
        if c["pick"]:
            x = x[s["rows"].long()]
        q = _exact_codes(x.view(c["M"], -1, 128), 2)[0].view(c["M"], -1)
        if c["pick"]:
            q[int(s["n"]):] = 0.0
        return {"q": q, "scale": None}
    if c["kind"] == "product":
        y = torch.empty(c["M"], c["N"], dtype=torch.float64, device="cuda")
        x = _exact_value(s["x"], s["xs"].permute(1, 0, 2).reshape(c["M"], -1))
        for n in range(0, c["N"], 16384):
            w = s["w"][n:n + 16384]
            y[:, n:n + 16384] = x @ _exact_value(w, s["ws"][n // 128:n // 128 + 128].repeat_interleave(128, 0)[:len(w)]).t()
        return y
    if c["kind"] == "experts":
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
        x = _exact_value(s["h"], s["hs"].permute(1, 0, 2).reshape(c["T"], -1))
        off = s["offsets"].tolist()
        for i in range(c["E"]):
            lo, hi = off[i], off[i + 1]
            if lo == hi:
                continue
            gate, up, down = (_exact_value(s["w_" + n][i], s["s_" + n][i].repeat_interleave(128, 0)) for n in ("gate", "up", "down"))
            xi = x[s["token"][lo:hi].long()]
            g = xi @ gate.t()
            q, e = _exact_codes((g * torch.sigmoid(g) * (xi @ up.t())).view(hi - lo, -1, 128), 2)
            y[lo:hi] = (q * torch.exp2(e)).view(hi - lo, -1) @ down.t()
        return y
    # tokens row by row: each kept set from a threshold on the value and a count of ties
    token, conf = [], []
    for i in range(c["M"]):
        x = s["x"][i].double()
        p = torch.softmax(x, 0)
        t = int((x == x.max()).nonzero()[0])
        if c["temperature"] > 0:
            order = torch.argsort(-x, stable=True)
            w = torch.softmax(x / _f32(c["temperature"]), 0)[order]
            n = min(c["top_k"], c["V"]) if c["top_k"] > 0 else c["V"]
            if c["top_p"] < 1.0:
                n = min(n, int((torch.cumsum(w[:n], 0) < _f32(c["top_p"]) * w[:n].sum()).sum()) + 1)
            n = min(n, max(1, int((w >= _f32(c["min_p"]) * w[0]).sum())))
            at = order[:n].sort().values
            cum = torch.cumsum(torch.softmax(x / _f32(c["temperature"]), 0)[at], 0)
            t = int(at[min(n - 1, int((cum <= float(s["u"][i]) * cum[-1]).sum()))])
        token.append(t)
        conf.append(float(p[t]))
    return {"token": torch.tensor(token, dtype=torch.int32), "conf": torch.tensor(conf, dtype=torch.float64)}


def _exact_value(q, e):
    """float64 numbers of codes [R, K] whose block b of row r has the scale byte e[r, b]."""
    R, K = q.shape
    return (q.double().view(R, K // 128, 128) * torch.exp2(e[:, :K // 128].double() - 127.0)[:, :, None]).view(R, K)
