"""The layer with 8-bit experts, the head that reads the masked rows, and a decode with both, against
the float64 oracle; calls of them captured, beside each other and past 32-bit offsets."""
from __future__ import annotations

import numpy as np
import pytest

import oracle
from gpu_common import note, require_gpu
from oracle import eight_bit as eb
from oracle import tokens as tk
from synth import generation_start, make_workload
from synth.device import state_tensors, to_device, weight_tensors
from test_gpu_fp8 import bf16, check_experts, check_product, codes, expert_case, f64, product_case, quant_rows, run_experts
from test_gpu_tokens import check as check_tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


class P:
    """Counts of at most k_max."""
    def __init__(self, k_max):
        self.k_base, self.delta_role, self.delta_cur, self.k_min, self.k_max = 2, 1, 1, 1, k_max
        self.q, self.theta, self.w_cf, self.v_ref, self.tau = 0.5, 0.9, 0.5, 0.1, 0.1


def random_weights(torch, E, d, f, fs, seed):
    from paper_2608_01784_amd.layer import ExpertWeights, ExpertWeights8
    rng = np.random.default_rng([E, d, f, fs, seed])

    def w(*shape):
        return bf16(torch, rng.normal(size=shape) * 0.05).cuda()
    more = {} if fs == 0 else dict(ws_gate=w(fs, d), ws_up=w(fs, d), ws_down=w(d, fs))
    router = torch.from_numpy(rng.normal(size=(E, d)).astype(np.float32) * 0.05).cuda()
    return ExpertWeights8.quantize(ExpertWeights(w(E, f, d), w(E, f, d), w(E, d, f), router, **more))


def value(w, name, e=None):
    q, s = getattr(w, name), getattr(w, name.replace("w", "s", 1))
    if e is not None:
        q, s = q[e], s[e]
    return eb.weight_value(codes(q), s.cpu().numpy())


def check_layer(lay, h, out, extra=(), k=None):
    """out against float64 from the layer's own scores and counts (k: the caller's).  Beyond the experts' bounds: their
    rows and the result are rounded to bf16 (half a step, 2^-8); the fp32 weights and the sum of at
    most 65 terms are off by at most 2^-17 of the terms' magnitudes."""
    w = lay.w
    x = eb.quantize_rows(f64(h))[0]
    route = oracle.topk_route(lay.logits.cpu().numpy(), (lay.k if k is None else k).cpu().numpy(), lay.norm_topk)
    ref, tol, size = np.zeros((lay.T, lay.d)), np.zeros((lay.T, lay.d)), np.zeros((lay.T, lay.d))

    def add(rows, weight, mats):
        y, t = eb.swiglu_rows(x[rows], *mats)
        t = t + 2.0 ** -8 * (np.abs(y) + t)
        for i, r in enumerate(rows):
            ref[r] += weight[i] * y[i]
            tol[r] += weight[i] * t[i]
            size[r] += weight[i] * (np.abs(y[i]) + t[i])
    for e in range(w.E):
        on = route.expert == e
        if on.any():
            add(route.token[on], route.weight[on], [value(w, n, e) for n in ("w_gate", "w_up", "w_down")])
    if w.f_shared:
        add(np.arange(lay.T), np.ones(lay.T), [value(w, n) for n in ("ws_gate", "ws_up", "ws_down")])
    for r in extra:
        ref += f64(r)
        size += np.abs(f64(r))
    tol += 2.0 ** -17 * size
    tol += 2.0 ** -8 * (np.abs(ref) + tol)
    err = np.abs(f64(out) - ref)
    assert (err <= tol).all(), f"{(err / tol).max():.3g} of the bound"
    return float((err / tol).max())


# T * k <= 5 E with fs = f: the shared expert's rows ride in the routed launches
@pytest.mark.parametrize("T, d, E, f, fs, k", [
    (1, 128, 4, 128, 0, 2), (1, 256, 8, 128, 128, 8), (7, 384, 3, 256, 0, 1), (16, 256, 8, 128, 128, 2),
    (33, 512, 8, 256, 0, 3), (65, 256, 8, 128, 128, 2), (100, 256, 8, 128, 256, 2), (150, 640, 5, 384, 128, 5),
    (300, 256, 2, 256, 256, 1), (40, 128, 64, 128, 128, 8), (520, 256, 4, 128, 0, 4)])
def test_layer(torch, T, d, E, f, fs, k):
    from paper_2608_01784_amd.layer import MoELayer8
    rng = np.random.default_rng([T, d, E])
    lay = MoELayer8(T, d, random_weights(torch, E, d, f, fs, 1), P(k), uniform_k=k)
    h = bf16(torch, rng.normal(size=(T, d)) * np.exp(rng.normal(size=(T, 1)))).cuda()
    lay.ws.fill_(255)
    out = lay.forward(h)
    assert (lay.k == k).all() and int(lay.pairs) == T * k
    worst = check_layer(lay, h, out)
    # residuals, the caller's counts (0 too), a result elsewhere
    k_in = torch.from_numpy(rng.integers(0, k + 1, T).astype(np.int32)).cuda()
    a, b = (bf16(torch, rng.normal(size=(T, d))).cuda() for _ in range(2))
    to = torch.full_like(out, float("nan"))
    assert lay.forward(h, k_in=k_in, residual_a=a, residual_b=b, out=to) is to
    check_layer(lay, h, to, (a, b), k_in)
    note(f"8-bit layer T={T} d={d} E={E} f={f} fs={fs}: {worst:.3f} of the bound")


@pytest.mark.parametrize("name", ["tiny_t128_e8", "tiny_roles_t128_e8"])
def test_layer_routes_as_the_bf16_one(torch, name):
    from paper_2608_01784_amd.layer import ExpertWeights, ExpertWeights8, MoELayer, MoELayer8, TokenState
    w = make_workload(name)
    st, h = TokenState(**state_tensors(w)), to_device(w.h)
    plain = ExpertWeights(**weight_tensors(w))
    a, b = MoELayer(w.T, w.d, plain, w.params), MoELayer8(w.T, w.d, ExpertWeights8.quantize(plain), w.params)
    ya, yb = a.forward(h, st), b.forward(h, st)
    assert torch.equal(a.k, b.k) and torch.equal(a.pairs, b.pairs) and torch.equal(a.logits, b.logits)
    check_layer(b, h, yb)
    # Rounding to e4m3 is off by 2.6 percent in the mean square (at most 2^-4, evenly).  Rows and weights
    # of gate, up and down, and those of g and u enter the activation together: sqrt(6) of that, 6.3
    err = np.linalg.norm(f64(ya) - f64(yb)) / np.linalg.norm(f64(ya))
    note(f"{name}: 8-bit experts {err:.3f} from bf16 ones")
    assert err < 0.1


def test_layer_without_tokens(torch):
    from paper_2608_01784_amd.layer import MoELayer8
    lay = MoELayer8(0, 256, random_weights(torch, 4, 256, 128, 0, 2), P(2), uniform_k=2)
    assert lay.forward(torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")).shape == (0, 256)


def test_calls_of_nothing(torch, lib):
    """No rows, no columns: accepted, and nothing is written but the count."""
    def new(*shape, dtype=torch.uint8):
        return torch.full(shape, 3, dtype=dtype, device="cuda")
    n, S = new(1, dtype=torch.int32), lib.fp8_scale_shape
    lib.reflex_select_rows(new(0), new(0, dtype=torch.int32), n)
    assert int(n) == 0
    lib.reflex_quantize_fp8(new(0, 128, dtype=torch.bfloat16), new(0, 128), new(*S(0, 128)))
    lib.reflex_quantize_fp8_weight(new(0, 128, dtype=torch.bfloat16), new(0, 128), new(0, 4))
    out = new(0, 5, dtype=torch.float32)
    lib.reflex_matmul_fp8(new(0, 128), new(*S(0, 128)), new(5, 128), new(1, 4), out)
    lib.reflex_matmul_fp8(new(5, 128), new(*S(5, 128)), new(0, 128), new(0, 4), new(5, 0, dtype=torch.float32))
    tokens = new(4, dtype=torch.int32)
    lib.reflex_sample_tokens(out, new(4, dtype=torch.float32), lib.SampleParamsC(1.0, 0, 1.0, 0.0), tokens)
    lib.reflex_grouped_swiglu_fp8(new(0, 128), new(*S(0, 128)), new(0, dtype=torch.int32), new(3, dtype=torch.int32),
                                  *[new(2, 128, 128) for _ in range(3)], *[new(2, 1, 4) for _ in range(3)],
                                  new(0, 128, dtype=torch.bfloat16), new(lib.reflex_swiglu_fp8_workspace_size(0, 2, 128)))
    torch.cuda.synchronize()
    assert (tokens == 3).all()


# ---- the head ----------------------------------------------------------------------------------
def check_head(head, x, masked, u, before, params):
    """A forward's list, logits, tokens and confidences; before: tokens and confidences ahead of it."""
    rows = np.nonzero(masked.cpu().numpy())[0]
    assert int(head.n_rows) == len(rows)
    np.testing.assert_array_equal(head.rows.cpu().numpy()[:len(rows)], rows)
    tokens, conf = head.tokens.cpu().numpy(), head.conf.cpu().numpy()
    rest = np.setdiff1d(np.arange(head.T), rows)
    np.testing.assert_array_equal(tokens[rest], before[0][rest])
    np.testing.assert_array_equal(conf[rest], before[1][rest])
    if len(rows) == 0:
        return
    logits = f64(head.logits[:len(rows)])
    from paper_2608_01784_amd import _lib
    import torch
    q, s = quant_rows(torch, _lib, x[masked.bool()].contiguous())
    check_product(logits, q, s, head.w, head.w_scale, 0.0 if head.logits.dtype == torch.float32 else 2.0 ** -8)
    check_tokens(logits, u.cpu().numpy()[rows], params, tokens[rows], conf[rows])


@pytest.mark.parametrize("T, d, V, dtype", [(1, 128, 7, "float32"), (37, 256, 1003, "float32"), (64, 384, 512, "bfloat16"),
                                            (300, 128, 2001, "bfloat16"), (20000, 128, 40, "float32")])
@pytest.mark.parametrize("params", [(0.0, 0, 1.0, 0.0), (0.8, 20, 0.9, 0.01)])
def test_head(torch, T, d, V, dtype, params):
    from paper_2608_01784_amd.head import TokenHead
    rng = np.random.default_rng([T, V])
    head = TokenHead(T, bf16(torch, rng.normal(size=(V, d)) * 0.2).cuda(), *params, logits_dtype=getattr(torch, dtype))
    for share in (1.0, 0.4, 0.0):
        x = bf16(torch, rng.normal(size=(T, d))).cuda()
        masked = torch.from_numpy((rng.random(T) < share).astype(np.uint8)).cuda()
        x[~masked.bool()] = float("nan")      # (what is not masked is not read)
        u = torch.from_numpy(rng.random(T, dtype=np.float32)).cuda()
        before = head.tokens.cpu().numpy(), head.conf.cpu().numpy()
        head.forward(x, masked, u)
        if T <= 1000:
            check_head(head, x, masked, u, before, params)
        else:
            assert int(head.n_rows) == int(masked.sum())


@pytest.mark.parametrize("apart", [False, True])
def test_decode_with_the_head(torch, apart):
    """Layer, head and state to the last position: each forward against the oracle, each position with
    the token of the forward that committed it."""
    from paper_2608_01784_amd.head import TokenHead
    from paper_2608_01784_amd.layer import ExpertWeights, ExpertWeights8, MoELayer8, TokenState
    from paper_2608_01784_amd.trajectory import run_trajectory
    w = make_workload("tiny_t128_e8")
    st = TokenState(**{k: to_device(v) for k, v in generation_start(w).items()})
    lay = MoELayer8(w.T, w.d, ExpertWeights8.quantize(ExpertWeights(**weight_tensors(w))), w.params)
    rng = np.random.default_rng(3)
    params = (0.9, 50, 0.95, 0.0)
    head = TokenHead(w.T, bf16(torch, rng.normal(size=(777, w.d)) * 0.5).cuda(), *params)
    draw = head.confidence(lay.out, st.masked, lambda t: torch.from_numpy(
        np.random.default_rng([9, t]).random(w.T, dtype=np.float32)).cuda())
    h, first = to_device(w.h), st.masked.cpu().numpy().copy()
    last = {}

    def confidence(t):
        before = head.tokens.cpu().numpy(), head.conf.cpu().numpy()
        masked = st.masked.clone()
        conf = draw(t)
        u = torch.from_numpy(np.random.default_rng([9, t]).random(w.T, dtype=np.float32))
        if t % 4 == 0:
            check_layer(lay, h, lay.out)
            check_head(head, lay.out, masked, u, before, params)
        for i in np.nonzero(masked.cpu().numpy())[0]:
            last[i] = int(head.tokens[i])
        return conf
    stats = run_trajectory(lay, h, st, confidence, 0.9, min_commit=1, stream=torch.cuda.Stream() if apart else None)
    assert stats.masked_left[-1] == 0 and int(st.masked.sum()) == 0
    tokens = head.tokens.cpu().numpy()
    assert set(last) == set(np.nonzero(first)[0]) and all(tokens[i] == v for i, v in last.items())
    assert (tokens[first == 0] == -1).all() and (tokens[first != 0] >= 0).all()
    note(f"decoded {int(first.sum())} positions in {stats.forwards} forwards, {stats.total_pairs} pairs")


# ---- captured, beside each other, on other streams ------------------------------------------------
def step_case(torch, T=70, V=1501, fs=128, seed=0):
    from paper_2608_01784_amd.head import TokenHead
    from paper_2608_01784_amd.layer import MoELayer8
    rng = np.random.default_rng([T, V, seed])
    lay = MoELayer8(T, 256, random_weights(torch, 8, 256, 128, fs, seed), P(3), uniform_k=3)
    head = TokenHead(T, bf16(torch, rng.normal(size=(V, 256)) * 0.3).cuda(), 1.0, 0, 0.9, 0.001)
    h = torch.empty(T, 256, dtype=torch.bfloat16, device="cuda")
    masked, u = torch.empty(T, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")

    def fill(n):
        g = np.random.default_rng([seed, n])
        h.copy_(bf16(torch, g.normal(size=(T, 256))))
        masked.copy_(torch.from_numpy((g.random(T) < [0.7, 0.0, 1.0, 0.2][n % 4]).astype(np.uint8)))
        u.copy_(torch.from_numpy(g.random(T, dtype=np.float32)))

    def step(stream=None):
        lay.forward(h, stream=stream)
        head.forward(lay.out, masked, u, stream=stream)

    def results():
        n = int(head.n_rows)
        return [t.clone() for t in (lay.out, head.tokens, head.conf, head.n_rows, head.rows[:n], head.logits[:n])]
    return fill, step, results, head


def same(torch, a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("fs", [0, 128])
def test_captured_step(torch, fs):
    fill, step, results, head = step_case(torch, fs=fs)
    want = []
    for n in range(5):
        fill(n)
        step()
        want.append(results())
    head.tokens.fill_(-1)
    head.conf.zero_()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    for n in range(5):
        fill(n)
        graph.replay()
        torch.cuda.synchronize()
        assert same(torch, results(), want[n]), n
        other = torch.randn(1000, 100, device="cuda").sum()      # (eager work between the replays)
        assert torch.isfinite(other)


def test_two_at_once(torch):
    cases = [step_case(torch, T=200, V=20011, seed=s) for s in (1, 2)]
    want = []
    for fill, step, results, head in cases:
        fill(0)
        step()
        want.append(results())
        head.tokens.fill_(-1)
        head.conf.zero_()
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for (fill, step, results, head), s in zip(cases, streams):
            step(s)
    torch.cuda.synchronize()
    for (fill, step, results, head), w in zip(cases, want):
        assert same(torch, results(), w)


# ---- offsets that pass 31 and 32 bits ---------------------------------------------------------------
def test_rows_past_32_bits(torch, lib):
    """Quantised rows and a product from 2^31 bytes of codes on."""
    M, K, N = 131072 + 300, 16384, 256
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(0)
    at = np.array([0, 1, 65535, 65536, 131071, 131072, 131073, M - 1])
    some = bf16(torch, rng.normal(size=(len(at), K)))
    x[torch.from_numpy(at).cuda()] = some.cuda()
    q, s = quant_rows(torch, lib, x)
    del x
    vals = eb.quantize_rows(some.double().numpy())[0]
    pick = torch.from_numpy(at).cuda()
    np.testing.assert_array_equal(eb.rows_value(codes(q[pick]), s[:, pick].cpu().numpy()), vals)
    wq, wscale = product_case(torch, lib, 1, N, K)[2:]
    for dtype, eps in ((torch.bfloat16, 2.0 ** -8), (torch.float32, 0.0)):
        y = torch.full((M, N), 5.0, dtype=dtype, device="cuda")
        lib.reflex_matmul_fp8(q, s, wq, wscale, y)
        check_product(f64(y[pick]), q[pick], s[:, pick].contiguous(), wq, wscale, eps)
        y[pick] = 0
        assert not y.any()


def test_experts_past_32_bits(torch, lib):
    """Gathered rows, then activations, from 2^31 bytes on."""
    T, d, f = 131072 + 40, 16384, 128
    rng = np.random.default_rng(1)
    c = expert_case(torch, lib, 1, d, f, [5, 0, 9])
    c["T"] = T
    at = np.array([0, 77, 131071, 131072, 131073, T - 1])
    q, s = quant_rows(torch, lib, bf16(torch, rng.normal(size=(len(at), d))).cuda())
    c["h"] = torch.zeros(T, d, dtype=torch.uint8, device="cuda")
    c["hs"] = torch.full(lib.fp8_scale_shape(T, d), 127, dtype=torch.uint8, device="cuda")
    pick = torch.from_numpy(at).cuda()
    c["h"][pick], c["hs"][:, pick] = q, s
    c["token"] = at[rng.integers(0, len(at), c["cap"])].astype(np.int32)
    y = run_experts(torch, lib, c)
    # (the check reads the rows that are there)
    small = dict(c, h=q, hs=s, token=np.searchsorted(at, c["token"]))
    check_experts(small, y)
    del c["h"], c["hs"]
    rows = 131072 + 100
    c = expert_case(torch, lib, 8, 128, 16384, [rows])
    y = run_experts(torch, lib, c)
    keep = np.array([0, 1, 255, 256, 65536, 131071, 131072, rows - 1])
    part = dict(c, offsets=np.array([0, len(keep)], dtype=np.int32), token=c["token"][keep], P=len(keep))
    check_experts(part, y[torch.from_numpy(keep).cuda()])


def test_logits_past_32_bits(torch, lib):
    M, V = 4100, 1 << 20
    logits = torch.zeros(M, V, dtype=torch.bfloat16, device="cuda")
    best = torch.randint(0, V, (M,), device="cuda", dtype=torch.int32, generator=torch.Generator("cuda").manual_seed(0))
    logits[torch.arange(M, device="cuda"), best.long()] = 40.0
    tokens = torch.full((M,), -9, dtype=torch.int32, device="cuda")
    conf = torch.zeros(M, device="cuda")
    ws = torch.empty(lib.reflex_sample_workspace_size(M, V), dtype=torch.uint8, device="cuda")
    u = torch.full((M,), 0.5, device="cuda")
    for params in ((0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (1.0, 0, 0.9, 0.0)):
        tokens.fill_(-9)
        lib.reflex_sample_tokens(logits, u, lib.SampleParamsC(*params), tokens, conf, ws=ws)
        assert torch.equal(tokens, best), params
        assert float((conf - 1.0).abs().max()) < 1e-6
    # flat rows at the end: a plain draw counts, equal logits have exact borders
    logits[-2:] = 0.0
    lib.reflex_sample_tokens(logits, u, lib.SampleParamsC(1.0, 0, 1.0, 0.0), tokens, conf, ws=ws)
    assert tokens[-2:].tolist() == [V // 2, V // 2]
    lib.reflex_sample_tokens(logits, u, lib.SampleParamsC(1.0, 0, 0.5, 0.0), tokens, conf, ws=ws)
    assert tokens[-2:].tolist() == [V // 4, V // 4] and torch.equal(tokens[:-2], best[:-2])
