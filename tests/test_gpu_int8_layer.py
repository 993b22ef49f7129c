"""The layer with 8-bit integer experts, its norm, the head, a stack and a decode of them, against the oracle;
calls captured, beside each other and past 32-bit offsets."""
from __future__ import annotations

import numpy as np
import pytest

import oracle
from gpu_common import note, require_gpu
from oracle import int8 as oi
from synth import generation_start, make_workload
from synth.device import state_tensors, to_device, weight_tensors
from test_gpu_fp8_layer import P, same
from test_gpu_int8 import bf16, check_experts, check_product, expert_case, host, int8_case, quant_rows, run_experts, same_rows
from test_gpu_tokens import check as check_tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def random_weights(torch, E, d, f, fs, seed):
    from paper_2608_01784_amd.layer import ExpertWeights, ExpertWeightsInt8
    rng = np.random.default_rng([E, d, f, fs, seed])

    def w(*shape):
        return bf16(torch, rng.normal(size=shape) * 0.05)
    more = {} if fs == 0 else dict(ws_gate=w(fs, d), ws_up=w(fs, d), ws_down=w(d, fs))
    router = torch.from_numpy(rng.normal(size=(E, d)).astype(np.float32) * 0.05).cuda()
    return ExpertWeightsInt8.quantize(ExpertWeights(w(E, f, d), w(E, f, d), w(E, d, f), router, **more))


def value(w, name, e=None):
    pair = getattr(w, name), getattr(w, name.replace("w", "s", 1))
    return [(t if e is None else t[e]).cpu().numpy() for t in pair]


def layer_rows(lay, h, k=None):
    """Float64 sums of the experts' rows from the layer's own scores and counts (k: the caller's), how far the layer's
    may be from them, and the sum of the terms' magnitudes.  Beyond the experts' bounds: their rows are rounded to bf16
    (half a step, 2^-8); the fp32 weights and the sum of at most 65 terms are off by at most 2^-17 of the magnitudes."""
    w = lay.w
    q, s = oi.quantize_rows(host(h))
    route = oracle.topk_route(lay.logits.cpu().numpy(), (lay.k if k is None else k).cpu().numpy(), lay.norm_topk)
    ref, tol, size = np.zeros((lay.T, lay.d)), np.zeros((lay.T, lay.d)), np.zeros((lay.T, lay.d))

    def add(rows, weight, mats):
        y, t = oi.swiglu_rows(q[rows], s[rows], *mats)
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
    return ref, tol + 2.0 ** -17 * size


def inside(got, ref, tol, rounding=2.0 ** -8):
    tol = tol + rounding * (np.abs(ref) + tol)
    err = np.abs(host(got) - ref)
    assert (err <= tol).all(), f"{(err / tol).max():.3g} of the bound"
    return float((err / tol).max())


# T * k <= 5 E with fs = f: the shared expert's rows ride in the routed launches
@pytest.mark.parametrize("T, d, E, f, fs, k", [
    (1, 128, 4, 128, 0, 2), (1, 256, 8, 128, 128, 8), (7, 384, 3, 256, 0, 1), (16, 256, 8, 128, 128, 2),
    (33, 512, 8, 256, 0, 3), (65, 256, 8, 128, 128, 2), (100, 256, 8, 128, 256, 2), (150, 640, 5, 384, 128, 5),
    (300, 256, 2, 256, 256, 1), (40, 128, 64, 128, 128, 8), (520, 256, 4, 128, 0, 4),
    (150, 256, 64, 128, 128, 2),       # (its rows in the tiles of the routed ones)
    (5000, 256, 4, 128, 1280, 1)])     # (a shared expert of whole tiles)
def test_layer(torch, lib, T, d, E, f, fs, k):
    from paper_2608_01784_amd.layer import MoELayerInt8
    rng = np.random.default_rng([T, d, E])
    lay = MoELayerInt8(T, d, random_weights(torch, E, d, f, fs, 1), P(k), uniform_k=k)
    h = bf16(torch, rng.normal(size=(T, d)) * np.exp(rng.normal(size=(T, 1))))
    lay.ws.fill_(255)
    out = lay.forward(h)
    assert (lay.k == k).all() and int(lay.pairs) == T * k
    worst = inside(out, *layer_rows(lay, h))
    # rows that are in 8 bits already, residuals, the caller's counts (0 too), a result elsewhere
    q, s = quant_rows(torch, lib, h)
    again = torch.empty_like(out)
    lay.ws.fill_(255)
    assert torch.equal(lay.forward(h, h_q=q, h_scale=s, out=again), out)
    k_in = torch.from_numpy(rng.integers(0, k + 1, T).astype(np.int32)).cuda()
    a, b = (bf16(torch, rng.normal(size=(T, d))) for _ in range(2))
    to = torch.full_like(out, float("nan"))
    assert lay.forward(h, k_in=k_in, residual_a=a, residual_b=b, out=to) is to
    ref, tol = layer_rows(lay, h, k_in)
    extra = host(a).astype(np.float64) + host(b)
    inside(to, ref + extra, tol + 2.0 ** -22 * (np.abs(host(a)) + np.abs(host(b)) + np.abs(ref)))
    note(f"integer layer T={T} d={d} E={E} f={f} fs={fs}: {worst:.3f} of the bound")


@pytest.mark.parametrize("name", ["tiny_t128_e8", "tiny_roles_t128_e8"])
def test_layer_routes_as_the_bf16_one(torch, name):
    from paper_2608_01784_amd.layer import ExpertWeights, ExpertWeightsInt8, MoELayer, MoELayerInt8, TokenState
    w = make_workload(name)
    st, h = TokenState(**state_tensors(w)), to_device(w.h)
    plain = ExpertWeights(**weight_tensors(w))
    a, b = MoELayer(w.T, w.d, plain, w.params), MoELayerInt8(w.T, w.d, ExpertWeightsInt8.quantize(plain), w.params)
    ya, yb = a.forward(h, st), b.forward(h, st)
    assert torch.equal(a.k, b.k) and torch.equal(a.pairs, b.pairs) and torch.equal(a.logits, b.logits)
    inside(yb, *layer_rows(b, h))
    # A step is the largest of a row over 127, an even error 0.29 steps: with a largest of 3 to 5 root mean
    # squares (rows of 256 to 512 normal numbers; the activation's tail is longer, up to 15) 0.7 to 1.1 percent,
    # 3.4 for the activation.  Rows and weights of gate and up, the activation and down's weights: under 5
    err = np.linalg.norm(host(ya) - host(yb)) / np.linalg.norm(host(ya))
    note(f"{name}: integer experts {err:.4f} from bf16 ones")
    assert err < 0.05


def test_nothing(torch, lib):
    """No rows, no columns, no tokens: accepted, and nothing is written."""
    from paper_2608_01784_amd.layer import BlockNorm, MoELayerInt8

    def new(*shape, dtype=torch.int8):
        return torch.full(shape, 3, dtype=dtype, device="cuda")
    f32, i32, b16 = torch.float32, torch.int32, torch.bfloat16
    lib.reflex_quantize_int8(new(0, 128, dtype=b16), new(0, 128), new(0, dtype=f32))
    lib.reflex_quantize_int8_weight(new(0, 128, dtype=b16), new(0, 128), new(0, dtype=f32))
    lib.reflex_matmul_int8(new(0, 128), new(0, dtype=f32), new(5, 128), new(5, dtype=f32), new(0, 5, dtype=f32))
    lib.reflex_matmul_int8(new(5, 128), new(5, dtype=f32), new(0, 128), new(0, dtype=f32), new(5, 0, dtype=f32))
    lib.reflex_grouped_swiglu_int8(new(0, 128), new(0, dtype=f32), new(0, dtype=i32), new(3, dtype=i32),
                                   *[new(2, 128, 128) for _ in range(3)], *[new(2, 128, dtype=f32) for _ in range(3)],
                                   new(0, 128, dtype=b16), new(lib.reflex_swiglu_int8_workspace_size(0, 2, 128), dtype=torch.uint8))
    norm = BlockNorm(0, 128, new(128, dtype=f32))
    assert norm.forward(new(0, 128, dtype=b16), new(0, 128, dtype=b16)).shape == (0, 128)
    lay = MoELayerInt8(0, 256, random_weights(torch, 4, 256, 128, 0, 2), P(2), uniform_k=2)
    assert lay.forward(new(0, 256, dtype=b16)).shape == (0, 256)
    # no pairs at all: the stream alone goes through the norm
    lay = MoELayerInt8(5, 256, random_weights(torch, 4, 256, 128, 0, 2), P(2), uniform_k=2)
    x, one = bf16(torch, np.random.default_rng(0).normal(size=(5, 256))), torch.ones(256, device="cuda")
    norm = BlockNorm(5, 256, one, one, eps=1e-5)
    keep = x.clone()
    lay.forward(x.clone(), k_in=new(5, dtype=i32).zero_(), join=norm.arrays(x))
    assert torch.equal(x, keep)
    np.testing.assert_array_equal(host(norm.n), oi.next_input(host(x), host(one), 1e-5))


# ---- with the norm in place of the combine -------------------------------------------------------
@pytest.mark.parametrize("T, d, E, f, fs, k", [(1, 256, 8, 128, 0, 2), (16, 256, 8, 128, 128, 2), (100, 256, 8, 128, 256, 3),
                                               (64, 2304, 4, 128, 128, 4)])
def test_join_adds_as_the_combine(torch, T, d, E, f, fs, k):
    """Without a norm after and a gate, the stream is the combine's result with the stream as a residual."""
    from paper_2608_01784_amd.layer import BlockNorm, MoELayerInt8
    rng = np.random.default_rng([T, d])
    lay = MoELayerInt8(T, d, random_weights(torch, E, d, f, fs, 3), P(k), uniform_k=k)
    norm = BlockNorm(T, d, torch.from_numpy(rng.normal(size=d).astype(np.float32)).cuda(), eps=1e-5)
    h, x = (bf16(torch, rng.normal(size=(T, d))) for _ in range(2))
    want = lay.forward(h, residual_a=x).clone()
    lay.ws.fill_(255)
    assert lay.forward(h, join=norm.arrays(x)) is norm.n
    assert torch.equal(x, want)
    n = oi.next_input(host(x), host(norm.w_pre), 1e-5)
    np.testing.assert_array_equal(host(norm.n), n)
    same_rows(norm.q.cpu().numpy(), norm.scale.cpu().numpy(), n)


def stack_case(torch, T=70, L=3, wide=False, seed=0, fs=128):
    """L layers of norm, experts, norm: the stream and each layer's input."""
    from paper_2608_01784_amd.layer import BlockNorm, MoELayerInt8
    rng = np.random.default_rng([T, L, seed])
    d = 256
    lays = [MoELayerInt8(T, d, random_weights(torch, 8, d, 128, fs, 10 * seed + i), P(3), uniform_k=3) for i in range(L)]

    def weight():
        return torch.from_numpy((1 + 0.2 * rng.normal(size=d)).astype(np.float32)).cuda()
    norms = [BlockNorm(T, d, weight(), weight() if i else None, eps=1e-5, residual_scale=0.75) for i in range(L + 1)]
    x = torch.empty(T, d, dtype=torch.float32 if wide else torch.bfloat16, device="cuda")
    gate = torch.empty(3, d, dtype=torch.bfloat16, device="cuda")
    seq = torch.tensor([0, T // 3, T // 3, T], dtype=torch.int32, device="cuda")

    def fill(n):
        g = np.random.default_rng([seed, n, 7])
        x.copy_(torch.from_numpy(g.normal(size=(T, d)).astype(np.float32)))
        gate.copy_(torch.from_numpy(g.normal(size=(3, d)).astype(np.float32)))

    def step(stream=None, after=None):
        norms[0].start(x, stream=stream)
        for i, lay in enumerate(lays):
            before = None if after is None else x.clone()
            lay.forward(norms[i].n, h_q=norms[i].q, h_scale=norms[i].scale, stream=stream,
                        join=norms[i + 1].arrays(x, gate, seq))
            if after is not None:
                after(lay, norms[i], norms[i + 1], before)
    return fill, step, lambda: [t.clone() for t in (x, norms[-1].n, norms[-1].q, norms[-1].scale)], (x, gate, seq)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("T, fs", [(1, 0), (70, 128), (200, 256)])
def test_stack(torch, wide, T, fs):
    fill, step, _, (x, gate, seq) = stack_case(torch, T, wide=wide, fs=fs)
    fill(0)
    at = np.repeat(np.arange(3), np.diff(seq.cpu().numpy()))
    g = host(gate)[at].astype(np.float64)

    def after(lay, prev, norm, before):
        u0 = host(before)
        if lay is not None and prev.w_post is None:      # (the first: from the stream as it was)
            np.testing.assert_array_equal(host(prev.n), oi.next_input(u0, host(prev.w_pre), 1e-5))
        y, ey = layer_rows(lay, prev.n)
        # 1 / root moves with the mean of 2 y ey; some ten fp32 roundings
        ms = (y ** 2).mean(1, keepdims=True) + 1e-5
        er = 1.1 * (np.abs(y) * ey + ey ** 2).mean(1, keepdims=True) / ms
        f = g * host(norm.w_post) / np.sqrt(ms)
        u = 0.75 * u0.astype(np.float64) + f * y
        tol = np.abs(f) * (ey + (np.abs(y) + ey) * er) + 2.0 ** -20 * (np.abs(f * y) + np.abs(u0))
        inside(x, u, tol, 0.0 if wide else 2.0 ** -8)
        n = oi.next_input(host(x), host(norm.w_pre), 1e-5)
        np.testing.assert_array_equal(host(norm.n), n)
        same_rows(norm.q.cpu().numpy(), norm.scale.cpu().numpy(), n)
    step(after=after)


@pytest.mark.parametrize("T, fs", [(8, 128), (70, 0), (70, 128), (300, 256)])
def test_join_over_the_layers_own_input(torch, T, fs):
    """One norm for every layer: the join writes the rows that the layer has read."""
    from paper_2608_01784_amd.layer import BlockNorm, MoELayerInt8
    rng = np.random.default_rng([T, fs])
    lay = MoELayerInt8(T, 256, random_weights(torch, 8, 256, 128, fs, 5), P(3), uniform_k=3)
    w = [torch.from_numpy((1 + 0.2 * rng.normal(size=256)).astype(np.float32)).cuda() for _ in range(2)]
    x = bf16(torch, rng.normal(size=(T, 256)))
    a, b = x.clone(), x.clone()
    one, turns = BlockNorm(T, 256, *w, eps=1e-5), [BlockNorm(T, 256, *w, eps=1e-5) for _ in range(2)]
    one.start(a)
    turns[0].start(b)
    for i in range(4):
        lay.forward(one.n, h_q=one.q, h_scale=one.scale, join=one.arrays(a))
        now, then = turns[i % 2], turns[(i + 1) % 2]
        lay.forward(now.n, h_q=now.q, h_scale=now.scale, join=then.arrays(b))
        assert torch.equal(a, b) and torch.equal(one.n, then.n) and torch.equal(one.q, then.q) and torch.equal(one.scale, then.scale)


@pytest.mark.parametrize("used", [0, 1, 40, 69, 70, 200])
def test_join_of_counted_rows(torch, used):
    """Rows behind the count keep their stream and their input."""
    fill, step, results, (x, gate, seq) = stack_case(torch, L=1)
    from paper_2608_01784_amd.layer import BlockNorm, MoELayerInt8
    T = 70
    lay = MoELayerInt8(T, 256, random_weights(torch, 8, 256, 128, 128, 6), P(3), uniform_k=3)
    fill(0)
    one = torch.ones(256, device="cuda")
    norm, full = (BlockNorm(T, 256, one, one, eps=1e-5) for _ in range(2))
    norm.start(x)
    h, q, s, keep = norm.n.clone(), norm.q.clone(), norm.scale.clone(), x.clone()
    want = x.clone()
    lay.forward(h, h_q=q, h_scale=s, join=full.arrays(want, gate, seq))
    lay.forward(h, h_q=q, h_scale=s, join=norm.arrays(x, gate, seq, torch.tensor([used], dtype=torch.int32, device="cuda")))
    n = min(used, T)
    for got, all_, before in ((x, want, keep), (norm.n, full.n, h), (norm.q, full.q, q), (norm.scale, full.scale, s)):
        assert torch.equal(got[:n], all_[:n]) and torch.equal(got[n:], before[n:])


def test_captured_stack(torch):
    fill, step, results, _ = stack_case(torch)
    want = []
    for n in range(5):
        fill(n)
        step()
        want.append(results())
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


def test_two_stacks_at_once(torch):
    cases = [stack_case(torch, T=300, seed=s, wide=s == 2) for s in (1, 2)]
    want = []
    for fill, step, results, _ in cases:
        fill(0)
        step()
        want.append(results())
        fill(0)
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for (fill, step, results, _), s in zip(cases, streams):
        step(s)
    torch.cuda.synchronize()
    for (fill, step, results, _), w in zip(cases, want):
        assert same(torch, results(), w)


# ---- the head, a decode ----------------------------------------------------------------------------
@pytest.mark.parametrize("T, d, V, dtype", [(1, 128, 7, "float32"), (37, 256, 1003, "float32"), (64, 384, 512, "bfloat16"),
                                            (300, 128, 2001, "bfloat16")])
def test_head(torch, lib, T, d, V, dtype):
    from paper_2608_01784_amd.head import TokenHead
    from paper_2608_01784_amd.layer import quantize_weight_int8
    rng = np.random.default_rng([T, V])
    params = (0.8, 20, 0.9, 0.01)
    head = TokenHead(T, quantize_weight_int8(bf16(torch, rng.normal(size=(V, d)) * 0.2)), *params,
                     logits_dtype=getattr(torch, dtype))
    for share in (1.0, 0.4, 0.0):
        x = bf16(torch, rng.normal(size=(T, d)))
        masked = torch.from_numpy((rng.random(T) < share).astype(np.uint8)).cuda()
        x[~masked.bool()] = float("nan")      # (what is not masked is not read)
        u = torch.from_numpy(rng.random(T, dtype=np.float32)).cuda()
        head.forward(x, masked, u)
        rows = np.nonzero(masked.cpu().numpy())[0]
        assert int(head.n_rows) == len(rows)
        if len(rows):
            logits = host(head.logits[:len(rows)]).astype(np.float64)
            q, s = quant_rows(torch, lib, x[masked.bool()].contiguous())
            check_product(logits, (q, s, head.w, head.w_scale), 0.0 if dtype == "float32" else 2.0 ** -8)
            check_tokens(logits, u.cpu().numpy()[rows], params, head.tokens.cpu().numpy()[rows], head.conf.cpu().numpy()[rows])


@pytest.mark.parametrize("apart", [False, True])
def test_decode(torch, apart):
    from paper_2608_01784_amd.head import TokenHead
    from paper_2608_01784_amd.layer import ExpertWeights, ExpertWeightsInt8, MoELayerInt8, TokenState, quantize_weight_int8
    from paper_2608_01784_amd.trajectory import run_trajectory
    w = make_workload("tiny_t128_e8")
    st = TokenState(**{k: to_device(v) for k, v in generation_start(w).items()})
    lay = MoELayerInt8(w.T, w.d, ExpertWeightsInt8.quantize(ExpertWeights(**weight_tensors(w))), w.params)
    rng = np.random.default_rng(3)
    head = TokenHead(w.T, quantize_weight_int8(bf16(torch, rng.normal(size=(777, w.d)) * 0.5)), 0.9, 50, 0.95, 0.0)
    draw = head.confidence(lay.out, st.masked, lambda t: torch.from_numpy(
        np.random.default_rng([9, t]).random(w.T, dtype=np.float32)).cuda())
    h, first = to_device(w.h), st.masked.cpu().numpy().copy()

    def confidence(t):
        if t % 4 == 0:
            inside(lay.out, *layer_rows(lay, h))
        return draw(t)
    stats = run_trajectory(lay, h, st, confidence, 0.9, min_commit=1, stream=torch.cuda.Stream() if apart else None)
    assert stats.masked_left[-1] == 0 and int(st.masked.sum()) == 0
    tokens = head.tokens.cpu().numpy()
    assert (tokens[first == 0] == -1).all() and (tokens[first != 0] >= 0).all()


# ---- offsets that pass 31 and 32 bits, the most rows --------------------------------------------------
def test_rows_past_32_bits(torch, lib):
    """Quantised rows and a product from 2^31 bytes of codes on."""
    M, K, N = 131072 + 300, 16384, 256
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(0)
    at = np.array([0, 1, 65535, 65536, 131071, 131072, 131073, M - 1])
    some = bf16(torch, rng.normal(size=(len(at), K)))
    pick = torch.from_numpy(at).cuda()
    x[pick] = some
    q, s = quant_rows(torch, lib, x)
    del x
    same_rows(q[pick].cpu().numpy(), s[pick].cpu().numpy(), host(some))
    w, ws = int8_case(torch, 1, N, K)[2:]
    for dtype, eps in ((torch.bfloat16, 2.0 ** -8), (torch.float32, 0.0)):
        y = torch.full((M, N), 5.0, dtype=dtype, device="cuda")
        lib.reflex_matmul_int8(q, s, w, ws, y)
        check_product(host(y[pick]).astype(np.float64), (q[pick], s[pick], w, ws), eps)
        y[pick] = 0
        assert not y.any()


@pytest.mark.parametrize("sizes", [[5, 0, 9], [70, 0, 90]])      # (few rows, and tiles)
def test_gathered_rows_past_32_bits(torch, lib, sizes):
    T, d, f = 131072 + 40, 16384, 128
    rng = np.random.default_rng(1)
    c = expert_case(torch, lib, 1, d, f, sizes)
    c["T"] = T
    at = np.array([0, 77, 131071, 131072, 131073, T - 1])
    q, s = quant_rows(torch, lib, bf16(torch, rng.normal(size=(len(at), d))))
    c["h"] = torch.zeros(T, d, dtype=torch.int8, device="cuda")
    c["hs"] = torch.ones(T, dtype=torch.float32, device="cuda")
    pick = torch.from_numpy(at).cuda()
    c["h"][pick], c["hs"][pick] = q, s
    c["token"] = at[rng.integers(0, len(at), c["cap"])].astype(np.int32)
    y = run_experts(torch, lib, c)
    check_experts(dict(c, h=q, hs=s, token=np.searchsorted(at, c["token"])), y)      # (of the rows that are there)


def test_activations_past_32_bits(torch, lib):
    rows = 131072 + 100
    c = expert_case(torch, lib, 8, 128, 16384, [rows])
    y = run_experts(torch, lib, c)
    keep = np.array([0, 1, 255, 256, 65536, 131071, 131072, rows - 1])
    part = dict(c, offsets=np.array([0, len(keep)], dtype=np.int32), token=c["token"][keep], P=len(keep))
    check_experts(part, y[torch.from_numpy(keep).cuda()])


def test_norm_past_32_bits(torch, lib):
    T, d = 131072 + 50, 16384
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(2)
    pick = torch.from_numpy(np.array([0, 1, 65535, 65536, 131071, 131072, T - 1])).cuda()
    x[pick] = bf16(torch, rng.normal(size=(len(pick), d)))
    w = torch.from_numpy((1 + 0.1 * rng.normal(size=d)).astype(np.float32)).cuda()
    q, s = torch.ones(T, d, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda")
    lib.reflex_block_norm(x=x, y=x, w_pre=w, x_out=x, q_out=q, q_scale=s, eps=1e-6, residual_scale=0.5)
    n = oi.next_input(host(x[pick]), host(w), 1e-6)
    same_rows(q[pick].cpu().numpy(), s[pick].cpu().numpy(), n)
    q[pick] = 0
    assert not q.any()


@pytest.mark.parametrize("used", [None, (1 << 24) - 5, 3 << 21])
def test_the_most_rows(torch, lib, used):
    M, K, p = 1 << 24, 2048, 64
    x = bf16(torch, np.random.default_rng(1).normal(size=(p, K)))
    want_q, want_s = quant_rows(torch, lib, x)
    q = torch.full((M, K), 0x55, dtype=torch.int8, device="cuda")
    s = torch.full((M,), 5.0, device="cuda")
    rows = (torch.arange(M, device="cuda", dtype=torch.int32) * 7) % p
    n = None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    lib.reflex_quantize_int8(x, q, s, rows=rows, n_rows=n)
    step = 1 << 20
    for i in range(0, M, step):
        here = min(max((M if used is None else used) - i, 0), step)
        at = rows[i:i + here].long()
        assert torch.equal(q[i:i + here], want_q[at]) and torch.equal(s[i:i + here], want_s[at]), i
        assert bool((q[i + here:i + step] == 0x55).all()) and bool((s[i + here:i + step] == 5.0).all()), i


@pytest.mark.parametrize("used", [None, (1 << 24) - 3])
def test_the_most_rows_of_a_norm(torch, lib, used):
    T, d, p = 1 << 24, 128, 64
    y = bf16(torch, np.random.default_rng(1).normal(size=(p, d)))
    w = torch.ones(d, device="cuda")
    want = torch.zeros(p, d, dtype=torch.bfloat16, device="cuda")
    lib.reflex_block_norm(x=y, w_pre=w, n_out=want, eps=1e-6)
    x, out = y.repeat(T // p, 1), torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    n = None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    lib.reflex_block_norm(x=x, w_pre=w, n_out=out, eps=1e-6, n_rows=n)
    m = T if used is None else used
    assert (out[m:] == 7.0).all()
    out[m:] = want.repeat(T // p, 1)[m:]
    assert torch.equal(out.view(-1, p, d), want.expand(T // p, p, d))
