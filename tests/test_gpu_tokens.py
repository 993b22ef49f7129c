"""reflex_sample_tokens against the float64 oracle.

The kernel's weights are within 4e-11 of theirs, so shares of a row's weight within 1e-10: a token
is right if the oracle takes it for some u, top_p and min_p within that of the given ones, and
rows whose borders are exact numbers (equal logits) have to be equal.  A confidence is a quotient of
fp32 powers whose arguments (up to 60 from a thread's reference) are rounded to fp32:
(60 ln 2 + 2) 2^-24 = 2.6e-6, and one rounding."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import require_gpu
from oracle import tokens as tk

pytestmark = pytest.mark.gpu

SLACK, CONF = 1e-10, 3e-6


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def f32(v):
    return float(np.float32(v))


def sample(torch, lib, x, u, params, T=None, **kw):
    """tokens, conf as numpy; positions not written hold -9."""
    M, V = x.shape
    T = M if T is None else T
    tokens = torch.full((T,), -9, dtype=torch.int32, device="cuda")
    conf = torch.full((T,), -9.0, dtype=torch.float32, device="cuda")
    size = lib.reflex_sample_workspace_size(M, V)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    lib.reflex_sample_tokens(x, torch.from_numpy(np.asarray(u, dtype=np.float32)).cuda(), lib.SampleParamsC(*params),
                             tokens, conf, ws=ws, **kw)
    return tokens.cpu().numpy(), conf.cpu().numpy()


def check(x, u, params, tokens, conf, slack=SLACK):
    t, k, p, q = params
    t, p, q = f32(t), f32(p), f32(q)
    for j in range(len(x)):
        l = np.asarray(x[j], dtype=np.float64)
        uj = float(np.float32(u[j]))
        token, c, _, _ = tk.sample_row(l, t, k, p, q, uj)
        if tokens[j] != token:
            assert slack and tokens[j] in tk.allowed(l, t, k, p, q, uj, slack), \
                f"row {j}: token {tokens[j]}, not {token} ({params}, u = {uj})"
            m = l.max()
            c = float(np.exp(l[tokens[j]] - m) / np.exp(l - m).sum())
        assert abs(conf[j] - c) <= CONF * c + 1e-45, f"row {j}: confidence {conf[j]}, not {c}"


def rows(rng, M, V, dtype):
    """From flat rows to nearly sure ones, a tail of tokens that are never allowed."""
    import torch
    x = rng.normal(size=(M, V)) * rng.uniform(0.1, 4.0, (M, 1))
    for j in range(M):
        at = rng.integers(0, V, 4)
        x[j, at] += rng.uniform(0, 15, 4)
        if V > 60:
            x[j, V - V // 60:] = -np.inf
    return torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype))


PARAMS = [(1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.7, 0, 1.0, 0.0), (1.0, 1, 1.0, 0.0), (1.0, 5, 1.0, 0.0),
          (1.5, 50, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.7, 0, 0.3, 0.0), (1.0, 0, 1.0, 0.1), (0.8, 40, 0.95, 0.02),
          (1.0, 1000000, 0.999, 0.0001), (0.05, 3, 0.5, 0.0), (30.0, 0, 0.5, 0.9)]


@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 65, 1000, 4097, 16385])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_tokens(torch, lib, V, dtype):
    rng = np.random.default_rng([V, len(dtype)])
    x = rows(rng, 12, V, dtype)
    host = x.double().numpy()
    dev = x.cuda()
    for params in PARAMS:
        u = rng.random(12).astype(np.float32)
        u[:2] = [0.0, 1.0 - 2.0 ** -24]
        check(host, u, params, *sample(torch, lib, dev, u, params))


@pytest.mark.parametrize("V", [100003, 131072, 1 << 20])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_tokens_of_large_vocabularies(torch, lib, V, dtype):
    rng = np.random.default_rng([V, 1])
    x = rows(rng, 3, V, dtype)
    host, dev = x.double().numpy(), x.cuda()
    for params in [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.02), (1.0, 0, 0.95, 0.0), (1.0, 30000, 1.0, 0.0)]:
        u = rng.random(3).astype(np.float32)
        check(host, u, params, *sample(torch, lib, dev, u, params))


@pytest.mark.parametrize("V", [10, 1024, 5000])
@pytest.mark.parametrize("value", [0.0, 3.5, -3.3895313892515355e38, 3.3895313892515355e38])
def test_equal_logits(torch, lib, V, value):
    """Every border is an exact number: the first token past u V, of the first kept ones by index."""
    x = torch.full((4, V), value, dtype=torch.bfloat16)
    u = np.array([0.0, 0.25, 0.5, 0.96875], dtype=np.float32)
    for params, n in (((1.0, 0, 1.0, 0.0), V), ((1.0, 0, 0.5, 0.0), V // 2), ((2.0, 7, 1.0, 0.0), 7),
                      ((1.0, 8, 0.25, 1.0), 2), ((1.0, 0, 1.0, 1.0), V)):
        tokens, conf = sample(torch, lib, x.cuda(), u, params)
        np.testing.assert_array_equal(tokens, np.floor(u * n).astype(int))
        np.testing.assert_allclose(conf, 1.0 / V, rtol=CONF)


def test_rows_at_the_ends_of_the_range(torch, lib):
    inf, nan, low = np.inf, np.nan, -3.4028234663852886e38
    V = 300
    x = np.random.default_rng(7).normal(size=(10, V)).astype(np.float32)
    x[0] = -inf
    x[1] = nan
    x[2] = -inf
    x[2, 123] = -7.0                       # one token
    x[3, 5] = inf
    x[4, [9, 200]] = inf
    x[5, ::2] = nan
    x[6] = low                             # masked by the type's lowest number, all of it
    x[7, 1:] = low
    x[8] = -0.0
    x[8, ::3] = 0.0
    x[9] *= 1e30                           # only the largest has weight
    for params in [(1.0, 0, 1.0, 0.0), (0.5, 4, 1.0, 0.0), (1.0, 0, 0.7, 0.0), (1.0, 3, 0.9, 0.3), (0.0, 0, 1.0, 0.0)]:
        u = np.linspace(0.05, 0.9, 10).astype(np.float32)
        tokens, conf = sample(torch, lib, torch.from_numpy(x).cuda(), u, params)
        assert list(tokens[:2]) == [-1, -1] and list(conf[:2]) == [0.0, 0.0]
        check(x[2:], u[2:], params, tokens[2:], conf[2:])


def test_uniform_numbers_outside_the_range_are_clamped(torch, lib):
    x = torch.zeros(5, 16)
    tokens, _ = sample(torch, lib, x.cuda(), [-1.0, 1.0, 2.0, np.nan, np.inf], (1.0, 0, 1.0, 0.0))
    assert list(tokens) == [0, 15, 15, 0, 15]


@pytest.mark.parametrize("used", [0, 1, 4, 6, 50, -2])
def test_listed_rows(torch, lib, used):
    """Rows of logits to positions by a list and a count on the device; u by position."""
    T, V = 20, 77
    rng = np.random.default_rng(11)
    where = np.array([4, 19, 0, -1, 20, 7], dtype=np.int32)
    x = rows(rng, len(where), V, "float32")
    u = rng.random(T).astype(np.float32)
    params = (0.9, 20, 0.95, 0.0)
    tokens, conf = sample(torch, lib, x.cuda(), u, params, T=T, rows=torch.from_numpy(where).cuda(),
                          n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    n = min(max(used, 0), len(where))
    on = [j for j in range(n) if 0 <= where[j] < T]
    at = where[on]
    rest = np.setdiff1d(np.arange(T), at)
    assert (tokens[rest] == -9).all() and (conf[rest] == -9.0).all()
    check(x.double().numpy()[on], u[at], params, tokens[at], conf[at])


@pytest.mark.parametrize("dtype, width", [("bfloat16", 8), ("float32", 4)])
def test_rows_of_every_alignment(torch, lib, dtype, width):
    """A matrix that starts at any element of a 16-byte group."""
    V = 1001
    rng = np.random.default_rng(13)
    flat = rows(rng, 1, 3 * V + width, dtype)[0]
    flat[torch.isinf(flat)] = 0.0
    for shift in range(width):
        x = flat[shift:shift + 3 * V].clone().view(3, V)
        room = torch.zeros(3 * V + width, dtype=x.dtype, device="cuda")
        dev = room[shift:shift + 3 * V].view(3, V)
        dev.copy_(x)
        u = rng.random(3).astype(np.float32)
        check(x.double().numpy(), u, (1.0, 0, 0.9, 0.0), *sample(torch, lib, dev, u, (1.0, 0, 0.9, 0.0)))


def test_confidence_is_optional(torch, lib):
    x = rows(np.random.default_rng(3), 4, 100, "float32").cuda()
    u = torch.rand(4, device="cuda")
    a, b = (torch.zeros(4, dtype=torch.int32, device="cuda") for _ in range(2))
    p = lib.SampleParamsC(1.0, 0, 1.0, 0.0)
    ws = torch.empty(max(1, lib.reflex_sample_workspace_size(4, 100)), dtype=torch.uint8, device="cuda")
    lib.reflex_sample_tokens(x, u, p, a, ws=ws)
    lib.reflex_sample_tokens(x, u, p, b, torch.empty(4, device="cuda"), ws=ws)
    assert torch.equal(a, b)


@pytest.mark.parametrize("params", [(1.0, 0, 0.9, 0.0), (1.5, 0, 0.5, 0.01), (1.0, 5000, 0.7, 0.0), (1.0, 0, 1.0, 0.05)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_flat_rows_of_every_order(torch, lib, dtype, params):
    """Rows in which the tokens around a border lie together, repeat, or are few: ascending, descending, of
    five values, with one token far above the others, with two levels, and next to the border of a wave's share."""
    V = 40013
    rng = np.random.default_rng(V)
    x = rng.normal(size=(6, V)) * 2.0
    x[0], x[1] = np.sort(x[0]), -np.sort(x[1])
    x[2] = np.round(x[2] / 2.0)
    x[3, 777] = 12.0
    x[4] = np.where(rng.random(V) < 0.3, 1.0, 0.0)
    x[5] = np.where(np.arange(V) % 2501 < 40, 3.0, 0.0) + 1e-3 * x[5]
    dev = torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype)).cuda()
    for k in range(3):
        u = rng.random(6, dtype=np.float32)
        check(dev.double().cpu().numpy(), u, params, *sample(torch, lib, dev, u, params))


@pytest.mark.parametrize("top_k", [33, 60, 113, 129, 197, 400, 1025])
@pytest.mark.parametrize("M, V", [(40, 20011), (300, 5003), (2, 40000)])
def test_top_k_of_many(torch, lib, M, V, top_k):
    """A top-k beyond the numbers of parts of a row, of their groups and of their pairs."""
    rng = np.random.default_rng([M, V, top_k])
    dev = torch.from_numpy((rng.normal(size=(M, V)) * 3.0).astype(np.float32)).cuda()
    for params in ((0.7, top_k, 1.0, 0.0), (1.0, top_k, 0.8, 0.01)):
        u = rng.random(M, dtype=np.float32)
        tokens, conf = sample(torch, lib, dev, u, params)
        some = rng.choice(M, min(M, 12), replace=False)
        check(dev.double().cpu().numpy()[some], u[some], params, tokens[some], conf[some])
