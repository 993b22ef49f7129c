"""Calls within the documented sizes that are larger than one launch of a thread an item can be."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import require_gpu
from test_gpu_fp8 import bf16, quant_rows
from test_gpu_tokens import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


@pytest.mark.parametrize("used", [None, (1 << 24) - 5, 3 << 21])
def test_quantize_the_most_rows(torch, lib, used):
    """2^24 rows of 2048 by a list: 2^32 lanes of work."""
    M, K, P = 1 << 24, 2048, 64
    x = bf16(torch, np.random.default_rng(1).normal(size=(P, K)))
    x[5] = 0.0
    x = x.cuda()
    want_q, want_s = quant_rows(torch, lib, x)
    q = torch.full((M, K), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full(lib.fp8_scale_shape(M, K), 0x55, dtype=torch.uint8, device="cuda")
    rows = (torch.arange(M, device="cuda", dtype=torch.int32) * 7) % P
    n = None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    lib.reflex_quantize_fp8(x, q, s, rows=rows, n_rows=n)
    step = 1 << 20
    for i in range(0, M, step):
        here = min(max((M if used is None else used) - i, 0), step)
        at = rows[i:i + here].long()
        assert torch.equal(q[i:i + here], want_q[at]) and torch.equal(s[:, i:i + here], want_s[:, at]), i
        assert bool((q[i + here:i + step] == 0x55).all()) and bool((s[:, i + here:i + step] == 0x55).all()), i


def draw(torch, lib, x, u, params, T, rows=None, n_rows=None):
    tokens = torch.full((T,), -9, dtype=torch.int32, device="cuda")
    conf = torch.full((T,), -9.0, device="cuda")
    ws = torch.empty(lib.reflex_sample_workspace_size(*x.shape), dtype=torch.uint8, device="cuda")
    lib.reflex_sample_tokens(x, u, lib.SampleParamsC(*params), tokens, conf, rows=rows, n_rows=n_rows, ws=ws)
    return tokens, conf


@pytest.mark.parametrize("params", [(1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (0.7, 3, 0.9, 0.01), (1.0, 0, 0.8, 0.0)])
@pytest.mark.parametrize("M", [(1 << 22) + 7, 1 << 24])
def test_sample_the_most_rows(torch, lib, M, params):
    """Rows that repeat: the results of one period, everywhere."""
    P, V = 60, 5
    rng = np.random.default_rng(2)
    x, u = rng.normal(size=(P, V)).astype(np.float32), rng.random(P, dtype=np.float32)
    dx, du = torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda()
    want = draw(torch, lib, dx, du, params, P)
    check(x.astype(np.float64), u, params, want[0].cpu().numpy(), want[1].cpu().numpy())
    at = torch.arange(M, device="cuda") % P
    got = draw(torch, lib, dx[at], du[at], params, M)
    assert torch.equal(got[0], want[0][at]) and torch.equal(got[1], want[1][at])


@pytest.mark.parametrize("params", [(1.0, 0, 1.0, 0.0), (0.7, 30, 0.9, 0.01), (1.0, 0, 0.95, 0.0)])
@pytest.mark.parametrize("used", [None, 0, 1, 65535, 65536, 65537, 70001, 140000])
def test_sample_listed_rows_of_two_launches(torch, lib, used, params):
    M, V, T = 70001, 1301, 80000
    g = torch.Generator("cuda").manual_seed(3)
    x = 2.0 * torch.randn(M, V, generator=g, device="cuda", dtype=torch.bfloat16)
    u = torch.rand(T, generator=g, device="cuda")
    rows = torch.randperm(T, generator=g, device="cuda")[:M].int()
    n = None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    tokens, conf = draw(torch, lib, x, u, params, T, rows, n)
    n = M if used is None else min(used, M)
    on = rows[:n].long()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[on] = False
    assert bool((tokens[rest] == -9).all()) and bool((conf[rest] == -9.0).all())
    # (each launch alone gives the same bits)
    for lo, hi in ((0, min(n, 65536)), (65536, n)):
        if lo < hi:
            part = draw(torch, lib, x[lo:hi], u[rows[lo:hi].long()], params, hi - lo)
            assert torch.equal(tokens[rows[lo:hi].long()], part[0]) and torch.equal(conf[rows[lo:hi].long()], part[1])
    some = [j for j in (0, 1, 65534, 65535, 65536, 65537, 70000) if j < n]
    at = rows[some].long()
    check(x[some].double().cpu().numpy(), u[at].cpu().numpy(), params, tokens[at].cpu().numpy(), conf[at].cpu().numpy())
