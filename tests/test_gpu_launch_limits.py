"""Calls within the documented sizes that are larger than one launch of a thread an item can be."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import require_gpu
from test_gpu_fp8 import bf16, quant_rows

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
