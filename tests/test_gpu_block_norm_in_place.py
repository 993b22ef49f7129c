"""reflex_block_norm with the new stream in the memory of the block's output, and of both its inputs at once."""
from __future__ import annotations

import pytest

from gpu_common import require_gpu
from test_gpu_block_norm import EPS, case, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


# (every count of waves a row; rows that fill a workgroup and that do not; more rows than the grid holds at once)
@pytest.mark.parametrize("T, d", [(1, 128), (6, 1024), (9, 1152), (5, 2048), (7, 4096), (3, 8192), (3, 16384), (70001, 256),
                                  (9001, 2176)])
@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("used", [None, 3])
def test_stream_into_the_blocks_output(torch, lib, T, d, both, used):
    a, b = case(torch, T, d, gate="one"), case(torch, T, d, gate="one")
    if both:
        a["x"] = a["y"]
        b["x"] = b["y"]
    before = b["y"].clone()
    n_rows = None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    run(lib, a, 0.75, n_rows=n_rows)
    lib.reflex_block_norm(**{k: b[k] for k in ("x", "y", "w_post", "w_pre", "gate")}, x_out=b["y"], n_out=b["n_out"][:T],
                          q_out=b["q_out"][:T], q_scale=b["q_scale"][:T], n_rows=n_rows, eps=EPS, residual_scale=0.75)
    n = T if used is None else min(T, used)
    assert torch.equal(b["y"][:n], a["x_out"][:n]) and torch.equal(b["y"][n:], before[n:])
    assert all(torch.equal(a[k], b[k]) for k in ("n_out", "q_out", "q_scale"))
