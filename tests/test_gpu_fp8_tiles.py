"""The tile kernels of the 8-bit products in the shapes that large calls run in: several tiles a workgroup,
K loops longer than the copies' lookahead, experts of uneven and no rows.  Which kernel a shape reaches
is read from the names of what it launches, so that a changed rule cannot empty these tests."""
from __future__ import annotations

import re

import numpy as np
import pytest

from gpu_common import note, require_gpu
from test_gpu_fp8 import check_experts, check_product, expert_case, f64, product_case, run_experts

pytestmark = pytest.mark.gpu

UP, DOWN, PLAIN = 0, 1, 2


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def launched(torch, call):
    """(mode, rows of a tile) of the 8-bit products that a call launches; small tiles: ("slim", rows)."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    found = []
    for e in prof.events():
        m = re.search(r"fp8_gemm_kernel<.*?(\d)(?:\)|,).*?Shape8<(\d+),", e.name)
        n = re.search(r"fp8_slim_kernel<(\d+),", e.name)
        if m:
            found.append((int(m[1]), 64 * int(m[2])))
        if n:
            found.append(("slim", 32 * int(n[1])))
    return found


# (256 CUs; a slice of K is 128 columns, and 3 or 4 of them are in flight)
@pytest.mark.parametrize("M, N, K, rows", [
    (64, 70001, 384, 64), (50, 66003, 1152, 64), (128, 70001, 384, 128), (65, 66003, 640, 128),
    (200, 30003, 640, 128),      # (few tiles of 256 rows)
    (300, 40003, 384, 256), (300, 40003, 640, 256), (520, 35009, 1152, 256)])
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_product_of_many_tiles(torch, lib, M, N, K, rows, out):
    x, xs, w, ws = product_case(torch, lib, M, N, K)
    room = torch.full((M * N + 64,), 5.0, dtype=getattr(torch, out), device="cuda")
    y = room[:M * N].view(M, N)
    assert launched(torch, lambda: lib.reflex_matmul_fp8(x, xs, w, ws, y)) == [(PLAIN, rows)]
    worst = check_product(f64(y), x, xs, w, ws, 2.0 ** -8 if out == "bfloat16" else 0.0)
    assert (room[M * N:] == 5.0).all()
    again = torch.empty_like(y)
    lib.reflex_matmul_fp8(x, xs, w, ws, again)
    assert torch.equal(y, again)
    # fewer rows in use: the same kernel, other tiles
    used = M - 37
    y.fill_(5.0)
    lib.reflex_matmul_fp8(x, xs, w, ws, y, n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    assert (y[used:] == 5.0).all()
    check_product(f64(y[:used]), x[:used], xs[:, :used].contiguous(), w, ws, 2.0 ** -8 if out == "bfloat16" else 0.0)
    note(f"product {M} x {N} x {K} {out}: {worst:.3f} of the bound")


def uneven(seed, E, first, most):
    sizes = np.random.default_rng(seed).integers(0, most, E)
    sizes[:len(first)] = first
    return [int(n) for n in sizes]


# extra: room for pairs past the last expert's (the rule goes by the room an expert has)
@pytest.mark.parametrize("T, d, f, sizes, extra, up, down", [
    (300, 640, 512, uneven(1, 130, [0, 1, 31, 64, 65, 130, 0, 0], 70), 0, 64, 64),
    (400, 512, 1024, uneven(2, 70, [0, 128, 129, 1, 300, 0, 64, 65], 180), 0, 128, 128),
    (300, 1664, 1024, uneven(3, 40, [0, 1, 256, 257, 300, 0, 255, 33], 300), 500, 256, 256),
    (400, 512, 512, uneven(4, 70, [400, 0, 0, 1, 257, 32, 129, 64], 330), 100, 256, 256),
])
def test_experts_of_many_tiles(torch, lib, T, d, f, sizes, extra, up, down):
    c = expert_case(torch, lib, T, d, f, sizes, extra)
    assert launched(torch, lambda: run_experts(torch, lib, c)) == [(UP, up), (DOWN, down)]
    y = run_experts(torch, lib, c)
    worst = check_experts(c, y)
    assert torch.equal(y, run_experts(torch, lib, c))
    note(f"experts T={T} d={d} f={f} E={len(sizes)} rows={sum(sizes)}: {worst:.3f} of the bound")


@pytest.mark.parametrize("M, N, K, rows", [(33, 70, 512, 32), (256, 300, 384, 32), (300, 2000, 1024, 64)])
def test_product_of_small_tiles(torch, lib, M, N, K, rows):
    x, xs, w, ws = product_case(torch, lib, M, N, K)
    y = torch.empty(M, N, dtype=torch.float32, device="cuda")
    assert launched(torch, lambda: lib.reflex_matmul_fp8(x, xs, w, ws, y)) == [("slim", rows)]
    check_product(f64(y), x, xs, w, ws, 0.0)
