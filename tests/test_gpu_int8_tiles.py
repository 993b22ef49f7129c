"""The kernels of the 8-bit integer products in the shapes that large calls run in: several tiles a workgroup, K loops
longer than the copies' lookahead, strips of M tiles, last rounds that are cut, experts of uneven and no rows.  Which
kernel a shape reaches is read from the names of what it launches, so that a changed rule cannot empty these tests."""
from __future__ import annotations

import re

import numpy as np
import pytest

from gpu_common import note, require_gpu
from test_gpu_int8 import check_experts, check_product, expert_case, host, int8_case, run_experts

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
    """(mode, rows of a tile) of the integer products that a call launches; ("slim", rows) and ("few", mode) of the
    kernels for few tiles and for experts of few rows."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    found = []
    for e in prof.events():
        m = re.search(r"int8_gemm_kernel<.*?(\d)(?:\)|,).*?Shape8<(\d+),", e.name)
        n = re.search(r"int8_slim_kernel<(\d+),", e.name)
        f = re.search(r"int8_few_kernel<.*?(\d)(?:\)|,)", e.name)
        if m:
            found.append((int(m[1]), 64 * int(m[2])))
        if n:
            found.append(("slim", 32 * int(n[1])))
        if f:
            found.append(("few", int(f[1])))
    return found


# (256 CUs; a slice of K is 128 columns, and 3 or 4 of them are in flight)
@pytest.mark.parametrize("M, N, K, rows", [
    (64, 70001, 384, 64), (50, 66003, 1152, 64), (128, 70001, 384, 128), (65, 66003, 640, 128),
    (200, 30003, 640, 128),      # (few tiles of 256 rows)
    (300, 40003, 384, 256), (300, 40003, 640, 256), (520, 35009, 1152, 256),
    (1000, 17000, 256, 256),     # (268 tiles: a last round cut into four)
    (1024, 20000, 128, 256),     # (316 tiles: into four)
    (1030, 21000, 384, 256),     # (415 tiles: not cut)
    (1100, 19300, 256, 256),     # (380 tiles: into two)
    (2400, 8000, 640, 256),      # (10 M tiles: a strip of eight and one of two)
    (4400, 5003, 256, 256)])     # (18: two strips and a part)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_product_of_many_tiles(torch, lib, M, N, K, rows, out):
    case = int8_case(torch, M, N, K)
    room = torch.full((M * N + 64,), 5.0, dtype=getattr(torch, out), device="cuda")
    y = room[:M * N].view(M, N)
    assert launched(torch, lambda: lib.reflex_matmul_int8(*case, y)) == [(PLAIN, rows)]
    check_product(host(y).astype(np.float64), case, 2.0 ** -8 if out == "bfloat16" else 0.0)
    assert (room[M * N:] == 5.0).all()


@pytest.mark.parametrize("M, N, K, rows", [(16, 4096, 256, 32), (33, 5000, 2048, 32), (256, 2048, 1152, 32), (256, 2100, 1152, 64),
                                           (64, 16384, 384, 64)])
def test_product_of_few_tiles(torch, lib, M, N, K, rows):
    case = int8_case(torch, M, N, K)
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    assert launched(torch, lambda: lib.reflex_matmul_int8(*case, y)) == [("slim", rows)]
    check_product(host(y).astype(np.float64), case, 2.0 ** -8)


@pytest.mark.parametrize("used", [0, 1, 700, 1025, 2399, 2400])
def test_counted_rows_of_strips_and_cut_rounds(torch, lib, used):
    M, N, K = 2400, 8000, 256
    case = int8_case(torch, M, N, K)
    full, y = (torch.full((M, N), 5.0, dtype=torch.float32, device="cuda") for _ in range(2))
    lib.reflex_matmul_int8(*case, full)
    lib.reflex_matmul_int8(*case, y, n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    assert torch.equal(y[:used], full[:used]) and (y[used:] == 5.0).all()


@pytest.mark.parametrize("T, d, f, sizes, extra, kind", [
    (300, 640, 512, [40] * 60 + [0, 64, 33], 0, 64),
    (400, 512, 1024, [100] * 30 + [0, 128, 3, 65], 0, 128),
    (300, 1664, 1024, [200, 0, 513, 256, 1, 257, 900, 130], 500, 128),      # (tiles of 256 rows would be few)
    (400, 512, 512, [300] * 12 + [0, 0, 700], 100, 128),
    (500, 1280, 640, [300] * 12 + [0, 0, 700, 257], 100, 128),
    (500, 2048, 896, [300] * 12 + [0, 0, 700, 257], 100, 256),
    (700, 1408, 1152, [256] * 9 + [513, 600, 1, 0, 511, 255, 129, 64], 64, 256),
    (900, 384, 128, [5000], 0, 128)])
def test_experts_of_many_tiles(torch, lib, T, d, f, sizes, extra, kind):
    c = expert_case(torch, lib, T, d, f, sizes, extra)
    found = launched(torch, lambda: run_experts(torch, lib, c))
    assert found == [(UP, kind), (DOWN, kind)], found
    worst = check_experts(c, run_experts(torch, lib, c))
    note(f"experts T={T} d={d} f={f} rows={sum(sizes)}: {worst:.3f} of the bound")


@pytest.mark.parametrize("T, d, f, sizes, extra", [
    (5, 2048, 1024, [0] * 20 + [1, 0, 3, 2] + [0] * 40, 30), (3, 640, 128, [2, 0, 1], 0), (40, 1152, 2432, [33, 0, 50, 20], 3),
    (20, 16384, 256, [7, 9], 0), (9, 256, 16384, [4, 5], 0), (1, 128, 384, [0] * 255 + [1], 0)])
def test_experts_of_few_rows(torch, lib, T, d, f, sizes, extra):
    c = expert_case(torch, lib, T, d, f, sizes, extra)
    found = launched(torch, lambda: run_experts(torch, lib, c))
    assert found == [("few", UP), ("few", DOWN)], found
    check_experts(c, run_experts(torch, lib, c))


def test_both_kernels_of_experts_give_the_same(torch, lib):
    """The rows of an expert alone and among many: sums are exact, so the kernels agree to the bit."""
    T, d, f = 700, 512, 640
    c = expert_case(torch, lib, T, d, f, [600, 20])
    c["token"][:600] = np.arange(600)
    many = run_experts(torch, lib, c)
    few = dict(c, cap=20, P=20, token=c["token"][:20], offsets=np.array([0, 20, 20], dtype=np.int32))
    few["h"], few["hs"], few["T"] = c["h"][:20].contiguous(), c["hs"][:20].contiguous(), 20
    assert launched(torch, lambda: run_experts(torch, lib, few)) == [("few", UP), ("few", DOWN)]
    assert torch.equal(run_experts(torch, lib, few)[:20], many[:20])


def test_room_for_more_rows_than_tokens(torch, lib):
    """A large pair capacity with few rows in use: a grid that goes by the rows there are."""
    c = expert_case(torch, lib, 2, 128, 128, [3, 0, 1], 1 << 22)
    y = torch.full((c["cap"], 128), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(lib.reflex_swiglu_int8_workspace_size(c["cap"], 3, 128), dtype=torch.uint8, device="cuda")
    args = (c["h"], c["hs"], torch.from_numpy(c["token"]).cuda(), torch.from_numpy(c["offsets"]).cuda(), c["w_gate"], c["w_up"],
            c["w_down"], c["s_gate"], c["s_up"], c["s_down"], y, ws)
    assert launched(torch, lambda: lib.reflex_grouped_swiglu_int8(*args)) == [(UP, 64), (DOWN, 64)]
    assert (y[4:] == 5.0).all()
    check_experts(dict(c, cap=4), host(y[:4]).astype(np.float64))
