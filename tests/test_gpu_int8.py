"""8-bit integer rows, weights, products and experts against the oracle.  Codes and scales are exact;
products are held to the roundings of the sum, the scales' product and the result."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import note, require_gpu
from oracle import int8 as oi

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def bf16(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).cuda()


def host(t):
    return t.float().cpu().numpy()


def random_rows(rng, M, K):
    return rng.normal(size=(M, K)) * np.exp(2.0 * rng.normal(size=(M, 1)))


def quant_rows(torch, lib, x, **kw):
    q = torch.zeros(x.shape, dtype=torch.int8, device="cuda")
    s = torch.zeros(x.shape[0], dtype=torch.float32, device="cuda")
    lib.reflex_quantize_int8(x, q, s, **kw)
    return q, s


def same_rows(q, s, x):
    want_q, want_s = oi.quantize_rows(x)
    np.testing.assert_array_equal(q, want_q)
    np.testing.assert_array_equal(s, want_s)


# ---- rows and weights -----------------------------------------------------------------------
@pytest.mark.parametrize("M, K", [(1, 128), (3, 256), (7, 384), (5, 512), (33, 640), (16, 2048), (5, 2176), (9, 4096), (3, 4224),
                                  (2, 8192), (3, 8320), (3, 16384), (1000, 1152)])
def test_quantize_rows(torch, lib, M, K):
    x = bf16(torch, random_rows(np.random.default_rng([M, K]), M, K))
    q, s = quant_rows(torch, lib, x)
    same_rows(q.cpu().numpy(), s.cpu().numpy(), host(x))


@pytest.mark.parametrize("K", [256, 4096, 16384])
def test_quantize_rows_at_the_ends_of_the_range(torch, lib, K):
    x = np.random.default_rng(3).normal(size=(14, K)).astype(np.float32)
    x[0] = 0.0
    x[1, :128] = 0.0
    x[2, 5], x[3, K - 1], x[4, 9] = np.nan, np.inf, -np.inf
    x[5] = np.nan
    x[6] *= 1e-38                      # near the smallest normal numbers
    x[7] *= 1e-40                      # subnormal
    x[8] *= 1e38
    x[9, 0] = 3.3895e38                # the largest bf16
    x[10] = np.where(np.arange(K) % 2, 0.5, -127.0)      # ties: 0.5 to 0
    x[11] = np.where(np.arange(K) % 3, 1.5, 127.0)
    x[12] = 2.0 ** -100
    x[13] = 2.0 ** -101
    t = bf16(torch, x)
    q, s = quant_rows(torch, lib, t)
    same_rows(q.cpu().numpy(), s.cpu().numpy(), host(t))


@pytest.mark.parametrize("K", [384, 2304, 6144])
@pytest.mark.parametrize("used", [0, 1, 5, 9, 100, -3])
def test_quantize_listed_rows(torch, lib, used, K):
    """Rows by a list, some outside the matrix, one twice, and a count on the device."""
    T = 20
    x = bf16(torch, random_rows(np.random.default_rng(5), T, K))
    rows = np.array([3, 3, 19, 0, -1, 7, 20, 18, 2], dtype=np.int32)
    M = len(rows)
    q = torch.full((M + 1, K), 0x55, dtype=torch.int8, device="cuda")
    s = torch.full((M + 1,), 5.0, dtype=torch.float32, device="cuda")
    lib.reflex_quantize_int8(x, q[:M], s[:M], rows=torch.from_numpy(rows).cuda(),
                             n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    n = min(max(used, 0), M)
    assert (q[n:] == 0x55).all() and (s[n:] == 5.0).all()
    inside = (rows >= 0) & (rows < T)
    want = np.where(inside[:, None], host(x)[np.clip(rows, 0, T - 1)], 0.0)
    same_rows(q[:n].cpu().numpy(), s[:n].cpu().numpy(), want[:n]) if n else None


@pytest.mark.parametrize("shape", [(1, 128), (127, 256), (130, 640), (3, 64, 128), (2, 201, 1152), (2, 7, 4096)])
def test_quantize_weight(torch, lib, shape):
    w = np.random.default_rng(shape).normal(size=shape) * 0.02
    w.reshape(-1, shape[-1])[0, 0] = np.nan
    w = bf16(torch, w)
    q = torch.zeros(shape, dtype=torch.int8, device="cuda")
    s = torch.zeros(shape[:-1], dtype=torch.float32, device="cuda")
    lib.reflex_quantize_int8_weight(w, q, s)
    same_rows(q.cpu().numpy().reshape(-1, shape[-1]), s.cpu().numpy().reshape(-1), host(w).reshape(-1, shape[-1]))


# ---- product ----------------------------------------------------------------------------------
def int8_case(torch, M, N, K, seed=0):
    rng = np.random.default_rng([M, N, K, seed])
    put = [rng.integers(-127, 128, (M, K)).astype(np.int8), np.exp(rng.normal(size=M)).astype(np.float32),
           rng.integers(-127, 128, (N, K)).astype(np.int8), np.exp(rng.normal(size=N) - 5).astype(np.float32)]
    put[0][0] = 127      # the largest sums
    put[2][0] = 127
    return [torch.from_numpy(a).cuda() for a in put]


def check_product(got, case, out_eps):
    y = oi.product(*(t.cpu().numpy() for t in case))
    tol = oi.PRODUCT_EPS * np.abs(y)
    tol += out_eps * (np.abs(y) + tol)
    err = np.abs(got - y)
    assert (err <= tol).all(), f"{(err - tol).max():.3g} over the bound at {np.argwhere(err > tol)[:4].tolist()}"


SHAPES = [(1, 1, 128), (1, 7, 256), (2, 100, 384), (5, 256, 512), (31, 257, 640), (33, 128, 2048), (64, 129, 896),
          (65, 300, 1152), (96, 511, 128), (127, 64, 1024), (129, 255, 256), (200, 513, 640), (256, 256, 512),
          (257, 1003, 384), (300, 77, 1280), (513, 260, 128), (777, 900, 256), (1030, 40, 4096), (3, 33, 16384)]


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_product(torch, lib, M, N, K, out):
    case = int8_case(torch, M, N, K)
    room = torch.full((M * N + 64,), 5.0, dtype=getattr(torch, out), device="cuda")
    y = room[:M * N].view(M, N)
    lib.reflex_matmul_int8(*case, y)
    check_product(host(y).astype(np.float64), case, 2.0 ** -8 if out == "bfloat16" else 0.0)
    assert (room[M * N:] == 5.0).all()


# (products of few 256-column tiles may have a kernel of their own: these have many)
@pytest.mark.parametrize("M, N, K", [(1, 16500, 128), (33, 16641, 256), (64, 20003, 640), (70, 17003, 384), (128, 16392, 1152),
                                     (129, 16400, 512), (300, 33001, 128), (513, 8450, 256), (2000, 9001, 256)])
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_product_of_many_columns(torch, lib, M, N, K, out):
    case = int8_case(torch, M, N, K)
    y = torch.full((M, N), float("nan"), dtype=getattr(torch, out), device="cuda")
    lib.reflex_matmul_int8(*case, y)
    check_product(host(y).astype(np.float64), case, 0.0 if out == "float32" else 2.0 ** -8)


@pytest.mark.parametrize("M, N, used", [(70, 201, 0), (70, 201, 1), (70, 201, 64), (70, 201, 69), (70, 201, 500), (70, 201, -1),
                                        (400, 201, 129), (400, 16897, 0), (400, 16897, 65), (400, 16897, 129), (400, 16897, 399),
                                        (400, 16897, 1000)])
def test_product_of_counted_rows(torch, lib, M, N, used):
    case = int8_case(torch, M, N, 640)
    full, y = (torch.full((M, N), 5.0, dtype=torch.float32, device="cuda") for _ in range(2))
    lib.reflex_matmul_int8(*case, full)
    lib.reflex_matmul_int8(*case, y, n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    n = min(max(used, 0), M)
    assert (y[n:] == 5.0).all()
    assert torch.equal(y[:n], full[:n])      # (the sums are exact: no tile changes them)
    check_product(host(full).astype(np.float64), case, 0.0)


@pytest.mark.parametrize("N", [150, 17000])
def test_product_passes_nan_through_its_row_and_column_only(torch, lib, N):
    M, K = 70, 256
    x, xs, w, ws = int8_case(torch, M, N, K)
    xs[3] = float("nan")
    ws[140] = float("nan")
    y = torch.empty(M, N, dtype=torch.float32, device="cuda")
    lib.reflex_matmul_int8(x, xs, w, ws, y)
    want = np.zeros((M, N), bool)
    want[3], want[:, 140] = True, True
    np.testing.assert_array_equal(np.isnan(host(y)), want)


def test_product_of_the_lowest_codes(torch, lib):
    """-128 is no code that the library makes, but is multiplied as what it is."""
    M, N, K = 40, 300, 16384
    x, w = (torch.full((n, K), -128, dtype=torch.int8, device="cuda") for n in (M, N))
    one = torch.ones(N, device="cuda")
    y = torch.empty(M, N, dtype=torch.float32, device="cuda")
    lib.reflex_matmul_int8(x, one[:M], w, one, y)
    assert (y == 2.0 ** 28).all()


# ---- experts ----------------------------------------------------------------------------------
def expert_case(torch, lib, T, d, f, sizes, cap_extra=0, seed=0):
    E, P = len(sizes), int(sum(sizes))
    rng = np.random.default_rng([T, d, f, P, seed])
    c = dict(T=T, d=d, f=f, E=E, P=P, cap=P + cap_extra)
    c["h"], c["hs"] = quant_rows(torch, lib, bf16(torch, random_rows(rng, T, d)))
    for name, n, k in (("gate", f, d), ("up", f, d), ("down", d, f)):
        w = bf16(torch, rng.normal(size=(E, n, k)) * 0.05 * np.exp(0.5 * rng.normal(size=(E, n, 1))))
        c["w_" + name] = torch.zeros(w.shape, dtype=torch.int8, device="cuda")
        c["s_" + name] = torch.zeros(w.shape[:2], dtype=torch.float32, device="cuda")
        lib.reflex_quantize_int8_weight(w, c["w_" + name], c["s_" + name])
    c["token"] = rng.integers(0, T, c["cap"]).astype(np.int32)
    c["offsets"] = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    return c


def run_experts(torch, lib, c):
    y = torch.full((c["cap"], c["d"]), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(lib.reflex_swiglu_int8_workspace_size(c["cap"], c["E"], c["f"]), dtype=torch.uint8, device="cuda")
    lib.reflex_grouped_swiglu_int8(c["h"], c["hs"], torch.from_numpy(c["token"]).cuda(),
                                   torch.from_numpy(c["offsets"]).cuda(), c["w_gate"], c["w_up"], c["w_down"],
                                   c["s_gate"], c["s_up"], c["s_down"], y, ws)
    return y


def check_experts(c, y):
    got = y if isinstance(y, np.ndarray) else host(y).astype(np.float64)
    assert (got[c["P"]:] == 5.0).all(), "rows past the last expert's were written"
    h, hs = c["h"].cpu().numpy(), c["hs"].cpu().numpy()
    worst = 0.0
    for e in range(c["E"]):
        lo, hi = c["offsets"][e], c["offsets"][e + 1]
        if lo == hi:
            continue
        w = [(c["w_" + n][e].cpu().numpy(), c["s_" + n][e].cpu().numpy()) for n in ("gate", "up", "down")]
        at = c["token"][lo:hi]
        ref, tol = oi.swiglu_rows(h[at], hs[at], *w)
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol) + 2.0 ** -134      # (half the least bf16 number)
        err = np.abs(got[lo:hi] - ref)
        assert (err <= tol).all(), f"expert {e}: {(err / tol).max():.3g} of the bound"
        worst = max(worst, float((err / tol).max()))
    return worst


EXPERTS = [
    (1, 128, 128, [1], 0),
    (3, 256, 128, [0, 2, 0, 1], 5),
    (20, 384, 256, [5, 0, 17, 1], 2),
    (64, 640, 384, [32, 33, 0, 31], 100),
    (50, 128, 640, [64, 65, 1], 0),
    (100, 1152, 128, [127, 129], 7),
    (300, 512, 512, [255, 0, 257], 0),
    (40, 256, 1152, [300, 20], 33),
    (10, 2048, 256, [9, 0, 0, 0, 10, 3, 0, 1], 0),
    (200, 256, 256, [513], 0),
    (33, 256, 256, [1] * 256, 0),
    (60, 256, 2432, [40, 61], 0),
    (300, 640, 512, [700, 0, 64, 300, 1], 64),
]


@pytest.mark.parametrize("T, d, f, sizes, extra", EXPERTS)
def test_experts(torch, lib, T, d, f, sizes, extra):
    c = expert_case(torch, lib, T, d, f, sizes, extra)
    worst = check_experts(c, run_experts(torch, lib, c))
    note(f"experts T={T} d={d} f={f} rows={sum(sizes)}: {worst:.3f} of the bound")


def test_experts_without_rows(torch, lib):
    c = expert_case(torch, lib, 4, 128, 128, [0, 0], 3)
    assert (run_experts(torch, lib, c) == 5.0).all()


@pytest.mark.parametrize("T, d, f, sizes", [(20, 256, 256, [9, 0, 11]), (90, 256, 128, [70, 60]), (300, 384, 256, [300])])
def test_experts_keep_what_is_not_finite_in_its_row(torch, lib, T, d, f, sizes):
    """Rows with the scale NaN, and rows whose activation overflows: their results are NaN, all others within
    the bound."""
    c = expert_case(torch, lib, T, d, f, sizes)
    c["token"] = (np.arange(c["cap"]) % T).astype(np.int32)
    bad = [3 % T, T // 2]
    c["hs"][bad[0]] = float("nan")
    c["hs"][bad[1]] = 2.0 ** 100      # (the product of gate and up is past fp32)
    y = host(run_experts(torch, lib, c)).astype(np.float64)
    hit = np.isin(c["token"][:c["P"]], bad)
    assert np.isnan(y[:c["P"]][hit]).all()
    good = dict(c, token=c["token"][:c["P"]][~hit], P=int((~hit).sum()))
    owner = np.repeat(np.arange(len(sizes)), sizes)[~hit]
    good["offsets"] = np.searchsorted(owner, np.arange(len(sizes) + 1)).astype(np.int32)
    check_experts(good, np.concatenate([y[:c["P"]][~hit], y[c["P"]:]]))
