"""8-bit rows, weights, products and experts, and the list of masked rows, against the float64
oracle.  Codes, scales and row lists are exact; products are held to the bound of an fp32 sum
(n terms: n 2^-23 of the sum of their magnitudes), for bf16 results the bits that the 8-bit MFMA drops,
and the output's rounding."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import note, require_gpu
from oracle import eight_bit as eb
from oracle import bf16_to_f64
from synth.device import bf16_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def bf16(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def f64(t):
    return t.double().cpu().numpy()


def codes(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def random_rows(rng, M, K):
    return rng.normal(size=(M, K)) * np.exp(2.0 * rng.normal(size=(M, 1)))


def quant_rows(torch, lib, x, **kw):
    """x: bf16 device tensor -> codes and scales by the library."""
    M = kw.pop("M", x.shape[0])
    q = torch.zeros(M, x.shape[1], dtype=torch.uint8, device="cuda")
    s = torch.zeros(lib.fp8_scale_shape(M, x.shape[1]), dtype=torch.uint8, device="cuda")
    lib.reflex_quantize_fp8(x, q, s, **kw)
    return q, s


def quant_weight(torch, lib, w):
    q = torch.zeros(w.shape, dtype=torch.uint8, device="cuda")
    s = torch.zeros(lib.fp8_weight_scale_shape(*w.shape), dtype=torch.uint8, device="cuda")
    lib.reflex_quantize_fp8_weight(w, q, s)
    return q, s


# ---- masked rows --------------------------------------------------------------------------
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 1000, 16383, 16384, 16385, 50001, 1 << 18])
@pytest.mark.parametrize("share", [0.0, 0.01, 0.5, 1.0])
@pytest.mark.parametrize("shift", [0, 3])
def test_select_rows(torch, lib, T, share, shift):
    rng = np.random.default_rng([T, int(100 * share)])
    m = (rng.random(T + shift) < share) * rng.integers(1, 256, T + shift)
    masked = torch.from_numpy(m.astype(np.uint8)).cuda()[shift:]
    rows = torch.full((T,), -7, dtype=torch.int32, device="cuda")
    n = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    size = lib.reflex_select_rows_workspace_size(T)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    lib.reflex_select_rows(masked, rows, n, ws)
    want = np.nonzero(m[shift:])[0]
    assert int(n.item()) == len(want)
    got = rows.cpu().numpy()
    np.testing.assert_array_equal(got[:len(want)], want)
    assert (got[len(want):] == -7).all()


def test_select_rows_of_nothing(torch, lib):
    n = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    some = torch.zeros(1, dtype=torch.uint8, device="cuda")
    assert lib.lib().reflex_select_rows(some.data_ptr(), 0, n.data_ptr(), n.data_ptr(), None, 0,
                                        lib.stream_handle()) == 0
    assert int(n.item()) == 0


# ---- rows and weights -----------------------------------------------------------------------
def check_rows(q, s, x):
    """Codes q and scales s of x (float64, exactly bf16)."""
    M, K = x.shape
    vals, exps = eb.quantize_rows(x)
    kb = K // 128
    e = s.transpose(1, 0, 2).reshape(M, -1)
    np.testing.assert_array_equal(e[:, :kb].astype(int) - 127, exps)
    assert (e[:, kb:] == 0).all()
    np.testing.assert_array_equal(eb.rows_value(q, s), vals)
    assert (q[~np.isfinite(x)] == 0x7f).all()


@pytest.mark.parametrize("M, K", [(1, 128), (3, 256), (7, 384), (5, 512), (33, 640), (16, 2048), (2, 16384)])
def test_quantize_rows(torch, lib, M, K):
    x = bf16(torch, random_rows(np.random.default_rng([M, K]), M, K)).cuda()
    q, s = quant_rows(torch, lib, x)
    check_rows(codes(q), s.cpu().numpy(), f64(x))


def test_quantize_rows_at_the_ends_of_the_range(torch, lib):
    x = np.random.default_rng(3).normal(size=(12, 256)).astype(np.float32)
    x[0] = 0.0
    x[1, :128] = 0.0
    x[2, 5], x[3, 7], x[4, 9] = np.nan, np.inf, -np.inf
    x[5] = np.nan
    x[6] *= 1e-38                      # near the smallest normal numbers
    x[7] *= 1e-40                      # subnormal
    x[8] *= 1e38
    x[9, 0] = 3.3895e38                # the largest bf16
    x[10, :] = 448.0                   # on the border of a scale
    x[11, :] = np.where(np.arange(256) % 2, -0.0, 450.0)
    t = bf16(torch, x).cuda()
    q, s = quant_rows(torch, lib, t)
    check_rows(codes(q), s.cpu().numpy(), f64(t))


@pytest.mark.parametrize("used", [0, 1, 5, 9, 100, -3])
def test_quantize_listed_rows(torch, lib, used):
    """Rows by a list, some outside the matrix, and a count on the device."""
    T, K = 20, 384
    x = bf16(torch, random_rows(np.random.default_rng(5), T, K)).cuda()
    rows = np.array([3, 3, 19, 0, -1, 7, 20, 18, 2], dtype=np.int32)
    M = len(rows)
    q = torch.full((M + 1, K), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((1, M, 4), 0x55, dtype=torch.uint8, device="cuda")
    n = torch.tensor([used], dtype=torch.int32, device="cuda")
    lib.reflex_quantize_fp8(x, q[:M], s, rows=torch.from_numpy(rows).cuda(), n_rows=n)
    n_used = min(max(used, 0), M)
    got, gs = codes(q), s.cpu().numpy()
    assert (got[n_used:] == 0x55).all() and (gs[0, n_used:] == 0x55).all()
    inside = (rows >= 0) & (rows < T)
    want = np.where(inside[:, None], f64(x)[np.clip(rows, 0, T - 1)], 0.0)
    if n_used:
        check_rows(got[:n_used], np.ascontiguousarray(gs[:, :n_used]), want[:n_used])


@pytest.mark.parametrize("shape", [(1, 128), (127, 256), (128, 512), (130, 640), (3, 64, 128), (2, 200, 1152)])
def test_quantize_weight(torch, lib, shape):
    rng = np.random.default_rng(shape)
    w = rng.normal(size=shape) * 0.02
    w.reshape(-1, shape[-1])[0, 0] = np.nan
    w = bf16(torch, w).cuda()
    q, s = quant_weight(torch, lib, w)
    q3, s3, w3 = (a.reshape(-1, *a.shape[-2:]) for a in (codes(q), s.cpu().numpy(), f64(w)))
    for i in range(len(w3)):
        vals, exps = eb.quantize_weight(w3[i])
        kb = shape[-1] // 128
        np.testing.assert_array_equal(s3[i][:, :kb].astype(int) - 127, exps)
        assert (s3[i][:, kb:] == 0).all()
        np.testing.assert_array_equal(eb.weight_value(q3[i], s3[i]), vals)


# ---- product ----------------------------------------------------------------------------------
def product_case(torch, lib, M, N, K, seed=0, spread=True):
    rng = np.random.default_rng([M, N, K, seed])
    x = bf16(torch, random_rows(rng, M, K)).cuda()
    w = rng.normal(size=(N, K)) * 0.02
    if spread:      # every 128 x 128 block its own magnitude
        w *= np.exp(3.0 * np.repeat(np.repeat(rng.normal(size=(-(-N // 128), K // 128)), 128, 0), 128, 1))[:N]
    w = bf16(torch, w).cuda()
    return quant_rows(torch, lib, x) + quant_weight(torch, lib, w)


def check_product(got, x, xs, w, ws, out_eps):
    xv, wv = eb.rows_value(codes(x), xs.cpu().numpy()), eb.weight_value(codes(w), ws.cpu().numpy())
    y, ay = eb.product(xv, wv)
    tol = x.shape[1] * 2.0 ** -23 * ay
    if out_eps:      # bf16 results come from the 8-bit MFMA
        tol += eb.dropped_bits(xv, wv)
    tol += out_eps * (np.abs(y) + tol)
    err = np.abs(got - y)
    assert np.isfinite(got).all() and (err <= tol).all(), f"{(err / np.maximum(tol, 1e-300)).max():.3g} of the bound"
    return float((err / np.maximum(tol, 1e-300)).max())


SHAPES = [(1, 1, 128), (1, 7, 256), (2, 100, 384), (5, 256, 512), (31, 257, 640), (33, 128, 2048), (64, 129, 896),
          (65, 300, 1152), (96, 511, 128), (127, 64, 1024), (129, 255, 256), (200, 513, 640), (256, 256, 512),
          (257, 1003, 384), (300, 77, 1280), (513, 260, 128), (777, 900, 256), (1030, 40, 4096)]


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_product(torch, lib, M, N, K, out):
    x, xs, w, ws = product_case(torch, lib, M, N, K)
    room = torch.full((M * N + 64,), 5.0, dtype=getattr(torch, out), device="cuda")
    y = room[:M * N].view(M, N)
    lib.reflex_matmul_fp8(x, xs, w, ws, y)
    worst = check_product(f64(y), x, xs, w, ws, 2.0 ** -8 if out == "bfloat16" else 0.0)
    assert (room[M * N:] == 5.0).all()
    note(f"product {M} x {N} x {K} {out}: {worst:.3f} of the bound")


# (products of few 256-column tiles have a kernel of their own: these have many)
@pytest.mark.parametrize("M, N, K", [(1, 16500, 128), (33, 16641, 256), (64, 20003, 640), (70, 17003, 384), (128, 16392, 1152),
                                     (129, 16400, 512), (300, 33001, 128), (513, 8450, 256)])
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
def test_product_of_many_columns(torch, lib, M, N, K, out):
    x, xs, w, ws = product_case(torch, lib, M, N, K)
    y = torch.full((M, N), float("nan"), dtype=getattr(torch, out), device="cuda")
    lib.reflex_matmul_fp8(x, xs, w, ws, y)
    check_product(f64(y), x, xs, w, ws, 0.0 if out == "float32" else 2.0 ** -8)


@pytest.mark.parametrize("used", [0, 1, 64, 65, 129, 399, 400, 1000])
def test_product_of_counted_rows_and_many_columns(torch, lib, used):
    x, xs, w, ws = product_case(torch, lib, 400, 16897, 256)
    y = torch.full((400, 16897), 5.0, device="cuda")
    lib.reflex_matmul_fp8(x, xs, w, ws, y, n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    n = min(used, 400)
    assert (y[n:] == 5.0).all()
    if n:
        check_product(f64(y[:n]), x[:n], xs[:, :n].contiguous(), w, ws, 0.0)


@pytest.mark.parametrize("M, used", [(70, 0), (70, 1), (70, 64), (70, 69), (70, 70), (70, 500), (70, -1), (400, 129), (400, 3)])
def test_product_of_counted_rows(torch, lib, M, used):
    N, K = 201, 640
    x, xs, w, ws = product_case(torch, lib, M, N, K)
    y = torch.full((M, N), 5.0, dtype=torch.float32, device="cuda")
    lib.reflex_matmul_fp8(x, xs, w, ws, y, n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    n = min(max(used, 0), M)
    assert (y[n:] == 5.0).all()
    if n:
        full = torch.empty(M, N, dtype=torch.float32, device="cuda")
        lib.reflex_matmul_fp8(x, xs, w, ws, full)
        check_product(f64(full), x, xs, w, ws, 0.0)
        # the tiles differ with the count, and with them the order of the sums
        xv, wv = eb.rows_value(codes(x), xs.cpu().numpy()), eb.weight_value(codes(w), ws.cpu().numpy())
        z, az = eb.product(xv[:n], wv)
        assert (np.abs(f64(y[:n]) - z) <= K * 2.0 ** -23 * az).all()


def test_product_passes_nan_through_its_row_and_column_only(torch, lib):
    M, N, K = 70, 150, 256
    x, xs, w, ws = product_case(torch, lib, M, N, K)
    x[3, 200] = 0x7f
    w[140, 10] = 0xff
    y = torch.empty(M, N, dtype=torch.float32, device="cuda")
    lib.reflex_matmul_fp8(x, xs, w, ws, y)
    bad = np.isnan(f64(y))
    want = np.zeros((M, N), bool)
    want[3], want[:, 140] = True, True
    np.testing.assert_array_equal(bad, want)


def test_product_is_repeatable(torch, lib):
    x, xs, w, ws = product_case(torch, lib, 300, 700, 1024)
    y = [torch.empty(300, 700, dtype=torch.float32, device="cuda") for _ in range(2)]
    for t in y:
        lib.reflex_matmul_fp8(x, xs, w, ws, t)
    assert torch.equal(y[0], y[1])


# ---- experts ----------------------------------------------------------------------------------
def expert_case(torch, lib, T, d, f, sizes, cap_extra=0, seed=0):
    E, P = len(sizes), int(sum(sizes))
    rng = np.random.default_rng([T, d, f, P, seed])
    h = bf16(torch, random_rows(rng, T, d)).cuda()
    c = dict(T=T, d=d, f=f, E=E, P=P, cap=P + cap_extra)
    c["h"], c["hs"] = quant_rows(torch, lib, h)
    for name, n, k in (("gate", f, d), ("up", f, d), ("down", d, f)):
        w = bf16(torch, rng.normal(size=(E, n, k)) * 0.05).cuda()
        c["w_" + name], c["s_" + name] = quant_weight(torch, lib, w)
    c["token"] = rng.integers(0, T, c["cap"]).astype(np.int32)
    c["offsets"] = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    return c


def run_experts(torch, lib, c):
    y = torch.full((c["cap"], c["d"]), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(1, lib.reflex_swiglu_fp8_workspace_size(c["cap"], c["E"], c["f"])), dtype=torch.uint8,
                     device="cuda")
    lib.reflex_grouped_swiglu_fp8(c["h"], c["hs"], torch.from_numpy(c["token"]).cuda(),
                                  torch.from_numpy(c["offsets"]).cuda(), c["w_gate"], c["w_up"], c["w_down"],
                                  c["s_gate"], c["s_up"], c["s_down"], y, ws)
    return y


def check_experts(c, y):
    got = f64(y)
    assert (got[c["P"]:] == 5.0).all(), "rows past the last expert's were written"
    x = eb.rows_value(codes(c["h"]), c["hs"].cpu().numpy())
    worst = 0.0
    for e in range(c["E"]):
        lo, hi = c["offsets"][e], c["offsets"][e + 1]
        if lo == hi:
            continue
        w = [eb.weight_value(codes(c["w_" + n][e]), c["s_" + n][e].cpu().numpy()) for n in ("gate", "up", "down")]
        ref, tol = eb.swiglu_rows(x[c["token"][lo:hi]], *w)
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
        err = np.abs(got[lo:hi] - ref)
        assert (err <= tol).all(), f"expert {e}: {(err / tol).max():.3g} of the bound"
        worst = max(worst, float((err / tol).max()))
    return worst


@pytest.mark.parametrize("T, d, f, sizes, extra", [
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
])
def test_experts(torch, lib, T, d, f, sizes, extra):
    c = expert_case(torch, lib, T, d, f, sizes, extra)
    worst = check_experts(c, run_experts(torch, lib, c))
    note(f"experts T={T} d={d} f={f} rows={sum(sizes)}: {worst:.3f} of the bound")


def test_experts_without_rows(torch, lib):
    c = expert_case(torch, lib, 4, 128, 128, [0, 0], 3)
    assert (run_experts(torch, lib, c) == 5.0).all()


@pytest.mark.parametrize("T, d, f, sizes", [(20, 256, 256, [9, 0, 11]), (90, 256, 128, [70, 60]), (300, 384, 256, [300])])
def test_experts_keep_what_is_not_finite_in_its_row(torch, lib, T, d, f, sizes):
    """Rows of NaN, and rows whose activation overflows in some columns: their results are NaN, all others
    within the bound."""
    c = expert_case(torch, lib, T, d, f, sizes)
    c["token"] = (np.arange(c["cap"]) % T).astype(np.int32)
    bad = [3 % T, T // 2]
    c["h"][bad[0], 5] = 0x7f
    c["hs"][:, bad[1]] = 247      # (2^120: the product of gate and up is past fp32)
    y = f64(run_experts(torch, lib, c))
    hit = np.isin(c["token"][:c["P"]], bad)
    assert np.isnan(y[:c["P"]][hit]).all()
    good = dict(c, token=c["token"][:c["P"]][~hit], P=int((~hit).sum()))
    owner = np.repeat(np.arange(len(sizes)), sizes)[~hit]
    good["offsets"] = np.searchsorted(owner, np.arange(len(sizes) + 1)).astype(np.int32)
    check_experts(good, torch.from_numpy(np.concatenate([y[:c["P"]][~hit], y[c["P"]:]])))
