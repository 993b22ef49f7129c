"""SwiGLU experts in 8 bits where gates are far below zero.  SiLU is as near itself as elsewhere down to -87; below, where e^-g
nears the end of fp32, it may be 0.  With a large u a row of the activation may hold nothing larger than such values, so that
its codes are they."""
from __future__ import annotations

import numpy as np
import pytest

import test_gpu_fp8 as e4m3
import test_gpu_int8 as int8
from gpu_common import note, require_gpu
from oracle import eight_bit as eb
from test_gpu_int8_tiles import DOWN, UP, launched

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def offsets(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


# (an expert's gates lie around the first number, its up values have the scale 2^second: SiLU(g) u is 2^-90 or more, above
# the least maximum of a row)
FAR = [(-85.0, 60), (-96.0, 80), (-80.0, 100), (-140.0, 108), (-86.5, 70)]


def int8_far_case(torch, T, d, f, sizes):
    """Column 0 of h makes the gates, column 1 the up values; every third token is scaled down to ordinary gates."""
    E, P = len(sizes), int(sum(sizes))
    rng = np.random.default_rng([T, d, f, P])
    h = np.zeros((T, d), np.int8)
    h[:, 0], h[:, 1] = 127, rng.integers(40, 128, T) * rng.choice([-1, 1], T)
    hs = rng.uniform(0.99, 1.01, T) / np.where(np.arange(T) % 3 == 1, 64.0, 1.0)
    w = {n: np.zeros((E, f, d), np.int8) for n in ("gate", "up")}
    s = {n: np.zeros((E, f), np.float32) for n in ("gate", "up")}
    for e in range(E):
        center, exponent = FAR[e % len(FAR)]
        w["gate"][e, :, 0] = rng.integers(-127, -99, f)
        s["gate"][e] = (center + rng.uniform(-1.5, 1.5, f)) / (127.0 * w["gate"][e, :, 0])
        w["up"][e, :, 1] = rng.integers(1, 128, f) * rng.choice([-1, 1], f)
        s["up"][e] = np.exp2(exponent + rng.uniform(-1, 1, f))
    w["down"] = rng.integers(-127, 128, (E, d, f)).astype(np.int8)
    s["down"] = (2.0 ** -8 * rng.uniform(0.5, 2.0, (E, d))).astype(np.float32)
    put = {"h": h, "hs": hs.astype(np.float32)}
    put.update({"w_" + n: a for n, a in w.items()})
    put.update({"s_" + n: a for n, a in s.items()})
    c = {n: torch.from_numpy(a).cuda() for n, a in put.items()}
    c.update(T=T, d=d, f=f, E=E, P=P, cap=P + 3, offsets=offsets(sizes))
    c["token"] = rng.integers(0, T, c["cap"]).astype(np.int32)
    return c


@pytest.mark.parametrize("T, d, f, sizes, kernels", [
    (20, 256, 256, [9, 0, 11, 3, 8], [("few", UP), ("few", DOWN)]),
    (9, 128, 2176, [5, 4, 3, 7, 6], [("few", UP), ("few", DOWN)]),
    (300, 128, 256, [40] * 60 + [0, 64, 33], [(UP, 64), (DOWN, 64)]),
    (400, 128, 1024, [100] * 30 + [0, 128, 3, 65], [(UP, 128), (DOWN, 128)]),
    (400, 256, 512, [300] * 12 + [0, 0, 700], [(UP, 128), (DOWN, 128)]),
    (700, 128, 1152, [256] * 9 + [513, 600, 1, 0, 511, 255, 129, 64], [(UP, 256), (DOWN, 128)])])
def test_integer_experts_of_far_gates(torch, lib, T, d, f, sizes, kernels):
    c = int8_far_case(torch, T, d, f, sizes)
    assert launched(torch, lambda: int8.run_experts(torch, lib, c)) == kernels
    y = int8.run_experts(torch, lib, c)
    worst = int8.check_experts(c, y)
    note(f"far gates T={T} d={d} f={f} rows={c['P']}: {worst:.3f} of the bound")


def e4m3_far_case(torch, T, d, f, sizes):
    """As above: all numbers e4m3 codes, blocks of 128 with the scale 1 but for the up weights'."""
    E, P = len(sizes), int(sum(sizes))
    rng = np.random.default_rng([T, d, f, P])
    values = eb.e4m3_values()
    fine = np.nonzero(np.isfinite(values))[0]
    fine = fine[np.argsort(values[fine], kind="stable")]

    def code(v):      # of the e4m3 number above or below
        at = np.clip(np.searchsorted(values[fine], v), 0, len(fine) - 1)
        return fine[at].astype(np.uint8)
    h = np.zeros((T, d), np.uint8)
    h[:, 0] = code(np.where(np.arange(T) % 3 == 1, 2.0 ** -6, 1.0))
    h[:, 1] = code(rng.choice([-1.5, -1.0, 1.0, 1.5], T))
    w = {n: np.zeros((E, f, d), np.uint8) for n in ("gate", "up")}
    s = {n: np.full((E, -(-f // 128), 4 * -(-d // 512)), 127, np.uint8) for n in ("gate", "up")}
    far = [((-80.0, -72.0), 60), ((-96.0, -104.0), 80), ((-120.0, -128.0), 100), ((-80.0, -88.0), 70)]
    for e in range(E):
        gate, exponent = far[e % len(far)]
        w["gate"][e, :, 0] = code(rng.choice(gate, f))
        w["up"][e, :, 1] = code(rng.choice([-1.0, 1.0], f) * rng.uniform(1, 4, f))
        s["up"][e] = 127 + exponent
    w["down"] = code(rng.choice([-1.0, 1.0], (E, d, f)) * rng.uniform(0.25, 4, (E, d, f)))
    s["down"] = np.full((E, -(-d // 128), 4 * -(-f // 512)), 127, np.uint8)
    put = {"h": h, "hs": np.full((-(-d // 512), T, 4), 127, np.uint8)}
    put.update({"w_" + n: a for n, a in w.items()})
    put.update({"s_" + n: a for n, a in s.items()})
    c = {n: torch.from_numpy(a).cuda() for n, a in put.items()}
    c.update(T=T, d=d, f=f, E=E, P=P, cap=P + 3, offsets=offsets(sizes))
    c["token"] = rng.integers(0, T, c["cap"]).astype(np.int32)
    return c


@pytest.mark.parametrize("T, d, f, sizes", [
    (20, 256, 256, [9, 0, 11, 3]), (64, 128, 384, [32, 33, 0, 64]), (100, 128, 256, [127, 129, 100, 96]),
    (300, 128, 1152, [256] * 9 + [513, 400, 1, 0, 511, 255, 129, 64])])
def test_e4m3_experts_of_far_gates(torch, lib, T, d, f, sizes):
    c = e4m3_far_case(torch, T, d, f, sizes)
    y = e4m3.run_experts(torch, lib, c)
    worst = e4m3.check_experts(c, y)
    note(f"far gates T={T} d={d} f={f} rows={c['P']}: {worst:.3f} of the bound")


def test_gates_down_to_the_end_of_the_range(torch, lib):
    """Gates from -87 on as near as all others, those below them right or 0, seen through a unit matrix."""
    d = f = 128
    gate = -87.0 + np.arange(-64, 64) * 2.0 ** -6
    h = np.zeros((1, d), np.int8)
    h[0, :2] = 1
    w = {n: np.zeros((1, f, d), np.int8) for n in ("gate", "up", "down")}
    w["gate"][0, :, 0], w["up"][0, :, 1] = -1, 1
    w["down"][0] = np.eye(d, f, dtype=np.int8)
    s = {"gate": -gate[None].astype(np.float32), "up": np.full((1, f), 2.0 ** 125, np.float32),
         "down": np.ones((1, d), np.float32)}
    c = {"h": torch.from_numpy(h).cuda(), "hs": torch.ones(1, device="cuda")}
    c.update({"w_" + n: torch.from_numpy(a).cuda() for n, a in w.items()})
    c.update({"s_" + n: torch.from_numpy(a).cuda() for n, a in s.items()})
    c.update(T=1, d=d, f=f, E=1, P=1, cap=1, offsets=offsets([1]), token=np.zeros(1, np.int32))
    y = int8.run_experts(torch, lib, c)
    int8.check_experts(c, y)
    y, a = int8.host(y)[0], gate * np.exp(gate) * 2.0 ** 125
    step = np.abs(a).max() / 127      # half a code, and a rounding to bf16 before and after it
    near = np.abs(y - a) <= 0.51 * step + 2.02 * 2.0 ** -8 * np.abs(a)
    assert near[gate >= -87.0].all() and (near | (y == 0.0)).all()
