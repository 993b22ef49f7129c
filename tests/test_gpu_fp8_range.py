"""Products of 8-bit numbers at the ends of the scales' range, against the float64 oracle: the largest and
the smallest numbers that rows and weights can hold, beside operands that bring the results back
into fp32's range."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import require_gpu
from test_gpu_fp8 import bf16, check_product, f64, quant_rows, quant_weight

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


# one shape of every kernel: small tiles of 32 and 64 rows, tiles of 64, 128 and 256 rows
SHAPES = [(33, 70, 512), (300, 2000, 384), (64, 20003, 256), (128, 17003, 256), (300, 17003, 256)]


def product(torch, lib, x, xs, w, ws, out):
    y = torch.full((x.shape[0], w.shape[0]), float("nan"), dtype=getattr(torch, out), device="cuda")
    lib.reflex_matmul_fp8(x, xs, w, ws, y)
    return check_product(f64(y), x, xs, w, ws, 2.0 ** -8 if out == "bfloat16" else 0.0)


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
@pytest.mark.parametrize("large", ["rows", "weights"])
def test_largest_numbers(torch, lib, M, N, K, out, large):
    """Numbers next to bf16's largest, whose codes stand for 2^128, beside small ones and zeros."""
    rng = np.random.default_rng([M, N, K])
    big, small = ((M, K), (N, K)) if large == "rows" else ((N, K), (M, K))
    a = rng.choice([3.3895e38, -3.32e38, 2.0e38, 1.0, 0.0], size=big)
    a[::3] = rng.normal(size=a[::3].shape)      # (weights: blocks that hold both)
    b = rng.normal(size=small) * 1e-12
    b[:, ::7] = 0.0
    x, w = (a, b) if large == "rows" else (b, a)
    product(torch, lib, *quant_rows(torch, lib, bf16(torch, x).cuda()), *quant_weight(torch, lib, bf16(torch, w).cuda()), out)


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
@pytest.mark.parametrize("small", ["rows", "weights"])
def test_smallest_numbers(torch, lib, M, N, K, out, small):
    """Numbers next to the smallest normal one and below it."""
    rng = np.random.default_rng([M, N, K, 1])
    low, high = ((M, K), (N, K)) if small == "rows" else ((N, K), (M, K))
    a = rng.normal(size=low) * 10.0 ** -rng.integers(37, 41, (low[0], 1))
    b = rng.normal(size=high) * 1e32
    x, w = (a, b) if small == "rows" else (b, a)
    product(torch, lib, *quant_rows(torch, lib, bf16(torch, x).cuda()), *quant_weight(torch, lib, bf16(torch, w).cuda()), out)


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("out", ["float32", "bfloat16"])
@pytest.mark.parametrize("low", ["rows", "weights"])
def test_codes_at_the_ends_of_the_scales(torch, lib, M, N, K, out, low):
    """All finite codes, the subnormal ones too, under the smallest scales on one side and large ones on the other."""
    rng = np.random.default_rng([M, N, K, 2])

    def operand(shape, scale_shape, bytes_):
        q = rng.integers(0, 127, shape) | (rng.integers(0, 2, shape) << 7)
        q[rng.random(shape) < 0.3] &= 0x83       # (subnormal numbers)
        return (torch.from_numpy(q.astype(np.uint8)).cuda(),
                torch.from_numpy(rng.choice(bytes_, scale_shape).astype(np.uint8)).cuda())
    few, many = [1, 2, 3, 4], [225, 227, 230]
    x = operand((M, K), lib.fp8_scale_shape(M, K), few if low == "rows" else many)
    w = operand((N, K), lib.fp8_weight_scale_shape(N, K), many if low == "rows" else few)
    product(torch, lib, *x, *w, out)
