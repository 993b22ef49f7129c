"""Token sampling where a row's logits reach the ends of fp32: the type's lowest number beside tokens
without weight, and temperatures so high that it has weight too."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import require_gpu
from test_gpu_tokens import check, sample

pytestmark = pytest.mark.gpu

LOW = -3.4028234663852886e38


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


@pytest.mark.parametrize("V", [300, 5003, 40013])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_lowest_logits_beside_tokens_without_weight(torch, lib, V, dtype):
    """-inf and NaN have no weight, however near to the type's lowest number the row's maximum is and however
    high the temperature."""
    rng = np.random.default_rng([V, 5])
    low = LOW if dtype == "float32" else -3.3895313892515355e38
    some = np.sort(rng.choice(V, V // 30, replace=False))
    x = np.full((8, V), -np.inf)
    x[0, some] = low                                    # few tokens have weight, the same each
    x[1, some] = low
    x[1, some[0] + 1:some[1]] = np.nan
    x[2] = np.where(rng.random(V) < 0.5, np.nan, low)   # half of them
    x[3] = np.where(rng.random(V) < 0.5, -np.inf, low)
    x[4, some[3:]], x[4, some[2]] = low, low * (1 - 2.0 ** -7)      # one token has all of the weight
    x[5] = rng.normal(size=V)                           # ordinary logits beside all of those
    x[5, ::3], x[5, 1::5], x[5, 2::7] = -np.inf, np.nan, low
    x[6] = np.nan
    x[6, some] = np.where(np.arange(len(some)) % 2, 0.0, low)
    x[7, V - 1] = low
    dev = torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype)).cuda()
    host = dev.double().cpu().numpy()
    for params in [(1.0, 0, 1.0, 0.0), (0.5, 4, 1.0, 0.0), (1.0, 0, 0.7, 0.0), (1.0, 3, 0.9, 0.3), (0.0, 0, 1.0, 0.0),
                   (1e38, 0, 1.0, 0.0), (1e38, 0, 0.6, 0.0), (1e38, 0, 1.0, 0.02), (3e38, 7, 0.9, 0.0),
                   (1e38, 2000, 0.9, 0.5), (1e-38, 0, 0.9, 0.0)]:
        for u in (np.linspace(0.03, 0.95, 8), np.full(8, 0.55)):
            u = u.astype(np.float32)
            check(host, u, params, *sample(torch, lib, dev, u, params))
