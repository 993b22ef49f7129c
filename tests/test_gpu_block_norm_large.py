"""reflex_block_norm on more than the Infinity Cache holds, where its rows pass the caches by: bit for bit what the same rows
give in small calls, and those of a sample held against the formulas."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import require_gpu
from test_gpu_block_norm import EPS, OUTPUTS, check_after_stream, check_rows, host, join_bound

pytestmark = pytest.mark.gpu
CACHE = 256 << 20
SCALE = 0.75


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def large_case(torch, T, d, stream, pairs):
    """Rows of given or (pairs) of joined ones, ragged gates, both norms."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T + d)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=g, dtype=dtype, device="cuda")
    c = dict(T=T, d=d, x=normal(T, d).to(getattr(torch, stream)) * 3, w_post=1 + 0.3 * normal(d, dtype=torch.float32),
             w_pre=1 + 0.3 * normal(d, dtype=torch.float32), gate=normal(5, d))
    cuts = torch.randint(0, T + 1, (4,), generator=g, device="cuda").sort().values
    c["seq_offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), T)]).int()
    c["at"] = np.repeat(np.arange(5), np.diff(c["seq_offsets"].cpu().numpy()))
    c["y"] = c["shared_y"] = None
    if pairs:
        n = torch.randint(0, pairs + 1, (T,), generator=g, device="cuda")
        c["pair_offsets"] = torch.cat([n.new_zeros(1), n.cumsum(0)]).int()
        P = int(c["pair_offsets"][-1])
        c["pair_to_sorted"] = torch.randperm(P, generator=g, device="cuda").int()
        c["pair_weight"] = torch.rand(P, generator=g, device="cuda")
        c["y_sorted"], c["shared_y"] = normal(P, d), normal(T, d)
    else:
        c["y"] = normal(T, d)
    return outputs(torch, c)


def outputs(torch, c):
    T, d = c["T"], c["d"]
    for name, kind, shape in (("x_out", c["x"].dtype, (T + 1, d)), ("n_out", torch.bfloat16, (T + 1, d)),
                              ("q_out", torch.int8, (T + 1, d)), ("q_scale", torch.float32, (T + 1,))):
        c[name] = torch.full(shape, 7, dtype=kind, device="cuda")
    return c


def moved(c):
    """Bytes that a call reads and writes once."""
    names = ["x", "y", "y_sorted", "shared_y", *OUTPUTS]
    return sum(t.numel() * t.element_size() for t in (c.get(n) for n in names) if t is not None)


def some_rows(torch, c, rows):
    """The case of these rows alone, a gate for each."""
    at = torch.as_tensor(rows, device="cuda")
    part = dict(c, T=len(rows), seq_offsets=None, at=np.arange(len(rows)))
    part["gate"] = c["gate"][torch.from_numpy(c["at"]).cuda()[at]]
    for name in ("x", "y", "shared_y"):
        part[name] = None if c[name] is None else c[name][at]
    if "y_sorted" in c:
        n = c["pair_offsets"].diff()[at].long()
        part["pair_offsets"] = torch.cat([n.new_zeros(1), n.cumsum(0)]).int()
        first = torch.repeat_interleave(c["pair_offsets"][at].long() - part["pair_offsets"][:-1].long(), n)
        pair = first + torch.arange(len(first), device="cuda")
        part["y_sorted"] = c["y_sorted"][c["pair_to_sorted"][pair].long()]
        part["pair_to_sorted"] = torch.arange(len(first), device="cuda").int()
        part["pair_weight"] = c["pair_weight"][pair]
    return outputs(torch, part)


def run(lib, c):
    names = ("x", "y", "w_post", "w_pre", "gate", "seq_offsets", "y_sorted", "pair_offsets", "pair_to_sorted", "pair_weight",
             "shared_y")
    lib.reflex_block_norm(**{k: c.get(k) for k in names}, **{k: c[k][:c["T"]] for k in OUTPUTS}, eps=EPS,
                          residual_scale=SCALE)


@pytest.mark.parametrize("T, d", [(40001, 1024), (17000, 2048), (8500, 4096), (4201, 8192), (2100, 16384)])
@pytest.mark.parametrize("stream", ["bfloat16", "float32"])
@pytest.mark.parametrize("pairs", [0, 4])
def test_large_calls_give_the_rows_of_small_ones(torch, lib, T, d, stream, pairs):
    c = large_case(torch, T, d, stream, pairs)
    assert moved(c) > CACHE + (1 << 20)
    run(lib, c)
    assert all((c[name][T:] == 7).all() for name in OUTPUTS)
    step = -(-T // 8)
    for first in range(0, T, step):
        rows = list(range(first, min(first + step, T)))
        part = some_rows(torch, c, rows)
        assert moved(part) < CACHE - (1 << 20)
        run(lib, part)
        for name in OUTPUTS:
            assert torch.equal(part[name][:len(rows)], c[name][first:first + len(rows)]), (name, first)
    rows = np.random.default_rng(T).choice(T, 24, replace=False)
    part = some_rows(torch, c, rows)
    for name in OUTPUTS:
        part[name][:24] = c[name][torch.from_numpy(rows).cuda()]
    if pairs:
        u, tol = join_bound(part, SCALE)
        assert (np.abs(host(part["x_out"])[:24] - u) <= tol).all()
        check_after_stream(part, 24)
    else:
        check_rows(part, SCALE)


def test_twelve_experts_rows_a_token_and_in_place(torch, lib):
    """Eight sequences' join, the stream replaced in place."""
    T, d = 8192, 2048
    c = large_case(torch, T, d, "bfloat16", 12)
    assert moved(c) > CACHE + (1 << 20)
    run(lib, c)
    want = {name: c[name].clone() for name in OUTPUTS}
    before = c["x"].clone()
    outputs(torch, c)
    c["x_out"] = c["x"]
    run(lib, c)
    assert torch.equal(c["x"], want["x_out"][:T]) and all(torch.equal(c[n], want[n]) for n in OUTPUTS[1:])
    c["x"] = before
    rows = np.random.default_rng(1).choice(T, 24, replace=False)
    part = some_rows(torch, c, rows)
    for name in OUTPUTS:
        part[name][:24] = want[name][torch.from_numpy(rows).cuda()]
    u, tol = join_bound(part, SCALE)
    assert (np.abs(host(part["x_out"])[:24] - u) <= tol).all()
    check_after_stream(part, 24)
