"""reflex_block_norm against its formulas: rows given as such, operation by operation (exact); the experts'
rows to the bound of their fp32 sum, and what follows exactly from the stream that came out."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import require_gpu
from oracle import int8 as oi

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def torch():
    return require_gpu()


@pytest.fixture(scope="module")
def lib(torch):
    from paper_2608_01784_amd import _lib
    return _lib


def host(t):
    return None if t is None else t.float().cpu().numpy()


def case(torch, T, d, stream="bfloat16", gate="none", post=True, x=True, y=True, seed=0, pairs=None):
    rng = np.random.default_rng([T, d, seed])

    def put(a, dtype=torch.bfloat16):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dtype).cuda()
    c = dict(T=T, d=d)
    kind = getattr(torch, stream)
    c["x"] = put(rng.normal(size=(T, d)) * np.exp(rng.normal(size=(T, 1))), kind) if x else None
    c["y"] = put(rng.normal(size=(T, d)) * np.exp(2 * rng.normal(size=(T, 1)))) if y and pairs is None else None
    c["w_post"] = put(1 + 0.3 * rng.normal(size=d), torch.float32) if post else None
    c["w_pre"] = put(1 + 0.3 * rng.normal(size=d), torch.float32)
    c["gate"] = c["seq_offsets"] = None
    c["at"] = None
    if gate == "one":
        c["gate"], c["at"] = put(rng.normal(size=(1, d))), np.zeros(T, int)
    elif gate == "token":
        c["gate"], c["at"] = put(rng.normal(size=(T, d))), np.arange(T)
    elif gate != "none":      # so many sequences, some of them empty
        B = int(gate)
        cuts = np.sort(rng.integers(0, T + 1, B - 1))
        seq = np.concatenate([[0], cuts, [T]]).astype(np.int32)
        c["gate"], c["seq_offsets"] = put(rng.normal(size=(B, d))), torch.from_numpy(seq).cuda()
        c["at"] = np.repeat(np.arange(B), np.diff(seq))
    if pairs is not None:
        n = rng.integers(0, pairs + 1, T)
        n[0] = pairs
        P, cap = int(n.sum()), T * pairs + 3
        c["y_sorted"] = put(rng.normal(size=(cap, d)))
        c["pair_offsets"] = torch.from_numpy(np.concatenate([[0], n.cumsum()]).astype(np.int32)).cuda()
        at = np.zeros(cap, np.int32)
        at[:P] = rng.permutation(cap)[:P]
        c["pair_to_sorted"] = torch.from_numpy(at).cuda()
        c["pair_weight"] = put(rng.random(cap), torch.float32)
        c["shared_y"] = put(rng.normal(size=(T, d))) if seed % 2 else None
    c["x_out"] = torch.full((T + 1, d), 7.0, dtype=kind, device="cuda")
    c["n_out"] = torch.full((T + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    c["q_out"] = torch.full((T + 1, d), 7, dtype=torch.int8, device="cuda")
    c["q_scale"] = torch.full((T + 1,), 7.0, dtype=torch.float32, device="cuda")
    return c


INPUTS = ("x", "y", "w_post", "w_pre", "gate", "seq_offsets", "y_sorted", "pair_offsets", "pair_to_sorted",
          "pair_weight", "shared_y")
OUTPUTS = ("x_out", "n_out", "q_out", "q_scale")


def run(lib, c, scale=1.0, outputs=OUTPUTS, **more):
    T = c["T"]
    lib.reflex_block_norm(**{k: c.get(k) for k in INPUTS}, **{k: c[k][:T] for k in outputs}, eps=EPS,
                          residual_scale=scale, **more)


def check_after_stream(c, n, outputs=OUTPUTS):
    """n_out and q_out from x_out's rows, exactly; everything from row n on as it was."""
    u = host(c["x_out"])
    ref = oi.next_input(u[:n], host(c["w_pre"]), EPS)
    q, s = oi.quantize_rows(ref)
    for name, want in (("n_out", ref), ("q_out", q), ("q_scale", s)):
        if name in outputs:
            got = c[name].float().cpu().numpy() if name == "n_out" else c[name].cpu().numpy()
            np.testing.assert_array_equal(got[:n], want, err_msg=name)
    for name in OUTPUTS:
        assert (c[name][n if name in outputs else 0:] == 7).all(), name


def check_rows(c, scale, n=None, **kw):
    n = c["T"] if n is None else n
    gate = None if c["gate"] is None else host(c["gate"])[c["at"]]
    ref = oi.stream(host(c["x"]), host(c["y"]), host(c["w_post"]), gate, scale, EPS, c["x_out"].dtype.itemsize == 4)
    np.testing.assert_array_equal(host(c["x_out"])[:n], ref[:n])
    check_after_stream(c, n, **kw)


SIZES = [(1, 128), (2, 256), (5, 640), (33, 2048), (7, 2176), (3, 4096), (6, 4224), (3, 8192), (2, 8320), (3, 16384), (2500, 384)]


@pytest.mark.parametrize("T, d", SIZES)
@pytest.mark.parametrize("stream", ["bfloat16", "float32"])
@pytest.mark.parametrize("gate, post, scale", [("none", False, 1.0), ("one", True, 0.75), ("token", True, -1.5), ("3", False, 0.0)])
def test_rows(torch, lib, T, d, stream, gate, post, scale):
    c = case(torch, T, d, stream, gate, post)
    run(lib, c, scale)
    check_rows(c, scale)


@pytest.mark.parametrize("T, B", [(1, 1), (1, 5), (40, 64), (40, 65), (500, 66), (300, 129), (2000, 4097), (700, 10000)])
@pytest.mark.parametrize("d", [128, 2304])
def test_gates_of_many_sequences(torch, lib, T, B, d):
    c = case(torch, T, d, gate=str(B))
    run(lib, c)
    check_rows(c, 1.0)


@pytest.mark.parametrize("d", [256, 4096])
@pytest.mark.parametrize("x, y", [(True, False), (False, True)])
def test_one_input_alone(torch, lib, d, x, y):
    c = case(torch, 9, d, gate="token" if y else "none", post=y, x=x, y=y)
    run(lib, c, 0.5)
    check_rows(c, 0.5)


@pytest.mark.parametrize("d", [384, 6144])
@pytest.mark.parametrize("used", [0, 1, 3, 9, 100, -2])
def test_counted_rows(torch, lib, d, used):
    c = case(torch, 9, d, gate="2")
    run(lib, c, n_rows=torch.tensor([used], dtype=torch.int32, device="cuda"))
    check_rows(c, 1.0, min(max(used, 0), 9))


@pytest.mark.parametrize("outputs", [("x_out",), ("x_out", "n_out"), ("x_out", "q_out", "q_scale")])
@pytest.mark.parametrize("d", [640, 4096])
def test_some_outputs(torch, lib, outputs, d):
    c = case(torch, 11, d)
    run(lib, c, outputs=outputs)
    check_rows(c, 1.0, outputs=outputs)


def test_outputs_without_the_stream(torch, lib):
    a, b = case(torch, 11, 640), case(torch, 11, 640)
    run(lib, a)
    run(lib, b, outputs=("n_out", "q_out", "q_scale"))
    assert all(torch.equal(a[k], b[k]) for k in ("n_out", "q_out", "q_scale")) and (b["x_out"] == 7.0).all()


@pytest.mark.parametrize("stream", ["bfloat16", "float32"])
def test_stream_in_place(torch, lib, stream):
    a, b = case(torch, 50, 2304, stream), case(torch, 50, 2304, stream)
    run(lib, a)
    args = {k: b.get(k) for k in INPUTS}
    for _ in range(2):      # the second pass goes on from the first one's stream
        lib.reflex_block_norm(**args, x_out=b["x"], n_out=b["n_out"][:50], eps=EPS)
        if _ == 0:
            assert torch.equal(b["x"], a["x_out"][:50]) and torch.equal(b["n_out"], a["n_out"])
    a["x"] = a["x_out"][:50].clone()
    run(lib, a)
    assert torch.equal(b["x"], a["x_out"][:50]) and torch.equal(b["n_out"], a["n_out"])


@pytest.mark.parametrize("d", [256, 4096])
def test_rows_at_the_ends_of_the_range(torch, lib, d):
    """Zeros, subnormal and huge numbers, and what is not finite stays in its row."""
    c = case(torch, 9, d, "float32", "one")
    c["x"][0], c["y"][0] = 0.0, 0.0
    c["x"][1], c["y"][1] = 0.0, 1e-40
    c["x"][2] = 1e-42
    c["y"][2] = 0.0
    c["y"][3] = 3e38
    c["x"][4] = 3e38
    c["x"][5, 3], c["y"][6, 5], c["y"][7, 7] = float("inf"), float("nan"), float("-inf")
    run(lib, c)
    with np.errstate(all="ignore"):
        check_rows(c, 1.0)
    q, s, n = c["q_out"].cpu().numpy(), c["q_scale"].cpu().numpy(), host(c["n_out"])
    assert not q[0].any() and s[0] == np.float32(2.0 ** -100) / np.float32(127)
    bad = np.isnan(s)
    assert bad[5:8].all() and not bad[:5].any() and not bad[8] and np.isnan(n[5:8]).any(1).all()


def join_bound(c, scale):
    """x_out in fp64 and how far fp32 sums of the experts' rows (and the roundings after) may be from it."""
    y, ay = oi.joined(host(c["y_sorted"]), c["pair_offsets"].cpu().numpy(), c["pair_to_sorted"].cpu().numpy(),
                      c["pair_weight"].cpu().numpy(), host(c["shared_y"]))
    most = int(np.diff(c["pair_offsets"].cpu().numpy()).max()) + 1
    ey = most * 2.0 ** -24 * 1.01 * ay
    rel = 0.0
    if c["w_post"] is not None:
        ms = (y ** 2).mean(1, keepdims=True) + EPS
        r = 1.0 / np.sqrt(ms)
        # the root moves with the mean of 2 y ey; two products and r are rounded
        er = (np.abs(y) * ey + ey ** 2).mean(1, keepdims=True) / ms + 2.0 ** -24
        w = host(c["w_post"]).astype(np.float64)
        y, ey = y * r * w, np.abs(r * w) * (ey + np.abs(y) * (1.1 * er))
        rel = 2.1 * 2.0 ** -24
    if c["gate"] is not None:
        g = host(c["gate"])[c["at"]].astype(np.float64)
        y, ey, rel = y * g, ey * np.abs(g), rel + 1.1 * 2.0 ** -24
    s = scale * host(c["x"]).astype(np.float64) if c["x"] is not None else 0.0
    u = s + y
    tol = ey + rel * np.abs(y) + 2.0 ** -24 * (np.abs(s) + np.abs(u)) * 1.01
    if c["x_out"].dtype.itemsize == 2:
        tol += 2.0 ** -8 * (np.abs(u) + tol)
    return u, tol


@pytest.mark.parametrize("T, d", [(1, 128), (5, 640), (40, 2048), (7, 2176), (6, 4224), (3, 16384), (1500, 256)])
@pytest.mark.parametrize("stream, gate, post, pairs, seed", [
    ("bfloat16", "none", False, 12, 0), ("float32", "one", True, 4, 1), ("float32", "token", True, 32, 3),
    ("bfloat16", "3", True, 1, 0), ("float32", "none", False, 7, 1)])
def test_experts_rows(torch, lib, T, d, stream, gate, post, pairs, seed):
    c = case(torch, T, d, stream, gate, post, seed=seed, pairs=pairs)
    run(lib, c, 0.5)
    u, tol = join_bound(c, 0.5)
    err = np.abs(host(c["x_out"])[:T] - u)
    assert (err <= tol).all(), f"{(err / tol).max():.3g} of the bound"
    check_after_stream(c, T)


def test_experts_rows_without_a_stream_and_more_pairs_than_lanes(torch, lib):
    c = case(torch, 5, 384, x=False, pairs=150, seed=1)
    run(lib, c)
    u, tol = join_bound(c, 1.0)
    assert (np.abs(host(c["x_out"])[:5] - u) <= tol).all()
    check_after_stream(c, 5)


def test_join_is_the_combine_and_the_norm(torch, lib):
    """Without a norm after, the stream is the combine's with the stream as a residual."""
    c = case(torch, 60, 512, pairs=8, post=False)
    out = torch.empty(60, 512, dtype=torch.bfloat16, device="cuda")
    lib.reflex_combine(c["y_sorted"], c["pair_offsets"], c["pair_to_sorted"], c["pair_weight"], None, out)
    c["x"].zero_()
    run(lib, c)
    assert torch.equal(c["x_out"][:60], out)


def test_pair_arrays_out_of_range_are_clamped(torch, lib):
    c = case(torch, 6, 256, pairs=4)
    c["pair_to_sorted"][:8] = torch.tensor([-5, 1 << 30, -1, 99999, 2, 3, 4, 5], dtype=torch.int32)
    c["pair_offsets"][3] = 1 << 30
    c["pair_offsets"][5] = -7
    run(lib, c)      # (whatever comes out, nothing outside is touched)
    assert (c["x_out"][6:] == 7.0).all() and (c["q_scale"][6:] == 7.0).all()


@pytest.mark.parametrize("seq", [[5, 2, 9, -3], [0, 0, 0, 0], [100, 100, 100, 100], [-4, -3, -2, -1]])
def test_odd_sequence_offsets_stay_inside_the_gate(torch, lib, seq):
    c = case(torch, 6, 256, gate="3")
    c["seq_offsets"].copy_(torch.tensor(seq, dtype=torch.int32))
    run(lib, c)
    gates = [oi.stream(host(c["x"]), host(c["y"]), host(c["w_post"]), np.tile(host(c["gate"])[g], (6, 1)), 1.0, EPS, False)
             for g in range(3)]
    got = host(c["x_out"])[:6]
    assert all(any(np.array_equal(got[i], g[i]) for g in gates) for i in range(6))
