"""MoELayer8 reads the weights it is given at the time of a forward, and refuses tensors that the C call,
which sees addresses alone, would read past their end or as another type (no GPU needed)."""
import dataclasses
import os

import pytest

_lib = pytest.importorskip("paper_2608_01784_amd._lib")
torch = pytest.importorskip("torch")

from test_abi_fp8 import bf, i32, u8, weights8  # noqa: E402

T, d = 16, 256


class P:
    k_base, delta_role, delta_cur, k_min, k_max = 2, 1, 1, 1, 2
    q, theta, w_cf, v_ref, tau = 0.5, 0.9, 0.5, 0.1, 0.1


@pytest.fixture
def layer():
    from paper_2608_01784_amd.layer import MoELayer8
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libreflex.so is not built (python -m paper_2608_01784_amd.build)")
    return MoELayer8(T, d, weights8(fs=128), P(), uniform_k=2, device="cpu")


def state(**kw):
    from paper_2608_01784_amd.layer import TokenState
    s = TokenState(i32(T), u8(T), torch.zeros(T, dtype=torch.int8), torch.zeros(T), torch.zeros(T), i32(2), i32(1))
    return dataclasses.replace(s, **kw)


@pytest.fixture
def calls(monkeypatch):
    """The structs of the calls that a forward would make."""
    made = []
    monkeypatch.setattr(_lib, "reflex_moe_forward_fp8", lambda args, experts, ws, stream=None: made.append((args, experts)))
    return made


NAMES = [n for n, _ in _lib.Fp8ExpertsC._fields_]


def test_forward_reads_the_weights_it_holds(layer, calls):
    layer.forward(bf(T, d))
    for name in NAMES:
        setattr(layer.w, name, torch.zeros_like(getattr(layer.w, name)))
        layer.forward(bf(T, d))
        got = [getattr(calls[-1][1], n) for n in NAMES]
        assert got == [getattr(layer.w, n).data_ptr() for n in NAMES], name
    layer.w.w_router = torch.zeros(2, d)
    layer.forward(bf(T, d))
    assert calls[-1][0].w_router == layer.w.w_router.data_ptr() and calls[-1][0].w_gate is None
    layer.w.w_up.data = torch.zeros_like(layer.w.w_up)      # (the same tensor with other memory)
    layer.forward(bf(T, d))
    assert calls[-1][1].w_up == layer.w.w_up.data_ptr()
    layer.w = weights8(fs=128)      # (all of them)
    layer.forward(bf(T, d))
    assert [getattr(calls[-1][1], n) for n in NAMES] == [getattr(layer.w, n).data_ptr() for n in NAMES]


@pytest.mark.parametrize("name, bad", [("w_gate", u8(2, 128, 384)), ("ws_down", None), ("s_up", u8(2, 2, 4)),
                                       ("w_router", torch.zeros(2, 128)), ("router_bias", torch.zeros(3)),
                                       ("w_down", bf(2, 256, 128))])
def test_replaced_weights_are_checked(layer, calls, name, bad):
    setattr(layer.w, name, bad)
    with pytest.raises((ValueError, TypeError)):
        layer.forward(bf(T, d))
    assert not calls


def test_weights_of_other_sizes_are_refused(layer, calls):
    for w in (weights8(E=3, fs=128), weights8(f=256, fs=128), weights8()):
        layer.w = w
        with pytest.raises(ValueError, match="made for"):
            layer.forward(bf(T, d))
    assert not calls


@pytest.mark.parametrize("name, bad", [
    ("h", torch.zeros(T, d)), ("h", bf(T - 1, d)), ("h", bf(T, 2 * d)[:, ::2]), ("h", bf(T, 128)),
    ("residual_a", torch.zeros(T, d)), ("residual_b", bf(T + 1, d)), ("out", bf(d, T).t()),
    ("out", torch.zeros(T, d, dtype=torch.float16)), ("k_in", torch.zeros(T, dtype=torch.int64)), ("k_in", i32(T - 1)),
    ("state", state(block_idx=i32(T - 1))), ("state", state(masked=i32(T))), ("state", state(hist_len=i32(T))),
    ("state", state(conf_prev1=torch.zeros(T, dtype=torch.float64))), ("state", state(conf_prev2=torch.zeros(1))),
    ("state", state(seq_offsets=i32(1))), ("state", state(active_block=torch.zeros(1)))])
def test_operands_are_checked(layer, calls, name, bad):
    good = dict(h=bf(T, d), state=state(), k_in=i32(T), residual_a=bf(T, d), residual_b=bf(T, d), out=bf(T, d))
    assert layer.forward(**good) is good["out"] and len(calls) == 1
    with pytest.raises((ValueError, TypeError), match=None if name == "state" else name):
        layer.forward(**dict(good, **{name: bad}))
    assert len(calls) == 1


def test_positions_in_several_dimensions(layer, calls):
    """(sequences, positions, d): what counts is the memory."""
    s = state(block_idx=i32(4, 4), masked=torch.zeros(T, dtype=torch.bool), conf_prev1=torch.zeros(4, 4))
    layer.forward(bf(4, 4, d), s, residual_a=bf(2, 8, d), out=bf(1, T, d))
    assert len(calls) == 1
    with pytest.raises(ValueError, match="rows of"):
        layer.forward(bf(d, T))


def test_host_memory_is_refused(layer):
    with pytest.raises(ValueError, match="device memory"):
        layer.forward(bf(T, d))


def test_layer_is_on_its_weights_device():
    from paper_2608_01784_amd.layer import MoELayer8
    lay = MoELayer8(T, d, weights8(), P(), uniform_k=2)
    assert lay.ws.device == lay.out.device == torch.device("cpu")
    with pytest.raises(ValueError, match="device"):
        MoELayer8(T, d, weights8(), P(), uniform_k=2, device="meta")


def test_layer_without_tokens_has_no_pairs(calls):
    from paper_2608_01784_amd.layer import MoELayer8
    lay = MoELayer8(0, d, weights8(), P(), uniform_k=2)
    lay.pairs.fill_(7)
    lay.forward(bf(0, d))
    assert int(lay.pairs) == 0 and not calls
