"""MoELayerInt8, BlockNorm and the head hand on the tensors they are given, and refuse those that the C call, which sees
addresses alone, would read past their end or as another type (no GPU needed)."""
import os

import pytest

_lib = pytest.importorskip("paper_2608_01784_amd._lib")
torch = pytest.importorskip("torch")

from test_abi_fp8 import bf, i32, u8  # noqa: E402
from test_layer8_host import P, state  # noqa: E402

T, d = 16, 256
NAMES = [n for n, _ in _lib.Int8ExpertsC._fields_]


def i8(*shape):
    return torch.zeros(shape, dtype=torch.int8)


def weights(E=2, f=128, fs=0):
    from paper_2608_01784_amd.layer import ExpertWeightsInt8
    w = dict(w_gate=i8(E, f, d), w_up=i8(E, f, d), w_down=i8(E, d, f), s_gate=torch.zeros(E, f), s_up=torch.zeros(E, f),
             s_down=torch.zeros(E, d), w_router=torch.zeros(E, d))
    if fs:
        w.update(ws_gate=i8(fs, d), ws_up=i8(fs, d), ws_down=i8(d, fs), ss_gate=torch.zeros(fs), ss_up=torch.zeros(fs),
                 ss_down=torch.zeros(d))
    return ExpertWeightsInt8(**w)


@pytest.fixture
def layer():
    from paper_2608_01784_amd.layer import MoELayerInt8
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libreflex.so is not built (python -m paper_2608_01784_amd.build)")
    return MoELayerInt8(T, d, weights(fs=128), P(), uniform_k=2)


@pytest.fixture
def calls(monkeypatch):
    """The arguments of the calls that a forward would make."""
    made = []
    monkeypatch.setattr(_lib, "reflex_moe_forward_int8", lambda args, experts, ws, h_q=None, h_scale=None, join=None,
                        stream=None: made.append((args, experts, h_q, h_scale, join)))
    return made


def test_expert_weights_check():
    w = weights(fs=128)
    assert (w.E, w.f, w.f_shared) == (2, 128, 128)
    w.check(d)
    for name, bad, error in [("w_up", i8(2, 128, 384), ValueError), ("w_down", u8(2, d, 128), TypeError),
                             ("s_down", torch.zeros(2, 128), ValueError), ("s_gate", None, ValueError),
                             ("s_up", torch.zeros(2, 128, dtype=torch.float64), TypeError), ("ss_up", None, ValueError),
                             ("ss_down", torch.zeros(d, 1), ValueError), ("ws_down", i8(128, d).t(), ValueError)]:
        w = weights(fs=128)
        setattr(w, name, bad)
        with pytest.raises(error, match="ExpertWeightsInt8"):
            w.check(d)


def test_forward_reads_the_weights_it_holds(layer, calls):
    for name in NAMES:
        setattr(layer.w, name, torch.zeros_like(getattr(layer.w, name)))
        layer.forward(bf(T, d))
        assert [getattr(calls[-1][1], n) for n in NAMES] == [getattr(layer.w, n).data_ptr() for n in NAMES], name
        assert isinstance(calls[-1][1], _lib.Int8ExpertsC) and calls[-1][0].w_gate is None
    layer.w = weights(f=256, fs=128)
    with pytest.raises(ValueError, match="made for"):
        layer.forward(bf(T, d))


def norm(**kw):
    from paper_2608_01784_amd.layer import BlockNorm
    return BlockNorm(T, d, torch.ones(d), torch.ones(d), **kw)


def test_join_in_place_of_the_combine(layer, calls):
    x, n, q, s = bf(T, d), norm(), i8(T, d), torch.zeros(T)
    assert layer.forward(bf(T, d), h_q=q, h_scale=s, join=n.arrays(x)) is n.n
    args, _, got_q, got_s, join = calls[-1]
    assert args.out is None and got_q is q and got_s is s
    assert (join.x, join.x_out, join.n_out, join.q_out, join.q_scale) == tuple(
        t.data_ptr() for t in (x, x, n.n, n.q, n.scale))
    assert (join.T, join.d, join.gate_rows, join.residual_scale) == (T, d, 0, 1.0) and join.y is None is join.y_sorted
    y = bf(T, d)
    stream_alone = dict(x=x, x_out=y, eps=1e-6)
    assert layer.forward(bf(T, d), join=stream_alone) is y
    n = len(calls)
    for error, kw in [(ValueError, dict(out=bf(T, d))), (ValueError, dict(residual_a=bf(T, d))),
                      (ValueError, dict(join=dict(stream_alone, x=bf(T - 1, d), x_out=bf(T - 1, d)))),
                      (TypeError, dict(join=dict(stream_alone, x=torch.zeros(T, d)))),
                      (ValueError, dict(join=dict(stream_alone, gate=bf(2, d), seq_offsets=i32(2)))),
                      (TypeError, dict(h=torch.zeros(T, d)))]:
        with pytest.raises(error):
            layer.forward(**dict(dict(h=bf(T, d), join=stream_alone), **kw))
    assert len(calls) == n


def test_rows_in_8_bits_are_checked(layer):
    for error, kw in [(TypeError, dict(h_q=u8(T, d), h_scale=torch.zeros(T))), (ValueError, dict(h_q=i8(T, 128), h_scale=torch.zeros(T))),
                      (ValueError, dict(h_q=i8(T, d), h_scale=torch.zeros(T - 1))),
                      (TypeError, dict(h_q=i8(T, d), h_scale=torch.zeros(T, dtype=torch.float64))),
                      (ValueError, dict(h_q=i8(T, d), h_scale=torch.zeros(T)))]:      # (the last: host memory)
        with pytest.raises(error):
            layer.forward(bf(T, d), **kw)


def test_layer_without_tokens_has_no_pairs(calls):
    from paper_2608_01784_amd.layer import MoELayerInt8
    lay = MoELayerInt8(0, d, weights(), P(), uniform_k=2)
    lay.pairs.fill_(7)
    lay.forward(bf(0, d))
    assert int(lay.pairs) == 0 and not calls


def test_operands_are_checked(layer, calls):
    good = dict(h=bf(T, d), state=state(), k_in=i32(T), residual_a=bf(T, d), residual_b=bf(T, d), out=bf(T, d))
    assert layer.forward(**good) is good["out"] and len(calls) == 1
    for name, bad in [("h", bf(T - 1, d)), ("residual_b", bf(T + 1, d)), ("out", torch.zeros(T, d)), ("k_in", i32(T - 1)),
                      ("state", state(masked=i32(T)))]:
        with pytest.raises((ValueError, TypeError)):
            layer.forward(**dict(good, **{name: bad}))
    assert len(calls) == 1


def test_block_norm_hands_on_its_arrays(monkeypatch):
    made = []
    monkeypatch.setattr(_lib, "reflex_block_norm", lambda **kw: made.append(kw))
    n, x, y, g = norm(residual_scale=0.5, eps=1e-3), bf(T, d), bf(T, d), bf(1, d)
    assert n.forward(x, y, gate=g) is n.n
    kw = made[-1]
    assert kw["x"] is x is kw["x_out"] and kw["y"] is y and kw["gate"] is g and kw["q_out"] is n.q and kw["q_scale"] is n.scale
    assert (kw["eps"], kw["residual_scale"]) == (1e-3, 0.5)
    n.start(x)
    assert "x_out" not in made[-1] and made[-1]["n_out"] is n.n and "residual_scale" not in made[-1]
    from paper_2608_01784_amd.layer import BlockNorm
    alone = BlockNorm(T, d, None, torch.ones(d))
    assert alone.forward(x, y) is None and made[-1]["n_out"] is None is made[-1]["q_out"]
    assert norm(quantize=False).q is None


def test_head_takes_integer_weights(monkeypatch):
    from paper_2608_01784_amd.head import TokenHead
    head = TokenHead(T, (i8(40, d), torch.zeros(40)))
    assert head.q.dtype == torch.int8 and head.scale.shape == (T,)
    made = []
    for name in ("reflex_select_rows", "reflex_quantize_int8", "reflex_matmul_int8", "reflex_sample_tokens"):
        monkeypatch.setattr(_lib, name, lambda *a, name=name, **kw: made.append(name))
    head.forward(bf(T, d), u8(T), torch.zeros(T))
    assert made == ["reflex_select_rows", "reflex_quantize_int8", "reflex_matmul_int8", "reflex_sample_tokens"]
