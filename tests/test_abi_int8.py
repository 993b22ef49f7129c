"""The 8-bit integer and block-norm entry points reject invalid arguments on the host before launching
anything, and the binding what the C call cannot see (so these run without a GPU)."""
import ctypes
import os

import pytest

_lib = pytest.importorskip("paper_2608_01784_amd._lib")
torch = pytest.importorskip("torch")

FAKE, ODD, MIS2, MIS4, MIS8 = 0x100000, 0x100001, 0x100002, 0x100004, 0x100008
NULL, SHAPE, PARAM, SPACE = -1, -2, -3, -4
MAX_T, MAX_D, MAX_E = 1 << 24, 16384, 256


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libreflex.so is not built (python -m paper_2608_01784_amd.build)")
    return _lib.lib()


def with_arg(good, i, value):
    return good[:i] + [value] + good[i + 1:]


def refuses(f, good, cases):
    for i, value, rc in cases:
        assert f(*with_arg(good, i, value)) == rc, (i, value)


def test_struct_layouts_and_sizes(L):
    assert L.reflex_sizeof_int8_experts() == ctypes.sizeof(_lib.Int8ExpertsC) == 12 * ctypes.sizeof(ctypes.c_void_p)
    assert L.reflex_sizeof_norm_args() == ctypes.sizeof(_lib.NormArgsC) == 32 + 16 * ctypes.sizeof(ctypes.c_void_p)
    assert L.reflex_swiglu_int8_workspace_size(100, 8, 256) >= 100 * 256 * 3 + 100 * 4
    assert L.reflex_swiglu_int8_workspace_size(0, 8, 256) > 0
    assert L.reflex_swiglu_int8_workspace_size(100, 8, 192) == L.reflex_swiglu_int8_workspace_size(-1, 8, 256) == 0
    assert 0 < L.reflex_workspace_int8_size(16, 8, 256, 128, 0, 4) < L.reflex_workspace_int8_size(16, 8, 256, 128, 128, 4)
    assert L.reflex_workspace_int8_size(16, 8, 256, 192, 0, 4) == L.reflex_workspace_int8_size(16, 8, 256, 128, 192, 4) == 0


def test_quantize_validation(L):
    good = [FAKE, FAKE, FAKE, 64, 32, 256, FAKE, FAKE, None]
    refuses(L.reflex_quantize_int8, good, [
        (0, None, NULL), (6, None, NULL), (7, None, NULL), (0, MIS8, SHAPE), (6, MIS4, SHAPE), (7, MIS2, SHAPE),
        (1, MIS2, SHAPE), (2, ODD, SHAPE), (3, -1, SHAPE), (3, MAX_T + 1, SHAPE), (4, -1, SHAPE), (5, 192, SHAPE),
        (5, 0, SHAPE), (5, MAX_D + 128, SHAPE)])
    assert L.reflex_quantize_int8(FAKE, None, None, 31, 32, 256, FAKE, FAKE, None) == SHAPE     # too few rows
    assert L.reflex_quantize_int8(*with_arg(good, 4, 0)) == 0
    good = [FAKE, 8, 256, 256, FAKE, FAKE, None]
    refuses(L.reflex_quantize_int8_weight, good, [
        (0, None, NULL), (4, None, NULL), (5, None, NULL), (0, MIS8, SHAPE), (5, ODD, SHAPE), (1, 0, SHAPE),
        (1, MAX_E + 1, SHAPE), (2, -1, SHAPE), (3, 130, SHAPE)])
    assert L.reflex_quantize_int8_weight(FAKE, 128, MAX_T, 128, FAKE, FAKE, None) == SHAPE      # 2^31 rows
    assert L.reflex_quantize_int8_weight(*with_arg(good, 2, 0)) == 0


def test_matmul_validation(L):
    good = [FAKE, FAKE, FAKE, FAKE, FAKE, 32, 256, 256, _lib.TYPE_F32, FAKE, None]
    refuses(L.reflex_matmul_int8, good, [
        (0, None, NULL), (1, None, NULL), (2, None, NULL), (3, None, NULL), (9, None, NULL), (0, MIS8, SHAPE),
        (1, MIS2, SHAPE), (2, MIS4, SHAPE), (3, ODD, SHAPE), (4, MIS2, SHAPE), (9, MIS8, SHAPE), (5, -1, SHAPE),
        (6, -1, SHAPE), (7, 64, SHAPE), (7, MAX_D + 128, SHAPE), (8, 2, PARAM), (8, -1, PARAM)])
    assert L.reflex_matmul_int8(*with_arg(good, 5, 0)) == L.reflex_matmul_int8(*with_arg(good, 6, 0)) == 0


def test_grouped_swiglu_validation(L):
    cap, E, f = 64, 8, 128
    need = L.reflex_swiglu_int8_workspace_size(cap, E, f)
    good = [FAKE] * 10 + [16, E, 256, f, cap, FAKE, FAKE, need, None]
    refuses(L.reflex_grouped_swiglu_int8, good, [(i, None, NULL) for i in (*range(10), 15, 16)] + [
        (0, MIS8, SHAPE), (1, MIS2, SHAPE), (2, MIS2, SHAPE), (3, MIS2, SHAPE), (4, MIS8, SHAPE), (7, ODD, SHAPE),
        (15, MIS8, SHAPE), (16, MIS8, SHAPE), (10, -1, SHAPE), (11, 0, SHAPE), (11, MAX_E + 1, SHAPE),
        (12, 192, SHAPE), (13, 192, SHAPE), (14, -1, SHAPE), (17, need - 1, SPACE)])
    assert L.reflex_grouped_swiglu_int8(*with_arg(good, 14, 0)) == 0


def norm(**kw):
    a = _lib.NormArgsC(T=16, d=256, eps=1e-6, residual_scale=1.0)
    a.x = a.x_out = FAKE
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


PAIRS = dict(y_sorted=FAKE, pair_offsets=FAKE, pair_to_sorted=FAKE, pair_weight=FAKE, pair_capacity=64)


@pytest.mark.parametrize("rc, kw", [
    (NULL, dict(x=None)), (NULL, dict(x_out=None)), (NULL, dict(n_out=FAKE)), (NULL, dict(q_out=FAKE, q_scale=FAKE)),
    (NULL, dict(q_out=FAKE, w_pre=FAKE)), (NULL, dict(q_scale=FAKE, w_pre=FAKE)), (NULL, dict(y=FAKE, seq_offsets=FAKE)),
    (NULL, {**PAIRS, "pair_offsets": None}), (NULL, {**PAIRS, "pair_to_sorted": None}), (NULL, {**PAIRS, "y_sorted": None}),
    (NULL, {**PAIRS, "pair_weight": None}),
    (PARAM, {**PAIRS, "y": FAKE}), (PARAM, dict(y=FAKE, shared_y=FAKE)), (PARAM, dict(w_post=FAKE)),
    (PARAM, dict(gate=FAKE, gate_rows=1)), (PARAM, dict(stream_type=2)), (PARAM, dict(stream_type=-1)), (PARAM, dict(eps=0.0)), (PARAM, dict(reserved=1)),
    (PARAM, dict(eps=-1e-6)), (PARAM, dict(eps=float("nan"))), (PARAM, dict(eps=float("inf"))),
    (PARAM, dict(residual_scale=float("inf"))), (PARAM, dict(residual_scale=float("nan"))),
    (SHAPE, dict(T=-1)), (SHAPE, dict(T=MAX_T + 1)), (SHAPE, dict(d=192)), (SHAPE, dict(d=0)), (SHAPE, dict(d=MAX_D + 128)),
    (SHAPE, {**PAIRS, "pair_capacity": -1}), (SHAPE, dict(y=FAKE, gate=FAKE, gate_rows=0)),
    (SHAPE, dict(y=FAKE, gate=FAKE, gate_rows=2)), (SHAPE, dict(y=FAKE, gate=FAKE, gate_rows=-1, seq_offsets=FAKE)),
    (SHAPE, dict(x=MIS8)), (SHAPE, dict(x_out=MIS8)), (SHAPE, dict(y=MIS8)), (SHAPE, dict(y=FAKE, w_post=MIS4)),
    (SHAPE, dict(w_pre=MIS8, n_out=FAKE)), (SHAPE, dict(w_pre=FAKE, n_out=MIS8)), (SHAPE, dict(y=FAKE, gate=MIS8, gate_rows=1)),
    (SHAPE, dict(w_pre=FAKE, q_out=MIS8, q_scale=FAKE)), (SHAPE, dict(w_pre=FAKE, q_out=FAKE, q_scale=MIS2)),
    (SHAPE, {**PAIRS, "y_sorted": MIS8}), (SHAPE, {**PAIRS, "shared_y": MIS8}), (SHAPE, {**PAIRS, "pair_weight": MIS2}),
    (SHAPE, dict(n_rows=ODD)), (SHAPE, dict(y=FAKE, gate=FAKE, gate_rows=2, seq_offsets=MIS2)),
])
def test_block_norm_validation(L, rc, kw):
    assert L.reflex_block_norm(norm(**kw), None) == rc


def test_block_norm_of_nothing(L):
    assert L.reflex_block_norm(None, None) == NULL
    assert L.reflex_block_norm(norm(T=0), None) == 0


def moe_args(**kw):
    a = _lib.MoeArgsC()
    a.T, a.d, a.E, a.f, a.f_shared, a.norm_topk, a.uniform_k, a.B = 16, 256, 8, 128, 0, 1, 2, 0
    a.h = a.w_router = a.out = FAKE
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_moe_forward_validation(L):
    need = L.reflex_workspace_int8_size(16, 8, 256, 128, 0, 2)
    names = [n for n, _ in _lib.Int8ExpertsC._fields_]
    experts = _lib.Int8ExpertsC(*[FAKE] * 6)

    def call(a=None, x=experts, q=None, s=None, join=None, ws=FAKE, n=need):
        return L.reflex_moe_forward_int8(ctypes.byref(moe_args() if a is None else a),
                                         None if x is None else ctypes.byref(x), q, s, join, ws, n, None)
    assert call(n=need - 1) == SPACE
    assert L.reflex_moe_forward_int8(None, ctypes.byref(experts), None, None, None, FAKE, need, None) == NULL
    assert call(x=None) == call(ws=None) == call(moe_args(h=None)) == call(moe_args(out=None)) == NULL
    for i, name in enumerate(names[:6]):
        assert call(x=_lib.Int8ExpertsC(*with_arg([FAKE] * 6, i, None))) == NULL, name
        assert call(x=_lib.Int8ExpertsC(*with_arg([FAKE] * 6, i, MIS2))) == SHAPE, name
    assert call(q=FAKE) == call(s=FAKE) == NULL
    assert call(q=MIS8, s=FAKE) == call(q=FAKE, s=MIS2) == SHAPE
    assert call(moe_args(f=192)) == SHAPE
    need_shared = L.reflex_workspace_int8_size(16, 8, 256, 128, 128, 2)
    assert call(moe_args(f_shared=128), n=need_shared) == NULL
    # a join instead of the combine
    free = moe_args(out=None)
    assert call(join=norm()) == call(moe_args(out=None, residual_a=FAKE), join=norm()) == PARAM
    assert call(free, join=norm(T=15)) == call(free, join=norm(d=128)) == call(free, join=norm(y=FAKE)) == PARAM
    assert call(free, join=norm(**PAIRS)) == call(free, join=norm(shared_y=FAKE)) == PARAM
    assert call(free, join=norm(x_out=None)) == NULL
    assert call(free, join=norm(x_out=MIS8)) == SHAPE
    assert call(free, join=norm(), n=need - 1) == SPACE


def test_binding_checks():
    def zeros(*shape, dtype=torch.int8):
        return torch.zeros(shape, dtype=dtype)
    f32, i32, b16 = torch.float32, torch.int32, torch.bfloat16
    x, q, s = zeros(4, 128, dtype=b16), zeros(4, 128), zeros(4, dtype=f32)
    with pytest.raises(ValueError, match="device memory"):
        _lib.reflex_quantize_int8(x, q, s)
    for bad in (dict(x=x.float()), dict(q=q.view(torch.uint8)), dict(scale=s.double())):
        with pytest.raises(TypeError):
            _lib.reflex_quantize_int8(**{**dict(x=x, q=q, scale=s), **bad})
    for bad in (dict(x=zeros(4, 256, dtype=b16)), dict(scale=zeros(5, dtype=f32)), dict(rows=zeros(3, dtype=i32)),
                dict(n_rows=zeros(2, dtype=i32)), dict(x=zeros(4, 256, dtype=b16)[:, ::2])):
        with pytest.raises(ValueError):
            _lib.reflex_quantize_int8(**{**dict(x=x, q=q, scale=s), **bad})
    with pytest.raises(ValueError, match="scale"):
        _lib.reflex_quantize_int8_weight(zeros(2, 4, 128, dtype=b16), zeros(2, 4, 128), zeros(2, dtype=f32))
    with pytest.raises(ValueError, match="w_scale"):
        _lib.reflex_matmul_int8(q, s, zeros(7, 128), zeros(8, dtype=f32), zeros(4, 7, dtype=f32))
    with pytest.raises(TypeError, match="out"):
        _lib.reflex_matmul_int8(q, s, zeros(7, 128), zeros(7, dtype=f32), zeros(4, 7, dtype=torch.float16))
    w, o = zeros(128, dtype=f32), zeros(4, 128, dtype=b16)
    for error, kw in ((ValueError, dict()), (ValueError, dict(x=x, y=zeros(5, 128, dtype=b16), x_out=o)),
                      (TypeError, dict(x=x, x_out=o.float())), (TypeError, dict(x=x.half(), x_out=o.half())),
                      (ValueError, dict(x=x, x_out=o, w_pre=zeros(64, dtype=f32), n_out=o)),
                      (TypeError, dict(x=x, x_out=o, w_pre=zeros(128, dtype=b16), n_out=o)),
                      (TypeError, dict(x=x, w_pre=w, q_out=zeros(4, 128, dtype=torch.uint8), q_scale=s)),
                      (ValueError, dict(x=x, w_pre=w, q_out=q, q_scale=zeros(3, dtype=f32))),
                      (ValueError, dict(x=x, y=x, gate=zeros(2, 128, dtype=b16), seq_offsets=zeros(2, dtype=i32), x_out=o)),
                      (ValueError, dict(x=zeros(128, dtype=b16), x_out=zeros(128, dtype=b16)))):
        with pytest.raises(error):
            _lib.reflex_block_norm(**kw, eps=1e-6)
    with pytest.raises(TypeError):
        _lib.reflex_block_norm(x=x, x_out=o)      # (eps has no default)
