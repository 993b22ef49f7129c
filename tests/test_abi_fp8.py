"""The 8-bit, masked-row and token entry points reject invalid arguments on the host before
launching anything, and the binding what the C call cannot see (so these run without a GPU)."""
import ctypes
import math
import os

import pytest

_lib = pytest.importorskip("paper_2608_01784_amd._lib")
torch = pytest.importorskip("torch")

FAKE, ODD, MIS2, MIS4, MIS8 = 0x100000, 0x100001, 0x100002, 0x100004, 0x100008
NULL, SHAPE, PARAM, SPACE = -1, -2, -3, -4
MAX_T, MAX_D, MAX_E, MAX_V = 1 << 24, 16384, 256, 1 << 20


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


def test_struct_layouts(L):
    assert L.reflex_sizeof_fp8_experts() == ctypes.sizeof(_lib.Fp8ExpertsC) == 12 * ctypes.sizeof(ctypes.c_void_p)
    assert L.reflex_sizeof_sample_params() == ctypes.sizeof(_lib.SampleParamsC) == 16


def test_sizes(L):
    assert L.reflex_fp8_scale_bytes(5, 640) == math.prod(_lib.fp8_scale_shape(5, 640)) == 2 * 5 * 4
    assert L.reflex_fp8_weight_scale_bytes(130, 512) == math.prod(_lib.fp8_weight_scale_shape(130, 512)) == 2 * 4
    assert _lib.fp8_weight_scale_shape(7, 130, 640) == (7, 2, 8)
    for f in (L.reflex_fp8_scale_bytes, L.reflex_fp8_weight_scale_bytes):
        assert f(-1, 128) == f(1, 64) == f(1, 0) == f(1, MAX_D + 128) == 0
    assert L.reflex_select_rows_workspace_size(1000) == 0 < L.reflex_select_rows_workspace_size(1 << 20)
    assert L.reflex_sample_workspace_size(3, 0) == L.reflex_sample_workspace_size(3, MAX_V + 1) == 0
    assert 0 < L.reflex_sample_workspace_size(1, 1) <= L.reflex_sample_workspace_size(9, MAX_V)
    assert L.reflex_swiglu_fp8_workspace_size(100, 8, 256) >= 100 * 256 + 100 * 4
    assert L.reflex_swiglu_fp8_workspace_size(100, 8, 192) == L.reflex_swiglu_fp8_workspace_size(-1, 8, 256) == 0
    assert 0 < L.reflex_workspace_fp8_size(16, 8, 256, 128, 0, 4) < L.reflex_workspace_fp8_size(16, 8, 256, 128, 128, 4)
    assert L.reflex_workspace_fp8_size(16, 8, 256, 192, 0, 4) == 0
    assert L.reflex_workspace_fp8_size(16, 8, 256, 128, 192, 4) == 0


def test_select_rows_validation(L):
    T = 1 << 20
    need = L.reflex_select_rows_workspace_size(T)
    good = [FAKE, T, FAKE, FAKE, FAKE, need, None]
    refuses(L.reflex_select_rows, good, [
        (0, None, NULL), (2, None, NULL), (3, None, NULL), (4, None, NULL), (2, MIS2, SHAPE), (3, ODD, SHAPE),
        (4, MIS8, SHAPE), (1, -1, SHAPE), (1, MAX_T * 2, SHAPE), (5, need - 1, SPACE)])


def test_quantize_validation(L):
    good = [FAKE, FAKE, FAKE, 64, 32, 256, FAKE, FAKE, None]
    refuses(L.reflex_quantize_fp8, good, [
        (0, None, NULL), (6, None, NULL), (7, None, NULL), (0, MIS8, SHAPE), (6, MIS4, SHAPE), (7, MIS2, SHAPE),
        (1, MIS2, SHAPE), (2, ODD, SHAPE), (3, -1, SHAPE), (4, -1, SHAPE), (5, 192, SHAPE), (5, 0, SHAPE),
        (5, MAX_D + 128, SHAPE)])
    assert L.reflex_quantize_fp8(FAKE, None, None, 31, 32, 256, FAKE, FAKE, None) == SHAPE     # too few rows
    assert L.reflex_quantize_fp8(*with_arg(good, 4, 0)) == 0
    good = [FAKE, 8, 256, 256, FAKE, FAKE, None]
    refuses(L.reflex_quantize_fp8_weight, good, [
        (0, None, NULL), (4, None, NULL), (5, None, NULL), (0, MIS8, SHAPE), (5, ODD, SHAPE), (1, 0, SHAPE),
        (1, MAX_E + 1, SHAPE), (2, -1, SHAPE), (3, 130, SHAPE)])
    assert L.reflex_quantize_fp8_weight(*with_arg(good, 2, 0)) == 0


def test_matmul_validation(L):
    good = [FAKE, FAKE, FAKE, FAKE, FAKE, 32, 256, 256, _lib.TYPE_F32, FAKE, None]
    refuses(L.reflex_matmul_fp8, good, [
        (0, None, NULL), (1, None, NULL), (2, None, NULL), (3, None, NULL), (9, None, NULL), (0, MIS8, SHAPE),
        (1, MIS2, SHAPE), (2, MIS4, SHAPE), (3, ODD, SHAPE), (4, MIS2, SHAPE), (9, MIS8, SHAPE), (5, -1, SHAPE),
        (6, -1, SHAPE), (7, 64, SHAPE), (7, MAX_D + 128, SHAPE), (8, 2, PARAM), (8, -1, PARAM)])
    assert L.reflex_matmul_fp8(*with_arg(good, 5, 0)) == L.reflex_matmul_fp8(*with_arg(good, 6, 0)) == 0


def test_grouped_swiglu_validation(L):
    cap, E, f = 64, 8, 128
    need = L.reflex_swiglu_fp8_workspace_size(cap, E, f)
    good = [FAKE] * 10 + [16, E, 256, f, cap, FAKE, FAKE, need, None]
    refuses(L.reflex_grouped_swiglu_fp8, good, [(i, None, NULL) for i in (*range(10), 15, 16)] + [
        (0, MIS8, SHAPE), (1, MIS2, SHAPE), (2, MIS2, SHAPE), (3, MIS2, SHAPE), (4, MIS8, SHAPE), (7, ODD, SHAPE),
        (15, MIS8, SHAPE), (16, MIS8, SHAPE), (10, -1, SHAPE), (11, 0, SHAPE), (11, MAX_E + 1, SHAPE),
        (12, 192, SHAPE), (13, 192, SHAPE), (14, -1, SHAPE), (17, need - 1, SPACE)])
    assert L.reflex_grouped_swiglu_fp8(*with_arg(good, 14, 0)) == 0


def moe_args(**kw):
    a = _lib.MoeArgsC()
    a.T, a.d, a.E, a.f, a.f_shared, a.norm_topk, a.uniform_k, a.B = 16, 256, 8, 128, 0, 1, 2, 0
    a.h = a.w_router = a.out = FAKE
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_moe_forward_validation(L):
    need = L.reflex_workspace_fp8_size(16, 8, 256, 128, 0, 2)
    names = [n for n, _ in _lib.Fp8ExpertsC._fields_]
    experts = _lib.Fp8ExpertsC(*[FAKE] * 6)

    def call(a=None, x=experts, ws=FAKE, n=need):
        return L.reflex_moe_forward_fp8(ctypes.byref(moe_args() if a is None else a),
                                        None if x is None else ctypes.byref(x), ws, n, None)
    assert call(n=need - 1) == SPACE
    assert L.reflex_moe_forward_fp8(None, ctypes.byref(experts), FAKE, need, None) == NULL
    assert call(x=None) == call(ws=None) == call(moe_args(h=None)) == NULL
    for i, name in enumerate(names[:6]):
        assert call(x=_lib.Fp8ExpertsC(*with_arg([FAKE] * 6, i, None))) == NULL, name
        assert call(x=_lib.Fp8ExpertsC(*with_arg([FAKE] * 6, i, MIS2))) == SHAPE, name
    big = 1 << 30
    for i, name in enumerate(names):
        both = moe_args(f_shared=128)
        assert call(both, _lib.Fp8ExpertsC(*with_arg([FAKE] * 12, i, None)), n=big) == NULL, name
    assert call(moe_args(f=192), n=big) == SHAPE
    assert call(moe_args(f_shared=192), _lib.Fp8ExpertsC(*[FAKE] * 12), n=big) == SHAPE
    assert call(moe_args(d=200), n=big) == call(moe_args(uniform_k=9), n=big) == SHAPE
    assert call(moe_args(norm_topk=2)) == PARAM
    assert call(moe_args(T=0)) == 0


def test_sample_validation(L):
    M, V, T = 8, 1000, 32
    need = L.reflex_sample_workspace_size(M, V)
    P = _lib.SampleParamsC

    def call(i=None, value=None, params=P(1.0, 0, 1.0, 0.0)):
        good = [FAKE, _lib.TYPE_F32, FAKE, FAKE, M, V, FAKE, ctypes.byref(params), T, FAKE, FAKE, FAKE, need, None]
        return L.reflex_sample_tokens(*(good if i is None else with_arg(good, i, value)))
    for i, value, rc in [(0, None, NULL), (6, None, NULL), (7, None, NULL), (9, None, NULL), (11, None, NULL),
                         (0, MIS2, SHAPE), (2, MIS2, SHAPE), (3, ODD, SHAPE), (6, MIS2, SHAPE), (9, MIS2, SHAPE),
                         (10, ODD, SHAPE), (11, MIS8, SHAPE), (1, 2, PARAM), (4, -1, SHAPE), (5, 0, SHAPE),
                         (5, MAX_V + 1, SHAPE), (8, -1, SHAPE), (12, need - 1, SPACE)]:
        assert call(i, value) == rc, (i, value)
    nan, inf = float("nan"), float("inf")
    for bad in [P(-1.0, 0, 1.0, 0.0), P(inf, 0, 1.0, 0.0), P(nan, 0, 1.0, 0.0), P(1.0, -1, 1.0, 0.0),
                P(1.0, 0, 0.0, 0.0), P(1.0, 0, 1.1, 0.0), P(1.0, 0, nan, 0.0), P(1.0, 0, 1.0, -0.1),
                P(1.0, 0, 1.0, 1.5), P(1.0, 0, 1.0, nan)]:
        assert call(params=bad) == PARAM
    assert call(4, 0) == call(8, 0) == 0


# ---- the binding -------------------------------------------------------------------------------
def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_binding_checks_types_shapes_and_density(L):
    rows, n = i32(16), i32(1)
    with pytest.raises(TypeError):
        _lib.reflex_select_rows(i32(16), rows, n)
    with pytest.raises(ValueError, match="rows"):
        _lib.reflex_select_rows(u8(16), i32(15), n)
    with pytest.raises(ValueError, match="contiguous"):
        _lib.reflex_select_rows(u8(32)[::2], rows, n)
    q, s = u8(4, 256), u8(*_lib.fp8_scale_shape(4, 256))
    with pytest.raises(TypeError):
        _lib.reflex_quantize_fp8(torch.zeros(4, 256), q, s)
    with pytest.raises(ValueError, match="scale"):
        _lib.reflex_quantize_fp8(bf(4, 256), q, u8(4, 4))
    with pytest.raises(ValueError, match="listed"):
        _lib.reflex_quantize_fp8(bf(9, 256), q, s, rows=i32(3))
    with pytest.raises(ValueError, match="w has shape"):
        _lib.reflex_quantize_fp8_weight(bf(256), u8(256), u8(4))
    with pytest.raises(ValueError, match="w_scale"):
        _lib.reflex_matmul_fp8(q, s, u8(130, 256), u8(1, 4), bf(4, 130))
    with pytest.raises(ValueError, match="out has shape"):
        _lib.reflex_matmul_fp8(q, s, u8(130, 256), u8(2, 4), bf(4, 131))
    with pytest.raises(TypeError, match="out"):
        _lib.reflex_matmul_fp8(q, s, u8(130, 256), u8(2, 4), torch.zeros(4, 130, dtype=torch.float16))
    with pytest.raises(ValueError, match="u has shape"):
        _lib.reflex_sample_tokens(bf(4, 100), torch.zeros(5), _lib.SampleParamsC(1, 0, 1, 0), i32(4))
    with pytest.raises(TypeError, match="tokens"):
        _lib.reflex_sample_tokens(bf(4, 100), torch.zeros(4), _lib.SampleParamsC(1, 0, 1, 0), torch.zeros(4).long())


def test_binding_refuses_host_memory(L):
    with pytest.raises(ValueError, match="device memory"):
        _lib.reflex_select_rows(u8(16), i32(16), i32(1))
    with pytest.raises(ValueError, match="device memory"):
        _lib.reflex_quantize_fp8(bf(4, 256), u8(4, 256), u8(*_lib.fp8_scale_shape(4, 256)))
    with pytest.raises(ValueError, match="device memory"):
        _lib.reflex_sample_tokens(bf(4, 100), torch.zeros(4), _lib.SampleParamsC(1, 0, 1, 0), i32(4))


def weights8(E=2, f=128, d=256, fs=0):
    from paper_2608_01784_amd.layer import ExpertWeights8
    S = _lib.fp8_weight_scale_shape
    w = dict(w_gate=u8(E, f, d), w_up=u8(E, f, d), w_down=u8(E, d, f), s_gate=u8(*S(E, f, d)), s_up=u8(*S(E, f, d)),
             s_down=u8(*S(E, d, f)), w_router=torch.zeros(E, d))
    if fs:
        w.update(ws_gate=u8(fs, d), ws_up=u8(fs, d), ws_down=u8(d, fs), ss_gate=u8(*S(fs, d)), ss_up=u8(*S(fs, d)),
                 ss_down=u8(*S(d, fs)))
    return ExpertWeights8(**w)


def test_expert_weights_check():
    w = weights8(fs=128)
    assert (w.E, w.f, w.f_shared) == (2, 128, 128)
    w.check(256)
    for name, bad, error in [("w_up", u8(2, 128, 384), ValueError), ("w_down", torch.zeros(2, 256, 128), TypeError),
                             ("s_down", u8(2, 1, 4), ValueError), ("s_gate", None, ValueError),
                             ("ss_up", None, ValueError), ("ws_down", u8(128, 256).t(), ValueError)]:
        w = weights8(fs=128)
        setattr(w, name, bad)
        with pytest.raises(error):
            w.check(256)
