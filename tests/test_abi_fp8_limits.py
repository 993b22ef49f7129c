"""Sizes and operands that the 8-bit and token entry points refuse, or are bounded by, on the host
(no GPU needed)."""
import os

import pytest

_lib = pytest.importorskip("paper_2608_01784_amd._lib")
torch = pytest.importorskip("torch")

FAKE = 0x100000
OK, NULL, SHAPE, PARAM, SPACE = 0, -1, -2, -3, -4


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(_lib.LIB_PATH):
        pytest.fail("libreflex.so is not built (python -m paper_2608_01784_amd.build)")
    return _lib.lib()


def test_weights_past_a_launch_are_refused(L):
    # a workgroup of 256 threads a block of 128 x 128, less than 2^32 threads
    assert L.reflex_quantize_fp8_weight(FAKE, 8, 1 << 21, 16384, FAKE, FAKE, None) == SHAPE
    assert L.reflex_quantize_fp8_weight(FAKE, 256, 1 << 24, 16384, FAKE, FAKE, None) == SHAPE


def test_sampling_workspace_is_bounded(L):
    # rows are taken 2^16 at a time
    size, V = L.reflex_sample_workspace_size, 40
    assert 0 < size(1, V) < size(1 << 16, V) == size((1 << 16) + 1, V) == size(1 << 24, V) < 1 << 32


def test_workspaces_that_are_not_dense_are_refused(L):
    def zeros(*shape, dtype=torch.uint8):
        return torch.zeros(shape, dtype=dtype)

    def i32(*shape):
        return zeros(*shape, dtype=torch.int32)
    thin = zeros(1, 64).expand(1 << 20, 64)      # (64 bytes that count as 64 MB)
    S = _lib.fp8_weight_scale_shape
    with pytest.raises(ValueError, match="ws is not contiguous"):
        _lib.reflex_select_rows(zeros(40000), i32(40000), i32(1), thin)
    with pytest.raises(ValueError, match="ws is not contiguous"):
        _lib.reflex_sample_tokens(torch.zeros(4, 100), torch.zeros(4), _lib.SampleParamsC(1, 0, 1, 0), i32(4), ws=thin)
    with pytest.raises(ValueError, match="ws is not contiguous"):
        _lib.reflex_grouped_swiglu_fp8(zeros(4, 128), zeros(*_lib.fp8_scale_shape(4, 128)), i32(8), i32(3),
                                       *(zeros(2, 128, 128) for _ in range(3)), *(zeros(*S(2, 128, 128)) for _ in range(3)),
                                       torch.zeros(8, 128, dtype=torch.bfloat16), thin)
    with pytest.raises(ValueError, match="ws is not contiguous"):
        _lib.reflex_moe_forward_fp8(_lib.MoeArgsC(), _lib.Fp8ExpertsC(), thin)
