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
