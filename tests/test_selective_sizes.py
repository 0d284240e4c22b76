"""Sizes of the selective leaky block that no launch takes, or that do not fit their
counters, are refused on the host before any launch (no GPU needed; the addresses are never
dereferenced)."""
import ctypes

import pytest

import paper_2211_10725_amd as snn
from tests.test_block_abi import ALIGN, OK, SHAPE

torch = pytest.importorskip("torch")
BIG = 1 << 62


def _sc(T, B, n, width=8):
    S = ctypes.c_int64 * 2
    return snn.ShortconvDesc(T, B, n, width, snn.GATE_SILU, snn.F32, S(B * n, n), S(B * n, n))


def _sc_bwd(d, gw=16, gb=16):
    # a call that is right otherwise stops at grad_state_in's alignment
    return snn.lib().snn_shortconv_bwd(ctypes.byref(d), 16, 16, 16, None, None, 16, None, 16, gw, gb,
                                       17, 16, BIG, None)


@pytest.mark.parametrize("width", [2, 4, 8])
def test_sums_of_the_convolution_of_one_launch(width):
    most = ((1 << 22) - 1) * 64 // (width + 1)  # 16 threads a tap and channel, below 2^32
    assert _sc_bwd(_sc(1, 1, most, width)) == ALIGN
    over = _sc(1, 1, most + 1, width)
    assert _sc_bwd(over) == SHAPE
    assert _sc_bwd(over, gw=None) == SHAPE and _sc_bwd(over, gb=None) == SHAPE
    assert _sc_bwd(over, None, None) == ALIGN  # no sum is launched
    assert snn.lib().snn_shortconv_fwd(ctypes.byref(over), 16, 16, 16, None, None, 16, 17,
                                       None) == ALIGN


def test_channels_of_the_convolution_are_counted_in_32_bits():
    for n, want in ((2 ** 31 - 1, SHAPE), (2 ** 31 - 1023, SHAPE), (2 ** 31 - 1024, ALIGN)):
        d = _sc(1, 1, n)
        got = snn.lib().snn_shortconv_fwd(ctypes.byref(d), 16, 16, 16, None, None, 16, 17, None)
        assert got == want, n
        assert snn.lib().snn_shortconv_step(ctypes.byref(d), 16, 16, None, None, 1, 16, 17, 16,
                                            None) == want
        assert (snn.snn_shortconv_workspace_bytes(d) == 0) == (want == SHAPE)
    assert snn.lib().snn_shortconv_fwd(ctypes.byref(_sc(1, 0, 2 ** 31 - 1024)), 16, 16, 16, None,
                                       None, 16, None, None) == OK


@pytest.mark.parametrize("shape", [((1 << 32) + 5, 2, 8), (2, (1 << 32) + 5, 8), ((1 << 31), 1, 8),
                                   (1, 1, (1 << 32) + 8)], ids=str)
def test_descriptors_refuse_sizes_past_32_bits(shape):
    """The fields would hold what is left of them, and the call do that much."""
    x = torch.empty(shape, device="meta")
    v = torch.empty(*shape[:2], 1, 4, device="meta")
    with pytest.raises(ValueError):
        snn.selscan_desc(x, x, v, v, x, x)
    with pytest.raises(ValueError):
        snn.shortconv_desc(x, x, 4)
    with pytest.raises(ValueError):
        snn.layer_norm_desc(x)
    with pytest.raises(ValueError):
        snn.layer_norm_desc(x, x)


def test_descriptors_refuse_other_fields_past_32_bits():
    x = torch.empty(4, 2, 8)
    with pytest.raises(ValueError):
        snn.shortconv_desc(x, x, (1 << 32) + 4)
    v = torch.empty(4, 2, 1, (1 << 32) + 16, device="meta")
    with pytest.raises(ValueError):
        snn.selscan_desc(x, x, v, v, x)
    v = torch.empty(4, 2, (1 << 32) + 1, 16, device="meta")
    with pytest.raises(ValueError):
        snn.selscan_desc(x, x, v, v, x)
