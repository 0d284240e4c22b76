"""Sizes that no launch takes are refused on the host (no GPU needed; the
addresses are never dereferenced)."""
import ctypes

import pytest

import paper_2211_10725_amd as snn

torch = pytest.importorskip("torch")
OK, NULL, SHAPE, DTYPE, ALIGN = range(5)


def _desc(T, B, H, KV, dk=8, dv=8):
    S = ctypes.c_int64 * 3
    return snn.LinattnDesc(T, B, H, KV, dk, dv, snn.F32, 1.0, S(B * H * dk, H * dk, dk),
                           S(B * KV * dk, KV * dk, dk), S(B * KV * dv, KV * dv, dv),
                           S(B * H * dv, H * dv, dv))


def _calls(d):
    """The three calls, which stop at a misaligned state where nothing else is wrong."""
    L, big = snn.lib(), 1 << 62
    return (L.snn_linattn_fwd(ctypes.byref(d), 16, 16, 16, 16, None, None, 16, 17, 16, big, None),
            L.snn_linattn_bwd(ctypes.byref(d), 16, 16, 16, 16, None, None, 16, None, 16, 16, 16,
                              17, 16, big, None),
            L.snn_linattn_step(ctypes.byref(d), 16, 16, 16, 16, None, d.B, 16, 17, 16, None))


def test_heads_of_one_launch():
    assert _calls(_desc(1, 1 << 20, 16, 16)) == (SHAPE,) * 3         # 2^32 threads
    assert _calls(_desc(1, (1 << 20) - 1, 16, 16)) == (ALIGN,) * 3
    assert snn.lib().snn_linattn_workspace_bytes(ctypes.byref(_desc(1, 1 << 20, 16, 16))) == 0


def test_sums_over_shared_heads_of_one_launch():
    # 2^28 tokens and key heads of 128 values: 2^32 runs of 8
    assert _calls(_desc(1 << 14, 1 << 10, 32, 16, 128, 128))[:2] == (ALIGN, SHAPE)
    assert _calls(_desc(1 << 14, 1 << 10, 32, 16, 128, 8))[1] == SHAPE
    assert _calls(_desc(1 << 14, 1 << 10, 32, 16, 120, 120))[1] == ALIGN
    assert _calls(_desc(1 << 14, 1 << 10, 32, 32, 128, 128))[1] == ALIGN  # none is shared
