"""Strides that would have several rows of an output in one place are refused on
the host (no GPU needed; the addresses are never dereferenced)."""
import ctypes

import pytest

import paper_2211_10725_amd as snn

torch = pytest.importorskip("torch")
OK, NULL, SHAPE, DTYPE, ALIGN = range(5)
BIG = 1 << 62


def _desc(q, k, v, o):
    return snn.linattn_desc(q, k, v, o)


def _fwd(d):  # state_out 17: a call that is right otherwise stops at its alignment
    return snn.lib().snn_linattn_fwd(ctypes.byref(d), 16, 16, 16, 16, None, None, 16, 17, 16, BIG,
                                     None)


def _bwd(d):
    return snn.lib().snn_linattn_bwd(ctypes.byref(d), 16, 16, 16, 16, None, None, 16, None, 16, 16,
                                     16, 17, 16, BIG, None)


def _step(d):
    return snn.lib().snn_linattn_step(ctypes.byref(d), 16, 16, 16, 16, None, d.B, 16, 17, 16, None)


def _tensors(T=6, B=4, H=4, KV=2, dk=64, dv=32):
    return dict(q=torch.empty(T, B, H, dk), k=torch.empty(T, B, KV, dk),
                v=torch.empty(T, B, KV, dv), o=torch.empty(T, B, H, dv))


def _broadcasts(t):
    """The tensor's shape over fewer elements: along each dimension, as a window
    that slides over time, and with two dimensions that step alike."""
    T, B, H, d = t.shape
    out = {f"dim {i}": t.narrow(i, 0, 1).expand(t.shape) for i in range(3)}
    out["window"] = torch.empty(T + B, H, d).unfold(0, B, 1)[:T].permute(0, 3, 1, 2)
    out["window by two"] = torch.empty(2 * T + B, H, d).unfold(0, B, 2)[:T].permute(0, 3, 1, 2)
    out["steps below the row"] = torch.as_strided(t, t.shape, (B * H * d, H * d, 8, 1))
    out["alike"] = torch.as_strided(t, t.shape, (H * d, H * d, d, 1))
    return {n: x for n, x in out.items() if x.shape == t.shape and x.stride(3) == 1}


CASES = list(_broadcasts(_tensors()["q"]))


def test_every_kind_of_broadcast_is_there():
    assert len(CASES) == 7


@pytest.mark.parametrize("how", [c for c in CASES if c != "dim 0"])
def test_outputs(how):
    t = _tensors()
    t["o"] = _broadcasts(t["o"])[how]
    d = _desc(**t)
    assert _fwd(d) == SHAPE
    assert _bwd(d) == ALIGN          # the backward reads o's gradient alone
    one = {n: x[:1] for n, x in t.items()}
    if how in ("dim 1", "dim 2", "steps below the row"):
        assert _step(_desc(**one)) == SHAPE


def test_output_broadcast_over_time():
    t = _tensors()
    t["o"] = _broadcasts(t["o"])["dim 0"]
    assert _fwd(_desc(**t)) == SHAPE
    assert _step(_desc(**{n: x[:1] for n, x in t.items()})) == ALIGN  # one token: no other row


@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("how", CASES)
def test_gradients(how, what):
    t = _tensors()
    t[what] = _broadcasts(t[what])[how]
    d = _desc(**t)
    assert _fwd(d) == ALIGN          # reading it is fine
    assert _bwd(d) == SHAPE


def test_layouts_without_shared_rows_are_taken():
    for order in ((0, 1, 2), (1, 0, 2), (2, 1, 0), (1, 2, 0), (0, 2, 1), (2, 0, 1)):
        t = {n: x.permute(*order, 3).contiguous().permute(*[order.index(i) for i in range(3)], 3)
             for n, x in _tensors().items()}
        assert _fwd(_desc(**t)) == ALIGN and _bwd(_desc(**t)) == ALIGN
    packed = torch.empty(6, 4, 4 * 64 + 2 * 64 + 2 * 32 + 8)[:, :, 8:].split([256, 128, 64], 2)
    t = dict(zip("qkv", (x.unflatten(2, (-1, w)) for x, w in zip(packed, (64, 64, 32)))))
    assert _bwd(_desc(**t, o=torch.empty(6, 4, 4, 32))) == ALIGN
    every_other = {n: torch.empty(12, 8, x.shape[2] * 2, x.shape[3])[::2, ::2, ::2]
                   for n, x in _tensors().items()}
    assert _fwd(_desc(**every_other)) == ALIGN and _bwd(_desc(**every_other)) == ALIGN
    # rows of two tensors in turn, in either nesting
    turns = torch.empty(6, 4, 4, 3, 64)
    t = dict(_tensors(KV=4), q=turns[..., 0, :], k=turns[..., 1, :])
    assert _bwd(_desc(**t)) == ALIGN
    # dimensions of one element have any stride
    t = {n: torch.as_strided(x, (1, 1, 1, x.shape[3]), (0, 8, 0, 1)) for n, x in _tensors().items()}
    assert _fwd(_desc(**t)) == ALIGN and _bwd(_desc(**t)) == ALIGN and _step(_desc(**t)) == ALIGN
    # no tokens: no rows at all
    t = _tensors(T=0)
    assert _fwd(_desc(**t)) == ALIGN and _bwd(_desc(**t)) == ALIGN
