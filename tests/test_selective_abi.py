"""The selective leaky block's refusals: every argument is checked on the host, before any
launch (no GPU needed; the addresses are never dereferenced)."""
import ctypes

import pytest

import paper_2211_10725_amd as snn
from tests.test_block_abi import (ALIGN, DTYPE, NULL, OK, SHAPE, UNSUPPORTED, WORKSPACE,
                                  _changed)

torch = pytest.importorskip("torch")
BIG = 1 << 50


def _ss(T=40, B=2, n=96, N=16, G=2, forward_only=False):
    x, v = torch.empty(T, B, n), torch.empty(T, B, G, N)
    return snn.selscan_desc(x, x, v, v, x, x, forward_only=forward_only)


def _fwd(d, u=16, dt=16, a=16, b=16, c=16, skip=16, bias=16, z=16, lens=None, s=None, y=16, so=17,
         saved=16, ws=16, size=BIG):
    # state_out 17: a call that is right otherwise stops at its alignment
    return snn.lib().snn_selscan_fwd(ctypes.byref(d) if d else None, u, dt, a, b, c, skip, bias, z,
                                     lens, s, y, so, saved, ws, size, None)


def test_selscan_descriptor():
    d = _ss()
    assert _fwd(None) == NULL and _fwd(d) == ALIGN
    for bad in (dict(T=-1), dict(B=-1), dict(n=-2), dict(states=0), dict(states=65),
                dict(groups=0), dict(groups=5), dict(u_stride=(0, -1)), dict(b_stride=(2, -1)),
                dict(c_stride=(1, (1 << 32) + 1)), dict(y_stride=(0, 95)), dict(y_stride=(1, 0)),
                dict(z_stride=(1, -5)), dict(dt_stride=(0, 1 << 33)), dict(B=1 << 23),
                dict(T=1 << 30, B=1 << 10), dict(n=1 << 30)):
        assert _fwd(_changed(d, **bad)) == SHAPE, bad
        if "y_stride" not in bad:
            assert snn.lib().snn_selscan_workspace_bytes(_changed(d, **bad)) == 0
            assert snn.lib().snn_selscan_saved_bytes(_changed(d, **bad)) == 0
    for dt in (snn.U8, 7, -1):
        assert _fwd(_changed(d, dtype=dt)) == DTYPE
    for bad in (dict(delta_softplus=2), dict(forward_only=-1)):
        assert _fwd(_changed(d, **bad)) == UNSUPPORTED
    assert _fwd(_changed(d, B=0)) == OK and _fwd(_changed(d, n=0)) == OK


def test_selscan_pointers_and_workspace():
    d = _ss(T=3000)
    for name in ("u", "dt", "a", "b", "c", "y", "saved"):
        assert _fwd(d, **{name: None}) == NULL, name
    for name in ("u", "dt", "b", "c", "y", "z"):
        assert _fwd(d, so=None, **{name: 18}) == ALIGN, name
    for name in ("a", "skip", "bias", "lens", "s", "saved", "ws"):
        assert _fwd(d, so=None, **{name: 24}) == ALIGN, name
    need = snn.snn_selscan_workspace_bytes(d)
    assert need > 0
    assert _fwd(d, so=None, size=need - 1) == WORKSPACE and _fwd(d, so=None, ws=None) == WORKSPACE
    only = _ss(T=3000, forward_only=True)
    assert _fwd(only) == UNSUPPORTED and _fwd(only, saved=None) == ALIGN
    # u dt a b c skip bias z lens saved gy gs du ddt da db dc dskip dbias dz ds
    ptr = [16] * 8 + [None, 16, 16, None] + [16] * 8 + [17]
    call = snn.lib().snn_selscan_bwd
    assert call(ctypes.byref(d), *ptr, 16, BIG, None) == ALIGN
    assert call(ctypes.byref(only), *ptr, 16, BIG, None) == UNSUPPORTED
    for i in (0, 1, 2, 3, 4, 9, 10, 12, 13, 15, 16, 19):
        assert call(ctypes.byref(d), *ptr[:i], None, *ptr[i + 1:], 16, BIG, None) == NULL, i
    for i in (5, 6, 7):  # a gradient of what is not there
        assert call(ctypes.byref(d), *ptr[:i], None, *ptr[i + 1:], 16, BIG, None) == UNSUPPORTED, i
    ptr[-1] = 16
    assert call(ctypes.byref(d), *ptr, 16, need - 1, None) == WORKSPACE
    for bad in (dict(u_stride=(0, 0)), dict(b_stride=(2, 15)), dict(c_stride=(1, 0)),
                dict(z_stride=(1, 10)), dict(dt_stride=(0, 100))):
        assert call(ctypes.byref(_changed(d, **bad)), *ptr, 16, BIG, None) == SHAPE, bad


def test_selscan_step():
    d = _ss(T=1)

    def step(d, u=16, a=16, slots=16, n=9, s=16, so=17, y=16):
        return snn.lib().snn_selscan_step(ctypes.byref(d), u, 16, a, 16, 16, None, None, None,
                                          slots, n, s, so, y, None)

    assert step(d) == ALIGN and step(_ss(T=2)) == SHAPE and step(d, n=-1) == SHAPE
    assert step(d, slots=None, n=1) == SHAPE and step(d, slots=None, n=2) == ALIGN
    for name in ("u", "a", "s", "so", "y"):
        assert step(d, **{name: None}) == NULL
    assert step(_changed(d, B=0)) == OK


def _sc(T=40, B=2, n=96, K=4, act="silu"):
    x = torch.empty(T, B, n)
    return snn.shortconv_desc(x, x, K, act)


def test_shortconv():
    d = _sc()

    def fwd(d, x=16, w=16, bias=None, lens=None, s=None, y=16, so=17):
        return snn.lib().snn_shortconv_fwd(ctypes.byref(d) if d else None, x, w, bias, lens, s, y,
                                           so, None)

    assert fwd(None) == NULL and fwd(d) == ALIGN
    for bad in (dict(T=-1), dict(B=-1), dict(n=-1), dict(width=1), dict(width=9),
                dict(x_stride=(0, -1)), dict(y_stride=(1, 95)), dict(x_stride=(1, 1 << 33)),
                dict(B=1 << 24), dict(T=1 << 30, B=1 << 10)):
        assert fwd(_changed(d, **bad)) == SHAPE, bad
    assert fwd(_changed(d, dtype=snn.U8)) == DTYPE
    assert fwd(_changed(d, act=snn.GATE_SIGMOID)) == UNSUPPORTED
    assert fwd(_changed(d, B=0)) == OK and fwd(_changed(d, n=0)) == OK
    for name in ("x", "w", "y"):
        assert fwd(d, **{name: None}) == NULL
    for bad in (dict(x=18), dict(w=20), dict(bias=20), dict(lens=20), dict(s=20), dict(y=18)):
        assert fwd(d, so=None, **bad) == ALIGN
    # x w bias lens state gy gs gx gw gb gstate
    ptr = [16, 16, 16, None, 16, 16, 32, 16, 16, 16, 17]
    call = snn.lib().snn_shortconv_bwd
    need = snn.snn_shortconv_workspace_bytes(d)
    assert need > 0 and call(ctypes.byref(d), *ptr, 16, BIG, None) == ALIGN
    for i in (0, 1, 5, 7):
        assert call(ctypes.byref(d), *ptr[:i], None, *ptr[i + 1:], 16, BIG, None) == NULL, i
    assert call(ctypes.byref(d), *ptr[:2], None, *ptr[3:], 16, BIG, None) == UNSUPPORTED
    ptr[-1] = 32
    assert call(ctypes.byref(d), *ptr, 16, BIG, None) == UNSUPPORTED  # in place
    ptr[-1] = 16
    assert call(ctypes.byref(d), *ptr, 16, need - 1, None) == WORKSPACE
    assert call(ctypes.byref(d), *ptr, None, need, None) == WORKSPACE
    assert call(ctypes.byref(_changed(d, x_stride=(1, 0))), *ptr, 16, BIG, None) == SHAPE

    def step(d, x=16, slots=16, n=9, s=16, so=17, y=16):
        return snn.lib().snn_shortconv_step(ctypes.byref(d), x, 16, None, slots, n, s, so, y, None)

    one = _sc(T=1)
    assert step(one) == ALIGN and step(d) == SHAPE and step(one, n=-1) == SHAPE
    assert step(one, slots=None, n=1) == SHAPE
    for name in ("x", "s", "so", "y"):
        assert step(one, **{name: None}) == NULL


def test_layer_norm():
    d = snn.layer_norm_desc(torch.empty(5, 96), torch.empty(5, 96))

    def fwd(d, x=16, w=17, b=None, y=32):
        return snn.lib().snn_layer_norm_fwd(ctypes.byref(d) if d else None, x, w, b, y, None)

    assert fwd(None) == NULL and fwd(d) == ALIGN
    for bad in (dict(rows=-1), dict(n=0), dict(n=16385), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(ld_x=95), dict(ld_y=1 << 33)):
        assert fwd(_changed(d, **bad)) == SHAPE, bad
        assert snn.lib().snn_layer_norm_workspace_bytes(_changed(d, **bad)) == 0
    for bad in (dict(x_dtype=snn.F16), dict(y_dtype=snn.U8)):
        assert fwd(_changed(d, **bad)) == DTYPE
    assert fwd(_changed(d, rows=0)) == OK
    assert fwd(d, x=None) == NULL and fwd(d, y=None) == NULL
    assert fwd(d, w=None, x=18) == ALIGN and fwd(d, w=None, y=34) == ALIGN
    assert fwd(_changed(d, ld_y=100), x=16, y=16, w=None) == UNSUPPORTED
    # x gy gres w gx gw gb
    ptr = [16, 16, 16, 17, 16, 16, 16]
    call, need = snn.lib().snn_layer_norm_bwd, snn.snn_layer_norm_workspace_bytes(d)
    assert need > 0 and call(ctypes.byref(d), *ptr, 16, BIG, None) == ALIGN
    ptr[3] = None
    for i in (0, 1, 4):
        assert call(ctypes.byref(d), *ptr[:i], None, *ptr[i + 1:], 16, BIG, None) == NULL, i
    assert call(ctypes.byref(d), *ptr, 16, need - 1, None) == WORKSPACE
    assert call(ctypes.byref(d), *ptr, None, need, None) == WORKSPACE


def test_binding_checks_tensors():
    x, v, ws = torch.empty(4, 2, 40), torch.empty(4, 2, 2, 8), torch.empty(64, dtype=torch.uint8)
    d = snn.selscan_desc(x, x, v, v, x, x, forward_only=True)
    a, s = torch.empty(8, 40), torch.empty(2, 8, 40)

    def call(u=x, dt=x, a=a, b=v, c=v, skip=None, bias=None, z=x, lens=None, s=s, y=x):
        snn.snn_selscan_fwd(d, u, dt, a, b, c, skip, bias, z, lens, s, y, None, None, ws, 0)

    for bad in (dict(u=x[:3]), dict(dt=x.half()), dict(a=a.t().contiguous().t()), dict(a=a[:4]),
                dict(b=v[:, :, :1]), dict(c=v.transpose(0, 1)), dict(skip=torch.empty(39)),
                dict(bias=torch.empty(40).double()), dict(z=torch.empty(4, 2, 80)[..., ::2]),
                dict(lens=torch.empty(2)), dict(s=s[:1]), dict(y=torch.empty(4, 2, 48)[..., :40])):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in ((x, x[:3], v, v, x), (x, x, v, v[:, :1], x), (x, x.half(), v, v, x),
                (x, x, x, x, x), (torch.empty(4, 2, 80)[..., ::2], x, v, v, x)):
        with pytest.raises(ValueError):
            snn.selscan_desc(*bad)
    with pytest.raises(ValueError):
        snn.snn_selscan_fwd(snn.selscan_desc(x, x, v, v, x), x, x, a, v, v, None, None, None, None,
                            s, x, None, torch.empty(8, dtype=torch.uint8), ws, 0)
    sc = snn.shortconv_desc(x, x, 4)
    w, st = torch.empty(4, 40), torch.empty(2, 3, 40)
    for bad in (dict(x=x[:3]), dict(w=w[:3]), dict(w=w.t()), dict(bias=w[0, :39]),
                dict(lens=torch.empty(2)), dict(s=st[:1]), dict(y=x.half())):
        k = dict(dict(x=x, w=w, bias=None, lens=None, s=st, y=x), **bad)
        with pytest.raises(ValueError):
            snn.snn_shortconv_fwd(sc, k["x"], k["w"], k["bias"], k["lens"], k["s"], k["y"], None, 0)
    with pytest.raises(ValueError):
        snn.shortconv_desc(x, x.half(), 4)
    r = torch.empty(6, 40)
    ln = snn.layer_norm_desc(r)
    for bad in (dict(x=r[:5]), dict(w=r[0, :39]), dict(y=r.half()), dict(b=r[:, 0].double())):
        k = dict(dict(x=r, w=None, b=None, y=r), **bad)
        with pytest.raises(ValueError):
            snn.snn_layer_norm_fwd(ln, k["x"], k["w"], k["b"], k["y"], 0)
    with pytest.raises(ValueError):
        snn.layer_norm_desc(r, r[:, :8])
