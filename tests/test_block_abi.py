"""The leaky sequence block's refusals: every argument is checked on the host,
before any launch (no GPU needed; the addresses are never dereferenced)."""
import ctypes

import pytest

import paper_2211_10725_amd as snn

torch = pytest.importorskip("torch")
OK, NULL, SHAPE, DTYPE, ALIGN, UNSUPPORTED, WORKSPACE = range(7)


def _la(T=4, B=2, H=4, KV=2, dk=64, dv=32, dt=torch.float32):
    q, k = torch.empty(T, B, H, dk, dtype=dt), torch.empty(T, B, KV, dk, dtype=dt)
    v, o = torch.empty(T, B, KV, dv, dtype=dt), torch.empty(T, B, H, dv, dtype=dt)
    return snn.linattn_desc(q, k, v, o)


def _changed(d, **fields):
    c = type(d)()
    ctypes.pointer(c)[0] = d
    for name, value in fields.items():
        if isinstance(value, tuple):
            getattr(c, name)[value[0]] = value[1]
        else:
            setattr(c, name, value)
    return c


def _fwd(d, q=16, k=16, v=16, decay=16, lens=None, s=None, o=16, so=17, ws=16, size=1 << 62):
    # state_out 17: a call that is right otherwise stops at its alignment
    return snn.lib().snn_linattn_fwd(ctypes.byref(d) if d else None, q, k, v, decay, lens, s, o,
                                     so, ws, size, None)


def test_linattn_descriptor():
    d = _la()
    assert _fwd(None) == NULL
    assert _fwd(d) == ALIGN
    for bad in (dict(T=-1), dict(B=-1), dict(heads=-4), dict(kv_heads=0), dict(kv_heads=3),
                dict(d_k=0), dict(d_k=12), dict(d_k=136), dict(d_v=4), dict(d_v=256),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride=(0, -8)),
                dict(k_stride=(1, 4)), dict(v_stride=(2, 1)), dict(o_stride=(0, 1 << 33)),
                dict(B=1 << 23), dict(T=1 << 30, B=1 << 10)):
        assert _fwd(_changed(d, **bad)) == SHAPE, bad
        assert snn.lib().snn_linattn_workspace_bytes(_changed(d, **bad)) == 0
    for dt in (snn.U8, 7, -1):
        assert _fwd(_changed(d, dtype=dt)) == DTYPE
    assert _fwd(_changed(d, B=0)) == OK and _fwd(_changed(d, heads=0, kv_heads=0)) == OK


def test_linattn_pointers_and_workspace():
    d = _la(T=3000)
    for name in ("q", "k", "v", "decay", "o"):
        assert _fwd(d, **{name: None}) == NULL, name
        assert _fwd(d, so=None, **{name: 24}) == ALIGN, name
    assert _fwd(d, lens=20) == ALIGN and _fwd(d, s=40) == ALIGN
    need = snn.snn_linattn_workspace_bytes(d)
    assert need > 0
    assert _fwd(d, so=None, size=need - 1) == WORKSPACE
    assert _fwd(d, so=None, ws=None) == WORKSPACE
    ptr = [16] * 4 + [None, None, 16, None, 16, 16, 16, 17]
    call = snn.lib().snn_linattn_bwd
    assert call(ctypes.byref(d), *ptr, 16, 1 << 62, None) == ALIGN
    for i in (0, 1, 2, 3, 6, 8, 9, 10):
        assert call(ctypes.byref(d), *ptr[:i], None, *ptr[i + 1:], 16, 1 << 62, None) == NULL, i
    ptr[-1] = 16
    assert call(ctypes.byref(d), *ptr, 16, need - 1, None) == WORKSPACE
    ptr[7] = 16  # the state's gradient in place
    assert call(ctypes.byref(d), *ptr, 16, need, None) == UNSUPPORTED


def test_linattn_step():
    d = _la(T=1)

    def step(d, q=16, decay=16, slots=16, n=9, s=16, so=17, o=16):
        return snn.lib().snn_linattn_step(ctypes.byref(d), q, 16, 16, decay, slots, n, s, so, o,
                                          None)

    assert step(d) == ALIGN
    assert step(_la(T=2)) == SHAPE and step(d, n=-1) == SHAPE
    assert step(d, slots=None, n=1) == SHAPE and step(d, slots=None, n=2) == ALIGN
    for name in ("q", "decay", "s", "so", "o"):
        assert step(d, **{name: None}) == NULL
    assert step(_changed(d, B=0)) == OK


def test_linattn_binding_checks_tensors():
    q, k, v = (torch.empty(4, 2, h, w) for h, w in ((4, 64), (2, 64), (2, 32)))
    o = torch.empty(4, 2, 4, 32)
    d = snn.linattn_desc(q, k, v, o)
    decay, ws = torch.empty(4), torch.empty(1 << 20, dtype=torch.uint8)

    def call(q=q, k=k, v=v, o=o, decay=decay, lens=None, s=None):
        snn.snn_linattn_fwd(d, q, k, v, decay, lens, s, o, None, ws, 0)

    for bad in (dict(q=q[:3]), dict(k=k.half()), dict(v=v.transpose(0, 1)), dict(o=o[..., :16]),
                dict(q=torch.empty(4, 2, 4, 128)[..., ::2]), dict(decay=decay[:3]),
                dict(decay=decay.double()), dict(decay=torch.empty(8)[::2]),
                dict(lens=torch.empty(1, dtype=torch.int32)), dict(lens=torch.empty(2)),
                dict(s=torch.empty(10))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        snn.linattn_desc(q, k[:, :1], v, o)
    with pytest.raises(ValueError):
        snn.linattn_desc(q, k.half(), v, o)
    with pytest.raises(ValueError):
        snn.linattn_desc(torch.empty(4, 2, 4, 128)[..., ::2], k, v, o)


def _gn(rows=5, n=96, groups=4, act="silu", x=torch.float32, y=torch.float32):
    t = torch.empty(rows, n, dtype=y)
    return snn.gate_norm_desc(torch.empty(rows, n, dtype=x), t, t if act != "none" else None,
                              groups, act)


def _gfwd(d, x=16, y=16, g=16, wp=None, s=None, wr=17, xo=16, h=16, y8=None, g8=None):
    # w_pre 17: a call that is right otherwise stops at its alignment
    return snn.lib().snn_gate_norm_fwd(ctypes.byref(d) if d else None, x, y, g, wp, s, wr, xo, h,
                                       y8, g8, None)


def test_gate_norm_descriptor():
    d = _gn()
    assert _gfwd(None) == NULL and _gfwd(d) == ALIGN
    for bad in (dict(rows=-1), dict(n=0), dict(n=16385, groups=1), dict(groups=0), dict(groups=5),
                dict(groups=24), dict(ckpt_block=0),
                dict(ckpt_block=48), dict(ckpt_block=256), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
                dict(ld_x=95), dict(ld_y=0), dict(ld_g=95), dict(ld_h=-96), dict(ld_x=1 << 33)):
        assert _gfwd(_changed(d, **bad)) == SHAPE, bad
        assert snn.lib().snn_gate_norm_workspace_bytes(_changed(d, **bad)) == 0
    for bad in (dict(x_dtype=snn.F16), dict(y_dtype=snn.U8), dict(x_dtype=snn.U8)):
        assert _gfwd(_changed(d, **bad)) == DTYPE
    assert _gfwd(_changed(d, gate=4)) == UNSUPPORTED
    assert _gfwd(_changed(d, rows=0)) == OK


def test_gate_norm_pointers():
    d = _gn()
    assert _gfwd(d, x=None) == NULL and _gfwd(d, xo=None) == NULL and _gfwd(d, g=None) == NULL
    assert _gfwd(d, y=None) == UNSUPPORTED                       # a gate without a block
    none = _gn(act="none")
    assert _gfwd(none, g=16) == UNSUPPORTED and _gfwd(none, g=None, g8=16) == UNSUPPORTED
    assert _gfwd(none, y=None, g=None, xo=None) == ALIGN
    assert _gfwd(none, y=None, g=None) == UNSUPPORTED             # x_out of nothing
    assert _gfwd(none, y=None, g=None, xo=None, h=None) == NULL
    assert _gfwd(d, wr=None, x=18) == ALIGN and _gfwd(d, wr=None, y8=24) == ALIGN

    def bwd(d, gx=16, gh=16, xo=16, y=16, g=16, y8=None, g8=None, wp=17, s=None, wr=None, dx=16,
            dy=16, dg=16, dwp=None, ds=None, dwr=None, ws=16, size=1 << 40):
        return snn.lib().snn_gate_norm_bwd(ctypes.byref(d), gx, gh, xo, y, g, y8, g8, wp, s, wr,
                                           dx, dy, dg, dwp, ds, dwr, ws, size, None)

    assert bwd(d) == ALIGN
    for bad in (dict(gx=None, gh=None), dict(xo=None), dict(dx=None), dict(dy=None),
                dict(dg=None), dict(g=None)):
        assert bwd(d, **bad) == NULL, bad
    for bad in (dict(y8=16), dict(g8=16), dict(y=None, y8=16), dict(gh=None, dwr=16),
                dict(y=None, g=None)):
        assert bwd(d, **bad) == UNSUPPORTED, bad
    assert bwd(d, y=None, g=None, y8=16, g8=16) == ALIGN
    need = snn.snn_gate_norm_workspace_bytes(d)
    assert need > 0
    assert bwd(d, wp=None, size=need - 1) == WORKSPACE
    assert bwd(d, wp=None, ws=None) == WORKSPACE


def test_gate_norm_binding_checks_tensors():
    x, y = torch.empty(6, 40), torch.empty(6, 40)
    d = snn.gate_norm_desc(x, y, y, 1, "silu")
    for bad in (dict(x=x[:5]), dict(y=y.half()), dict(h=torch.empty(6, 48)[:, :40]),
                dict(w=torch.empty(39)), dict(y8=torch.empty(10, dtype=torch.uint8))):
        a = dict(dict(x=x, y=y, h=y, w=None, y8=None), **bad)
        with pytest.raises(ValueError):
            snn.snn_gate_norm_fwd(d, a["x"], a["y"], y, a["w"], None, None, x, a["h"], a["y8"],
                                  None, 0)
    with pytest.raises(ValueError):
        snn.gate_norm_desc(x, y[:, :8])
    with pytest.raises(ValueError):
        snn.gate_norm_desc(x.t(), None)
    assert snn.gate_norm_desc(torch.empty(3, 4, 90)[:, :, :40]).ld_x == 90
    with pytest.raises(ValueError):
        snn.gate_norm_desc(torch.empty(3, 8, 40)[:, :4])


def test_checkpoint():
    L = snn.lib()
    assert L.snn_checkpoint_bytes(-1, 5, 128) == 0 and L.snn_checkpoint_bytes(3, -1, 128) == 0
    assert L.snn_checkpoint_bytes(2, 129, 128) == 512 + 256      # codes, then 4 scales
    assert L.snn_checkpoint_bytes(2, 1024, 8) == 2048 + 1024     # 256 scales
    assert all(L.snn_checkpoint_bytes(2, 129, b) == 0 for b in (0, 4, 24, 256, -8))
    for fn in (L.snn_checkpoint_save, L.snn_checkpoint_load):
        assert fn(-1, 8, 128, 8, snn.F32, 16, 16, None) == SHAPE
        assert fn(3, 8, 128, 7, snn.F32, 16, 16, None) == SHAPE
        assert fn(3, 8, 96, 8, snn.F32, 16, 16, None) == SHAPE
        assert fn(1 << 30, 1 << 20, 128, 1 << 20, snn.F32, 16, 16, None) == SHAPE
        assert fn(3, 8, 64, 8, snn.U8, 16, 16, None) == DTYPE
        assert fn(3, 8, 64, 8, snn.F32, None, 16, None) == NULL
        assert fn(3, 8, 64, 8, snn.F32, 16, None, None) == NULL
        assert fn(0, 8, 64, 8, snn.F32, None, None, None) == OK
    assert L.snn_checkpoint_save(3, 8, 128, 8, snn.F32, 18, 16, None) == ALIGN
    assert L.snn_checkpoint_load(3, 8, 128, 8, snn.F16, 24, 16, None) == ALIGN
    with pytest.raises(ValueError):
        snn.snn_checkpoint_save(torch.empty(4, 40), torch.empty(100, dtype=torch.uint8))
