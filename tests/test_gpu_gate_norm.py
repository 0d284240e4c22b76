"""Gated norms with their backward and 8-bit checkpoints against plain 64-bit
references.

Tolerance, per element: 64 x 2^-24 of the sum of the absolute values of the
result's terms (each is a handful of fp32 roundings of sums that a tree of at
most 16 + log2(1024) levels adds, and of an exponential, reciprocal or root
good to a few units), plus half a unit of the result's type; a column's sum
over R rows adds R 2^-24 of its terms."""
import numpy as np
import pytest

import paper_2211_10725_amd as snn
from tests import block_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
PAIRS = [("f32", "f32"), ("f32", "f16"), ("f32", "bf16"), ("f16", "f16"), ("bf16", "bf16")]
EPS = 1e-5


def _np(x):
    return x.detach().double().cpu().numpy()


def _rand(rng, shape, dt, std=1.0, mean=0.0, pad=0, off=0):
    """Normal values; with pad, rows of a wider tensor starting `off` in."""
    x = torch.as_tensor(rng.standard_normal((shape[0], shape[1] + pad)) * std + mean)
    return x.to(torch.float32).to(TYPES[dt]).cuda()[:, off:off + shape[1]]


def _nan_like(x):
    out = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)
    return out.fill_(float("nan"))


def _near(got, want, absolute, dt, rows=0, what=""):
    rel, least = ref.HALF_ULP[dt]
    bound = (64 + rows) * ref.EPS32 * absolute + rel * np.abs(want) + least
    got = _np(got)
    assert np.isfinite(got).all(), what
    err = np.abs(got - want)
    assert (err <= bound).all(), (what, float((err / np.maximum(bound, 1e-300)).max()))


class Case:
    def __init__(self, rows, n, groups=1, act="silu", x="f32", y="f32", pad=0, off=0, seed=0,
                 weights=True, ckpt=0):
        rng = np.random.default_rng(seed)
        self.xt, self.yt, self.n, self.rows = x, y, n, rows
        self.groups, self.act, self.ckpt = groups, act, ckpt
        more = dict(pad=pad, off=off)
        self.x = _rand(rng, (rows, n), x, **more)
        self.y = _rand(rng, (rows, n), y, 2.0, **more)
        self.g = _rand(rng, (rows, n), y, 2.0, **more) if act != "none" else None
        self.gx = _rand(rng, (rows, n), x, **more)
        self.h = _nan_like(self.y)
        self.gh = _rand(rng, (rows, n), y, **more)
        self.w = [_rand(rng, (1, n), "f32", 0.3, 1.0)[0].contiguous() if weights else None
                  for _ in range(3)]
        self.d = snn.gate_norm_desc(self.x, self.y, self.g, groups, act, EPS, self.h,
                                    ckpt_block=ckpt or 128)
        self.y8 = self.g8 = None
        if ckpt:
            size = snn.snn_checkpoint_bytes(rows, n, ckpt)
            self.y8 = torch.empty(size, dtype=torch.uint8, device="cuda")
            self.g8 = torch.empty(size, dtype=torch.uint8, device="cuda") if self.g is not None \
                else None

    def weights(self):
        return [_np(w) if w is not None else np.ones(self.n) for w in self.w]

    def fwd(self):
        self.xo = _nan_like(self.x)
        snn.snn_gate_norm_fwd(self.d, self.x, self.y, self.g, *self.w, self.xo, self.h, self.y8,
                              self.g8)
        g = _np(self.g) if self.g is not None else None
        w_post, scale, w_pre = self.weights()
        xo, h, ax, ah = ref.gate_norm(_np(self.x), _np(self.y), g, self.groups, self.act,
                                      self.d.eps, w_post, scale, w_pre)
        _near(self.xo, xo, ax, self.xt, what="x_out")
        _near(self.h, h, ah, self.yt, what="h")

    def bwd(self, weight_grads=True):
        dx, dy = _nan_like(self.x), _nan_like(self.y)
        dg = _nan_like(self.g) if self.g is not None else None
        dw = [torch.full((self.n,), float("nan"), device="cuda") if weight_grads else None
              for _ in range(3)]
        ws = torch.empty(max(16, snn.snn_gate_norm_workspace_bytes(self.d)), dtype=torch.uint8,
                         device="cuda")
        y, g = (None, None) if self.ckpt else (self.y, self.g)
        snn.snn_gate_norm_bwd(self.d, self.gx, self.gh, self.xo, y, g, self.y8, self.g8, *self.w,
                              dx, dy, dg, *dw, ws)
        y, g = _np(self.y), _np(self.g) if self.g is not None else None
        if self.ckpt:
            y = ref.quantised(y, self.ckpt).astype(np.float64)
            g = ref.quantised(g, self.ckpt).astype(np.float64) if g is not None else None
        w_post, scale, w_pre = self.weights()
        want = ref.gate_norm_grads(_np(self.gx), _np(self.gh), _np(self.xo), y, g, self.groups,
                                   self.act, self.d.eps, w_post, scale, w_pre)
        self.got = dict(dx=dx, dy=dy, dg=dg, dw_post=dw[0], ds=dw[1], dw_pre=dw[2])
        for name, t in self.got.items():
            if t is None:
                continue
            cols = name in ("dw_post", "ds", "dw_pre")
            _near(t, want[name], want["abs_" + name],
                  "f32" if cols else self.xt if name == "dx" else self.yt,
                  rows=self.rows if cols else 0, what=name)


# widths of one value, under a run of 8, odd, at and past each size that
# another number of threads takes, and the widest
WIDTHS = [1, 7, 8, 24, 100, 511, 512, 513, 1001, 1024, 1025, 2048, 2056, 4096, 4097, 8192, 8200,
          16383, 16384]


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("types", PAIRS, ids="-".join)
def test_widths(n, types):
    c = Case(7, n, 1, ("silu", "sigmoid", "mul", "none")[n % 4], *types, seed=n)
    c.fwd()
    c.bwd()


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 513, 2051, 9000])
def test_rows(rows):
    for n, types in ((96, ("f32", "f32")), (600, ("f32", "bf16")), (1030, ("f16", "f16"))):
        c = Case(rows, n, 1, "silu", *types, seed=rows)
        c.fwd()
        c.bwd()


# runs of 8 per group: 1, powers of two, others, more than a wave
@pytest.mark.parametrize("groups,d", [(4, 8), (8, 16), (3, 24), (12, 40), (16, 64), (16, 128),
                                      (5, 136), (7, 520), (3, 1000), (4, 2048), (2, 8192)])
@pytest.mark.parametrize("act", ["silu", "none"])
def test_groups(groups, d, act):
    for types in (("f32", "f32"), ("f32", "bf16")):
        c = Case(9, groups * d, groups, act, *types, seed=d)
        c.fwd()
        c.bwd()


@pytest.mark.parametrize("act", ["silu", "sigmoid", "mul", "none"])
@pytest.mark.parametrize("types", PAIRS, ids="-".join)
def test_gates_slices_and_absent_weights(act, types):
    for pad, off in ((8, 0), (13, 3)):
        c = Case(33, 200, 1, act, *types, pad=pad, off=off)
        c.fwd()
        c.bwd()
        c = Case(33, 200, 5, act, *types, pad=pad, off=off, weights=False)
        c.fwd()
        c.bwd(weight_grads=False)


@pytest.mark.parametrize("types", PAIRS, ids="-".join)
@pytest.mark.parametrize("n,groups", [(64, 1), (100, 1), (384, 3), (1001, 1), (2048, 16),
                                      (5000, 1)])
def test_backward_from_8_bit_checkpoints(n, groups, types):
    for act, block in (("silu", 128), ("none", 128), ("silu", 32), ("mul", 8)):
        c = Case(40, n, groups, act, *types, ckpt=block, seed=n)
        c.fwd()
        for t, kept in ((c.y, c.y8), (c.g, c.g8)):
            if t is None:
                continue
            back = torch.empty((40, n), device="cuda")
            snn.snn_checkpoint_load(kept, back, block)
            assert np.array_equal(back.cpu().numpy(),
                                  ref.quantised(t.float().cpu().numpy(), block))
        c.bwd()


def test_norm_alone_and_partial_gradients():
    rng = np.random.default_rng(3)
    x = _rand(rng, (50, 300), "f32")
    gh, gx = _rand(rng, (50, 300), "bf16"), _rand(rng, (50, 300), "f32")
    h = torch.empty((50, 300), dtype=torch.bfloat16, device="cuda")
    d = snn.gate_norm_desc(x, eps=EPS, h=h)
    w = _rand(rng, (1, 300), "f32", 0.2, 1.0)[0].contiguous()
    snn.snn_gate_norm_fwd(d, x, None, None, None, None, w, None, h)
    _, want, _, ah = ref.gate_norm(_np(x), None, None, 1, "none", d.eps, 1.0, 1.0, _np(w))
    _near(h, want, ah, "bf16")
    ws = torch.empty(snn.snn_gate_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    for upstream in (gx, None):
        dx, dw = torch.empty_like(x), torch.empty(300, device="cuda")
        snn.snn_gate_norm_bwd(d, upstream, gh, x, None, None, None, None, None, None, w, dx, None,
                              None, None, None, dw, ws)
        want = ref.gate_norm_grads(_np(upstream) if upstream is not None else np.zeros((50, 300)),
                                   _np(gh), _np(x), None, None, 1, "none", d.eps, 1.0, 1.0,
                                   _np(w))
        _near(dx, want["dx"], want["abs_dx"], "f32")
        _near(dw, want["dw_pre"], want["abs_dw_pre"], "f32", rows=50)
    # no norm after the block: h and its gradient absent
    c = Case(20, 136, 1, "silu")
    c.h = None
    c.xo = torch.empty_like(c.x)
    snn.snn_gate_norm_fwd(c.d, c.x, c.y, c.g, c.w[0], c.w[1], None, c.xo, None)
    w_post, scale, _ = c.weights()
    xo, _, ax, _ = ref.gate_norm(_np(c.x), _np(c.y), _np(c.g), 1, "silu", c.d.eps, w_post, scale,
                                 1.0)
    _near(c.xo, xo, ax, "f32")
    dx, dy, dg = (torch.empty_like(c.x) for _ in range(3))
    ws = torch.empty(snn.snn_gate_norm_workspace_bytes(c.d), dtype=torch.uint8, device="cuda")
    snn.snn_gate_norm_bwd(c.d, c.gx, None, None, c.y, c.g, None, None, c.w[0], c.w[1], None, dx,
                          dy, dg, None, None, None, ws)
    want = ref.gate_norm_grads(_np(c.gx), None, None, _np(c.y), _np(c.g), 1, "silu", c.d.eps,
                               w_post, scale, 1.0)
    for name, t in (("dx", dx), ("dy", dy), ("dg", dg)):
        _near(t, want[name], want["abs_" + name], "f32", what=name)


def test_in_place_and_no_rows():
    c = Case(30, 520, 1, "silu", "f32", "bf16")
    c.fwd()
    x, h = c.x.clone(), torch.empty_like(c.h)
    snn.snn_gate_norm_fwd(c.d, x, c.y, c.g, *c.w, x, h)
    assert torch.equal(x, c.xo) and torch.equal(h, c.h)
    c.bwd()
    first = {k: v.clone() for k, v in c.got.items()}
    c.bwd()
    assert all(torch.equal(first[k], c.got[k]) for k in first)
    dx = c.gx.clone()
    ws = torch.empty(snn.snn_gate_norm_workspace_bytes(c.d), dtype=torch.uint8, device="cuda")
    snn.snn_gate_norm_bwd(c.d, dx, c.gh, c.xo, c.y, c.g, None, None, *c.w, dx,
                          torch.empty_like(c.y), torch.empty_like(c.g), None, None, None, ws)
    assert torch.equal(dx, first["dx"])
    e = Case(0, 64, 1, "silu")
    e.fwd()
    e.bwd()  # column sums over no rows are zero
    assert all((e.got[k] == 0).all() for k in ("dw_post", "ds", "dw_pre"))


def test_rows_of_zeros_and_of_bad_values():
    c = Case(6, 312, 3, "silu")
    c.y[2] = 0
    c.x[2] = 0
    c.fwd()
    assert (c.h[2] == 0).all()
    c.bwd()
    c.y[4, 7] = float("nan")
    c.x[5, 0] = float("inf")
    snn.snn_gate_norm_fwd(c.d, c.x, c.y, c.g, *c.w, c.xo, c.h, None, None)
    assert torch.isfinite(c.xo[:4]).all() and torch.isfinite(c.h[:4]).all()
    # the NaN stays in its group of x_out, and in its row of h
    assert torch.isfinite(c.xo[4, 104:]).all() and not torch.isfinite(c.xo[4, :104]).any()
    assert not torch.isfinite(c.h[4]).any()


def test_gate_extremes():
    for act in ("silu", "sigmoid"):
        c = Case(4, 64, 1, act)
        c.g[0] = torch.linspace(-200, 200, 64)
        c.g[1] = torch.linspace(-30, 30, 64)
        c.g[2] = 0
        c.fwd()
        c.bwd()


def test_gradient_against_differences():
    """Central differences of the 64-bit loss <x_out, gx> + <h, gh> along random
    directions: their error at step 1e-5 is below 1e-8 of the sum of absolute
    terms, the gradients' as above."""
    for act, groups in (("silu", 4), ("sigmoid", 1), ("mul", 2), ("none", 1)):
        c = Case(12, 96, groups, act)
        c.fwd()
        c.bwd()
        rng = np.random.default_rng(1)
        args = dict(x=_np(c.x), y=_np(c.y), g=_np(c.g) if c.g is not None else None)
        args.update(zip(("w_post", "scale", "w_pre"), c.weights()))
        gx, gh = _np(c.gx), _np(c.gh)

        def loss(**a):
            xo, h, _, _ = ref.gate_norm(a["x"], a["y"], a["g"], groups, act, c.d.eps, a["w_post"],
                                        a["scale"], a["w_pre"])
            return (xo * gx).sum() + (h * gh).sum()

        for name, grad in (("x", "dx"), ("y", "dy"), ("g", "dg"), ("w_post", "dw_post"),
                           ("scale", "ds"), ("w_pre", "dw_pre")):
            if args[name] is None:
                continue
            step = rng.standard_normal(args[name].shape)
            e = 1e-5
            diff = (loss(**{**args, name: args[name] + e * step}) -
                    loss(**{**args, name: args[name] - e * step})) / (2 * e)
            terms = _np(c.got[grad]) * step
            # x_out as the kernel rounded it moves the gradients by fp32 roundings too
            assert abs(diff - terms.sum()) <= 256 * ref.EPS32 * np.abs(terms).sum() + 1e-5, name


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("block", [128, 64, 16, 8])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 127), (5, 128), (4, 129), (17, 1000), (300, 4104),
                                    (2000, 50)])
def test_checkpoint_values(rows, n, block, dt):
    rng = np.random.default_rng(n)
    wide = _rand(rng, (rows, n), dt, pad=5, off=2)
    scales = torch.as_tensor(10.0 ** rng.integers(-4, 4, (rows, 1)), device="cuda")
    wide.copy_(wide.float() * scales)
    for x in (wide, wide.contiguous()):
        kept = torch.full((snn.snn_checkpoint_bytes(rows, n, block) + 64,), 77,
                          dtype=torch.uint8, device="cuda")
        snn.snn_checkpoint_save(x, kept, block)
        assert (kept[-64:] == 77).all()
        want = ref.quantised(x.float().cpu().numpy(), block)
        back = torch.full((rows, n), float("nan"), device="cuda")
        snn.snn_checkpoint_load(kept, back, block)
        assert np.array_equal(back.cpu().numpy(), want)
        out = _nan_like(x)
        snn.snn_checkpoint_load(kept, out, block)
        assert torch.equal(out.cpu(), torch.as_tensor(want).to(TYPES[dt]))
    # at most half a step of the block's scale from the value itself
    x32 = x.float().cpu().numpy()
    for a in range(0, n, block):
        top = np.abs(x32[:, a:a + block]).max(1, keepdims=True)
        assert (np.abs(want[:, a:a + block] - x32[:, a:a + block]) <= top / 254 * (1 + 1e-4)).all()


def test_checkpoint_of_zeros_tiny_and_bad_values():
    x = torch.zeros((4, 300), device="cuda")
    x[1, :128] = 1e-35
    x[1, 130] = 3e38
    x[2, 5] = float("nan")
    x[2, 200] = float("-inf")
    x[3, 299] = 2.0
    kept = torch.empty(snn.snn_checkpoint_bytes(4, 300), dtype=torch.uint8, device="cuda")
    back = torch.empty_like(x)
    snn.snn_checkpoint_save(x, kept)
    snn.snn_checkpoint_load(kept, back)
    want = ref.quantised(x.cpu().numpy())
    assert np.array_equal(back.cpu().numpy(), want, equal_nan=True)
    assert (back[0] == 0).all() and (back[1, :128] == 0).all() and torch.isnan(back[2, :256]).all()
    assert (back[2, 256:] == 0).all() and abs(back[3, 299].item() - 2.0) < 1e-6


def test_checkpoint_offsets_past_32_bits():
    rows, n = 2200000, 1000  # over 2^31 codes
    x = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    x[-2:] = torch.linspace(-3, 5, 2 * n).view(2, n)
    x[:1] = 1.0
    kept = torch.empty(snn.snn_checkpoint_bytes(rows, n), dtype=torch.uint8, device="cuda")
    snn.snn_checkpoint_save(x, kept)
    want = ref.quantised(x[-2:].float().cpu().numpy())
    x[-2:] = 0
    snn.snn_checkpoint_load(kept, x)
    assert torch.equal(x[-2:].cpu(), torch.as_tensor(want).to(torch.bfloat16))
    assert (x[:1] == 1.0).all()


def test_graph_replays():
    c = Case(200, 768, 6, "silu", "f32", "f16", ckpt=128)
    c.fwd(), c.bwd()
    want = {k: v.clone() for k, v in c.got.items()}
    want["xo"], want["h"] = c.xo.clone(), c.h.clone()
    ws = torch.empty(snn.snn_gate_norm_workspace_bytes(c.d), dtype=torch.uint8, device="cuda")
    out = dict(c.got, xo=c.xo, h=c.h)

    def call():
        snn.snn_gate_norm_fwd(c.d, c.x, c.y, c.g, *c.w, c.xo, c.h, c.y8, c.g8)
        snn.snn_gate_norm_bwd(c.d, c.gx, c.gh, c.xo, None, None, c.y8, c.g8, *c.w,
                              *(c.got[k] for k in ("dx", "dy", "dg", "dw_post", "ds", "dw_pre")),
                              ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for k, t in out.items():
            assert torch.equal(t, want[k]), k
