"""Layer norm and its backward against the 64-bit reference and its tolerance
(``selective_reference``)."""
import numpy as np
import pytest

import paper_2211_10725_amd as snn
from tests import selective_reference as ref
from tests.test_gpu_selscan import TYPES, _dev, _nan_like, _np, _room

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PAIRS = [("f32", "f32"), ("f32", "f16"), ("f32", "bf16"), ("f16", "f16"), ("bf16", "bf16")]
EPS = 1e-5
WIDTHS = [1, 7, 8, 24, 511, 512, 513, 1001, 1024, 1025, 2048, 2056, 4096, 4097, 8192, 8200, 16383,
          16384]


class Case:
    def __init__(self, rows, n, x="f32", y="f32", pad=0, off=0, seed=0, weights=True, res=True,
                 mean=0.5):
        rng = np.random.default_rng(seed)

        def make(dt, shift=0.0):
            t = _dev(rng.standard_normal((rows, n + pad + off)) * 2 + shift, dt)
            return t[:, off:off + n]

        self.x, self.gy, self.xt, self.yt = make(x, mean), make(y), x, y
        self.gres = make(x) if res else None
        self.w, self.b = (_dev(rng.standard_normal(n) * 0.3 + 1) if weights else None
                          for _ in range(2))
        self.y, self.n, self.rows = _nan_like(self.gy), n, rows
        self.d = snn.layer_norm_desc(self.x, self.y, EPS)
        self.ws = _room(snn.snn_layer_norm_workspace_bytes(self.d))

    def run(self):
        snn.snn_layer_norm_fwd(self.d, self.x, self.w, self.b, self.y)
        self.dx = _nan_like(self.x)
        self.dw, self.db = (torch.full((self.n,), float("nan"), device="cuda") for _ in range(2))
        snn.snn_layer_norm_bwd(self.d, self.x, self.gy, self.gres, self.w, self.dx, self.dw,
                               self.db, self.ws)

    def check(self):
        self.run()
        w = _np(self.w) if self.w is not None else np.ones(self.n)
        b = _np(self.b) if self.b is not None else np.zeros(self.n)
        gres = _np(self.gres) if self.gres is not None else np.zeros((self.rows, self.n))
        y, g = ref.layer_norm(_np(self.x), w, b, self.d.eps, _np(self.gy), gres)
        ref.near(_np(self.y), y, self.yt, "y")
        ref.near(_np(self.dx), g["dx"], self.xt, "dx")
        ref.near(_np(self.dw), g["dw"], "f32", "dw")
        ref.near(_np(self.db), g["db"], "f32", "db")


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("types", PAIRS, ids="-".join)
def test_widths(n, types):
    Case(5, n, *types, seed=n).check()


@pytest.mark.parametrize("rows,n", [(1, 100), (3, 512), (1025, 40), (4099, 24), (600, 9000)])
def test_rows(rows, n):
    Case(rows, n, "f32", "bf16", seed=rows).check()


@pytest.mark.parametrize("pad,off", [(8, 0), (5, 3), (1, 1)])
@pytest.mark.parametrize("types", PAIRS, ids="-".join)
def test_slices_of_any_alignment(pad, off, types):
    Case(9, 333, *types, pad=pad, off=off).check()


def test_without_weights_and_residual():
    Case(20, 96, weights=False, res=False).check()


def test_a_mean_far_from_zero():
    """A mean of 1000 standard deviations costs ten bits, of x's own rounding alone."""
    Case(6, 700, mean=2000.0).check()


def test_constant_rows_and_rows_of_zeros():
    x = torch.zeros((3, 40), device="cuda")
    x[1] = 3.25
    y = torch.empty_like(x)
    b = torch.arange(40, device="cuda", dtype=torch.float32)
    snn.snn_layer_norm_fwd(snn.layer_norm_desc(x, y, EPS), x, None, b, y)
    assert torch.equal(y, b.expand(3, 40))


def test_in_place_and_residual_in_place():
    c = Case(50, 200)
    c.run()
    dx, x = c.dx.clone(), c.x.clone()
    snn.snn_layer_norm_bwd(c.d, c.x, c.gy, c.gres, c.w, c.gres, c.dw, c.db, c.ws)
    assert torch.equal(c.gres, dx)
    snn.snn_layer_norm_fwd(c.d, x, c.w, c.b, x)
    assert torch.equal(x, c.y)


def test_bad_values_stay_in_their_row():
    c = Case(6, 90)
    c.run()
    y = c.y.clone()
    c.x[2, 7] = float("nan")
    c.run()
    assert torch.isnan(c.y[2]).all() and torch.equal(c.y[[0, 1, 3, 4, 5]], y[[0, 1, 3, 4, 5]])


def test_no_rows_and_optional_outputs():
    c = Case(0, 30)
    c.run()
    assert (c.dw == 0).all() and (c.db == 0).all()
    c = Case(40, 30)
    c.run()
    dw, db = c.dw.clone(), c.db.clone()
    for w, b in ((c.dw, None), (None, c.db), (None, None)):
        c.dw.fill_(-1), c.db.fill_(-1)
        snn.snn_layer_norm_bwd(c.d, c.x, c.gy, c.gres, c.w, c.dx, w, b, c.ws)
        assert torch.equal(c.dw, dw if w is not None else torch.full_like(dw, -1))
        assert torch.equal(c.db, db if b is not None else torch.full_like(db, -1))


def test_replayed_graph_and_other_stream():
    c = Case(700, 130, "f32", "bf16")
    c.run()
    got = [c.y, c.dx, c.dw, c.db]
    want = [t.clone() for t in got]

    def both():
        snn.snn_layer_norm_fwd(c.d, c.x, c.w, c.b, c.y)
        snn.snn_layer_norm_bwd(c.d, c.x, c.gy, c.gres, c.w, c.dx, c.dw, c.db, c.ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    for t in got:
        t.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
