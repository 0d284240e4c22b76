"""Short causal convolution with its backward and single tokens against the 64-bit
reference, whose carried error is the tolerance (``selective_reference``)."""
import numpy as np
import pytest

import paper_2211_10725_amd as snn
from tests import selective_reference as ref
from tests.test_gpu_selscan import TYPES, _dev, _nan_like, _np, _room

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

GRADS = ["dx", "dw", "dbias", "dstate"]


class Case:
    def __init__(self, T, B, n, K, act="silu", dt="f32", ragged=False, pad=0, off=0, seed=0,
                 state=True, bias=True, poison=False):
        rng = np.random.default_rng(seed)
        self.T, self.B, self.n, self.K, self.act, self.dt = T, B, n, K, act, dt

        def rows():
            return _dev(rng.standard_normal((T, B, n + pad + off)), dt)[:, :, off:off + n]

        self.x, self.gy = rows(), rows()
        self.w = _dev(rng.standard_normal((K, n)))
        self.bias = _dev(rng.standard_normal(n)) if bias else None
        self.init = _dev(rng.standard_normal((B, K - 1, n))) if state else None
        self.gs = _dev(rng.standard_normal((B, K - 1, n))) if state else None
        lens = np.full(B, T)
        if ragged:  # T, then short ones (below the window too), then longer ones
            lens = np.array([T if i == 0 else i - 1 if i < K else (i * 5) % (T + 1)
                             for i in range(B)]).clip(max=T)
        self.lens = torch.as_tensor(lens, dtype=torch.int32).cuda() if ragged else None
        if poison:
            for x in (self.x, self.gy):
                for i in range(B):
                    x[lens[i]:, i] = [float("nan"), float("inf")][i % 2]
        zero = np.zeros((B, K - 1, n))
        self.args = [_np(self.x), _np(self.w), _np(self.bias) if bias else np.zeros(n), lens,
                     _np(self.init) if state else zero, act]
        self.grads_in = [_np(self.gy), _np(self.gs) if state else zero]
        self.y = _nan_like(self.gy)
        self.d = snn.shortconv_desc(self.x, self.y, K, act)
        self.ws = _room(snn.snn_shortconv_workspace_bytes(self.d))
        self.out = torch.full((B, K - 1, n), float("nan"), device="cuda")

    def fwd(self):
        snn.snn_shortconv_fwd(self.d, self.x, self.w, self.bias, self.lens, self.init, self.y,
                              self.out)

    def bwd(self):
        new = {"dx": self.x, "dw": self.w, "dbias": self.bias, "dstate": self.out}
        self.got = {k: None if t is None else _nan_like(t) for k, t in new.items()}
        snn.snn_shortconv_bwd(self.d, self.x, self.w, self.bias, self.lens, self.init, self.gy,
                              self.gs, *(self.got[k] for k in GRADS), self.ws)

    def check(self):
        self.fwd()
        self.bwd()
        y, state, want = ref.shortconv(*self.args, *self.grads_in)
        ref.near(_np(self.y), y, self.dt, "y")
        assert np.array_equal(_np(self.out), state)  # inputs, as they are
        for k in GRADS:
            if self.got[k] is not None:
                ref.near(_np(self.got[k]), want[k], self.dt if k == "dx" else "f32", k)


@pytest.mark.parametrize("K", range(2, 9))
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dt", list(TYPES))
def test_widths(K, act, dt):
    Case(45, 2, 40, K, act, dt, seed=K).check()


# one of each, a token less and more than a window, slice and workgroup, odd channels
@pytest.mark.parametrize("T,B,n", [(1, 1, 1), (2, 3, 5), (3, 1, 8), (4, 2, 9), (8, 1, 511),
                                   (9, 2, 512), (31, 1, 513), (33, 1, 3), (129, 2, 7),
                                   (300, 1, 1001), (40, 70, 1030)])
@pytest.mark.parametrize("dt", list(TYPES))
def test_sizes(T, B, n, dt):
    Case(T, B, n, 4, dt=dt, seed=T).check()


@pytest.mark.parametrize("K", [2, 4, 8])
@pytest.mark.parametrize("dt", list(TYPES))
def test_ragged_lengths_and_what_lies_behind(K, dt):
    Case(50, 12, 33, K, dt=dt, ragged=True, poison=True, seed=K).check()


@pytest.mark.parametrize("pad,off", [(8, 0), (5, 3), (1, 1)])
@pytest.mark.parametrize("dt", ["f32", "f16"])
def test_slices_of_any_alignment(pad, off, dt):
    Case(37, 2, 70, 4, dt=dt, pad=pad, off=off).check()


def test_without_state_and_bias():
    Case(30, 2, 24, 3, state=False, bias=False).check()


def test_no_tokens_and_no_sequences():
    for T, B in ((0, 3), (4, 0)):
        c = Case(T, B, 20, 4)
        c.fwd()
        c.bwd()
        assert torch.equal(c.out, c.init) or T
        assert torch.equal(c.got["dstate"], c.gs) or T
        assert (c.got["dw"] == 0).all() and (c.got["dbias"] == 0).all()


@pytest.mark.parametrize("T", [1, 2, 200])
def test_state_in_place(T):
    c = Case(T, 3, 40, 4, seed=T)
    c.fwd()
    y, out = c.y.clone(), c.out.clone()
    c.out = c.init
    c.fwd()
    assert torch.equal(c.y, y) and torch.equal(c.init, out)


@pytest.mark.parametrize("n", [513, 519, 1030, 261])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_state_in_place_where_a_row_ends_within_a_run(n, dt):
    """The last run's neighbour may belong to another workgroup."""
    c = Case(5, 64, n, 4, dt=dt, seed=n, ragged=True)
    c.fwd()
    y, out = c.y.clone(), c.out.clone()
    c.out = c.init
    c.fwd()
    assert torch.equal(c.y, y) and torch.equal(c.init, out)


def test_same_call_same_bits_and_optional_outputs():
    c = Case(600, 3, 96, 4, dt="bf16")
    c.fwd()
    c.bwd()
    first = {k: v.clone() for k, v in c.got.items()}
    c.bwd()
    assert all(torch.equal(first[k], c.got[k]) for k in GRADS)
    snn.snn_shortconv_bwd(c.d, c.x, c.w, c.bias, None, c.init, c.gy, None, c.got["dx"], None, None,
                          None, c.ws)
    c.grads_in[1] = np.zeros_like(c.grads_in[1])
    ref.near(_np(c.got["dx"]), ref.shortconv(*c.args, *c.grads_in)[2]["dx"], "bf16", "dx")


@pytest.mark.parametrize("K", range(2, 9))
@pytest.mark.parametrize("dt", list(TYPES))
def test_step(K, dt):
    B, n = 5, 1030
    c = Case(1, B, n, K, dt=dt, seed=K, pad=2, off=1)
    pool = torch.randn((B + 3, K - 1, n), device="cuda")
    slots = torch.randperm(B + 3, device="cuda")[:B].to(torch.int32)
    slots[1] = B + 3
    keep, at = [0, 2, 3, 4], slots.long()
    out = pool.clone()
    snn.snn_shortconv_step(c.d, c.x, c.w, c.bias, slots, out, out, c.y)
    c.args[4] = _np(pool[at.clamp(max=B + 2)])
    y, state = ref.shortconv(*c.args)
    ref.near(_np(c.y)[0][keep], y[0][keep], dt, "y")
    assert np.array_equal(_np(out[at[keep]]), state[keep])
    assert (c.y[0, 1] == 0).all()
    rest = torch.ones(B + 3, dtype=torch.bool, device="cuda")
    rest[at[keep]] = False
    assert torch.equal(out[rest], pool[rest])


def test_steps_continue_a_prompt():
    c = Case(9, 2, 30, 4, seed=2)
    c.fwd()
    state, y = c.init.clone(), torch.empty_like(c.y)
    d = snn.shortconv_desc(c.x[:1], y[:1], 4, "silu")
    for t in range(9):
        snn.snn_shortconv_step(d, c.x[t:t + 1], c.w, c.bias, None, state, state, y[t:t + 1])
    assert torch.equal(y, c.y) and torch.equal(state, c.out)


def test_far_apart_tokens():
    c = Case(3, 1, 40, 4, dt="bf16")
    far = torch.empty(2 * (1 << 31) + 64, dtype=torch.bfloat16, device="cuda")
    x = far.as_strided((3, 1, 40), (1 << 31, 40, 1))
    x.copy_(c.x)
    c.x = x
    c.d = snn.shortconv_desc(c.x, c.y, 4, "silu")
    c.fwd()
    ref.near(_np(c.y), ref.shortconv(*c.args)[0], "bf16", "y")


def test_infinities_reach_their_window_only():
    c = Case(30, 1, 12, 4, "none")
    c.fwd()
    y = c.y.clone()
    c.x[11, 0, 5] = float("nan")
    c.fwd()
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[11:15, 0, 5] = True
    assert torch.isnan(c.y[bad]).all() and torch.equal(c.y[~bad], y[~bad])


def test_replayed_graph_and_other_stream():
    c = Case(150, 2, 64, 4, dt="bf16", seed=6)
    c.fwd()
    c.bwd()
    got = [c.y, c.out] + [c.got[k] for k in GRADS]
    want = [t.clone() for t in got]

    def both():
        c.fwd()
        snn.snn_shortconv_bwd(c.d, c.x, c.w, c.bias, c.lens, c.init, c.gy, c.gs,
                              *(c.got[k] for k in GRADS), c.ws)

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
