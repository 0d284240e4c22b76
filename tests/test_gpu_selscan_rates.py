"""Rates of any finite size: integrators that forget at once, and steps of zero at which
they do not."""
import pytest

import paper_2211_10725_amd as snn
from tests import selective_reference as ref
from tests.test_gpu_selscan import Case, _np

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
FAST = (-1e30, -2.3e38, -2.4e38, -3.4028234e38)


# a part of a tile, segments, and sequences that end inside of them
@pytest.mark.parametrize("T,ragged", [(20, False), (20, True), (400, False), (400, True)])
@pytest.mark.parametrize("N", [4, 24])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_integrators_that_forget_at_once(T, ragged, N, dt):
    c = Case(T, 3, 40, N, dt=dt, ragged=ragged, seed=N)
    for i, a in enumerate(FAST):
        c.a[i % N, i::5] = a
    c.args[2] = _np(c.a)
    c.check()


def test_a_step_of_zero_keeps_the_state():
    """Raw steps of exactly zero: the state stays, whatever its rate."""
    c = Case(5, 2, 40, 16, soft=False, vecs=False, seed=1)
    c.step.zero_()
    for i, a in enumerate(FAST):
        c.a[i::4] = a
    c.fwd()
    assert torch.equal(c.out, c.init)
    d = snn.selscan_desc(c.u[:1], c.step[:1], c.b[:1], c.c[:1], c.y[:1], c.z[:1], False)
    state = c.init.clone()
    snn.snn_selscan_step(d, c.u[:1], c.step[:1], c.a, c.b[:1], c.c[:1], None, None, c.z[:1], None,
                         state, state, c.y[:1])
    assert torch.equal(state, c.init)


def test_a_rate_that_is_nan_shows():
    c = Case(20, 1, 40, 8, seed=2)
    c.fwd()
    y = c.y.clone()
    c.a[3, 7] = float("nan")
    c.fwd()
    assert torch.isnan(c.y[:, 0, 7]).all()
    same = torch.ones(40, dtype=torch.bool, device="cuda")
    same[7] = False
    assert torch.equal(c.y[..., same], y[..., same])
    ref.near(_np(c.y[..., same]), ref.V(_np(y[..., same])), "f32")
