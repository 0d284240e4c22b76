"""Scans that are cut into segments, in every type, against the 64-bit reference: sequences
that end long before their last segment, several groups, more integrators than one round."""
import numpy as np
import pytest

import paper_2211_10725_amd as snn
from tests import selective_reference as ref
from tests.test_gpu_selscan import GRADS, TYPES, Case, _nan_like

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _with_lengths(c, lens):
    c.lens = torch.as_tensor(lens, dtype=torch.int32).cuda()
    c.args[8] = np.asarray(lens)
    return c


# ragged: lengths of 700, 501, 301 and 101 tokens in segments of 64
@pytest.mark.parametrize("N,G", [(20, 1), (20, 2), (64, 1), (64, 2), (16, 3), (5, 2)])
@pytest.mark.parametrize("dt", list(TYPES))
def test_ragged_segments(N, G, dt):
    Case(700, 4, 66, N, G, dt=dt, ragged=True, poison=True, seed=N + G).check()


@pytest.mark.parametrize("lens", [[0, 640, 0], [1, 17, 640], [64, 128, 65], [0, 0, 0]], ids=str)
@pytest.mark.parametrize("N", [17, 64])
def test_sequences_that_end_at_and_beside_a_segment(N, lens):
    """Of the segments past a sequence's end each still has its own gradient to pass on:
    none."""
    _with_lengths(Case(640, 3, 40, N, seed=N), lens).check()


@pytest.mark.parametrize("gate,soft", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("N", [8, 16, 24])
@pytest.mark.parametrize("dt", list(TYPES))
def test_options(gate, soft, N, dt):
    Case(400, 2, 40, N, 2, dt=dt, gate=gate, soft=soft, ragged=True, seed=N).check()


def test_state_gradients_of_empty_segments_are_passed_on():
    """Of a sequence that ended in its first segment, or has no token, the gradient of the
    state after it enters the one before it: as it is over no tokens."""
    c = _with_lengths(Case(900, 3, 64, 40, seed=3), [0, 5, 900])
    c.fwd()
    c.bwd()
    assert torch.equal(c.got["dstate"][0], c.gs[0]) and torch.equal(c.out[0], c.init[0])
    for k in ("du", "ddt", "dz", "db", "dc"):
        assert (c.got[k][:, 0] == 0).all() and (c.got[k][5:, 1] == 0).all(), k
    # the same bits whatever ran before on the device
    first = {k: c.got[k].clone() for k in GRADS}
    for seed in range(3):
        other = Case(900, 3, 64, 40, seed=seed + 10)
        other.fwd()
        other.bwd()
        c.bwd()
        assert all(torch.equal(first[k], c.got[k]) for k in GRADS)


def test_a_plan_of_one_segment_agrees():
    """Two sequences' gradients among enough others to leave them uncut, and by themselves
    in segments: the same within twice the reference's error of each."""
    T, n, N = 256, 64, 20
    many = Case(T, 200, n, N, ragged=True, seed=1)
    many.fwd()
    many.bwd()
    few = Case(T, 2, n, N, ragged=True, seed=1)
    for name in ("u", "step", "z", "gy", "b", "c"):
        setattr(few, name, getattr(many, name)[:, :2].contiguous())
    few.a, few.skip, few.bias = many.a, many.skip, many.bias
    few.init, few.gs, few.lens = many.init[:2].clone(), many.gs[:2].clone(), many.lens[:2].clone()
    few.y = _nan_like(few.gy)
    few.d = snn.selscan_desc(few.u, few.step, few.b, few.c, few.y, few.z)
    few.fwd()
    few.bwd()

    def np64(x):
        return x.detach().double().cpu().numpy()

    want = ref.selscan(*(np64(x) for x in (few.u, few.step, few.a, few.b, few.c, few.skip,
                                           few.bias, few.z, few.lens, few.init)), True,
                       np64(few.gy), np64(few.gs))[2]
    for k in ("du", "ddt", "db", "dc", "dz"):
        ref.near(np64(few.got[k]), want[k], "f32", k)
        ref.near(np64(many.got[k][:, :2]), want[k], "f32", k)
    ref.near(np64(many.got["dstate"][:2]), want["dstate"], "f32", "dstate")
    ref.near(np64(few.got["dstate"]), want["dstate"], "f32", "dstate")
