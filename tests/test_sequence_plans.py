"""The buffers that the sequence model keeps between calls (no GPU needed: none
runs)."""
import pytest

import paper_2211_10725_amd as snn
from paper_2211_10725_amd.sequence import SequenceNet

torch = pytest.importorskip("torch")


def _net(**more):
    return SequenceNet(16, heads=2, kv_heads=1, d_k=16, d_v=16, blocks=2, n_out=4, T=20, B=3,
                       device="cpu", **more)


def _held(net, train=False):
    """Bytes of the distinct buffers that the kept plans hold."""
    seen = {}
    for key, p in net.plans.items():
        if key[2] != train:
            continue
        for x in vars(p).values():
            for t in x if isinstance(x, list) else [x]:
                if isinstance(t, torch.Tensor):
                    seen[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
    return sum(seen.values())


def test_prompts_of_many_lengths_do_not_grow_without_end():
    net = _net()
    net._plan(200, 8)
    one = _held(net)
    for T in range(1, 200):
        net._plan(T, 8)
        assert _held(net) <= 5 * one
    assert (199, 8, False) in net.plans                # the last ones stay


def test_steps_with_changing_numbers_of_requests_keep_their_plans():
    net = _net()
    net._plan(400, 8)
    plans = [net._plan(1, b) for b in range(1, 33)]
    assert [net._plan(1, b) for b in range(1, 33)] == plans


def test_the_longest_unused_goes_first():
    net = _net()
    first = net._plan(100, 8)
    for T in range(101, 140):
        net._plan(T, 8)
        assert net._plan(100, 8) is first              # in use all the time
    assert (101, 8, False) not in net.plans


def test_the_training_plan_and_those_of_graphs_stay():
    net = _net()
    train, graph = net._plan(20, 3, True), net._plan(50, 2)
    graph.stays = True
    for T in range(60, 160):
        net._plan(T, 8)
    assert net._plan(20, 3, True) is train and net._plan(50, 2) is graph


def test_buffers_of_a_shape_are_its_own():
    """Two shapes may run on two streams at a time."""
    net = _net()
    a, b = net._plan(30, 2), net._plan(1, 2)
    assert not {t.data_ptr() for t in a.bufs} & {t.data_ptr() for t in b.bufs}
    assert a.ws.numel() >= snn.snn_linattn_workspace_bytes(a.attn)
