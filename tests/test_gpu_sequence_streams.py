"""The sequence models on several streams and in several graphs at a time: calls of one
shape share no buffer unless one stream orders them."""
import pytest

from paper_2211_10725_amd.selective import SelectiveNet
from paper_2211_10725_amd.sequence import SequenceNet, spike_trains

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NETS = {
    "linear attention": lambda T, B: SequenceNet(32, heads=2, kv_heads=1, d_k=16, d_v=32, blocks=2,
                                                 n_out=4, T=T, B=B),
    "selective": lambda T, B: SelectiveNet(32, n=48, width=64, states=8, blocks=2, n_out=4, T=T,
                                           B=B),
}


@pytest.fixture(params=list(NETS))
def make(request):
    return NETS[request.param]


def _spikes(T, B, seed):
    return torch.as_tensor(spike_trains(T, B, 32, 4, seed=seed)[0]).cuda()


def _pointers(plan):
    return {t.data_ptr() for t in plan.bufs if t.numel()}


def _flat(states):
    return [t for s in states for t in (s if isinstance(s, tuple) else [s])]


def test_plans_of_two_streams_and_of_graphs_share_no_buffer(make):
    net, side = make(30, 3), torch.cuda.Stream()
    for T, train in ((1, False), (30, False), (30, True)):
        here = net._plan(T, 3, train)
        with torch.cuda.stream(side):
            there = net._plan(T, 3, train)
            assert net._plan(T, 3, train) is there
        assert net._plan(T, 3, train) is here
        assert not _pointers(here) & _pointers(there)
        seen = [_pointers(here), _pointers(there)]
        graphs, kept = [], []
        for _ in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                kept.append(net._plan(T, 3, train))
                kept[-1].ws.zero_()
            seen.append(_pointers(kept[-1]))
        assert len(set.union(*seen)) == sum(len(s) for s in seen)
        assert net._plan(T, 3, train) is here


def test_many_streams_keep_their_plans(make):
    """The bound on what is kept counts each stream's own."""
    net, streams, plans = make(200, 4), [torch.cuda.Stream() for _ in range(8)], []
    for s in streams:
        with torch.cuda.stream(s):
            plans.append(net._plan(200, 4))
    for s, p in zip(streams, plans):
        with torch.cuda.stream(s):
            assert net._plan(200, 4) is p


@pytest.mark.parametrize("T", [1, 60])
def test_two_streams_at_a_time(make, T):
    B, calls = 5, 24
    net = make(60, B)
    data = [[_spikes(60, B, 2 * i + k)[:T].contiguous() for i in range(calls)] for k in range(2)]

    def run(x, states):
        return net.step(x[0], states) if T == 1 else net.prompt(x, states)

    want, ends = [], []
    for k in range(2):
        states = net.states(B)
        want.append([run(x, states) for x in data[k]])
        ends.append(states)
    torch.cuda.synchronize()
    streams, states = [torch.cuda.Stream() for _ in range(2)], [net.states(B) for _ in range(2)]
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(calls):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(run(data[k][i], states[k]))
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[k], want[k]))
        assert all(torch.equal(a, b) for a, b in zip(_flat(states[k]), _flat(ends[k])))


def test_two_graphs_and_eager_steps_at_a_time(make):
    B, calls = 5, 20
    net = make(1, B)
    data = [_spikes(calls, B, k) for k in range(3)]
    want = []
    for x in data:
        states = net.states(B)
        want.append([net.step(x[t], states) for t in range(calls)])
    streams = [torch.cuda.Stream() for _ in range(2)]
    spikes, states = [x[0].clone() for x in data[:2]], [net.states(B) for _ in range(3)]
    graphs, out = [], []
    for k in range(2):
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[k]):
            out.append(net.step(spikes[k], states[k]))
    torch.cuda.synchronize()
    got = [[], [], []]
    for t in range(calls):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                spikes[k].copy_(data[k][t])
                graphs[k].replay()
                got[k].append(out[k].clone())
        got[2].append(net.step(data[2][t], states[2]))
    torch.cuda.synchronize()
    for k in range(3):
        for t in range(calls):
            assert torch.equal(got[k][t], want[k][t]), (k, t)


def test_a_captured_training_step_beside_an_eager_one(make):
    """Gradients of a replayed step, with eager prompts of another stream between."""
    T, B = 40, 4
    net = make(T, B)
    x, y = (torch.as_tensor(a).cuda() for a in spike_trains(T, B, 32, 4, seed=3))
    loss = net.train_step(x, y).item()
    want = [g.clone() for g in net.grads]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = net.train_step(x, y)
    before = net.prompt(x, net.states(B))
    torch.cuda.synchronize()
    for _ in range(3):
        for g in net.grads:
            g.fill_(float("nan"))
        states = net.states(B)
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            beside = net.prompt(x, states)
        torch.cuda.synchronize()
        assert captured.item() == loss and torch.equal(beside, before)
        assert all(torch.equal(g, w) for g, w in zip(net.grads, want))
