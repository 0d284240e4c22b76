"""The sequence models on slices of wider spike tensors, and on what is no spike train of
theirs."""
import pytest

from paper_2211_10725_amd.sequence import spike_trains
from tests.test_gpu_sequence_streams import NETS, _flat

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(params=list(NETS))
def net(request):
    return NETS[request.param](20, 3)


def _slices(x):
    """x [T,B,n] again, as slices of tensors that hold more."""
    T, B, n = x.shape
    more = torch.full((T + 2, B + 2, n + 3), 1, dtype=torch.uint8, device="cuda")
    for part in (more[:T, :B, :n], more[1:T + 1, 1:B + 1, 2:n + 2], more[2:, 2:, 3:]):
        part.copy_(x)
        yield part
        more.fill_(1)
    yield x.transpose(0, 1).contiguous().transpose(0, 1)
    flat = torch.ones(x.numel() + 5, dtype=torch.uint8, device="cuda")
    flat[5:] = x.flatten()
    yield flat[5:].view(T, B, n)


def test_slices_are_what_they_hold(net):
    x, y = (torch.as_tensor(a).cuda() for a in spike_trains(20, 3, 32, 4, seed=1))
    states = net.states(3)
    want, step = net.prompt(x, states), net.step(x[4].clone(), states)
    loss = net.train_step(x, y).item()
    grads = [g.clone() for g in net.grads]
    for part in _slices(x):
        again = net.states(3)
        assert torch.equal(net.prompt(part, again), want)
        assert torch.equal(net.step(part[4], again), step)
        assert all(torch.equal(a, b) for a, b in zip(_flat(again), _flat(states)))
        assert net.train_step(part, y).item() == loss
        assert all(torch.equal(g, w) for g, w in zip(net.grads, grads))


def test_other_shapes_and_types_are_refused(net):
    x, y = (torch.as_tensor(a).cuda() for a in spike_trains(20, 3, 32, 4))
    wide = torch.zeros((20, 3, 33), dtype=torch.uint8, device="cuda")
    for bad in (wide, x.float(), x[..., :31], x.cpu()):
        with pytest.raises(ValueError):
            net.prompt(bad, net.states(3))
        with pytest.raises(ValueError):
            net.step(bad[0], net.states(3))
        with pytest.raises(ValueError):
            net.train_step(bad, y)
    for bad in (x[:19], x[:, :2], torch.cat([x, x], 1)):  # of another length or batch
        with pytest.raises(ValueError):
            net.train_step(bad, y)
    for bad in (y.long(), y[:2], y.float(), y.cpu(), torch.stack([y, y], 1)[:, 0]):
        with pytest.raises(ValueError):
            net.train_step(x, bad)
