"""What the sequence model returns stays the caller's: later calls of the same
shape leave it alone."""
import pytest

from paper_2211_10725_amd.sequence import SequenceNet, spike_trains

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _net(T, B):
    net = SequenceNet(32, heads=2, kv_heads=1, d_k=16, d_v=32, blocks=2, n_out=4, T=T, B=B)
    data = [torch.as_tensor(spike_trains(T, B, 32, 4, seed=i)[0]).cuda() for i in range(3)]
    return net, data


def test_currents_of_a_prompt_and_of_steps_stay():
    net, data = _net(40, 3)
    states = net.states(3)
    for call in (lambda x: net.prompt(x, states), lambda x: net.step(x[0], states),
                 lambda x: net.prompt(x[:1], states)):
        got = [call(x) for x in data[:1]]
        kept = got[0].clone()
        got += [call(x) for x in data[1:]]
        assert torch.equal(got[0], kept)
        assert not torch.equal(got[1], got[0]) and not torch.equal(got[2], got[1])


def test_losses_of_several_steps_stay():
    net, data = _net(40, 3)
    labels = [torch.as_tensor(spike_trains(40, 3, 32, 4, seed=i)[1]).cuda() for i in range(3)]
    net.init_adamw(lr=1e-2)
    losses, kept = [], []
    for x, y in zip(data, labels):
        losses.append(net.train_step(x, y))
        kept.append(losses[-1].item())
        net.update()
    assert [v.item() for v in losses] == kept and len(set(kept)) > 1


def test_prompts_of_many_lengths_on_another_stream():
    """Buffers given up on one stream while another may still read them."""
    net, _ = _net(40, 3)
    x = torch.as_tensor(spike_trains(300, 3, 32, 4)[0]).cuda()
    want = {T: net.prompt(x[:T].contiguous(), net.states(3)) for T in range(200, 300, 9)}
    net.plans.clear()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = {}
    for T in want:
        net._plan(T, 3)  # made on this stream, run on the other
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got[T] = net.prompt(x[:T].contiguous(), net.states(3))
        torch.full((1 << 20,), float("nan"), device="cuda")  # takes what is free here
    torch.cuda.synchronize()
    for T in want:
        assert torch.equal(got[T], want[T]), T
