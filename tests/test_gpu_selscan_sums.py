"""Sums of the scan's gradients over many tokens in one sequence: the error of a sum of
terms of one sign grows with the longest chain of additions, which is a tile's and then the
tiles'."""
import pytest

import paper_2211_10725_amd as snn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("N", [1, 16, 20])
def test_gradient_of_the_rates_over_many_equal_tokens(N):
    """The same token 8192 times, in as many channels as leave the sequence uncut: from the
    first few on each adds the same term, g h exp(d a) d, and a rounding of the sum that
    goes the same way each time.  (T / 16 + 16) roundings of the sum; of a term, with
    exp(d a) <= 0.7, each of g and h has at most 4 of its own a token, summed over 1 / (1 -
    exp(d a)) <= 3.4 tokens, and their factors' few: 64."""
    T, n = 8192, 32 * 321
    full = dict(device="cuda", dtype=torch.float32)
    u, dt, gy = (torch.full((T, 1, n), v, **full) for v in (0.7, 0.55, 1.3))
    b, c = (torch.full((T, 1, 1, N), v, **full) for v in (0.9, 1.1))
    a = -(1 + torch.arange(N * n, device="cuda") % 4001 / 4001.0).view(N, n)
    y = torch.empty_like(u)
    d = snn.selscan_desc(u, dt, b, c, y, delta_softplus=False)
    saved = torch.empty(snn.snn_selscan_saved_bytes(d), dtype=torch.uint8, device="cuda")
    ws = torch.empty(snn.snn_selscan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    ins = (u, dt, a, b, c, None, None, None, None)
    snn.snn_selscan_fwd(d, *ins, None, y, None, saved, ws)
    da, gb, gc = torch.empty_like(a), torch.empty_like(b), torch.empty_like(c)
    snn.snn_selscan_bwd(d, *ins, saved, gy, None, torch.empty_like(u), torch.empty_like(u), da, gb,
                        gc, None, None, None, None, ws)
    # in 64 bits, where sums over tokens of geometric series have closed forms
    step, x, g = (t[0, 0, 0].double() for t in (dt, u, gy))
    bv, cv = b[0, 0, 0, 0].double(), c[0, 0, 0, 0].double()
    e = (step * a.double()).exp()
    assert e.max() <= 0.7
    # h before token t (from 0): step x b (1 - e^t) / (1 - e); g after it: c gy (1 - e^(T - t)) / (1 - e)
    geo = (1 - e ** T) / (1 - e)                 # sum over t of e^t, and of e^(T - 1 - t)
    total = T - geo - e * geo + T * e ** T       # of (1 - e^t) (1 - e^(T - t))
    want = step * e * (step * x * bv) * (cv * g) * total / (1 - e) ** 2
    err = ((da.double() - want).abs() / want).max().item()
    assert err <= (T / 16 + 16 + 64) * U, err / U
