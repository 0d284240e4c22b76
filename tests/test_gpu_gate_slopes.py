"""Slopes of the sigmoid and SiLU gates over their whole range, open gates
included: sigmoid'(g) = e^-|g| / (1 + e^-|g|)^2 in 64 bits, which cancels
nowhere.  Tolerance: 64 x 2^-24 of the sum of the absolute values of the slope's
terms (its exponential, reciprocal and products are good to a few units each)
times the factors beside it, and half a unit of the result's type."""
import numpy as np
import pytest

import paper_2211_10725_amd as snn
from tests import block_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
def test_gate_slope_over_its_range(act, dt, ckpt):
    rows, n, eps = 6, 1024, 1e-5
    t = torch.float32 if dt == "f32" else torch.bfloat16
    rng = np.random.default_rng(4)
    y = torch.as_tensor(rng.standard_normal((rows, n)), dtype=torch.float32).to(t).cuda()
    g = torch.linspace(-85, 85, n).repeat(rows, 1)
    g[1] = torch.linspace(-20, 20, n)
    g[2] = torch.linspace(8, 30, n)
    g[3] = torch.linspace(-400, 400, n)
    g = g.to(t).cuda()
    gx = torch.as_tensor(rng.standard_normal((rows, n)), dtype=torch.float32).cuda()
    d = snn.gate_norm_desc(gx, y, g, 1, act, eps)
    dx, dy, dg = torch.empty_like(gx), torch.empty_like(y), torch.empty_like(g)
    ws = torch.empty(snn.snn_gate_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    kept = [None, None]
    if ckpt:
        for i, x in enumerate((y, g)):
            kept[i] = torch.empty(snn.snn_checkpoint_bytes(rows, n), dtype=torch.uint8,
                                  device="cuda")
            snn.snn_checkpoint_save(x, kept[i])
    snn.snn_gate_norm_bwd(d, gx, None, None, *((None, None) if ckpt else (y, g)), *kept, None,
                          None, None, dx, dy, dg, None, None, None, ws)
    y, g = (x.float().cpu().numpy() for x in (y, g))
    if ckpt:
        y, g = ref.quantised(y), ref.quantised(g)
    y, g = y.astype(np.float64), g.astype(np.float64)
    e = np.exp(-np.abs(g))
    q = e / (1 + e) ** 2
    p = np.where(g >= 0, 1 / (1 + e), e / (1 + e))
    slope, terms = (q, q) if act == "sigmoid" else (p + g * q, p + np.abs(g) * q)
    beside = gx.double().cpu().numpy() * y / np.sqrt((y * y).mean(1, keepdims=True) +
                                                     np.float32(eps))
    want, absolute = beside * slope, np.abs(beside) * terms
    rel, least = ref.HALF_ULP[dt]
    err = np.abs(dg.double().cpu().numpy() - want)
    bound = 64 * ref.EPS32 * absolute + rel * np.abs(want) + least
    assert (err <= bound).all(), (float((err / bound).max()), g.ravel()[np.argmax(err / bound)])
