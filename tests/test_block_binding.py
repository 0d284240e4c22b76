"""What the binding of the leaky sequence block refuses and accepts beside
``test_block_abi`` (no GPU needed: every refusal comes before the call)."""
import pytest

import paper_2211_10725_amd as snn

torch = pytest.importorskip("torch")


def _rows(n):
    """One row of n values that do not lie next to each other."""
    return {"every other": torch.empty(1, 2 * n)[:, ::2], "expanded": torch.empty(1, 1).expand(1, n),
            "column": torch.empty(n, 3).t()[:1]}


@pytest.mark.parametrize("what", ["x", "y", "gate", "x_out", "h"])
@pytest.mark.parametrize("how", list(_rows(8)))
def test_one_row_must_be_contiguous(how, what):
    x = torch.empty(1, 40)
    d = snn.gate_norm_desc(x, x, x, 1, "silu")
    a = dict(dict.fromkeys(("x", "y", "gate", "x_out", "h"), x), **{what: _rows(40)[how]})
    with pytest.raises(ValueError):
        snn.snn_gate_norm_fwd(d, a["x"], a["y"], a["gate"], None, None, None, a["x_out"], a["h"],
                              None, None, 0)


@pytest.mark.parametrize("what", ["grad_x_out", "grad_h", "x_out", "y", "gate", "grad_x",
                                  "grad_y", "grad_gate"])
def test_one_row_of_a_gradient_must_be_contiguous(what):
    x = torch.empty(1, 40)
    d = snn.gate_norm_desc(x, x, x, 1, "silu")
    names = ("grad_x_out", "grad_h", "x_out", "y", "gate", "grad_x", "grad_y", "grad_gate")
    a = dict(dict.fromkeys(names, x), **{what: _rows(40)["every other"]})
    with pytest.raises(ValueError):
        snn.snn_gate_norm_bwd(d, a["grad_x_out"], a["grad_h"], a["x_out"], a["y"], a["gate"], None,
                              None, None, None, None, a["grad_x"], a["grad_y"], a["grad_gate"],
                              None, None, None, None, 0)


def test_single_rows_and_single_values_of_any_stride_go_through():
    d = snn.gate_norm_desc(torch.empty(1, 40))
    for t in (torch.empty(1, 40), torch.empty(40), torch.empty(5, 80)[2:3, 8:48],
              torch.empty(1, 1, 40), torch.empty(3, 40)[1]):
        snn._need_rows("fn", "x", t, d, torch.float32, d.ld_x)
    one = snn.gate_norm_desc(torch.empty(1, 1))
    snn._need_rows("fn", "x", torch.empty(1, 7)[:, ::3][:, :1], one, torch.float32, one.ld_x)


def test_current_stream_without_the_private_names(monkeypatch):
    """The quick way to the current stream's handle is torch's own business: where
    it is absent, the public one is taken."""
    class Stream:
        cuda_stream = 1234

    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream)
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        with monkeypatch.context() as m:
            m.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
            m.delattr(torch._C, name, raising=False)
            assert snn._stream(None) == 1234
