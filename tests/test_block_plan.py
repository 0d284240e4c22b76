"""How linear attention cuts sequences, seen from its workspace: the states of its
segments (no GPU needed)."""
import pytest

import paper_2211_10725_amd as snn

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads", [60, 128, 129, 192, 255, 256])
def test_long_sequences_are_cut_while_two_workgroups_fit_a_unit(heads, dt):
    """512 workgroups of heads of 128 are resident at once: up to 256 uncut ones
    leave room for a second segment, which long sequences gain from in every type."""
    q = torch.empty(4096, 1, 1, 128, dtype=dt).expand(4096, 1, heads, 128)
    d = snn.linattn_desc(q, q, q, q, forward_only=True)
    assert snn.snn_linattn_workspace_bytes(d) >= 2 * heads * 128 * 128 * 4


def test_more_heads_than_that_are_not():
    q = torch.empty(4096, 1, 1, 128).expand(4096, 1, 257, 128)
    assert snn.snn_linattn_workspace_bytes(snn.linattn_desc(q, q, q, q, forward_only=True)) == 0


@pytest.mark.parametrize("T,heads,cut", [(384, 129, True), (384, 192, False), (512, 255, False),
                                         (800, 255, True), (800, 129, True)])
def test_two_fp32_segments_only_of_long_sequences(T, heads, cut):
    q = torch.empty(T, 1, 1, 128).expand(T, 1, heads, 128)
    d = snn.linattn_desc(q, q, q, q, forward_only=True)
    assert (snn.snn_linattn_workspace_bytes(d) > 0) == cut
