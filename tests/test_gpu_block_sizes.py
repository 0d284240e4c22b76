"""Sizes whose threads pass 2^32, more than one dimension of a launch may have."""
import pytest

import paper_2211_10725_amd as snn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_checkpoint_of_more_rows_than_a_dimension_of_a_launch():
    """2^28 rows and a few, of 8 values: each row's largest value comes back as it
    was (127 of its scale's steps, rounded to 8 of fp16's 11 bits)."""
    rows = 2 ** 28 + 37
    x = torch.ones((rows, 8), dtype=torch.float16, device="cuda")
    x[::3, ::2] = -1.0
    x[-2:] = 4.0
    x[2 ** 27 - 1:2 ** 27 + 1] = 0.0
    kept = torch.empty(snn.snn_checkpoint_bytes(rows, 8), dtype=torch.uint8, device="cuda")
    snn.snn_checkpoint_save(x, kept)
    back = torch.full_like(x, float("nan"))
    snn.snn_checkpoint_load(kept, back)
    assert torch.equal(back, x)
