"""Sizes whose threads pass 2^32, more than one dimension of a launch may have."""
import pytest

import paper_2211_10725_amd as snn
from tests.test_gpu_linattn import Case

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


def test_linear_attention_backward_of_more_heads_than_one_launch():
    """5.6 million heads: three gradients of a workgroup of 256 threads each pass
    2^32.  One token of integer values, so that every sum is exact."""
    B, H, d = 349600, 16, 8
    assert 3 * B * H >= 2 ** 24
    gen = torch.Generator(device="cuda").manual_seed(0)
    q, k, v, go = (torch.randint(-3, 4, (1, B, H, d), generator=gen, device="cuda").half()
                   for _ in range(4))
    desc = snn.linattn_desc(q, k, v, go, 1.0)
    decay = torch.full((H,), 0.5, device="cuda")
    dq, dk, dv = (torch.full_like(x, float("nan")) for x in (q, k, v))
    ws = torch.empty(max(16, snn.snn_linattn_workspace_bytes(desc)), dtype=torch.uint8,
                     device="cuda")
    snn.snn_linattn_bwd(desc, q, k, v, decay, None, None, go, None, dq, dk, dv, None, ws)
    f = [x.float() for x in (q, k, v, go)]
    vg = (f[2] * f[3]).sum(3, keepdim=True)
    kq = (f[0] * f[1]).sum(3, keepdim=True)
    for got, want in ((dq, f[1] * vg), (dk, f[0] * vg), (dv, kq * f[3])):
        assert torch.equal(got.float(), want)


@pytest.mark.parametrize("H,T", [(131, 400), (200, 790)])
def test_segments_of_more_heads_than_half_the_units(H, T):
    c = Case(T, 1, H, H, 72, 104, "f32")
    c.check_fwd()


def test_segments_of_roles_and_heads_between_half_and_all_units():
    c = Case(400, 1, 45, 45, 72, 80, "f32", lens=[393])
    c.check_fwd()
    c.check_bwd()
