"""Layer norm of many rows, whose workgroups take several each, against the 64-bit
reference: narrow rows in half as many workgroups, wide ones in all of them."""
import pytest

from tests.test_gpu_layer_norm import Case

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n", [(16400, 24), (8200, 600), (4100, 1500), (4097, 2049),
                                    (2050, 4097), (1100, 8200)])
@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("f16", "f16")], ids="-".join)
def test_rows(rows, n, types):
    Case(rows, n, *types, seed=n).check()
