"""Workgroups of layer norm's backward, each with its own sums in the workspace (no GPU
needed)."""
import pytest

import paper_2211_10725_amd as snn

pytest.importorskip("torch")
UNITS = 256  # compute units


def _workgroups(rows, n):
    d = snn.LayerNormDesc(rows, n, snn.F32, snn.F32, 1e-5, n, n)
    return snn.snn_layer_norm_workspace_bytes(d) // (2 * n * 4)


@pytest.mark.parametrize("n", [1, 512, 1024, 1536, 2048, 2049, 4096, 4097, 8192, 8193, 12288, 16384])
@pytest.mark.parametrize("rows", [1024, 1100, 2048, 4096, 16384, 100000])
def test_many_rows_give_every_compute_unit_work(rows, n):
    threads = min(1024, max(64, 1 << (-(-n // 8) - 1).bit_length()))
    turns = -(-rows // max(1, 256 // threads))
    assert _workgroups(rows, n) >= min(turns, UNITS), "units without a row"
    # and eight waves to each, where there are rows for them
    assert _workgroups(rows, n) * max(256, threads) >= min(turns, 2 * UNITS) * 256
