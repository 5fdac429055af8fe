"""The linear cross-entropy's gradient for some dozens of rows under more classes than a tile of dz may have between two rows (2^21): they are
taken in pieces."""
import pytest

from tests.test_gpu_linear_xent import check, make


@pytest.mark.parametrize("rows,classes", [(3, 1 << 24), (4, 12000000), (16, 1 << 22), (20, 2500000), (31, 2200000)])
def test_rows_of_dz_stay_within_a_tile_s_reach(rows, classes):
    """(On the host: what the workspace holds beside the statistics of a tile of 64 classes, the tables of 256-byte places and parts of dx.)"""
    import paper_1811_01532_amd as wap
    features = 8
    asked = wap.wap_linear_xent_workspace_bytes(wap.linear_xent_desc(rows, features, classes), True)
    statistics = rows * ((classes + 63) // 64) * 8
    assert asked <= statistics + rows * (1 << 21) * 2 + 32 * rows * features * 4 + 16 * 1024


@pytest.mark.gpu
@pytest.mark.parametrize("rows,features,classes", [(17, 8, (1 << 21) + 777), (24, 6, 2100000)])
def test_against_the_formula(rows, features, classes):
    print(f"[case] linear_xent {rows} x {features} -> {classes}", flush=True)
    check(*make(rows, features, classes, 0.1), features)
