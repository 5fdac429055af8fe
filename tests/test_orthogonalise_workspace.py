"""What the orthogonalised updates ask for as workspace: what their way needs, and no more (no GPU)."""
import pytest

MIB = 1 << 20


@pytest.fixture(scope="module")
def wap():
    import paper_1811_01532_amd as w
    w.lib()
    return w


def asked(wap, *sizes):
    orth = wap.wap_orthogonalise_workspace_bytes(wap.ns_desc(), [wap.ns_matrix(r, c, None, None) for r, c in sizes])
    muon = wap.wap_muon_workspace_bytes(wap.muon_desc(), [wap.muon_matrix(r, c, 0.1, None, None, None, None) for r, c in sizes])
    assert orth == muon
    return orth


@pytest.mark.parametrize("rows,cols", [(1, 1), (64, 640), (640, 64), (64, 27), (1, 640)])
def test_one_work_group_keeps_everything_to_itself(wap, rows, cols):
    assert 0 < asked(wap, (rows, cols)) <= 4096
    assert asked(wap, *[(rows, cols)] * 16) <= 16 * 4096


@pytest.mark.parametrize("rows,cols", [(64, 641), (641, 64), (3, 20000), (64, 32768)])
def test_several_work_groups_keep_x_and_their_sums(wap, rows, cols):
    groups = (max(rows, cols) + 511) // 512
    assert asked(wap, (rows, cols)) <= groups * (64 * 512 * 4 + 2 * 10 * 1024) + 4096


@pytest.mark.parametrize("rows,cols", [(16, 1 << 20), (1 << 24, 8), (64, 32769), (65, 64), (65, 100000), (512, 4608), (4096, 4096), (25088, 4096)])
def test_tiles_keep_x_twice_its_rest_and_two_squares(wap, rows, cols):
    n = min(rows, cols)
    up8 = lambda v: (v + 7) // 8 * 8
    tiles = (n + 63) // 64 * ((n + 63) // 64 + 1) // 2
    parts = min(64 * MIB, 32 * tiles * 64 * 64 * 4)  # of X X^T, where it is divided
    assert asked(wap, (rows, cols)) <= 3 * 2 * rows * up8(cols) + 2 * 2 * n * up8(n) + parts + 8 * tiles + 16384


def test_a_small_matrix_takes_the_way_of_the_largest_of_its_set(wap):
    alone, beside = asked(wap, (16, 4096)), asked(wap, (16, 4096), (300, 300)) - asked(wap, (300, 300))
    assert beside < 3 * 2 * 16 * 4096 + 32 * 64 * 64 * 4 + 16384
    assert alone <= 8 * (64 * 512 * 4 + 2 * 10 * 1024) + 4096
