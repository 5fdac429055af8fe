"""GPU parity of the Newton-Schulz orthogonalisation and the Muon update over the range of fp32, with the formula in 64 bits: matrices and
columns whose norm, or its reciprocal, fp32 has no normal number for, on each way that a matrix can take (one work-group, several work-groups, tiles).

The bounds are those of the operators' other tests: a power of two that all of a matrix is multiplied by changes no rounding of the iteration."""
import pytest
import torch

from tests.test_gpu_orthogonalise import NORM_TOL, formula, matrix, near, orthogonalise

pytestmark = pytest.mark.gpu

WAYS = [(60, 200), (200, 60), (60, 1400), (1400, 60), (130, 264)]


@pytest.mark.parametrize("rows,cols", WAYS)
@pytest.mark.parametrize("factor", [1e-42, 1e-38, 1e-30, 1e30, 3e37])
def test_norms_at_the_ends_of_fp32(rows, cols, factor):
    """Without eps: the reciprocal of the norm is beyond fp32 at the lower end, a subnormal number at the upper one."""
    print(f"[case] orthogonalise {rows} x {cols} times {factor}", flush=True)
    u = matrix(rows, cols) * factor
    assert torch.isfinite(u).all() and (u != 0).any()
    near(orthogonalise([u], eps=0.0)[0], formula(u, eps=0.0))


@pytest.mark.parametrize("rows,cols", WAYS)
def test_a_subnormal_matrix_beside_eps_is_next_to_nothing(rows, cols):
    u = matrix(rows, cols) * 1e-42
    got = orthogonalise([u])[0]
    assert torch.isfinite(got).all() and got.float().abs().max() < 1e-30


SILENT = [(64, 1200, 512, 1024), (64, 1025, 1024, 1025), (1025, 64, 1024, 1025), (1200, 64, 0, 512), (16, 4096, 1024, 2048), (64, 1200, 0, 1200), (64, 1100, 1024, 1100)]


@pytest.mark.parametrize("level", [0.0, 1e-44, 1e-42, 1e-38])
@pytest.mark.parametrize("rows,cols,first,last", SILENT)
def test_inputs_that_fell_silent(rows, cols, first, last, level):
    """Places of the longer side, among them all of a work-group's, that hold next to nothing beside ordinary ones."""
    print(f"[case] orthogonalise {rows} x {cols}, {level} in {first} .. {last}", flush=True)
    u = matrix(rows, cols)
    (u if rows > cols else u.T)[first:last] = level
    near(orthogonalise([u])[0], formula(u))


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("rows,cols,first,last", SILENT)
def test_update_of_inputs_that_fell_silent(rows, cols, first, last, nesterov):
    """No gradient and a momentum that has decayed to the last subnormal numbers: 0.95 of them rounds back to what they were."""
    import paper_1811_01532_amd as wap
    print(f"[case] muon {rows} x {cols}, silent in {first} .. {last}", flush=True)
    g, m, w = matrix(rows, cols, "mixed", 1), 10 * matrix(rows, cols, "mixed", 2), matrix(rows, cols, seed=3) * 0.05
    for t, level in ((g, 0.0), (m, 1.3e-44)):
        (t if rows > cols else t.T)[first:last] = level
    lr, mu = 0.02, 0.95
    gd, md, wd = g.cuda(), m.cuda(), w.cuda()
    wb = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    d = wap.muon_desc(momentum=mu, nesterov=nesterov)
    entries = [wap.muon_matrix(rows, cols, lr, wd, wb, md, gd)]
    ws = torch.full((wap.wap_muon_workspace_bytes(d, entries),), 0xff, dtype=torch.uint8, device="cuda")
    wap.wap_muon_update(d, entries, ws)
    torch.cuda.synchronize()
    mref = mu * m.double() + g.double()
    o = formula(g.double() + mu * mref if nesterov else mref)
    assert (md.cpu().double() - mref).abs().max() <= 2.0 ** -22 * mref.abs().max() + 2.0 ** -149
    got, keep = wd.cpu().double(), w.double()
    assert torch.isfinite(got).all()
    assert (got - (keep - lr * o)).abs().max() <= lr * 10 * NORM_TOL * (o.norm() / o.numel() ** 0.5) + 2.0 ** -22 * w.abs().max()
    assert torch.equal(wb.view(torch.int16), wd.to(torch.bfloat16).view(torch.int16))
