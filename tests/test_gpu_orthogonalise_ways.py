"""GPU parity of the Newton-Schulz orthogonalisation and the Muon update on every way that a matrix can take: one work-group, several of them,
products on tiles of 64 (X X^T whole and divided), 128, 192 and 256, wide and tall, rows of whole groups of four and others; lists that share launches;
the sizes at which one way ends and the next begins.

Bounds as in the operator's other tests."""
import pytest
import torch

from tests.test_gpu_orthogonalise import NORM_TOL, formula, matrix, near, orthogonalise

pytestmark = pytest.mark.gpu

FEW = [(64, 640), (640, 64), (64, 641), (641, 63), (64, 1025), (1030, 33), (7, 5000), (65, 64), (64, 1152), (2048, 1), (16, 32768), (32768, 15), (16, 32769), (32769, 16)]
TILES = [
    (131, 260), (260, 131), (65, 65), (66, 3000),  # all on tiles of 64
    (130, 7000), (130, 7001), (7000, 130), (7001, 131), (512, 9000), (9000, 511),  # X X^T divided; X on 64 or 192
    (1000, 4004), (1001, 4002), (4004, 1000), (4002, 1001),  # X on 128
    (2001, 5003), (2000, 5004), (5003, 2001), (5004, 2000),  # X on 256
    (2301, 2502), (2300, 2504), (2502, 2301), (2504, 2300),  # A and B on 128, X on 192
    (3001, 3502), (3000, 3504), (3502, 3001), (3504, 3000),  # A and B on 192
    (4401, 4410), (4400, 4412), (4410, 4401), (4412, 4400),  # A and B on 256
]


class Update:
    """One matrix of a Muon update, its reference, and what surrounds its buffers."""

    def __init__(self, rows, cols, lr, seed=0, copy=True):
        self.shape, self.lr = (rows, cols), lr
        self.g, self.m = matrix(rows, cols, "mixed", 1 + seed), 10 * matrix(rows, cols, "mixed", 2 + seed)
        self.w = matrix(rows, cols, seed=3 + seed) * 0.05
        self.gd, self.md, self.wd = (torch.cat([t.flatten(), torch.full((8,), 7.0)]).cuda() for t in (self.g, self.m, self.w))
        self.wb = torch.full((rows * cols + 8,), 7.0, dtype=torch.bfloat16, device="cuda") if copy else None

    def entry(self, wap):
        return wap.muon_matrix(*self.shape, self.lr, self.wd, self.wb, self.md, self.gd)

    def check(self, mu, decay, nesterov):
        n = self.g.numel()
        for t in (self.gd, self.md, self.wd) + (() if self.wb is None else (self.wb,)):
            assert (t[n:] == 7.0).all()
        assert torch.equal(self.gd[:n].cpu(), self.g.flatten())
        g, m, w = self.g.cuda().double(), self.m.cuda().double(), self.w.cuda().double()
        moving = mu * m + g
        o = formula(g + mu * moving if nesterov else moving)
        got_m, got_w = self.md[:n].double().reshape(self.shape), self.wd[:n].double().reshape(self.shape)
        assert (got_m - moving).abs().max() <= 2.0 ** -22 * moving.abs().max()
        ref = w * (1.0 - self.lr * decay) - self.lr * o
        assert torch.isfinite(got_w).all()
        assert (got_w - ref).abs().max() <= self.lr * 10 * NORM_TOL * (o.norm() / n ** 0.5) + 2.0 ** -22 * w.abs().max()
        # what was taken off, as a whole: decay, product and store round by 2^-24 of the weights each
        assert (got_w - ref).norm() <= self.lr * NORM_TOL * o.norm() + 2.0 ** -22 * w.norm()
        if self.wb is not None:
            assert torch.equal(self.wb[:n].view(torch.int16), self.wd[:n].to(torch.bfloat16).view(torch.int16))


def update(updates, mu=0.95, decay=0.1, nesterov=True):
    import paper_1811_01532_amd as wap
    d = wap.muon_desc(momentum=mu, weight_decay=decay, nesterov=nesterov)
    entries = [u.entry(wap) for u in updates]
    ws = torch.full((wap.wap_muon_workspace_bytes(d, entries),), 0xff, dtype=torch.uint8, device="cuda")
    wap.wap_muon_update(d, entries, ws)
    torch.cuda.synchronize()
    for u in updates:
        u.check(mu, decay, nesterov)


@pytest.mark.parametrize("rows,cols", FEW + TILES)
def test_orthogonalise(rows, cols):
    print(f"[case] orthogonalise {rows} x {cols}", flush=True)
    u = matrix(rows, cols, "mixed")
    near(orthogonalise([u])[0], formula(u.cuda()).cpu())


@pytest.mark.parametrize("rows,cols", FEW + TILES)
def test_muon(rows, cols):
    print(f"[case] muon {rows} x {cols}", flush=True)
    update([Update(rows, cols, 0.02)], nesterov=(rows + cols) % 3 != 0)


@pytest.mark.parametrize("sizes", [
    [(64, 1025), (1030, 33), (7, 5000), (64, 64), (3, 3), (64, 2000)],  # several work-groups each
    [(64, 576), (27, 64), (1, 1), (640, 5), (64, 640)],  # one each
    [(64, 1025), (5, 9), (333, 1025), (1500, 250), (64, 27), (130, 7001)] * 3,  # tiles, and more than one set of launches
    [(64, 1152)] * 16 + [(300, 200)] * 3,  # a set of several work-groups, then one of tiles
    [(64, 64)] * 16 + [(64, 700)] * 2,
    [(2400, 2400), (2398, 2402), (2402, 2399)],  # tiles of 256 for three
    [(512, 4608), (4608, 511), (64, 27)],  # X X^T of all three divided
])
def test_lists(sizes):
    print(f"[case] lists of {len(sizes)}, from {sizes[0]}", flush=True)
    mats = [matrix(r, c, "mixed", seed=i) for i, (r, c) in enumerate(sizes)]
    for m, o in zip(mats, orthogonalise(mats)):
        near(o, formula(m.cuda()).cpu())
    update([Update(r, c, 0.005 * (1 + i), seed=10 * i, copy=i % 4 != 3) for i, (r, c) in enumerate(sizes)])
    update([Update(r, c, 0.005 * (1 + i), seed=10 * i + 5) for i, (r, c) in enumerate(sizes)], nesterov=False, decay=0.0)


@pytest.mark.parametrize("sizes", [[(64, 1100), (33, 2000), (1500, 64)], [(64, 576), (20, 30), (100, 5)], [(130, 264), (300, 70), (64, 1100)]])
def test_zeros_and_nan_stay_in_their_matrix(sizes):
    mats = [matrix(r, c, seed=i) for i, (r, c) in enumerate(sizes)]
    mats[0].zero_()
    mats[1][3, 4] = float("nan")
    zero, nan, whole = orthogonalise(mats)
    assert (zero == 0).all() and torch.isnan(nan).all()
    near(whole, formula(mats[2]))


@pytest.mark.parametrize("rows,cols", [(64, 1100), (64, 576), (130, 7001)])
def test_update_in_a_graph(rows, cols):
    """Replays, with other work in between, leave what eager calls leave."""
    import paper_1811_01532_amd as wap
    u = Update(rows, cols, 0.01)
    d = wap.muon_desc()
    entries = [u.entry(wap)]
    ws = torch.empty(wap.wap_muon_workspace_bytes(d, entries), dtype=torch.uint8, device="cuda")
    state = [u.wd, u.wb, u.md]
    start = [t.clone() for t in state]
    wap.wap_muon_update(d, entries, ws)  # attributes are set before a capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wap.wap_muon_update(d, entries, ws)
    seen = []
    for eager in (True, False):
        for t, s in zip(state, start):
            t.copy_(s)
        got = []
        for _ in range(4):
            wap.wap_muon_update(d, entries, ws) if eager else graph.replay()
            torch.cuda.synchronize()
            got.append([t.clone() for t in state])
            torch.ones(1 << 16, device="cuda").sum().item()  # the program's own work in between
        seen.append(got)
    for a, b in zip(*seen):
        assert all(torch.equal(p.view(torch.int16), q.view(torch.int16)) for p, q in zip(a, b))
