"""GPU parity of the linear cross-entropy on every way that its products take: logits on tiles of 64, 128 and 256, whole, divided, kept and made
again; dx and dw on each tile, divided or not, in one piece of the classes or several; weights of whole, even and odd row lengths; rows
copied, gathered or taken as they are.  The sizes were drawn on the host until each combination that the plan can reach was among them.
Every gradient that is asked for is compared, and the other one is untouched.

Bounds as in the operator's other tests, from the arithmetic: dz is rounded to bf16 once (2^-8 of it), the output once more unless it is
fp32, and logits, exponentials and sums in fp32 add less than 1e-4 of softmax and one-hot."""
import pytest
import torch

from tests.test_gpu_linear_xent import LOSS_TOL, make

pytestmark = pytest.mark.gpu

SIZES = [
    # up to 64 rows: one and two steps of 32 of them, dx whole and divided
    (17, 31, 2), (1, 2345, 2185), (1, 310, 2454), (4, 2082, 4), (38, 56, 2), (37, 166, 2), (33, 8, 2086), (36, 14, 1479),
    # logits divided, joined in one chunk of the classes and in several
    (138, 1903, 44), (71, 2748, 2156), (69, 4237, 9668), (6832, 3938, 66), (17185, 3824, 134), (132, 3902, 22779), (90, 34, 20602),
    # kept, or made again
    (5289, 1026, 2), (71, 312, 32766), (12742, 592, 2), (200, 770, 20004), (225, 160, 20450), (109, 26, 2), (99, 32, 21321), (96, 14, 42017), (158, 12, 33171),
    (7342, 9, 1035), (149, 2560, 28023), (5901, 3560, 4880),
    # several pieces of the classes
    (8769, 12, 7543), (774, 16, 87126), (1657, 80, 41168), (6258, 66, 14513), (3084, 402, 22353), (569, 166, 179453), (18501, 8, 3738), (19397, 112, 4266),
    (9157, 206, 8103), (903, 272, 76731), (18778, 450, 3598), (15760, 808, 4354),
]


def formula(x, w, labels, scale):
    """(loss, losses, dz, size of dz's terms), in 64 bits on the device."""
    z = x @ w.T
    counts = (labels >= 0) & (labels < w.shape[0])
    place = labels.clamp(0, w.shape[0] - 1).long()[:, None]
    lse = torch.logsumexp(z, 1)
    losses = torch.where(counts, lse - z.gather(1, place)[:, 0], 0.0)
    p = z.sub_(lse[:, None]).exp_()
    n = max(1, int(counts.sum()))
    f = (counts.double() * (scale / n))[:, None]
    one = torch.ones_like(place, dtype=torch.float64)
    dz = p.clone().scatter_add_(1, place, -one).mul_(f)
    return losses.sum() / n, losses, dz, p.scatter_add_(1, place, one).mul_(f.abs())


def within(got, dz, size, other, rounded):
    got, u = got.double(), 2.0 ** -8
    assert torch.isfinite(got).all()
    ref = dz @ other
    other = other.abs()
    bound = dz.abs() @ other * (1.01 * u) + size @ other * 1e-4
    if rounded:
        bound += u * (ref.abs() + bound)
    over = float(((got - ref).abs() / (bound + 1e-30)).max())
    assert over <= 1.0, over


def run(x, w, labels, scale, dw_f32, want_dx=True, want_dw=True):
    import paper_1811_01532_amd as wap
    (rows, features), classes = x.shape, w.shape[0]
    d = wap.linear_xent_desc(rows, features, classes, dw_f32=dw_f32)
    loss, losses = torch.full((4,), 7.0, device="cuda"), torch.full((rows + 4,), 7.0, device="cuda")
    dx = torch.full((rows * features + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((classes * features + 8,), 7.0, dtype=torch.float32 if dw_f32 else torch.bfloat16, device="cuda")
    ws = torch.full((wap.wap_linear_xent_workspace_bytes(d, True),), 0xff, dtype=torch.uint8, device="cuda")  # (NaN wherever something reads what nothing wrote)
    wap.wap_linear_xent_grad(d, x, w, labels, scale, loss, losses, dx if want_dx else None, dw if want_dw else None, ws)
    torch.cuda.synchronize()
    for t, n in ((loss, 1), (losses, rows), (dx, rows * features if want_dx else 0), (dw, classes * features if want_dw else 0)):
        assert (t[n:] == 7.0).all()
    return loss[:1], losses[:rows], dx[:rows * features].reshape(rows, features), dw[:classes * features].reshape(classes, features)


@pytest.mark.parametrize("rows,features,classes", SIZES)
def test_every_way_of_the_products(rows, features, classes):
    import paper_1811_01532_amd as wap
    print(f"[case] linear_xent {rows} x {features} -> {classes}", flush=True)
    x, w, labels = (t.cuda() for t in make(rows, features, classes, 0.1))
    dw_f32, scale = features % 4 < 2, 1.0 + (rows % 3)
    loss, losses, dx, dw = run(x, w, labels, scale, dw_f32)
    d = wap.linear_xent_desc(rows, features, classes)
    loss2, losses2 = torch.full((4,), 7.0, device="cuda"), torch.full((rows + 4,), 7.0, device="cuda")
    ws = torch.full((wap.wap_linear_xent_workspace_bytes(d, False),), 0xff, dtype=torch.uint8, device="cuda")
    wap.wap_linear_xent_fwd(d, x, w, labels, loss2, losses2, ws)
    torch.cuda.synchronize()
    assert (loss2[1:] == 7.0).all() and (losses2[rows:] == 7.0).all()
    rloss, rlosses, dz, size = formula(x.double(), w.double(), labels, scale)
    top = max(1.0, float(rlosses.abs().max()))
    for one, some in ((loss, losses), (loss2[0], losses2[:rows])):
        assert float((some.double() - rlosses).abs().max()) <= LOSS_TOL * top
        assert abs(float(one) - float(rloss)) <= LOSS_TOL * max(1.0, abs(float(rloss)))
    within(dx, dz, size, w.double(), True)
    within(dw, dz.T, size.T, x.double(), not dw_f32)


@pytest.mark.parametrize("rows,features,classes", [(20, 64, 300), (50, 66, 3000), (130, 72, 300), (700, 130, 3001), (774, 16, 87126)])
@pytest.mark.parametrize("dw_f32", [False, True])
def test_a_gradient_alone_is_what_it_is_beside_the_other(rows, features, classes, dw_f32):
    x, w, labels = (t.cuda() for t in make(rows, features, classes, 0.1))
    both = run(x, w, labels, 1.0, dw_f32)
    same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    alone = run(x, w, labels, 1.0, dw_f32, want_dw=False)
    assert all(same(p, q) for p, q in zip(both[:3], alone[:3]))
    alone = run(x, w, labels, 1.0, dw_f32, want_dx=False)
    assert all(same(p, q) for p, q in zip(both[:2] + both[3:], alone[:2] + alone[3:]))
