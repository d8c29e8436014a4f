"""GPU: surgeon_layer_norm and surgeon_layer_norm_grad against the formulas in 64 bits.

Tolerances count roundings, u = 2^-24 each, of sums that are taken sequentially over at most 32 elements of
a thread (rows in registers) or channels / 1024 (long rows) and then over trees of at most 15 levels; K below
bounds the number of roundings on any path.  Outputs are rounded once more to their type: half a step, finfo.eps / 2."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-6
# every kernel variant, its edges, odd widths, one channel; rows that do not fill a CTA
SHAPES = [(1, 1), (3, 2), (5, 7), (1, 8), (37, 8), (33, 64), (257, 65), (9, 72), (197, 256), (31, 257), (8, 264), (64, 320),
          (7, 512), (50, 513), (197, 768), (13, 769), (1000, 776), (5, 1000), (4, 1024), (3, 1032), (2, 1025), (9, 2048),
          (3, 2049), (2, 4096), (5, 4104), (2, 5003), (3, 8192), (2, 8200), (3, 8191), (2, 16391)]


def inputs(rows, channels, dt, seed=0, offset=2.0):
    g = torch.Generator().manual_seed(1000 * rows + channels + seed)
    x = (torch.randn(rows, channels, generator=g) * 1.5 + offset).to(dt)
    gamma = 1.0 + 0.3 * torch.randn(channels, generator=g)
    beta = 0.3 * torch.randn(channels, generator=g)
    return g, x, gamma, beta


def k_of(channels):
    return 64 + channels // 1024


def check_forward(x, gamma, beta, y, stats, eps=EPS):
    """x, y, stats: what the call had and gave, on the host."""
    rows, c = x.shape
    xd = x.double()
    mean = xd.mean(1, keepdim=True)
    r = (((xd - mean) ** 2).mean(1, keepdim=True) + eps).rsqrt()
    xh = (xd - mean) * r
    g = gamma.double() if gamma is not None else torch.ones(c, dtype=torch.float64)
    b = beta.double() if beta is not None else torch.zeros(c, dtype=torch.float64)
    want = xh * g + b
    k = k_of(c) * U
    size = xd.abs().mean(1, keepdim=True)
    # the mean is off by k * size; centring and its products by a rounding each
    err_mean = k * size
    # the variance: k relative, the square of the mean's error, and the rounding of each x - mean
    var = 1.0 / r ** 2
    rel_r = 0.5 * k + 0.5 * (err_mean ** 2) / var + 2 * U
    tol = g.abs() * r * (err_mean + U * (xd - mean).abs()) + (g * xh).abs() * (rel_r + 4 * U) + 2 * U * want.abs()
    tol = tol + torch.finfo(y.dtype).eps / 2 * (want.abs() + tol)
    assert ((y.double() - want).abs() <= tol).all(), ((y.double() - want).abs() / tol).max()
    if stats is not None:
        assert ((stats[0].double() - mean[:, 0]).abs() <= err_mean[:, 0] + U * mean[:, 0].abs()).all()
        assert ((stats[1].double() / r[:, 0] - 1).abs() <= rel_r[:, 0] + 2 * U).all()


@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows,channels", SHAPES)
def test_forward_matches_the_formula(rows, channels, dt):
    _, x, gamma, beta = inputs(rows, channels, dt)
    for g, b in ((gamma, beta), (None, None), (gamma, None), (None, beta)):
        pad = torch.full((rows * channels + 64,), 7.0, dtype=dt, device="cuda")     # canaries behind the output
        out = pad[:rows * channels].view(rows, channels)
        stats = torch.full((2, rows), -1.0, device="cuda")
        y = B.surgeon_layer_norm(x.cuda(), None if g is None else g.cuda(), None if b is None else b.cuda(), EPS, out=out,
                                 stats=stats)
        assert y is out and bool((pad[rows * channels:] == 7.0).all())
        check_forward(x, g, b, y.cpu(), stats.cpu())
    again = B.surgeon_layer_norm(x.cuda(), None, beta.cuda(), EPS)                  # without statistics, new output
    assert torch.equal(again, y)


def backward_reference(x, dy, gamma, stats, residual):
    """dx, dgamma, dbeta in 64 bits and what each may be off by."""
    rows, c = x.shape
    xd, d = x.double(), dy.double()
    mean, r = stats[0].double()[:, None], stats[1].double()[:, None]
    g = gamma.double() if gamma is not None else torch.ones(c, dtype=torch.float64)
    xh = (xd - mean) * r
    e_xh = 2 * U * xh.abs() + U * (xd - mean).abs() * r
    gd = d * g
    c1, c2 = gd.mean(1, keepdim=True), (gd * xh).mean(1, keepdim=True)
    dx = r * (gd - c1 - xh * c2)
    k = k_of(c) * U
    e_c1 = k * gd.abs().mean(1, keepdim=True)
    e_c2 = k * (gd * xh).abs().mean(1, keepdim=True) + (gd.abs() * e_xh).mean(1, keepdim=True)
    e_dx = r * (U * gd.abs() + e_c1 + xh.abs() * e_c2 + e_xh * c2.abs() + 4 * U * (gd.abs() + c1.abs() + (xh * c2).abs()))
    if residual is not None:
        dx = dx + residual.double()
        e_dx = e_dx + U * dx.abs()
    e_dx = e_dx + torch.finfo(dy.dtype).eps / 2 * (dx.abs() + e_dx)
    n = (100 + rows // 296) * U                   # rows of a thread, groups of a CTA, slices of the partial sums
    return (dx, e_dx, (d * xh).sum(0), n * (d * xh).abs().sum(0) + (d.abs() * e_xh).sum(0), d.sum(0), n * d.abs().sum(0))


TYPES = [(F32, F32), (BF16, F32), (BF16, BF16)]
IDS = ["fp32", "bf16-fp32", "bf16"]


@pytest.mark.parametrize("dt,gt", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,channels", SHAPES + [(5000, 64), (3001, 40), (700, 8200)])
def test_backward_matches_the_formula(rows, channels, dt, gt):
    gen, x, gamma, _ = inputs(rows, channels, dt, seed=1)
    dy = (0.1 * torch.randn(rows, channels, generator=gen)).to(gt)
    skip = (0.1 * torch.randn(rows, channels, generator=gen)).to(gt)
    stats = torch.stack([x.double().mean(1), (x.double().var(1, unbiased=False) + EPS).rsqrt()]).float()
    old = torch.randn(2, channels, generator=gen)
    for g, res in ((gamma, skip), (None, None)):
        dx, e_dx, dg, e_dg, db, e_db = backward_reference(x, dy, g, stats, res)
        dev = dict(gamma=None if g is None else g.cuda(), stats=stats.cuda(), residual_grad=None if res is None else res.cuda())
        dgamma, dbeta = torch.full((channels,), 9.0, device="cuda"), torch.full((channels,), 9.0, device="cuda")
        need = B.surgeon_layer_norm_grad_workspace(rows, channels)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")        # NaNs where nothing is written
        got = B.surgeon_layer_norm_grad(x.cuda(), dy.cuda(), dgamma=dgamma, dbeta=dbeta, workspace=ws, **dev)
        assert ((got.cpu().double() - dx).abs() <= e_dx).all(), ((got.cpu().double() - dx).abs() / e_dx).max()
        assert ((dgamma.cpu().double() - dg).abs() <= e_dg).all(), ((dgamma.cpu().double() - dg).abs() / e_dg).max()
        assert ((dbeta.cpu().double() - db).abs() <= e_db).all()
        assert bool((ws[need:] == 0xFF).all())
        # the same bits again; one output at a time; added to what is there
        g2, b2 = old[0].cuda(), old[1].cuda()
        again = B.surgeon_layer_norm_grad(x.cuda(), dy.cuda(), dgamma=g2, dbeta=b2, accumulate=True, **dev)
        assert torch.equal(again, got)
        assert torch.equal(g2, old[0].cuda() + dgamma) and torch.equal(b2, old[1].cuda() + dbeta)
        g3, b3 = torch.empty_like(dgamma), torch.empty_like(dbeta)
        assert B.surgeon_layer_norm_grad(x.cuda(), dy.cuda(), dgamma=g3, want_dx=False, **dev) is None
        assert B.surgeon_layer_norm_grad(x.cuda(), dy.cuda(), dbeta=b3, want_dx=False, **dev) is None
        assert torch.equal(g3, dgamma) and torch.equal(b3, dbeta)
        assert torch.equal(B.surgeon_layer_norm_grad(x.cuda(), dy.cuda(), **dev), got)


@pytest.mark.parametrize("channels", [48, 769, 8200])
def test_outputs_in_place_of_inputs(channels):
    gen, x, gamma, beta = inputs(21, channels, BF16, seed=2)
    x, gamma, beta = x.cuda(), gamma.cuda(), beta.cuda()
    stats = torch.empty(2, 21, device="cuda")
    want = B.surgeon_layer_norm(x, gamma, beta, EPS, stats=stats)
    own = x.clone()
    assert torch.equal(B.surgeon_layer_norm(own, gamma, beta, EPS, out=own), want)
    dy, skip = torch.randn(21, channels, generator=gen).cuda(), torch.randn(21, channels, generator=gen).cuda()
    dg, db = torch.empty(channels, device="cuda"), torch.empty(channels, device="cuda")
    dx = B.surgeon_layer_norm_grad(x, dy, gamma, stats, residual_grad=skip, dgamma=dg, dbeta=db)
    for which in (0, 1):
        d2, s2, dg2, db2 = dy.clone(), skip.clone(), torch.empty_like(dg), torch.empty_like(db)
        got = B.surgeon_layer_norm_grad(x, d2, gamma, stats, residual_grad=s2, dx=(d2, s2)[which], dgamma=dg2, dbeta=db2)
        assert torch.equal(got, dx) and torch.equal(dg2, dg) and torch.equal(db2, db)


@pytest.mark.parametrize("channels", [64, 513, 3000, 8200])
def test_nan_and_infinity_stay_in_their_row(channels):
    _, x, gamma, beta = inputs(9, channels, F32, seed=3)
    clean = B.surgeon_layer_norm(x.cuda(), gamma.cuda(), beta.cuda(), EPS)
    bad = x.clone()
    bad[2, channels // 2] = float("nan")
    bad[5, 0] = float("inf")
    y = B.surgeon_layer_norm(bad.cuda(), gamma.cuda(), beta.cuda(), EPS)
    rows = [i for i in range(9) if i not in (2, 5)]
    assert torch.equal(y[rows], clean[rows]) and bool(y[[2, 5]].isnan().all())


def test_constant_rows_and_a_large_mean():
    # every centred value is zero: beta is left
    x = torch.full((4, 768), 3.0, device="cuda")
    beta = torch.randn(768, device="cuda")
    assert torch.equal(B.surgeon_layer_norm(x, None, beta), beta.expand(4, 768))
    # a mean 4096 times the spread: squares minus the square of the mean would leave a few bits
    _, x, gamma, beta = inputs(16, 320, F32, seed=4, offset=4096.0)
    stats = torch.empty(2, 16, device="cuda")
    y = B.surgeon_layer_norm(x.cuda(), gamma.cuda(), beta.cuda(), EPS, stats=stats)
    check_forward(x, gamma, beta, y.cpu(), stats.cpu())


def test_no_rows():
    x = torch.empty(0, 768, device="cuda")
    assert B.surgeon_layer_norm(x).shape == (0, 768)
    dg, db = torch.full((768,), 4.0, device="cuda"), torch.full((768,), 4.0, device="cuda")
    stats = torch.empty(2, 0, device="cuda")
    B.surgeon_layer_norm_grad(x, x, None, stats, dgamma=dg, dbeta=db, accumulate=True)
    assert bool((dg == 4.0).all()) and bool((db == 4.0).all())
    B.surgeon_layer_norm_grad(x, x, None, stats, dgamma=dg, dbeta=db)
    assert not dg.any() and not db.any()


def test_gradient_against_differences():
    """The backward pass is the derivative of the forward pass: sum(w * y) along a direction, by a central difference in
    64 bits of the formula (the kernel's own roundings stay out of the quotient)."""
    gen, x, gamma, beta = inputs(6, 96, F32, seed=5)
    w = torch.randn(6, 96, generator=gen)
    stats = torch.empty(2, 6, device="cuda")
    B.surgeon_layer_norm(x.cuda(), gamma.cuda(), beta.cuda(), EPS, stats=stats)
    dg, db = torch.empty(96, device="cuda"), torch.empty(96, device="cuda")
    dx = B.surgeon_layer_norm_grad(x.cuda(), w.cuda(), gamma.cuda(), stats, dgamma=dg, dbeta=db)

    def value(x, gamma, beta):
        return (torch.nn.functional.layer_norm(x, (96,), gamma, beta, EPS) * w.double()).sum()

    at = [t.double() for t in (x, gamma, beta)]
    for i, got in enumerate((dx, dg, db)):
        step = torch.randn(at[i].shape, generator=gen, dtype=torch.float64)
        h = 1e-5
        up, down = [list(at), list(at)]
        up[i], down[i] = at[i] + h * step, at[i] - h * step
        want = (value(*up) - value(*down)) / (2 * h)
        have = (got.cpu().double() * step).sum()
        # 576 products with errors of some 64 u each, and h^2 of the third derivative
        assert abs(have - want) <= 64 * U * (got.cpu().double() * step).abs().sum() + 1e-7 * (1 + abs(want))


def test_many_rows_pass_32_bits():
    """2^31 - 2^20 elements of bf16 (4 GB each): the last rows lie behind 2^32 bytes."""
    rows, c = (1 << 21) - 1024, 1024
    x = torch.empty(rows, c, dtype=BF16, device="cuda")
    x[:4096].normal_()
    x[-4096:].normal_()
    x[4096:-4096] = 1.0
    stats = torch.empty(2, rows, device="cuda")
    y = B.surgeon_layer_norm(x, None, None, EPS, out=None, stats=stats)
    check_forward(x[-100:].cpu(), None, None, y[-100:].cpu(), stats[:, -100:].cpu())
    assert not y[4096:-4096].any()


def test_refusals():
    x = torch.randn(4, 64, device="cuda")
    stats = torch.empty(2, 4, device="cuda")
    for call in (lambda: B.surgeon_layer_norm(x.t()), lambda: B.surgeon_layer_norm(x.cpu()),
                 lambda: B.surgeon_layer_norm(x, gamma=torch.ones(63, device="cuda")),
                 lambda: B.surgeon_layer_norm(x, gamma=torch.ones(64, device="cuda", dtype=BF16)),
                 lambda: B.surgeon_layer_norm(x, out=torch.empty(4, 64, device="cuda", dtype=BF16)),
                 lambda: B.surgeon_layer_norm(x, stats=torch.empty(4, 2, device="cuda")),
                 lambda: B.surgeon_layer_norm_grad(x, x[:3], None, stats),
                 lambda: B.surgeon_layer_norm_grad(x, x, None, stats, residual_grad=x.to(BF16))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        B.surgeon_layer_norm(x.half())
    for call, status in ((lambda: B.surgeon_layer_norm(x, eps=0.0), B.SURGEON_ERR_INVALID_ARG),
                         (lambda: B.surgeon_layer_norm(x, eps=float("nan")), B.SURGEON_ERR_INVALID_ARG),
                         (lambda: B.surgeon_layer_norm(x.view(-1)[1:65].view(1, 64)), B.SURGEON_ERR_INVALID_ARG),
                         (lambda: B.surgeon_layer_norm_grad(x, x.to(BF16), None, stats), B.SURGEON_ERR_UNSUPPORTED),
                         (lambda: B.surgeon_layer_norm_grad(x, x, None, stats, dgamma=torch.empty(64, device="cuda"),
                                                            workspace=torch.empty(16, device="cuda")),
                          B.SURGEON_ERR_BUFFER_TOO_SMALL)):
        with pytest.raises(B.SurgeonError) as e:
            call()
        assert e.value.status == status
