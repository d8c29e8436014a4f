"""GPU: surgeon_group_norm and surgeon_group_norm_grad against the formulas in 64 bits.

Tolerances count roundings, u = 2^-24 each.  A thread sums at most `positions` numbers of a channel in fp32, groups and images are summed
in double; K bounds the number of roundings on any path.  Outputs are rounded once more to their type: half a step, finfo.eps / 2."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5
ACTS = {"none": B.SURGEON_ACT_NONE, "relu": B.SURGEON_ACT_RELU, "gelu": B.SURGEON_ACT_GELU, "silu": B.SURGEON_ACT_SILU}
# one position, odd channels, groups that no vector divides, held in registers or streamed, several blocks of channels, many images
SHAPES = [(1, 1, 1, 1), (2, 3, 6, 2), (1, 49, 2048, 32), (3, 5, 320, 32), (2, 100, 64, 64), (1, 300, 24, 3), (2, 1000, 320, 32), (1, 5000, 96, 1),
          (4, 3136, 256, 32), (1, 777, 4104, 8), (70, 9, 40, 5), (1, 4097, 33, 11), (2, 2500, 2056, 257), (300, 4, 8, 8), (1, 20000, 16, 4), (2, 3000, 2100, 2100),
          (3, 700, 515, 5)]


def inputs(b, p, c, dt, seed=0, offset=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * p + c)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = (rnd(b, p, c) * (0.5 + torch.rand(c, generator=g, device="cuda")) + rnd(c) * 0.5 + offset).to(dt)
    return g, x, 1.0 + 0.3 * rnd(c), 0.3 * rnd(c)


def act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: torch.nn.functional.gelu(z), "silu": lambda: torch.nn.functional.silu(z)}[act]()


def slope64(z, act):
    t = z.detach().requires_grad_()
    return torch.autograd.grad(act64(t, act).sum(), t)[0] if act != "relu" else (z > 0).double()


def terms(x, groups):
    b, p, c = x.shape
    xd = x.double().view(b, p, groups, c // groups)
    mean, var = xd.mean((1, 3)), xd.var((1, 3), unbiased=False)
    return xd, mean, 1 / (var + EPS).sqrt(), var


def check_forward(x, groups, gamma, beta, act, y, stats):
    b, p, c = x.shape
    xd, mean, r, var = terms(x, groups)
    k = (64 + 2 * min(p, 2000)) * U
    e_mean = U * mean.abs() + k * xd.abs().mean((1, 3))
    rel_r = 0.5 * (k * (var + e_mean ** 2) * r ** 2 + (e_mean * r) ** 2) + 4 * U
    if stats is not None:
        assert ((stats[0].double() - mean).abs() <= e_mean).all()
        assert ((stats[1].double() / r - 1).abs() <= rel_r).all(), ((stats[1].double() / r - 1).abs() / rel_r).max()
    wide = lambda t: t[:, None, :, None]
    xh = (xd - wide(mean)) * wide(r)
    g = (gamma.double() if gamma is not None else torch.ones(c, dtype=torch.float64, device="cuda")).view(groups, -1)
    o = (beta.double() if beta is not None else torch.zeros(c, dtype=torch.float64, device="cuda")).view(groups, -1)
    z = xh * g + o
    e_xh = wide(r) * (wide(e_mean) + U * (xd - wide(mean)).abs()) + xh.abs() * (wide(rel_r) + 2 * U)
    e_z = e_xh * g.abs() + 2 * U * ((xh * g).abs() + z.abs())
    want = act64(z, act)
    tol = 1.2 * e_z + (0 if act in ("none", "relu") else 2e-7 * (1 + z.abs()))       # slopes of the activations up to 1.13; GELU's Phi to 8e-8
    tol = tol + torch.finfo(y.dtype).eps / 2 * (want.abs() + tol)
    e = (y.double().view_as(want) - want).abs()
    assert (e <= tol).all(), (e / tol).max()


@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("b,p,c,groups", SHAPES)
def test_forward_matches_the_formula(b, p, c, groups, dt):
    _, x, gamma, beta = inputs(b, p, c, dt)
    need = B.surgeon_group_norm_workspace(b, p, c, groups)
    for act, (g, o) in zip(ACTS, ((gamma, beta), (gamma, beta), (None, beta), (gamma, None))):
        pad = torch.full((b * p * c + 64,), 7.0, dtype=dt, device="cuda")            # canaries behind the output and the scratch
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        out, stats = pad[:b * p * c].view(b, p, c), torch.full((2, b, groups), -1.0, device="cuda")
        y = B.surgeon_group_norm(x, groups, g, o, EPS, act=ACTS[act], out=out, stats=stats, workspace=ws)
        assert y is out and bool((pad[b * p * c:] == 7.0).all()) and bool((ws[need:] == 0xFF).all())
        check_forward(x, groups, g, o, act, y, stats)
        assert torch.equal(B.surgeon_group_norm(x, groups, g, o, EPS, act=ACTS[act]), y)           # without statistics, new output
        place = x.clone()
        assert torch.equal(B.surgeon_group_norm(place, groups, g, o, EPS, act=ACTS[act], out=place), y)


def test_positions_in_several_dimensions():
    _, x, gamma, beta = inputs(2, 12 * 20, 64, BF16)
    y = B.surgeon_group_norm(x.view(2, 12, 20, 64), 8, gamma, beta)
    assert y.shape == (2, 12, 20, 64) and torch.equal(y.view(2, 240, 64), B.surgeon_group_norm(x, 8, gamma, beta))


@pytest.mark.parametrize("p", [40, 6000])
def test_means_far_from_zero(p):
    """Numbers whose spread is a thousandth of their mean, and a first number far from the others."""
    _, x, gamma, beta = inputs(2, p, 64, F32)
    x = 1000.0 + 0.5 * x
    x[:, 0] = 5000.0
    stats = torch.empty(2, 2, 8, device="cuda")
    y = B.surgeon_group_norm(x, 8, gamma, beta, EPS, stats=stats)
    check_forward(x, 8, gamma, beta, "none", y, stats)


@pytest.mark.parametrize("p", [40, 6000])
def test_a_nan_stays_in_its_group(p):
    _, x, gamma, beta = inputs(2, p, 64, F32)
    clean = B.surgeon_group_norm(x, 8, gamma, beta)
    x[1, p // 2, 19] = float("nan")
    y = B.surgeon_group_norm(x, 8, gamma, beta)
    assert bool(torch.isnan(y[1, :, 16:24]).all())
    y[1, :, 16:24] = clean[1, :, 16:24]
    assert torch.equal(y, clean)


def test_activations_at_the_ends():
    x = torch.tensor([-3e38, -1e4, -200.0, 0.0, 200.0, 1e4], device="cuda").view(1, 1, 6)
    beta = torch.tensor([-float("inf"), -1e4, -200.0, 0.0, 200.0, 1e4], device="cuda")
    gamma = torch.zeros(6, device="cuda")
    for act in ("gelu", "silu"):
        y = B.surgeon_group_norm(torch.ones_like(x), 1, gamma, beta, act=ACTS[act]).view(-1)
        assert torch.equal(y, torch.tensor([0.0, 0.0, 0.0, 0.0, 200.0, 1e4], device="cuda")), (act, y)


TYPES = [(F32, F32), (BF16, F32), (BF16, BF16)]


@pytest.mark.parametrize("dt,gt", TYPES, ids=["fp32", "bf16-fp32", "bf16"])
@pytest.mark.parametrize("b,p,c,groups", SHAPES[1:])
def test_backward_matches_the_formula(b, p, c, groups, dt, gt):
    g, x, gamma, beta = inputs(b, p, c, dt, seed=1)
    dy = (0.1 * torch.randn(b, p, c, generator=g, device="cuda")).to(gt)
    xd, mean, r, _ = terms(x, groups)
    stats = torch.stack([mean, r]).float()
    old = torch.randn(2, c, generator=g, device="cuda")
    need = B.surgeon_group_norm_grad_workspace(b, p, c, groups)
    for act, (w, o) in zip(ACTS, ((gamma, beta), (gamma, beta), (None, beta), (gamma, None))):
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        dg, db = torch.full((c,), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")
        dx = B.surgeon_group_norm_grad(x, dy, groups, w, o, stats, act=ACTS[act], dgamma=dg, dbeta=db, workspace=ws)
        assert bool((ws[need:] == 0xFF).all())
        wide = lambda t: t.double()[:, None, :, None]
        m, s = wide(stats[0]), wide(stats[1])
        gw = (w.double() if w is not None else torch.ones(c, dtype=torch.float64, device="cuda")).view(groups, -1)
        ow = (o.double() if o is not None else torch.zeros(c, dtype=torch.float64, device="cuda")).view(groups, -1)
        d, xh = dy.double().view_as(xd), (xd - m) * s
        z = xh * gw + ow
        e_xh = 3 * U * xh.abs() + U * (xd - m).abs() * s
        e_z = e_xh * gw.abs() + 2 * U * ((xh * gw).abs() + z.abs())
        dz = d * slope64(z, act)
        e_dz = 2 * U * dz.abs() + d.abs() * (0 if act == "none" else (z.abs() <= e_z).double() if act == "relu" else e_z + 4e-7 * (1 + z.abs()))
        gd = dz * gw
        c1, c2 = gd.mean((1, 3), keepdim=True), (gd * xh).mean((1, 3), keepdim=True)
        k = (64 + 2 * min(p, 2000)) * U
        e_c1 = ((e_dz * gw.abs()) + k * gd.abs()).mean((1, 3), keepdim=True)
        e_c2 = ((e_dz * gw.abs() + k * gd.abs()) * xh.abs() + gd.abs() * e_xh).mean((1, 3), keepdim=True)
        want = s * (gd - c1 - xh * c2)
        tol = s * (e_dz * gw.abs() + e_c1 + xh.abs() * e_c2 + e_xh * c2.abs() + 6 * U * (gd.abs() + c1.abs() + (xh * c2).abs()))
        tol = tol + torch.finfo(gt).eps / 2 * (want.abs() + tol)
        e = (dx.double().view_as(want) - want).abs()
        assert (e <= tol).all(), (act, (e / tol).max())
        w_dg, w_db = (dz * xh).sum((0, 1)).view(-1), dz.sum((0, 1)).view(-1)
        t_dg = ((e_dz + k * dz.abs()) * xh.abs() + dz.abs() * e_xh).sum((0, 1)).view(-1) + U * w_dg.abs()
        t_db = (e_dz + k * dz.abs()).sum((0, 1)).view(-1) + U * w_db.abs()
        assert ((dg.double() - w_dg).abs() <= t_dg).all() and ((db.double() - w_db).abs() <= t_db).all()
        # added to what was there; without dx; in the place of dy
        ag, ab = old[0].clone(), old[1].clone()
        assert B.surgeon_group_norm_grad(x, dy, groups, w, o, stats, act=ACTS[act], dgamma=ag, dbeta=ab, accumulate=True, want_dx=False) is None
        assert ((ag.double() - old[0].double() - w_dg).abs() <= t_dg + 2 * U * (ag.abs() + old[0].abs())).all()
        assert ((ab.double() - old[1].double() - w_db).abs() <= t_db + 2 * U * (ab.abs() + old[1].abs())).all()
        place = dy.clone()
        assert torch.equal(B.surgeon_group_norm_grad(x, place, groups, w, o, stats, act=ACTS[act], dx=place), dx)


def test_no_rows():
    gamma = torch.ones(8, device="cuda")
    for b, p in ((0, 5), (3, 0)):
        x, stats = torch.empty(b, p, 8, device="cuda"), torch.zeros(2, b, 2, device="cuda")
        assert B.surgeon_group_norm(x, 2, gamma, gamma, stats=stats).shape == x.shape and bool((stats == 0).all())
        dg, db = torch.full((8,), 3.0, device="cuda"), torch.full((8,), 3.0, device="cuda")
        B.surgeon_group_norm_grad(x, x, 2, gamma, gamma, stats, dgamma=dg, dbeta=db, accumulate=True)
        assert bool((dg == 3).all()) and bool((db == 3).all())
        B.surgeon_group_norm_grad(x, x, 2, gamma, gamma, stats, dgamma=dg, dbeta=db)
        assert bool((dg == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_against_autograd(act):
    g, x, gamma, beta = inputs(2, 50, 48, F32, seed=2)
    dy = torch.randn(2, 50, 48, generator=g, device="cuda")
    t = [v.double().requires_grad_() for v in (x, gamma, beta)]
    y = act64(torch.nn.functional.group_norm(t[0].transpose(1, 2), 6, t[1], t[2], EPS).transpose(1, 2), act)
    y.backward(dy.double())
    stats, dg, db = torch.empty(2, 2, 6, device="cuda"), torch.empty(48, device="cuda"), torch.empty(48, device="cuda")
    B.surgeon_group_norm(x, 6, gamma, beta, EPS, act=ACTS[act], stats=stats)
    dx = B.surgeon_group_norm_grad(x, dy, 6, gamma, beta, stats, act=ACTS[act], dgamma=dg, dbeta=db)
    for got, want in ((dx, t[0].grad), (dg, t[1].grad), (db, t[2].grad)):
        assert ((got.double() - want).norm() / want.norm()).item() < 2e-6
