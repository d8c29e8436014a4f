"""GPU: surgeon_linear and surgeon_linear_grad against the formulas in 64 bits.

Tolerances.  Products of two bf16 numbers are exact in fp32; the tensor cores add 16 at a time to an fp32 accumulator, each
addition within 2^-23 of the largest partial sum, so a sum of K products is within K 2^-23 sum |a b| (the sum of one warp's lanes,
for few rows, is closer).  GELU: Phi within 7.5e-8 (the polynomial's error, halved) and 8 roundings of 2^-24.  An output or an operand
rounded to bf16 is off by 2^-8 of itself."""
import math

import pytest
import torch

from paper_2503_20354_b200 import binding as B
from paper_2503_20354_b200 import workloads as W

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
NONE, RELU, GELU = B.SURGEON_ACT_NONE, B.SURGEON_ACT_RELU, B.SURGEON_ACT_GELU
PHI = 7.5e-8 + 8 * U

# rows, c_in, c_out: few rows; one row behind them; tiles that are not full; widths that no 16-byte row holds
SHAPES = [(1, 1, 1), (1, 2048, 1000), (2, 64, 33), (3, 100, 9), (4, 768, 257), (4, 65, 64), (5, 8, 8), (5, 1, 1), (7, 16, 24),
          (33, 72, 40), (64, 512, 1000), (65, 63, 64), (100, 64, 63), (127, 200, 100), (128, 128, 128), (129, 136, 130), (200, 768, 96),
          (257, 320, 1280), (300, 1000, 72), (513, 65, 513), (1030, 256, 264), (2050, 264, 1032)]
LARGE = [(12608, 768, 768), (9000, 512, 2048), (37000, 64, 256), (5000, 1600, 384), (20000, 128, 192)]


def weights(c_in, c_out, gen):
    return (torch.randn(c_out, c_in, generator=gen) * c_in ** -0.5).to(BF16)


def phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def act_of(z, act):
    return z if act == NONE else z.clamp(min=0.0) if act == RELU else z * phi(z)


def slope_of(z, act):
    if act == NONE:
        return torch.ones_like(z)
    if act == RELU:
        return (z > 0).double()
    return phi(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def half_step(dt):
    return torch.finfo(dt).eps / 2


def product(a, b):
    """a b^T in 64 bits, and what a sum in fp32 may be off by."""
    a, b = a.double().cuda(), b.double().cuda()
    return (a @ b.t()).cpu(), (a.shape[1] * 2.0 ** -23 * (a.abs() @ b.abs().t())).cpu()


def check_forward(rows, c_in, c_out, act, bias, residual, keep, dt, seed=0):
    gen = torch.Generator().manual_seed(rows + 7 * c_in + 13 * c_out + seed)
    x, w = torch.randn(rows, c_in, generator=gen).to(BF16), weights(c_in, c_out, gen)
    b = 0.5 * torch.randn(c_out, generator=gen) if bias else None
    r = torch.randn(rows, c_out, generator=gen).to(dt) if residual else None
    n = rows * c_out
    pads = [torch.full((n + 64,), 7.0, dtype=t, device="cuda") for t in (dt, BF16)]
    out, pre = pads[0][:n].view(rows, c_out), pads[1][:n].view(rows, c_out) if keep else None
    desc = B.linear_desc(rows, c_in, c_out)
    need = B.surgeon_linear_workspace(desc)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    args = [None if t is None else t.cuda() for t in (b, r)]
    got = B.surgeon_linear(desc, x.cuda(), w.cuda(), args[0], act, args[1], out=out, pre=pre, workspace=ws)
    torch.cuda.synchronize()
    assert got is out and bool((ws[need:] == 0xFF).all())
    assert int(ws[:4].view(torch.int32)[0]) in (B.SURGEON_OK, -1)
    assert bool((pads[0][n:] == 7.0).all()) and bool((pads[1][n if keep else 0:] == 7.0).all())
    z, tol = product(x, w)
    if bias:
        z = z + b.double()
        tol = tol + U * z.abs()
    if keep:
        assert ((pre.cpu().double() - z).abs() <= tol + half_step(BF16) * (z.abs() + tol)).all()
    y = act_of(z, act)
    tol = 1.13 * tol + (PHI * z.abs() if act == GELU else 0.0)
    if residual:
        y = y + r.double()
        tol = tol + U * y.abs()
    tol = tol + half_step(dt) * (y.abs() + tol)
    off = (got.cpu().double() - y).abs()
    assert (off <= tol).all(), (off / tol).max()
    again = B.surgeon_linear(desc, x.cuda(), w.cuda(), args[0], act, args[1], out_dtype=dt)
    assert torch.equal(again, got)
    if residual:                                                     # the output in the residual's place
        own = r.cuda()
        assert torch.equal(B.surgeon_linear(desc, x.cuda(), w.cuda(), args[0], act, own, out=own), got)


@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,c_in,c_out", SHAPES)
def test_forward_matches_the_formula(rows, c_in, c_out, dt):
    check_forward(rows, c_in, c_out, NONE, False, False, False, dt)
    check_forward(rows, c_in, c_out, GELU, True, False, True, dt, 1)
    check_forward(rows, c_in, c_out, RELU, True, True, False, dt, 2)
    check_forward(rows, c_in, c_out, GELU, False, True, True, dt, 3)


@pytest.mark.parametrize("rows,c_in,c_out", LARGE)
def test_forward_on_many_tiles(rows, c_in, c_out):
    check_forward(rows, c_in, c_out, GELU, True, True, True, BF16, 4)
    check_forward(rows, c_in, c_out, NONE, True, True, False, F32, 5)
    check_forward(rows, c_in, c_out, RELU, True, False, False, BF16, 6)


def check_backward(rows, c_in, c_out, act, gt, xt, seed=0):
    gen = torch.Generator().manual_seed(rows + 3 * c_in + 5 * c_out + seed)
    w = weights(c_in, c_out, gen)
    dy = (0.1 * torch.randn(rows, c_out, generator=gen)).to(gt)
    pre = (1.5 * torch.randn(rows, c_out, generator=gen)).to(BF16)
    pre.view(-1)[::7] = 0.0
    old = torch.randn(c_out, generator=gen)
    desc = B.linear_desc(rows, c_in, c_out)
    need = B.surgeon_linear_grad_workspace(desc)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    dx_pad, dz_pad = torch.full((rows * c_in + 64,), 7.0, dtype=xt, device="cuda"), torch.full((rows * c_out + 64,), 7.0, device="cuda")
    dx, dz = dx_pad[:rows * c_in].view(rows, c_in), dz_pad[:rows * c_out].view(rows, c_out)
    db = torch.full((c_out,), 9.0, device="cuda")
    p = None if act == NONE else pre.cuda()
    got = B.surgeon_linear_grad(desc, dy.cuda(), w.cuda(), p, act, dx=dx, dz=dz, dbias=db, workspace=ws)
    torch.cuda.synchronize()
    assert got is dx and bool((ws[need:] == 0xFF).all())
    assert int(ws[:4].view(torch.int32)[0]) in (B.SURGEON_OK, -1)
    assert bool((dx_pad[rows * c_in:] == 7.0).all()) and bool((dz_pad[rows * c_out:] == 7.0).all())
    d = dy.double() * slope_of(pre.double(), act)
    e_d = (PHI + 8 * U) * dy.double().abs() + U * d.abs() if act == GELU else U * d.abs()
    assert ((dz.cpu().double() - d).abs() <= e_d).all()
    k = (100 + rows // 16) * U
    assert ((db.cpu().double() - d.sum(0)).abs() <= k * d.abs().sum(0) + e_d.sum(0)).all()
    want, tol = product(d, w.t())
    rounded = rows > 4 and not (act == NONE and gt == BF16)
    err = e_d + (half_step(BF16) * (d.abs() + e_d) if rounded else 0.0)
    tol = tol + product(err, w.t().abs())[0]
    tol = tol + half_step(xt) * (want.abs() + tol)
    off = (dx.cpu().double() - want).abs()
    assert (off <= tol).all(), (off / tol).max()
    # one output at a time, the same bits; added to what is there
    assert torch.equal(B.surgeon_linear_grad(desc, dy.cuda(), w.cuda(), p, act, dx=torch.empty_like(dx)), dx)
    dz2, db2 = torch.empty_like(dz), old.cuda()
    assert B.surgeon_linear_grad(desc, dy.cuda(), None, p, act, dz=dz2, want_dx=False) is None
    assert B.surgeon_linear_grad(desc, dy.cuda(), None, p, act, dbias=db2, accumulate=True, want_dx=False) is None
    assert torch.equal(dz2, dz)
    # with dx, dz's sums come from the product's tiles: grouped otherwise
    if act == NONE and gt == BF16 and c_out % 8 == 0 and rows > 4:
        assert ((db2 - old.cuda()).double().cpu() - d.sum(0)).abs().le(k * d.abs().sum(0) + e_d.sum(0) + U * (db2.cpu().abs() + old.abs())).all()
        again = torch.full_like(db, 9.0)
        B.surgeon_linear_grad(desc, dy.cuda(), w.cuda(), p, act, dx=torch.empty_like(dx), dbias=again)
        assert torch.equal(again, db)
        B.surgeon_linear_grad(desc, dy.cuda(), w.cuda(), p, act, dx=torch.empty_like(dx), dbias=again, accumulate=True)
        assert torch.equal(again, db + db)
    else:
        assert torch.equal(db2, old.cuda() + db)


@pytest.mark.parametrize("act", [NONE, RELU, GELU], ids=["none", "relu", "gelu"])
@pytest.mark.parametrize("rows,c_in,c_out", SHAPES)
def test_backward_matches_the_formula(rows, c_in, c_out, act):
    check_backward(rows, c_in, c_out, act, BF16, BF16)
    check_backward(rows, c_in, c_out, act, F32, F32, 1)


@pytest.mark.parametrize("rows,c_in,c_out", LARGE)
def test_backward_on_many_tiles(rows, c_in, c_out):
    check_backward(rows, c_in, c_out, NONE, BF16, BF16, 2)
    check_backward(rows, c_in, c_out, GELU, F32, BF16, 3)
    check_backward(rows, c_in, c_out, RELU, BF16, F32, 4)


@pytest.mark.parametrize("rows", [3, 300])
def test_numbers_that_are_not_finite(rows):
    """They stay in their row (of x) and column (of the weights); padding columns hold none of them."""
    gen = torch.Generator().manual_seed(5)
    c_in, c_out = 72, 80
    x, w = torch.randn(rows, c_in, generator=gen).to(BF16), weights(c_in, c_out, gen)
    desc = B.linear_desc(rows, c_in, c_out)
    clean = B.surgeon_linear(desc, x.cuda(), w.cuda(), act=GELU, out_dtype=F32)
    bad = x.clone()
    bad[1, 5] = float("nan")
    y = B.surgeon_linear(desc, bad.cuda(), w.cuda(), act=GELU, out_dtype=F32)
    keep = [i for i in range(rows) if i != 1]
    assert torch.equal(y[keep], clean[keep]) and bool(y[1].isnan().all())
    # z of infinity: GELU and ReLU give infinity and 0, and NaN for NaN
    bias = torch.zeros(c_out)
    bias[0], bias[1], bias[2] = float("inf"), float("-inf"), float("nan")
    for act in (GELU, RELU):
        y = B.surgeon_linear(desc, x.cuda(), w.cuda(), bias.cuda(), act, out_dtype=F32)
        assert bool((y[:, 0] == float("inf")).all()) and bool((y[:, 1] == 0).all()) and bool(y[:, 2].isnan().all())


def test_gradient_against_differences():
    """sum(g * y) along a direction of x and of the bias: a central difference in 64 bits."""
    gen = torch.Generator().manual_seed(6)
    rows, c_in, c_out = 40, 24, 56
    x, w = torch.randn(rows, c_in, generator=gen).to(BF16), weights(c_in, c_out, gen)
    b = (0.3 * torch.randn(c_out, generator=gen))
    g = torch.randn(rows, c_out, generator=gen).to(BF16)
    desc = B.linear_desc(rows, c_in, c_out)
    for act in (NONE, GELU):
        pre = torch.empty(rows, c_out, dtype=BF16, device="cuda")
        B.surgeon_linear(desc, x.cuda(), w.cuda(), b.cuda(), act, pre=pre)
        dx, db = torch.empty(rows, c_in, device="cuda"), torch.empty(c_out, device="cuda")
        B.surgeon_linear_grad(desc, g.cuda(), w.cuda(), pre, act, dx=dx, dbias=db)
        at = [x.double(), b.double()]

        def value(x, b):
            return (act_of(x @ w.double().t() + b, act) * g.double()).sum()

        for i, got in enumerate((dx, db)):
            step = torch.randn(at[i].shape, generator=gen, dtype=torch.float64)
            h = 1e-5
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * step, at[i] - h * step
            want = (value(*up) - value(*down)) / (2 * h)
            have = (got.cpu().double() * step).sum()
            # pre is stored with 8 bits: the slope (its derivative at most 0.8) and dz are off by 2^-8 of |z| and of themselves
            z = at[0] @ w.double().t() + at[1]
            err = g.double().abs() * (0.8 * z.abs() + 1.13) * 2.0 ** -8
            tol = ((err @ w.double().abs()) * step.abs()).sum() if i == 0 else (err.sum(0) * step.abs()).sum()
            assert abs(have - want) <= tol + 1e-6 * (1 + abs(want))


def test_a_block_around_the_store():
    """Layer norm, prune, linear with GELU, linear with residual, and back: as an adaptation step calls them, against the
    formulas in 64 bits."""
    rows, c, hidden = 394, 192, 768
    gen = torch.Generator().manual_seed(7)
    x = torch.randn(rows, c, generator=gen).to(BF16).cuda()
    gamma, beta = (1 + 0.1 * torch.randn(c, generator=gen)).cuda(), (0.1 * torch.randn(c, generator=gen)).cuda()
    w1, w2 = weights(c, hidden, gen).cuda(), weights(hidden, c, gen).cuda()
    b1, b2 = (0.1 * torch.randn(hidden, generator=gen)).cuda(), (0.1 * torch.randn(c, generator=gen)).cuda()
    dy = (0.01 * torch.randn(rows, c, generator=gen)).to(BF16).cuda()
    d1, d2 = B.linear_desc(rows, c, hidden), B.linear_desc(rows, hidden, c)
    stats = torch.empty(2, rows, device="cuda")
    h = B.surgeon_layer_norm(x, gamma, beta, 1e-6, stats=stats)
    store1 = B.surgeon_prune_compact(h, 0.6)
    pre = torch.empty(rows, hidden, dtype=BF16, device="cuda")
    a = B.surgeon_linear(d1, h, w1, b1, GELU, pre=pre)
    store2 = B.surgeon_prune_compact(a, 0.8)
    y = B.surgeon_linear(d2, a, w2, b2, residual=x)
    # backward
    dz2, db2 = torch.empty(rows, c, device="cuda"), torch.empty(c, device="cuda")
    da = B.surgeon_linear_grad(d2, dy, w2, dz=dz2, dbias=db2)
    dw2 = B.surgeon_weight_grad(store2, B.layer_desc(W.linear("fc2", rows, hidden, c), B.PATH_TENSOR_CORE), dz2)
    dz1, db1 = torch.empty(rows, hidden, device="cuda"), torch.empty(hidden, device="cuda")
    dh = B.surgeon_linear_grad(d1, da, w1, pre, GELU, dz=dz1, dbias=db1)
    dw1 = B.surgeon_weight_grad(store1, B.layer_desc(W.linear("fc1", rows, c, hidden), B.PATH_TENSOR_CORE), dz1)
    dg, dbt = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    dx = B.surgeon_layer_norm_grad(x, dh, gamma, stats, residual_grad=dy, dgamma=dg, dbeta=dbt)
    grads = [dw1, db1, dw2, db2, dg, dbt]
    before = [g.clone() for g in grads]
    norm = B.surgeon_clip_gradients(grads, 0.1)
    # the same step by autograd in 64 bits
    f = [t.double().requires_grad_() for t in (x, gamma, beta, w1, b1, w2, b2)]
    hn = torch.nn.functional.layer_norm(f[0], (c,), f[1], f[2], 1e-6)
    an = torch.nn.functional.gelu(hn @ f[3].t() + f[4])
    yn = an @ f[5].t() + f[6] + f[0]
    yn.backward(dy.double())

    def off(got, want):
        return float((got.double() - want).norm() / want.norm())

    # tensors rounded on the way (h, a, y, pre, da, dz, dh): each by 2^-8 of its values at most
    assert off(y, yn.detach()) < 3 * 2.0 ** -8 and off(dx, f[0].grad) < 5 * 2.0 ** -8
    for got, want in ((before[1], f[4].grad), (before[3], f[6].grad), (before[4], f[1].grad), (before[5], f[2].grad)):
        assert off(got, want) < 6 * 2.0 ** -8
    s1, s2 = B.surgeon_decompress(store1).view(rows, c).double(), B.surgeon_decompress(store2).view(rows, hidden).double()
    assert off(before[0], dz1.double().t() @ s1) < 5e-3 and off(before[2], dz2.double().t() @ s2) < 5e-3
    want = math.sqrt(sum(float(g.double().square().sum()) for g in before))
    assert abs(norm.item() - want) <= 1e-12 * want
    for g, g0 in zip(grads, before):
        assert torch.allclose(g.double(), g0.double() * min(1.0, 0.1 / (want + 1e-6)), rtol=4 * U, atol=0)


def test_refusals():
    gen = torch.Generator().manual_seed(8)
    d = B.linear_desc(8, 16, 24)
    x, w = torch.randn(8, 16, generator=gen).to(BF16).cuda(), weights(16, 24, gen).cuda()
    dy = torch.randn(8, 24, generator=gen).to(BF16).cuda()
    for call in (lambda: B.surgeon_linear(d, x.float(), w), lambda: B.surgeon_linear(d, x, w.float()), lambda: B.surgeon_linear(d, x[:4], w),
                 lambda: B.surgeon_linear(d, x, w.t()), lambda: B.surgeon_linear(d, x, w, bias=dy[0]),
                 lambda: B.surgeon_linear(d, x, w, residual=dy, out_dtype=F32), lambda: B.surgeon_linear(d, x, w, pre=dy.float()),
                 lambda: B.surgeon_linear_grad(d, dy[:, :16].contiguous(), w), lambda: B.surgeon_linear_grad(d, dy, w, dz=dy),
                 lambda: B.surgeon_linear_grad(d, dy, w, dx=torch.empty(8, 24, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    fp32 = B.linear_desc(8, 16, 24)
    fp32.path = B.PATH_FP32
    conv = B.layer_desc(W.conv("c", 1, 16, 8, 24, 1), B.PATH_TENSOR_CORE)
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for call, status in ((lambda: B.surgeon_linear(d, x, w, act=3), B.SURGEON_ERR_INVALID_ARG),
                         (lambda: B.surgeon_linear(fp32, x, w, workspace=ws), B.SURGEON_ERR_UNSUPPORTED),
                         (lambda: B.surgeon_linear(d, x, w, workspace=small), B.SURGEON_ERR_BUFFER_TOO_SMALL),
                         (lambda: B.surgeon_linear_grad(d, dy, w, act=GELU), B.SURGEON_ERR_INVALID_ARG),
                         (lambda: B.surgeon_linear_grad(d, dy, None), B.SURGEON_ERR_INVALID_ARG),
                         (lambda: B.surgeon_linear_grad(d, dy, w, workspace=small), B.SURGEON_ERR_BUFFER_TOO_SMALL)):
        with pytest.raises(B.SurgeonError) as e:
            call()
        assert e.value.status == status
    assert B.surgeon_linear_workspace(conv) == 0 and B.surgeon_linear_grad_workspace(conv) == 0
