"""GPU: many calls of linear layers whose tiles are taken by pairs of CTAs, some behind a short kernel (odd widths are padded first),
one behind the other.  The two CTAs of a pair allocate tensor memory together, and may start some time apart.

A sum of K products is within K 2^-23 of the sum of magnitudes, an output rounded to bf16 within half a step."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16 = torch.bfloat16
HALF = torch.finfo(BF16).eps / 2


def make(rows, c_in, c_out, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return rnd(rows, c_in).to(BF16), (rnd(c_out, c_in) * c_in ** -0.5).to(BF16), rnd(rows, c_out).to(BF16)


def within(got, want, tol):
    return bool(((got.double() - want).abs() <= tol + HALF * (want.abs() + tol)).all())


@pytest.mark.parametrize("rows,c_in,c_out,calls", [(44009, 839, 143, 12000), (30001, 515, 190, 6000), (16384, 2048, 2048, 600),
                                                   (12608, 768, 2304, 1500), (25000, 840, 144, 6000)])
def test_forward(rows, c_in, c_out, calls):
    d = B.linear_desc(rows, c_in, c_out)
    sets = [make(rows, c_in, c_out, k) for k in range(3)]
    ws = torch.empty(B.surgeon_linear_workspace(d), dtype=torch.uint8, device="cuda")
    wants = []
    for x, w, r in sets:
        y = B.surgeon_linear(d, x, w, residual=r)
        want, tol = x.double() @ w.double().t(), c_in * 2.0 ** -23 * (x.double().abs() @ w.double().abs().t())
        want += r.double()
        assert within(y, want, tol + U * want.abs())
        wants.append(y)
    out = torch.empty_like(wants[0])
    for i in range(calls):
        x, w, r = sets[i % 3]
        B.surgeon_linear(d, x, w, residual=r, out=out, workspace=ws)
        if i % 500 == 499:
            assert torch.equal(out, wants[i % 3]) and int(ws[:4].view(torch.int32)[0]) == B.SURGEON_OK


@pytest.mark.parametrize("rows,c_in,c_out,calls", [(16384, 2048, 2048, 600), (40001, 250, 840, 4000), (20000, 256, 1544, 4000)])
def test_input_gradient(rows, c_in, c_out, calls):
    d = B.linear_desc(rows, c_in, c_out)
    sets = [make(rows, c_in, c_out, k) for k in range(3)]
    ws = torch.empty(B.surgeon_linear_grad_workspace(d), dtype=torch.uint8, device="cuda")
    wants = []
    for _, w, dy in sets:
        dx = B.surgeon_linear_grad(d, dy, w)
        assert within(dx, dy.double() @ w.double(), c_out * 2.0 ** -23 * (dy.double().abs() @ w.double().abs()))
        wants.append(dx)
    out = torch.empty_like(wants[0])
    for i in range(calls):
        _, w, dy = sets[i % 3]
        B.surgeon_linear_grad(d, dy, w, dx=out, workspace=ws)
        if i % 500 == 499:
            assert torch.equal(out, wants[i % 3]) and int(ws[:4].view(torch.int32)[0]) == B.SURGEON_OK
