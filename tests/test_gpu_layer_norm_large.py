"""GPU: the layer norms' kernels for many rows against the formulas in 64 bits: CTAs that stay for many rows (forward), rings whose
stages are filled again and again (odd widths of bf16 forward, every backward pass).  The bounds are those of test_gpu_layer_norm.py."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B
from test_gpu_layer_norm import EPS, IDS, TYPES, backward_reference, check_forward

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def inputs(rows, channels, dt, seed=0):
    g = torch.Generator(device="cuda").manual_seed(rows + 7 * channels + seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return rnd, (rnd(rows, channels) * 1.5 + 2.0).to(dt), 1.0 + 0.3 * rnd(channels), 0.3 * rnd(channels)


# more rows than the SMs hold at once: each count of lanes a row, whole and part vectors; odd widths of bf16
FORWARD = [(12608, 768, BF16), (20000, 64, BF16), (20001, 40, BF16), (10000, 128, BF16), (5001, 256, BF16), (5003, 512, BF16),
           (5000, 1000, BF16), (5000, 1024, F32), (4000, 776, F32), (12608, 768, F32), (30000, 1021, BF16), (9000, 2047, BF16),
           (70001, 63, BF16), (5000, 8191, BF16), (12608, 767, F32)]


@pytest.mark.parametrize("rows,channels,dt", FORWARD)
def test_forward_of_many_rows(rows, channels, dt):
    _, x, gamma, beta = inputs(rows, channels, dt)
    ones, zeros = torch.ones_like(gamma), torch.zeros_like(beta)
    for g, b in ((gamma, beta), (None, None), (gamma, None), (None, beta)):
        pad = torch.full((rows * channels + 64,), 7.0, dtype=dt, device="cuda")
        out = pad[:rows * channels].view(rows, channels)
        stats = torch.full((2, rows), -1.0, device="cuda")
        y = B.surgeon_layer_norm(x, g, b, EPS, out=out, stats=stats)
        assert bool((pad[rows * channels:] == 7.0).all())
        check_forward(x, ones if g is None else g, zeros if b is None else b, y, stats)
        own = x.clone()                               # in place, without statistics
        assert torch.equal(B.surgeon_layer_norm(own, g, b, EPS, out=own), y)


BACKWARD = [(12608, 768), (4097, 1021), (3000, 2047), (20000, 64), (20001, 40), (6000, 257), (1500, 8192), (2500, 4100), (9000, 1024)]


@pytest.mark.parametrize("dt,gt", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,channels", BACKWARD)
def test_backward_of_many_rows(rows, channels, dt, gt):
    rnd, x, gamma, _ = inputs(rows, channels, dt, seed=1)
    dy, skip = (0.1 * rnd(rows, channels)).to(gt), (0.1 * rnd(rows, channels)).to(gt)
    ones = torch.ones_like(gamma)
    stats = torch.stack([x.double().mean(1), (x.double().var(1, unbiased=False) + EPS).rsqrt()]).float()
    for g, res in ((gamma, skip), (gamma, None), (None, skip)):
        dx, e_dx, dg, e_dg, db, e_db = backward_reference(x, dy, ones if g is None else g, stats, res)
        first = None
        for k in range(12):
            dgamma, dbeta = torch.full((channels,), 9.0, device="cuda"), torch.full((channels,), 9.0, device="cuda")
            got = B.surgeon_layer_norm_grad(x, dy, g, stats, residual_grad=res, dgamma=dgamma, dbeta=dbeta)
            if first is None:
                first = (got, dgamma, dbeta)
                assert ((got.double() - dx).abs() <= e_dx).all(), ((got.double() - dx).abs() / e_dx).max()
                assert ((dgamma.double() - dg).abs() <= e_dg).all(), ((dgamma.double() - dg).abs() / e_dg).max()
                assert ((dbeta.double() - db).abs() <= e_db).all(), ((dbeta.double() - db).abs() / e_db).max()
            else:
                assert all(torch.equal(p, q) for p, q in zip((got, dgamma, dbeta), first))
        g2, b2 = torch.empty_like(dgamma), torch.empty_like(dbeta)
        assert B.surgeon_layer_norm_grad(x, dy, g, stats, dgamma=g2, dbeta=b2, want_dx=False) is None
        assert torch.equal(g2, dgamma) and torch.equal(b2, dbeta)
        own = dy.clone()                              # in the place of dy
        assert torch.equal(B.surgeon_layer_norm_grad(x, own, g, stats, residual_grad=res, dx=own), first[0])
