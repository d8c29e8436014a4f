"""GPU: buffers of one allocation that touch without overlapping are taken, and what is left out is not compared."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


class Arena:
    """Tensors one right behind the other."""

    def __init__(self, n):
        self.all = torch.zeros(n, dtype=torch.uint8, device="cuda")
        self.at = 0

    def take(self, *shape, dt=F32):
        n = dt.itemsize
        for s in shape:
            n *= s
        assert n % 16 == 0
        t = self.all[self.at:self.at + n].view(dt).view(*shape)
        self.at += n
        return t


@pytest.mark.parametrize("rows", [4, 40, 1000])
def test_buffers_that_touch(rows):
    c, h = 64, 96
    g = torch.Generator().manual_seed(rows)
    rnd = lambda *s, dt=F32: torch.randn(*s, generator=g).to(dt).cuda()
    src = dict(x=rnd(rows, c, dt=BF16), gamma=rnd(c), beta=rnd(c), w=rnd(h, c, dt=BF16), bias=rnd(h), res=rnd(rows, h, dt=BF16),
               dy=rnd(rows, h, dt=BF16), skip=rnd(rows, c, dt=BF16))
    d = B.linear_desc(rows, c, h)
    need = max(B.surgeon_layer_norm_grad_workspace(rows, c), B.surgeon_linear_workspace(d), B.surgeon_linear_grad_workspace(d))

    def step(take):
        t = {}
        for k, v in src.items():
            t[k] = take(*v.shape, dt=v.dtype)
            t[k].copy_(v)
            if k == "x":
                t["y"], t["stats"] = take(rows, c, dt=BF16), take(2, rows)
            if k == "bias":
                t["z"], t["pre"], t["ws"] = take(rows, h, dt=BF16), take(rows, h, dt=BF16), take((need + 15) // 16 * 16, dt=torch.uint8)
            if k == "dy":
                t["dx"], t["dz"], t["db"] = take(rows, c, dt=BF16), take(rows, h), take(h)
            if k == "skip":
                t["out"], t["dg"], t["dbt"] = take(rows, c, dt=BF16), take(c), take(c)
        B.surgeon_layer_norm(t["x"], t["gamma"], t["beta"], 1e-6, out=t["y"], stats=t["stats"])
        B.surgeon_linear(d, t["y"], t["w"], t["bias"], B.SURGEON_ACT_GELU, t["res"], out=t["z"], pre=t["pre"], workspace=t["ws"])
        B.surgeon_linear_grad(d, t["dy"], t["w"], t["pre"], B.SURGEON_ACT_GELU, dx=t["dx"], dz=t["dz"], dbias=t["db"], workspace=t["ws"])
        B.surgeon_layer_norm_grad(t["x"], t["dx"], t["gamma"], t["stats"], t["skip"], dx=t["out"], dgamma=t["dg"], dbeta=t["dbt"], workspace=t["ws"])
        t.pop("ws")
        return t

    together, apart = step(Arena(1 << 25).take), step(lambda *s, dt=F32: torch.zeros(*s, dtype=dt, device="cuda"))
    torch.cuda.synchronize()
    for k in together:
        assert torch.equal(together[k], apart[k]), k


def test_what_is_not_read_is_not_compared():
    d = B.linear_desc(40, 64, 24)
    w, dy = torch.randn(24, 64, device="cuda").to(BF16), torch.randn(40, 24, device="cuda").to(BF16)
    pre = torch.zeros(40, 64, device="cuda").to(BF16)
    # z is not read without an activation: its place may be dx's
    dx = B.surgeon_linear_grad(d, dy, w, pre.view(-1)[:40 * 24].view(40, 24), B.SURGEON_ACT_NONE, dx=pre)
    assert torch.equal(dx, B.surgeon_linear_grad(d, dy, w))
    with pytest.raises(B.SurgeonError) as e:
        B.surgeon_linear_grad(d, dy, w, pre.view(-1)[:40 * 24].view(40, 24), B.SURGEON_ACT_RELU, dx=pre)
    assert e.value.status == B.SURGEON_ERR_INVALID_ARG
