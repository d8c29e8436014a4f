"""GPU: surgeon_gradient_norm and surgeon_clip_gradients against sums in 64 bits.

Both sides square and add in double (a product of two fp32 numbers is exact there): n additions of
positive numbers in any order are within n * 2^-53 of each other; 1e-12 covers the sizes below.  A clipped value has three
roundings of 2^-24 (the factor, the product, the stored fp32 number), or the last one to bf16, 2^-8 / 2."""
import math

import pytest
import torch

import oracle
from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
CLIP_EPS = 1e-6


def make(sizes, dt, seed=0, at=0):
    """Gradients one behind the other in one buffer that starts `at` elements behind a 16-byte boundary."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.empty(sum(sizes) + at + 64, dtype=dt, device="cuda")
    flat.copy_(torch.randn(flat.numel(), generator=g) * 1e-2)
    views, p = [], at
    for n in sizes:
        views.append(flat[p:p + n])
        p += n
    return flat, views


def check(views, before, norm, gi, outs, max_norm):
    squares = [float(v.double().square().sum()) for v in before]
    want = math.sqrt(sum(squares))
    assert abs(norm.item() - want) <= 1e-12 * want
    if gi is not None:
        for q, v, got in zip(squares, before, gi.tolist()):
            ref = math.sqrt(q / v.numel()) if v.numel() else 0.0
            assert abs(got - ref) <= 1e-12 * ref
    c = min(1.0, max_norm / (want + CLIP_EPS))
    for v, o in zip(before, outs):
        ref = v.double() * c
        if c == 1.0:
            assert torch.equal(o, v)
        else:
            tol = 3 * 2.0 ** -24 + (torch.finfo(o.dtype).eps / 2 * (1 + 2.0 ** -22) if o.dtype == BF16 else 0.0)
            assert ((o.double() - ref).abs() <= tol * ref.abs() + 1e-44).all()


LISTS = [[1], [0], [4096], [4095, 4097], [1, 2, 3, 4, 5, 6, 7, 8, 9], [0, 5, 0, 0, 8193, 0], [64, 64, 256, 256, 2048, 7],
         [100003, 1, 77, 65536, 12289], [1_000_003, 999_999, 3], [7] * 95, [7] * 96, [130] * 97, [33] * 1024, [9] * 1025,
         [5] * 2500]


@pytest.mark.parametrize("dt", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("at", [0, 1, 3])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: "%d_tensors_of_%d" % (len(s), s[0]))
def test_norm_and_clipping(sizes, at, dt):
    flat, grads = make(sizes, dt, at=at)
    before = [v.clone() for v in grads]
    image = flat.clone()
    norm, gi = B.surgeon_gradient_norm(grads)
    assert torch.equal(flat, image)
    check(grads, before, norm, gi, grads, math.inf)
    again, gi2 = B.surgeon_gradient_norm(B.GradientList(grads))
    assert again.item() == norm.item() and torch.equal(gi, gi2)          # fixed order
    # a place of their own, at another distance from a 16-byte boundary too
    for to in (at, at + 2):
        out_flat, outs = make(sizes, dt, seed=1, at=to)
        edge = out_flat.clone()
        gi3 = torch.full_like(gi, -1.0)
        n3 = B.surgeon_clip_gradients(B.GradientList(grads, outs), 0.25 * norm.item(), gi=gi3)
        assert n3.item() == norm.item() and torch.equal(gi3, gi) and torch.equal(flat, image)
        check(grads, before, n3, gi3, outs, 0.25 * norm.item())
        assert torch.equal(out_flat[:to], edge[:to]) and torch.equal(out_flat[to + sum(sizes):], edge[to + sum(sizes):])
    # nothing to clip; then in place
    B.surgeon_clip_gradients(B.GradientList(grads, outs), 2.0 * norm.item() + 1.0)
    assert all(torch.equal(o, v) for o, v in zip(outs, before))
    B.surgeon_clip_gradients(grads, 2.0 * norm.item() + 1.0)
    assert torch.equal(flat, image)
    n4 = B.surgeon_clip_gradients(grads, 0.5 * norm.item())
    assert n4.item() == norm.item()
    check(grads, before, n4, None, grads, 0.5 * norm.item())
    assert torch.equal(flat[:at], image[:at]) and torch.equal(flat[at + sum(sizes):], image[at + sum(sizes):])


def test_mixed_types_and_separate_tensors():
    g = torch.Generator().manual_seed(3)
    grads = [(torch.randn(n, generator=g)).to(dt).cuda() for n, dt in ((768, F32), (2304, BF16), (1, BF16), (30001, F32))]
    before = [v.clone() for v in grads]
    norm = B.surgeon_clip_gradients(grads, 1.0)
    check(grads, before, norm, None, grads, 1.0)


def test_importance_is_that_of_the_single_call_and_of_the_oracle():
    _, grads = make([640 * 9, 100_001, 1], F32, seed=5)
    _, gi = B.surgeon_gradient_norm(grads)
    for v, got in zip(grads, gi.tolist()):
        ref = oracle.gradient_importance(v.cpu().numpy())
        assert abs(got - ref) <= 1e-12 * ref
        one = B.surgeon_gradient_importance(v.clone()).item()
        assert abs(got - one) <= 1e-12 * one


def test_large_and_small_numbers():
    """Squares that no fp32 number holds."""
    big = torch.full((5000,), 3.0e38, device="cuda")
    tiny = torch.full((5000,), 1e-30, device="cuda")
    norm, gi = B.surgeon_gradient_norm([big, tiny])
    want = float(torch.tensor(3.0e38))
    assert abs(norm.item() / (want * math.sqrt(5000.0)) - 1) <= 1e-12
    assert abs(gi[1].item() / float(torch.tensor(1e-30)) - 1) <= 1e-12


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_norm_that_is_no_number_leaves_the_gradients(bad):
    _, grads = make([5000, 300], F32, seed=6)
    grads[1][7] = bad
    before = [v.clone() for v in grads]
    _, outs = make([5000, 300], F32, seed=7)
    norm = B.surgeon_clip_gradients(B.GradientList(grads, outs), 1e-3)
    assert not math.isfinite(norm.item()) and math.isnan(norm.item()) == math.isnan(bad)
    assert torch.equal(outs[0], before[0]) and torch.equal(outs[1].view(torch.int32), before[1].view(torch.int32))
    B.surgeon_clip_gradients(grads, 1e-3)
    assert torch.equal(grads[0], before[0]) and torch.equal(grads[1].view(torch.int32), before[1].view(torch.int32))


def test_limits_of_the_threshold():
    _, grads = make([513], F32, seed=8)
    before = grads[0].clone()
    B.surgeon_clip_gradients(grads, math.inf)
    assert torch.equal(grads[0], before)
    B.surgeon_clip_gradients(grads, 0.0)
    assert not grads[0].any()
    assert B.surgeon_clip_gradients(grads, 0.0).item() == 0.0             # a norm of zero
    assert B.surgeon_clip_gradients([], 1.0).item() == 0.0                # of an empty list
    norm, gi = B.surgeon_gradient_norm([])
    assert norm.item() == 0.0 and gi.numel() == 0


def test_a_list_of_a_network_of_many_elements():
    """More units than CTAs, tensors over many CTAs and many tensors in one."""
    sizes = [3_000_001, 17, 768, 5_000_000] + [64] * 700 + [8_000_003]
    _, grads = make(sizes, F32, seed=9, at=2)
    before = [v.clone() for v in grads]
    gi = torch.empty(len(sizes), dtype=torch.float64, device="cuda")
    norm = B.surgeon_clip_gradients(grads, 0.1, gi=gi)
    check(grads, before, norm, gi, grads, 0.1)


def test_refusals():
    _, grads = make([100, 200], F32)
    for bad in (-1.0, float("nan")):
        with pytest.raises(B.SurgeonError) as e:
            B.surgeon_clip_gradients(grads, bad)
        assert e.value.status == B.SURGEON_ERR_INVALID_ARG
    flat = torch.zeros(4000, device="cuda")
    for lst in (B.GradientList([flat, flat]),                                         # the same tensor twice
                B.GradientList([flat[:100], flat[50:150]]),                           # in part
                B.GradientList([flat[:100]], [flat[50:150]]),
                B.GradientList([flat[:100], flat[200:300]], [flat[100:200], flat[0:100]])):   # another one's gradient
        with pytest.raises(B.SurgeonError) as e:
            B.surgeon_clip_gradients(lst, 1.0)
        assert e.value.status == B.SURGEON_ERR_INVALID_ARG
        B.surgeon_gradient_norm(lst)                                                  # only read: allowed
    outs = torch.empty(8000, device="cuda")
    B.surgeon_clip_gradients(B.GradientList([flat, flat], [outs[:4000], outs[4000:]]), 1.0)   # read twice: allowed
    with pytest.raises(B.SurgeonError) as e:
        B.surgeon_gradient_norm(grads, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == B.SURGEON_ERR_BUFFER_TOO_SMALL
    for call in (lambda: B.GradientList([flat[::2]]), lambda: B.GradientList([flat], [outs]),
                 lambda: B.GradientList([flat], [flat.to(BF16)]), lambda: B.GradientList([flat.cpu()]),
                 lambda: B.GradientList([flat, flat], [outs]),
                 lambda: B.surgeon_gradient_norm([flat], norm=torch.empty(1, device="cuda")),
                 lambda: B.surgeon_gradient_norm([flat], gi=torch.empty(2, dtype=torch.float64, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        B.GradientList([flat.half()])
