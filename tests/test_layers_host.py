"""CPU-side checks of the layers around the store: scratch sizes and the refusals that are decided on the host.  No kernel is
launched: every call below is refused before anything reaches the device (the addresses are never touched)."""
import ctypes as C
import math

import pytest
import torch

from paper_2503_20354_b200 import binding as B
from paper_2503_20354_b200 import build as lib_build
from paper_2503_20354_b200 import workloads as W

OK, INVALID, SMALL, UNSUPPORTED = B.SURGEON_OK, B.SURGEON_ERR_INVALID_ARG, B.SURGEON_ERR_BUFFER_TOO_SMALL, B.SURGEON_ERR_UNSUPPORTED
F32, BF16 = B.SURGEON_F32, B.SURGEON_BF16
P = 1 << 20                                       # an aligned address that is not looked at


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


def norm(x=P, rows=4, channels=64, dt=F32, gamma=P, beta=P, eps=1e-5, y=P, stats=P):
    return B.lib().surgeon_layer_norm(x, rows, channels, dt, gamma, beta, eps, y, stats, None)


def norm_grad(x=P, dy=P, rows=4, channels=64, dt=F32, gdt=F32, gamma=P, stats=P, res=P, dx=P, dg=P, db=P, ws=P, size=1 << 30):
    return B.lib().surgeon_layer_norm_grad(x, dy, rows, channels, dt, gdt, gamma, stats, res, dx, dg, db, 0, ws, size, None)


def linear(d=None, x=P, w=2 * P, bias=P, act=0, res=P, dt=BF16, y=3 * P, pre=4 * P, ws=P, size=1 << 30):
    return B.lib().surgeon_linear(d or B.linear_desc(8, 16, 24), x, w, bias, act, res, dt, y, pre, ws, size, None)


def linear_grad(d=None, dy=P, gdt=BF16, w=P, pre=P, act=0, xdt=BF16, dx=2 * P, dz=3 * P, db=P, ws=P, size=1 << 30):
    return B.lib().surgeon_linear_grad(d or B.linear_desc(8, 16, 24), dy, gdt, w, pre, act, xdt, dx, dz, db, 0, ws, size, None)


def test_layer_norm_refusals():
    for bad in (dict(x=None), dict(y=None), dict(rows=-1), dict(channels=0), dict(channels=-3), dict(dt=2), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e-60), dict(x=P + 4), dict(y=P + 8), dict(gamma=P + 4), dict(beta=P + 8),
                dict(stats=P + 4)):
        assert norm(**bad) == INVALID, bad
    assert norm(rows=1 << 20, channels=1 << 12) == UNSUPPORTED
    assert norm(rows=(1 << 62), channels=1 << 12) == UNSUPPORTED
    assert norm(x=None, y=None, rows=0) == OK                                   # nothing to do


def test_layer_norm_grad_refusals():
    for bad in (dict(x=None), dict(dy=None), dict(stats=None), dict(rows=-1), dict(channels=0), dict(dt=3), dict(gdt=-1), dict(ws=None),
                dict(x=P + 2), dict(dy=P + 2), dict(dx=P + 2), dict(res=P + 2), dict(dg=P + 4), dict(db=P + 4), dict(ws=P + 8)):
        assert norm_grad(**bad) == INVALID, bad
    assert norm_grad(gdt=BF16) == UNSUPPORTED and norm_grad(rows=1 << 21, channels=1 << 12) == UNSUPPORTED
    need = B.surgeon_layer_norm_grad_workspace(4, 64)
    assert need > 0 and norm_grad(size=need - 1) == SMALL
    assert B.surgeon_layer_norm_grad_workspace(-1, 64) == 0 and B.surgeon_layer_norm_grad_workspace(4, 0) == 0
    # at most one row of partial sums per array for two CTAs an SM
    assert B.surgeon_layer_norm_grad_workspace(1 << 20, 768) == B.surgeon_layer_norm_grad_workspace(1000, 768) <= 296 * 2 * 768 * 4


def test_linear_refusals():
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(ws=None), dict(act=-1), dict(act=3), dict(dt=2), dict(x=P + 2), dict(w=P + 2),
                dict(bias=P + 4), dict(res=P + 2), dict(y=P + 2), dict(pre=P + 2), dict(ws=P + 8), dict(y=P), dict(pre=P), dict(pre=3 * P),
                dict(d=B.linear_desc(0, 16, 24)), dict(d=B.linear_desc(8, 0, 24)), dict(d=B.linear_desc(8, 16, -1)),
                dict(d=B.layer_desc(W.conv("c", 1, 16, 8, 24, 1), 0))):
        assert linear(**bad) == INVALID, bad
    fp32 = B.linear_desc(8, 16, 24)
    fp32.path = B.PATH_FP32
    assert linear(d=fp32) == UNSUPPORTED and linear(d=B.linear_desc(1 << 20, 1 << 12, 8)) == UNSUPPORTED
    assert linear(size=B.surgeon_linear_workspace(B.linear_desc(8, 16, 24)) - 1) == SMALL
    odd = B.linear_desc(8, 17, 24)                                               # padded copies of x and the weights
    assert B.surgeon_linear_workspace(odd) >= 256 + (8 + 24) * 24 * 2
    assert B.surgeon_linear_workspace(fp32) == 0 and B.lib().surgeon_linear_workspace(None) == 0


def test_linear_grad_refusals():
    for bad in (dict(dy=None), dict(ws=None), dict(w=None), dict(act=1, pre=None), dict(act=4), dict(gdt=2), dict(xdt=2), dict(dx=P),
                dict(dz=P), dict(dy=P + 2), dict(w=P + 2), dict(pre=P + 2, act=1), dict(dx=P + 2), dict(dz=P + 4), dict(db=P + 4),
                dict(ws=P + 8), dict(d=B.linear_desc(8, 16, 0))):
        assert linear_grad(**bad) == INVALID, bad
    d = B.linear_desc(8, 16, 24)
    assert linear_grad(size=B.surgeon_linear_grad_workspace(d) - 1) == SMALL
    assert B.surgeon_linear_grad_workspace(d) >= 256 + 8 * 24 * 2


def test_outputs_in_the_place_of_operands_are_refused():
    assert norm_grad(dx=P, dg=3 * P, db=4 * P) == INVALID                        # dx over x
    assert norm_grad(dx=2 * P, dg=3 * P, db=3 * P) == INVALID                    # dgamma over dbeta
    assert linear(pre=5 * P, res=5 * P) == INVALID
    for bad in (dict(dx=P), dict(dy=5 * P, dx=P), dict(dx=3 * P), dict(dy=5 * P, pre=6 * P, act=1, dx=6 * P),
                dict(dy=5 * P, pre=6 * P, act=2, dz=6 * P)):
        assert linear_grad(**bad) == INVALID, bad


def test_extents_beyond_what_the_kernels_count_are_refused():
    top = (1 << 30) + 1
    assert norm(rows=1, channels=top) == UNSUPPORTED and norm(rows=1, channels=(1 << 31) - 1) == UNSUPPORTED
    assert norm_grad(rows=1, channels=top) == UNSUPPORTED and B.surgeon_layer_norm_grad_workspace(1, top) == 0
    for d in (B.linear_desc(top, 1, 1), B.linear_desc(1, top, 1), B.linear_desc(1, 1, top), B.linear_desc((1 << 31) - 1, 1, 1)):
        assert linear(d=d) == UNSUPPORTED and linear_grad(d=d) == UNSUPPORTED
        assert B.surgeon_linear_workspace(d) == 0 and B.surgeon_linear_grad_workspace(d) == 0
    assert B.surgeon_linear_grad_workspace(B.linear_desc(1 << 30, 1, 1)) > 0


def test_a_gradient_list_keeps_its_length():
    assert B.GradientList([]).grads == () and len(B.GradientList([])) == 0


def grads(*entries):
    """(address, output, n, dt) each."""
    return (B.Gradient * max(len(entries), 1))(*[(g, o, n, dt, 0) for g, o, n, dt in entries])


def test_gradient_list_refusals():
    l = B.lib()

    def both(lst, count, norm=P, gi=P, ws=P, size=1 << 30, max_norm=1.0):
        a = C.addressof(lst) if lst is not None else None
        return (l.surgeon_gradient_norm(a, count, norm, gi, ws, size, None), l.surgeon_clip_gradients(a, count, max_norm, norm, gi, ws, size, None))

    one = grads((P, 2 * P, 100, F32))
    for bad in (dict(lst=None, count=1), dict(lst=one, count=-1), dict(lst=one, count=1, ws=None), dict(lst=one, count=1, ws=P + 4),
                dict(lst=one, count=1, norm=P + 4), dict(lst=one, count=1, gi=P + 4), dict(lst=grads((None, P, 5, F32)), count=1),
                dict(lst=grads((P, 2 * P, -1, F32)), count=1), dict(lst=grads((P, 2 * P, 5, 7)), count=1),
                dict(lst=grads((P + 2, 2 * P, 5, F32)), count=1), dict(lst=grads((P + 1, 2 * P, 5, BF16)), count=1)):
        assert both(**bad) == (INVALID, INVALID), bad
    assert both(one, 1, size=8) == (SMALL, SMALL)
    assert both(grads((P, 1 << 50, 1 << 31, F32)), 1) == (UNSUPPORTED, UNSUPPORTED)
    assert both(one, B.lib().surgeon_gradient_norm_workspace(1) and 65537) == (UNSUPPORTED, UNSUPPORTED)
    assert l.surgeon_gradient_norm(C.addressof(one), 1, None, None, P, 1 << 30, None) == INVALID        # nothing asked for
    for max_norm in (-1.0, math.nan):
        assert l.surgeon_clip_gradients(C.addressof(one), 1, max_norm, P, P, P, 1 << 30, None) == INVALID
    # outputs over outputs, over another's gradient, over their own in part; in any order of the list
    a, b, far = P, P + 4096, 8 * P
    for lst in (grads((a, a, 100, F32), (a, a, 100, F32)), grads((a, far, 100, F32), (b, far + 396, 100, F32)),
                grads((b, far + 396, 100, F32), (a, far, 100, F32)), grads((a, b, 100, F32), (b, far, 100, F32)),
                grads((b, far, 100, F32), (a, b + 100, 100, F32)), grads((a, a + 4, 100, F32)), grads((a, a - 4, 100, F32)),
                grads((a, a, 1000, BF16), (far, a + 1998, 4, BF16))):
        assert l.surgeon_clip_gradients(C.addressof(lst), len(lst), 1.0, P, P, P, 1 << 30, None) == INVALID
    assert l.surgeon_gradient_norm_workspace(-1) == 0 and l.surgeon_gradient_norm_workspace(65537) == 0
    assert l.surgeon_gradient_norm_workspace(1000) < 20000


def test_the_short_calls_leave_what_is_not_ordinary_to_the_binding():
    """Anything but tensors on the current device with the right types and shapes: None, and no exception."""
    lib_build.build_calls()
    from paper_2503_20354_b200 import _calls
    x, v = torch.zeros(4, 64), torch.zeros(64)
    d = B.linear_desc(4, 64, 8)
    for args in ((), (x,), (x, None, None, 1e-5, x, None), (None,) * 6, (x, "a", None, 1e-5, x, None), (x, v, v, "eps", x, None),
                 (object(),) * 6, (x.half(), None, None, 1e-5, x, None)):
        assert _calls.layer_norm(*args) is None
    assert _calls.layer_norm_grad(x, x, v, x, None, x, v, v, False, v) is None and _calls.layer_norm_grad(*[None] * 10) is None
    assert _calls.linear(d, x, x, None, 0, None, x, None, v) is None and _calls.linear(object(), *[x] * 8) is None
    assert _calls.linear(b"short", *[x] * 8) is None
    assert _calls.linear_grad(d, x, x, None, 0, x, None, None, False, v) is None and _calls.linear_grad(*[3] * 10) is None
    assert _calls.gradients(0, 1, 0, 1.0, v, None, v) is None and _calls.gradients("a", -1, 1 << 70, None, v, None, v) is None
    with pytest.raises(TypeError):
        _calls.bind(1, 2)
    with pytest.raises(ValueError):
        _calls.bind(0, 0, 0, 0, 0, 0)
    l = B.lib()                                       # (as the binding has bound them)
    _calls.bind(*(C.cast(f, C.c_void_p).value for f in (l.surgeon_layer_norm, l.surgeon_layer_norm_grad, l.surgeon_linear,
                                                        l.surgeon_linear_grad, l.surgeon_gradient_norm, l.surgeon_clip_gradients)))


def test_the_binding_refuses_host_tensors_and_wrong_types():
    x, v = torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError):
        B.GradientList([v])
    with pytest.raises(TypeError):
        B.dtype_code(torch.float16)
    with pytest.raises(ValueError):
        B._operand(x, "x", 0, (4, 64), torch.float32)
    with pytest.raises(ValueError):
        B._rows(torch.zeros(()), "x")
    with pytest.raises(ValueError):
        B._rows(torch.zeros(4, 0), "x")
    assert B._rows(torch.zeros(2, 3, 5), "x") == ((2, 3, 5), 6, 5)
    assert C.sizeof(B.Gradient) == 32
    d = B.linear_desc(7, 5, 3)
    same = B.layer_desc(W.linear("l", 7, 5, 3), B.PATH_TENSOR_CORE)
    assert all(getattr(d, n) == getattr(same, n) for n, _ in B.LayerDesc._fields_)
