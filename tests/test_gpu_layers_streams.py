"""GPU: the layers around the store on other streams, in captured graphs that are replayed on new data, and with scratch that
two graphs share."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
GELU = B.SURGEON_ACT_GELU


class Calls:
    """Every call once, on buffers of its own; `outputs` are what they write."""

    def __init__(self, rows, c, hidden, seed):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s, dt=F32, k=1.0: (torch.randn(*s, generator=g) * k).to(dt).cuda()
        self.x, self.dy, self.skip = rnd(rows, c, dt=BF16), rnd(rows, c), rnd(rows, c)
        self.gamma, self.beta = rnd(c), rnd(c)
        self.w, self.b, self.dh, self.res = rnd(hidden, c, dt=BF16, k=c ** -0.5), rnd(hidden), rnd(rows, hidden, dt=BF16), rnd(rows, hidden, dt=BF16)
        self.d = B.linear_desc(rows, c, hidden)
        e = lambda *s, dt=F32: torch.zeros(*s, dtype=dt, device="cuda")
        self.y, self.stats, self.h, self.pre = e(rows, c, dt=BF16), e(2, rows), e(rows, hidden, dt=BF16), e(rows, hidden, dt=BF16)
        self.dx, self.dg, self.db = e(rows, c), e(c), e(c)
        self.dxl, self.dz, self.dbl = e(rows, c, dt=BF16), e(rows, hidden), e(hidden)
        self.grads = [rnd(hidden * c + 3), rnd(77, dt=BF16), rnd(c)]
        self.outs = [torch.zeros_like(v) for v in self.grads]
        self.list = B.GradientList(self.grads, self.outs)
        self.norm, self.gi = e(1, dt=torch.float64), e(3, dt=torch.float64)
        self.need = max(B.surgeon_layer_norm_grad_workspace(rows, c), B.surgeon_linear_workspace(self.d),
                        B.surgeon_linear_grad_workspace(self.d), B.surgeon_gradient_norm_workspace(self.list))
        self.outputs = [self.y, self.stats, self.h, self.pre, self.dx, self.dg, self.db, self.dxl, self.dz, self.dbl, *self.outs, self.norm, self.gi]

    def run(self, ws=None, stream=None):
        k = dict(stream=stream)
        B.surgeon_layer_norm(self.x, self.gamma, self.beta, 1e-6, out=self.y, stats=self.stats, **k)
        B.surgeon_linear(self.d, self.y, self.w, self.b, GELU, self.res, out=self.h, pre=self.pre, workspace=ws, **k)
        B.surgeon_linear_grad(self.d, self.dh, self.w, self.pre, GELU, dx=self.dxl, dz=self.dz, dbias=self.dbl, workspace=ws, **k)
        B.surgeon_layer_norm_grad(self.x, self.dy, self.gamma, self.stats, residual_grad=self.skip, dx=self.dx, dgamma=self.dg,
                                  dbeta=self.db, workspace=ws, **k)
        B.surgeon_clip_gradients(self.list, 1.0, norm=self.norm, gi=self.gi, workspace=ws, **k)

    def take(self):
        torch.cuda.synchronize()
        got = [o.clone() for o in self.outputs]
        for o in self.outputs:
            o.zero_()
        torch.cuda.synchronize()
        return got


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


SIZES = [(3, 64, 72), (150, 100, 130), (1000, 256, 512), (70, 1000, 1000)]


@pytest.mark.parametrize("rows,c,hidden", SIZES)
def test_on_a_stream_of_their_own(rows, c, hidden):
    calls = Calls(rows, c, hidden, 1)
    calls.run()
    want = calls.take()
    s = torch.cuda.Stream()
    calls.run(stream=s)                              # named, scratch made by the call
    assert same(calls.take(), want)
    with torch.cuda.stream(s):                       # current
        calls.run(ws=torch.empty(calls.need, dtype=torch.uint8, device="cuda"))
    assert same(calls.take(), want)


def test_two_streams_at_once_with_scratch_of_their_own():
    a, b = Calls(1000, 256, 512, 2), Calls(777, 320, 640, 3)
    want = []
    for c in (a, b):
        c.run()
        want.append(c.take())
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        a.run(stream=s)
        b.run(stream=t)
    assert same(a.take(), want[0]) and same(b.take(), want[1])


@pytest.mark.parametrize("rows,c,hidden", SIZES)
def test_captured_and_replayed_on_new_data(rows, c, hidden):
    calls, other = Calls(rows, c, hidden, 4), Calls(rows, c, hidden, 5)
    other.run()
    want = other.take()
    ws = torch.empty(calls.need, dtype=torch.uint8, device="cuda")
    calls.run(ws)
    calls.take()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls.run(ws)
    calls.take()
    for name in ("x", "dy", "skip", "gamma", "beta", "w", "b", "dh", "res"):
        getattr(calls, name).copy_(getattr(other, name))
    for p, q in zip(calls.grads, other.grads):
        p.copy_(q)
    for _ in range(3):
        g.replay()
        ws.fill_(0xFF)                               # nothing is kept in the scratch from one replay to the next
        g.replay()
        assert same(calls.take(), want)


def test_two_graphs_share_their_scratch():
    a, b = Calls(500, 256, 512, 6), Calls(333, 192, 768, 7)
    want = []
    for c in (a, b):
        c.run()
        want.append(c.take())
    ws = torch.empty(max(a.need, b.need), dtype=torch.uint8, device="cuda")
    graphs = []
    for c in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run(ws)
        graphs.append(g)
    for c in (a, b):
        c.take()
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for i in order:
            graphs[i].replay()
    assert same(a.take(), want[0]) and same(b.take(), want[1])


def test_short_calls_are_the_bindings_calls():
    """The calls marshalled in C++ and those that go through the binding's own checks: the same bits."""
    from paper_2503_20354_b200 import build
    build.build_calls()
    B.lib()
    assert B._calls is not None
    calls = Calls(150, 104, 136, 8)
    ws = torch.empty(calls.need, dtype=torch.uint8, device="cuda")
    calls.run(ws)
    want = calls.take()
    module, B._calls = B._calls, None
    try:
        calls.run(ws)
    finally:
        B._calls = module
    assert same(calls.take(), want)
    with pytest.raises(B.SurgeonError):              # the library's own refusals come through
        B.surgeon_layer_norm(calls.x, eps=-1.0, out=calls.y)


def test_accumulate_is_any_true_value():
    """Sums are added to what is there for accumulate=1 as for accumulate=True, whichever way the call takes."""
    calls = Calls(40, 64, 72, 7)
    ws = torch.empty(calls.need, dtype=torch.uint8, device="cuda")
    calls.run(ws)
    first = [t.clone() for t in (calls.dg, calls.db, calls.dbl)]
    for accumulate in (1, True):
        for stream in (None, torch.cuda.current_stream()):
            for t, v in zip((calls.dg, calls.db, calls.dbl), first):
                t.copy_(v)
            B.surgeon_layer_norm_grad(calls.x, calls.dy, calls.gamma, calls.stats, calls.skip, calls.dx, calls.dg, calls.db, accumulate,
                                      ws, stream=stream)
            B.surgeon_linear_grad(calls.d, calls.dh, calls.w, calls.pre, GELU, calls.dxl, calls.dz, calls.dbl, accumulate, ws, stream=stream)
            assert same((calls.dg, calls.db, calls.dbl), [v + v for v in first])


def test_many_calls_in_a_row():
    """Rings and accumulators pass many rounds; each call's bits are the first call's."""
    for rows, c in ((12608, 768), (4097, 1021), (3000, 2047), (20000, 64)):
        g = torch.Generator(device="cuda").manual_seed(rows)
        x = torch.randn(rows, c, generator=g, device="cuda").to(BF16)
        dy = torch.randn(rows, c, generator=g, device="cuda")
        stats = torch.empty(2, rows, device="cuda")
        first = None
        for k in range(60):
            y = B.surgeon_layer_norm(x, stats=stats)
            dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
            dx = B.surgeon_layer_norm_grad(x, dy, None, stats, residual_grad=dy, dgamma=dg, dbeta=db)
            if first is None:
                first = (y, dx, dg, db)
            elif k % 10 == 9:
                assert same((y, dx, dg, db), first)
