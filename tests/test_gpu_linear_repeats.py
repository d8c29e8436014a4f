"""GPU: the backward pass of linear layers without an activation, bf16 gradients, call after call.  dz is dy in fp32 and dbias its
sums, both written from the operand tiles that the product holds in shared memory for a moment; every call's bits are compared, since a
tile that is given back too early shows only when memory is busy.

dz has to be dy exactly (bf16 numbers are fp32 numbers).  dbias against sums in 64 bits: a warp adds 32 rows one by one, then four
warps, at most rows / 4096 + 1 slabs one by one and 32 slices of them: K roundings of 2^-24 of the sum of magnitudes.  dx against
64 bits: products are exact in fp32, a sum of c_out of them within c_out 2^-23 of the sum of magnitudes, then half a step of bf16."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16 = torch.bfloat16
# many tiles a CTA with a ring that wraps; a wide layer; many rows of two tiles of k; tiles whose reduction a cluster shares;
# rows and columns that fill no whole tile
SIZES = [(12608, 768, 2304), (16384, 2048, 2048), (37000, 64, 256), (300, 256, 512), (64, 320, 4096), (4037, 328, 1288), (20001, 72, 64)]
KINDS = 3                                             # different dy, one after the other


class Backward:
    def __init__(self, rows, c_in, c_out, seed=0):
        g = torch.Generator(device="cuda").manual_seed(rows + c_in + c_out + seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.d = B.linear_desc(rows, c_in, c_out)
        self.w = (rnd(c_out, c_in) * c_in ** -0.5).to(BF16)
        self.dys = [(0.1 * rnd(rows, c_out)).to(BF16) for _ in range(KINDS)]
        self.dy = self.dys[0].clone()
        self.dx = torch.empty(rows, c_in, dtype=BF16, device="cuda")
        self.dz, self.db = torch.empty(rows, c_out, device="cuda"), torch.empty(c_out, device="cuda")
        self.need = B.surgeon_linear_grad_workspace(self.d)
        self.ws = torch.empty(self.need, dtype=torch.uint8, device="cuda")
        self.wants = [self.reference(dy) for dy in self.dys]

    def reference(self, dy):
        """dx and dbias of one call, checked against 64 bits."""
        self.clear()
        self.run(dy)
        rows, c_out = dy.shape
        d, w = dy.double(), self.w.double()
        k = (32 + 4 + rows // 4096 + 1 + 32) * U
        assert ((self.db.double() - d.sum(0)).abs() <= k * d.abs().sum(0)).all()
        want = d @ w
        tol = c_out * 2.0 ** -23 * (d.abs() @ w.abs())
        assert ((self.dx.double() - want).abs() <= tol + torch.finfo(BF16).eps / 2 * (want.abs() + tol)).all()
        # the same products where dx alone is wanted, and nothing is passed on
        assert torch.equal(B.surgeon_linear_grad(self.d, dy, self.w, dx=torch.empty_like(self.dx)), self.dx)
        return self.dx.clone(), dy.float(), self.db.clone()

    def clear(self):
        for t in (self.dx, self.dz, self.db):
            t.fill_(float("nan"))

    def run(self, dy=None, ws=None, stream=None):
        B.surgeon_linear_grad(self.d, self.dy if dy is None else dy, self.w, dx=self.dx, dz=self.dz, dbias=self.db,
                              workspace=self.ws if ws is None else ws, stream=stream)

    def off(self, kind):
        """How many numbers of each output are not the first call's (on the device)."""
        return torch.stack([(a != b).sum() for a, b in zip((self.dx, self.dz, self.db), self.wants[kind])])


@pytest.mark.parametrize("rows,c_in,c_out", SIZES)
def test_every_call_gives_the_same_bits(rows, c_in, c_out):
    t = Backward(rows, c_in, c_out)
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    for i in range(200):
        t.clear()
        t.run(t.dys[i % KINDS])
        off += t.off(i % KINDS)
    assert off.tolist() == [0, 0, 0]
    assert int(t.ws[:4].view(torch.int32)[0]) == B.SURGEON_OK


@pytest.mark.parametrize("rows,c_in,c_out", SIZES[:5])
def test_calls_without_a_pause_while_memory_is_busy(rows, c_in, c_out):
    """Calls one behind the other, beside a stream that copies all the time: stores of dz wait for memory."""
    t = Backward(rows, c_in, c_out)
    a = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    b = torch.empty_like(a)
    busy, s = torch.cuda.Stream(), torch.cuda.Stream()
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    for i in range(60):
        with torch.cuda.stream(busy):
            for _ in range(4):
                b.copy_(a)
        with torch.cuda.stream(s):
            t.clear()
            for _ in range(3):
                t.run(t.dys[i % KINDS])
            off += t.off(i % KINDS)
    torch.cuda.synchronize()
    assert off.tolist() == [0, 0, 0]


@pytest.mark.parametrize("rows,c_in,c_out", SIZES[:5])
def test_replayed_beside_another_stream(rows, c_in, c_out):
    """A captured call replayed on new data while another stream runs the same kernels."""
    t, other = Backward(rows, c_in, c_out), Backward(rows, c_in, c_out, seed=1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.run()
    s = torch.cuda.Stream()
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    for i in range(60):
        with torch.cuda.stream(s):
            other.run(other.dys[i % KINDS])
        t.dy.copy_(t.dys[i % KINDS])
        t.clear()
        t.ws.fill_(0xFF)                              # nothing is kept in the scratch
        graph.replay()
        off += t.off(i % KINDS)
    torch.cuda.synchronize()
    assert off.tolist() == [0, 0, 0] and other.off(59 % KINDS).tolist() == [0, 0, 0]
    assert int(t.ws[:4].view(torch.int32)[0]) == B.SURGEON_OK


def test_two_graphs_share_their_scratch():
    a, b = Backward(777, 320, 640), Backward(3000, 192, 768)
    ws = torch.empty(max(a.need, b.need), dtype=torch.uint8, device="cuda")
    graphs = []
    for t in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.run(ws=ws)
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        a.clear()
        b.clear()
        for i in order:
            graphs[i].replay()
        assert a.off(0).tolist() == [0, 0, 0] and b.off(0).tolist() == [0, 0, 0]


def test_streams_named_and_current():
    t = Backward(1000, 256, 512)
    s = torch.cuda.Stream()
    t.clear()
    s.wait_stream(torch.cuda.current_stream())
    t.run(t.dys[1], stream=s)
    torch.cuda.synchronize()
    assert t.off(1).tolist() == [0, 0, 0]
    t.clear()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        t.run(t.dys[2], ws=torch.empty(t.need, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert t.off(2).tolist() == [0, 0, 0]


@pytest.mark.parametrize("rows", [5, 128, 129, 3000])
def test_the_status_word_is_written(rows):
    """From 5 rows on both passes leave SURGEON_OK in the scratch's first word."""
    t = Backward(rows, 136, 264)
    x = torch.randn(rows, 136, device="cuda").to(BF16)
    for act in (B.SURGEON_ACT_NONE, B.SURGEON_ACT_GELU):
        pre = torch.empty(rows, 264, dtype=BF16, device="cuda")
        ws = torch.full((B.surgeon_linear_workspace(t.d),), 0xFF, dtype=torch.uint8, device="cuda")
        B.surgeon_linear(t.d, x, t.w, act=act, pre=pre, workspace=ws)
        assert int(ws[:4].view(torch.int32)[0]) == B.SURGEON_OK
        ws = torch.full((t.need,), 0xFF, dtype=torch.uint8, device="cuda")
        B.surgeon_linear_grad(t.d, t.dy, t.w, pre, act, dx=t.dx, dz=t.dz, dbias=t.db, workspace=ws)
        assert int(ws[:4].view(torch.int32)[0]) == B.SURGEON_OK
