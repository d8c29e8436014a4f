"""GPU: the new layers as an adaptation step uses them, beside the store, the norms and the linear layers: a transformer's attention sublayer and a
head with a group norm, forward and backward, against autograd in 64 bits; other streams, captured graphs, scratch that graphs share."""
import pytest
import torch

from paper_2503_20354_b200 import binding as B
from paper_2503_20354_b200 import workloads as W

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
SILU = B.SURGEON_ACT_SILU


class Block:
    """layer norm, qkv layer, attention, projection, dropout and skip connection, group norm with SiLU: every tensor its own buffer."""

    def __init__(self, batch, n, heads, d, seed, causal=False, p=0.2):
        g = torch.Generator().manual_seed(seed)
        c = heads * d
        self.b, self.n, self.h, self.d, self.c, self.p, self.seed, self.causal = batch, n, heads, d, c, p, seed, causal
        rnd = lambda *s, dt=F32, k=1.0: (torch.randn(*s, generator=g) * k).to(dt).cuda()
        self.x = rnd(batch * n, c, dt=BF16)
        self.gamma, self.beta, self.gamma2, self.beta2 = 1 + rnd(c, k=0.2), rnd(c, k=0.2), 1 + rnd(c, k=0.2), rnd(c, k=0.2)
        self.wqkv, self.wo, self.bo = rnd(3 * c, c, dt=BF16, k=c ** -0.5), rnd(c, c, dt=BF16, k=c ** -0.5), rnd(c, k=0.2)
        self.dy = rnd(batch, n, c, k=0.1)
        e = lambda *s, dt=F32: torch.zeros(*s, dtype=dt, device="cuda")
        rows = batch * n
        self.h0, self.stats = e(rows, c, dt=BF16), e(2, rows)
        self.qkv, self.o, self.lse = e(batch, n, 3, heads, d, dt=BF16), e(batch, n, heads, d, dt=BF16), e(batch, heads, n)
        self.proj, self.skip, self.y, self.stats2 = e(rows, c, dt=BF16), e(rows, c, dt=BF16), e(batch, n, c, dt=BF16), e(2, batch, heads)
        self.dskip, self.dproj, self.do, self.dqkv, self.dh, self.dx = e(batch, n, c), e(rows, c), e(rows, c, dt=BF16), e(batch, n, 3, heads, d, dt=BF16), e(rows, c), e(rows, c)
        self.dzo, self.dzq = e(rows, c), e(rows, 3 * c)
        self.dgamma, self.dbeta, self.dgamma2, self.dbeta2, self.dbo = e(c), e(c), e(c), e(c), e(c)
        self.l1, self.l2 = B.linear_desc(rows, c, 3 * c), B.linear_desc(rows, c, c)
        self.a = B.attention_desc(batch, heads, n, n, d, causal=causal)
        self.need = max(B.surgeon_linear_workspace(self.l1), B.surgeon_linear_grad_workspace(self.l1), B.surgeon_linear_grad_workspace(self.l2),
                        B.surgeon_attention_workspace(self.a), B.surgeon_attention_grad_workspace(self.a), B.surgeon_layer_norm_grad_workspace(rows, c),
                        B.surgeon_group_norm_workspace(batch, n, c, heads), B.surgeon_group_norm_grad_workspace(batch, n, c, heads))
        self.ws = torch.empty(self.need, dtype=torch.uint8, device="cuda")
        self.outputs = [self.h0, self.qkv, self.o, self.lse, self.proj, self.skip, self.y, self.stats2, self.dskip, self.dproj, self.do, self.dqkv, self.dh,
                        self.dx, self.dgamma, self.dbeta, self.dgamma2, self.dbeta2, self.dbo, self.dzo, self.dzq]

    def step(self, ws="own", stream=None):
        k, rows, c = dict(stream=stream), self.b * self.n, self.c
        w = dict(workspace=self.ws if isinstance(ws, str) else ws, **k)
        B.surgeon_layer_norm(self.x, self.gamma, self.beta, 1e-6, out=self.h0, stats=self.stats, **k)
        B.surgeon_linear(self.l1, self.h0, self.wqkv, out=self.qkv.view(rows, 3 * c), **w)
        q, kk, v = self.qkv.unbind(2)
        B.surgeon_attention(self.a, q, kk, v, out=self.o, lse=self.lse, **w)
        B.surgeon_linear(self.l2, self.o.view(rows, c), self.wo, self.bo, out=self.proj, **w)
        B.surgeon_dropout(self.proj, self.p, self.seed, 4, residual=self.x, out=self.skip, **k)
        B.surgeon_group_norm(self.skip.view(self.b, self.n, c), self.h, self.gamma2, self.beta2, 1e-5, act=SILU, out=self.y, stats=self.stats2, **w)
        # and back
        B.surgeon_group_norm_grad(self.skip.view(self.b, self.n, c), self.dy, self.h, self.gamma2, self.beta2, self.stats2, act=SILU, dx=self.dskip,
                                  dgamma=self.dgamma2, dbeta=self.dbeta2, **w)
        B.surgeon_dropout(self.dskip.view(rows, c), self.p, self.seed, 4, out=self.dproj, **k)
        B.surgeon_linear_grad(self.l2, self.dproj, self.wo, dx=self.do, dz=self.dzo, dbias=self.dbo, **w)
        dq, dk, dv = self.dqkv.unbind(2)
        B.surgeon_attention_grad(self.a, q, kk, v, self.o, self.do.view(self.b, self.n, self.h, self.d), self.lse, dq=dq, dk=dk, dv=dv, **w)
        B.surgeon_linear_grad(self.l1, self.dqkv.view(rows, 3 * c), self.wqkv, dx=self.dh, dz=self.dzq, **w)
        B.surgeon_layer_norm_grad(self.x, self.dh, self.gamma, self.stats, residual_grad=self.dskip.view(rows, c), dx=self.dx, dgamma=self.dgamma,
                                  dbeta=self.dbeta, **w)

    def take(self):
        torch.cuda.synchronize()
        got = [o.clone() for o in self.outputs]
        for o in self.outputs:
            o.zero_()
        torch.cuda.synchronize()
        return got


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("batch,n,heads,d,causal", [(3, 197, 4, 64, False), (2, 300, 3, 32, True), (1, 65, 2, 128, False)])
def test_a_step_against_autograd(batch, n, heads, d, causal):
    t = Block(batch, n, heads, d, 1, causal)
    t.step()
    rows, c = batch * n, heads * d
    store_h, store_o = B.surgeon_prune_compact(t.h0, 0.0), B.surgeon_prune_compact(t.o.view(rows, c), 0.0)
    dwqkv = B.surgeon_weight_grad(store_h, B.layer_desc(W.linear("qkv", rows, c, 3 * c), B.PATH_TENSOR_CORE), t.dzq)
    dwo = B.surgeon_weight_grad(store_o, B.layer_desc(W.linear("proj", rows, c, c), B.PATH_TENSOR_CORE), t.dzo)
    mask = (B.surgeon_dropout(torch.ones(rows, c, device="cuda"), t.p, t.seed, 4)).double()
    f = [v.double().requires_grad_() for v in (t.x, t.gamma, t.beta, t.wqkv, t.wo, t.bo, t.gamma2, t.beta2)]
    x, gamma, beta, wqkv, wo, bo, gamma2, beta2 = f
    h0 = torch.nn.functional.layer_norm(x, (c,), gamma, beta, 1e-6)
    q, k, v = (h0 @ wqkv.t()).view(batch, n, 3, heads, d).permute(2, 0, 3, 1, 4)
    s = q @ k.transpose(2, 3) * d ** -0.5
    if causal:
        s = s.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -float("inf"))
    o = (s.softmax(3) @ v).transpose(1, 2).reshape(rows, c)
    skip = (o @ wo.t() + bo) * mask + x
    z = torch.nn.functional.group_norm(skip.view(batch, n, c).transpose(1, 2), heads, gamma2, beta2, 1e-5).transpose(1, 2)
    y = torch.nn.functional.silu(z)
    y.backward(t.dy.double())
    # activations are rounded to bf16 some five times on the way, gradients some five times more: 2^-8 each, independent
    for name, got, want in (("y", t.y, y.detach()), ("dx", t.dx, x.grad), ("dgamma", t.dgamma, gamma.grad), ("dbeta", t.dbeta, beta.grad), ("dwqkv", dwqkv, wqkv.grad),
                            ("dwo", dwo, wo.grad), ("dbo", t.dbo, bo.grad), ("dgamma2", t.dgamma2, gamma2.grad), ("dbeta2", t.dbeta2, beta2.grad)):
        err = ((got.double().view_as(want) - want).norm() / want.norm()).item()
        assert err < 10 ** 0.5 * 2.0 ** -8, (name, err)
    norm = B.surgeon_clip_gradients([t.dgamma, t.dbeta, dwqkv, dwo, t.dbo, t.dgamma2, t.dbeta2], 1.0).item()
    assert norm > 0


SIZES = [(2, 70, 2, 64), (1, 300, 3, 128), (4, 197, 4, 32)]


@pytest.mark.parametrize("size", SIZES)
def test_on_a_stream_of_their_own(size):
    t = Block(*size, 2)
    t.step()
    want = t.take()
    s = torch.cuda.Stream()
    t.step(ws=None, stream=s)                         # named, scratch made by the calls
    assert same(t.take(), want)
    with torch.cuda.stream(s):                        # current
        t.step()
    assert same(t.take(), want)


def test_two_streams_at_once_with_scratch_of_their_own():
    a, b = Block(2, 500, 4, 64, 3), Block(3, 333, 2, 128, 4, causal=True)
    want = []
    for t in (a, b):
        t.step()
        want.append(t.take())
    s, u = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s):
            a.step()
        with torch.cuda.stream(u):
            b.step()
        got = a.take(), b.take()
        assert same(got[0], want[0]) and same(got[1], want[1])


def test_captured_and_replayed_on_new_data_with_scratch_that_graphs_share():
    a, b = Block(2, 197, 3, 64, 5), Block(1, 260, 2, 128, 6, causal=True)
    ws = torch.empty(max(a.need, b.need), dtype=torch.uint8, device="cuda")
    graphs = []
    for t in (a, b):
        t.step(ws=ws)                                 # (the first call of a kernel sets its shared memory)
        t.take()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.step(ws=ws)
        graphs.append(g)
    for i in range(3):
        new = [torch.randn(t.x.shape, generator=torch.Generator().manual_seed(i)).to(BF16).cuda() for t in (a, b)]
        for t, x in zip((a, b), new):
            t.x.copy_(x)
        ws.fill_(0xFF)
        for g in graphs:
            g.replay()
        got = [t.take() for t in (a, b)]
        for t, r in zip((a, b), got):
            t.step()                                  # eager, scratch of its own
            assert same(t.take(), r)


def test_few_queries_in_a_graph():
    """The path that shares the keys out: its parts and their sum, replayed on new queries and lengths."""
    q = torch.zeros(2, 1, 8, 128, dtype=BF16, device="cuda")
    k, v = (torch.randn(2, 3000, 2, 128, device="cuda").to(BF16) for _ in range(2))
    desc = B.attention_desc(2, 8, 1, 3000, 128, kv_heads=2)
    kl = torch.tensor([3000, 3000], dtype=torch.int32, device="cuda")
    ws = torch.empty(B.surgeon_attention_workspace(desc), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(2, 8, 1, device="cuda")
    B.surgeon_attention(desc, q, k, v, kv_lengths=kl, out=out, lse=lse, workspace=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.surgeon_attention(desc, q, k, v, kv_lengths=kl, out=out, lse=lse, workspace=ws)
    for lengths in ((3000, 3000), (1, 700), (0, 129)):
        q.copy_(torch.randn(q.shape, device="cuda"))
        kl.copy_(torch.tensor(lengths))
        ws.fill_(0xFF)
        g.replay()
        want = torch.empty_like(out)
        want_lse = torch.empty_like(lse)
        B.surgeon_attention(desc, q, k, v, kv_lengths=kl, out=want, lse=want_lse)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
