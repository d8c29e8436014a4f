"""GPU: surgeon_attention and surgeon_attention_grad against the formulas in 64 bits.

Tolerances count roundings, element by element.  u = 2^-24: the products' sums are taken in fp32 (2 u a term covers the tensor cores' truncation),
exponentials are good to 2^-21.  P and dS are rounded to bf16 for the products, results once more: half a step, finfo.eps / 2, each."""
import math

import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16 = torch.bfloat16
H = torch.finfo(BF16).eps / 2


def make(b, nq, nk, h, hk, d, layout="rows", seed=0, scale_q=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * nq + nk + d)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)
    if layout == "packed":
        q, k, v = rnd(b, nq, 3, h, d).unbind(2)
    elif layout == "heads":
        q, k, v = (rnd(b, n, m, d).transpose(1, 2) for n, m in ((h, nq), (hk, nk), (hk, nk)))
    else:
        q, k, v = rnd(b, nq, h, d), rnd(b, nk, hk, d), rnd(b, nk, hk, d)
    return q * scale_q if scale_q != 1.0 else q, k, v, g


def visible(b, nq, nk, ql, kl, causal):
    i, j = torch.arange(nq, device="cuda")[:, None], torch.arange(nk, device="cuda")[None]
    m = torch.zeros(b, nq, nk, dtype=torch.bool, device="cuda")
    for n in range(b):
        q_n, k_n = nq if ql is None else int(ql[n]), nk if kl is None else int(kl[n])
        m[n] = (i < q_n) & (j < k_n)
        if causal:
            m[n] &= j <= i + (k_n - q_n)
    return m[:, None]


def clean(t, lengths):
    """64 bits, heads first; what lies behind the lengths is 0."""
    t = t.double()
    if lengths is not None:
        keep = torch.arange(t.shape[1], device="cuda")[None] < lengths[:, None]
        t = torch.where(keep[:, :, None, None], t, torch.zeros_like(t))
    return t.transpose(1, 2)


class Reference:
    """Forward pass in 64 bits and what each result may be off by."""

    def __init__(self, q, k, v, causal, scale, ql=None, kl=None):
        b, nq, h, d = q.shape
        nk, hk = k.shape[1:3]
        self.times, self.scale, self.d, self.shape = h // hk, scale, d, (b, nq, nk, h, hk, d)
        rep = lambda t: t.repeat_interleave(self.times, 1)
        self.q, self.k, self.v = clean(q, ql), rep(clean(k, kl)), rep(clean(v, kl))
        self.m = visible(b, nq, nk, ql, kl, causal)
        s = self.q @ self.k.transpose(2, 3) * scale
        self.s = s.masked_fill(~self.m, -math.inf)
        top = self.s.amax(3, keepdim=True) if nk else torch.full((b, h, nq, 1), -math.inf, dtype=torch.float64, device="cuda")
        self.seen = self.m.any(3) if nk else torch.zeros(b, 1, nq, dtype=torch.bool, device="cuda")
        e = torch.exp(self.s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
        total = e.sum(3, keepdim=True)
        self.p = e / torch.where(total > 0, total, torch.ones_like(total))
        self.o = self.p @ self.v
        self.lse = torch.where(total[..., 0] > 0, torch.log(total[..., 0]) + top[..., 0], torch.full_like(total[..., 0], -math.inf))
        # the scores' error, in units of the exponent
        self.e_s = 2 * d * U * (self.q.abs() @ self.k.abs().transpose(2, 3)) * scale + 4 * U * s.abs()
        self.rel = self.e_s.masked_fill(~self.m, 0.0).amax(3, keepdim=True) if nk else torch.zeros_like(top)

    def check(self, out, lse):
        b, nq, nk, h, hk, d = self.shape
        size = self.p @ self.v.abs()
        rel = 2 * self.rel + 2.0 ** -20 + 2 * nk * U
        tol = size * (H + rel) * (1 + H) + H * self.o.abs() + 1e-30
        got = out.double().transpose(1, 2)
        assert torch.isfinite(got).all() and ((got - self.o).abs() <= tol).all(), ((got - self.o).abs() / tol).max()
        assert bool((got.masked_select(~self.seen[..., None].expand_as(got)) == 0).all())
        if lse is not None:
            gone = ~self.seen.expand_as(lse)
            assert bool((lse[gone] == -math.inf).all()) and bool(torch.isfinite(lse[~gone]).all())
            e = (lse.double() - self.lse)[~gone].abs()
            assert (e <= (self.rel[..., 0] + 2.0 ** -20 + 2 * nk * U + 4 * U * self.lse.abs()).expand_as(lse)[~gone]).all(), e.max()

    def gradients(self, out, dout, lse, ql=None):
        """dq, dk, dv from the `out` and `lse` that the call had, and their tolerances."""
        b, nq, nk, h, hk, d = self.shape
        o, do = clean(out, ql), clean(dout, ql)
        l = torch.where(torch.isfinite(lse.double()), lse.double(), torch.zeros_like(lse.double()))[..., None]
        p = torch.exp(self.s - l).masked_fill(~self.m, 0.0)
        rel = self.rel + 2.0 ** -20 + 8 * U * (l.abs() + 1)
        dp, delta = do @ self.v.transpose(2, 3), (do * o).sum(3, keepdim=True)
        ds = p * (dp - delta)
        e_dp = 2 * d * U * (do.abs() @ self.v.abs().transpose(2, 3) + (do * o).abs().sum(3, keepdim=True)) + 4 * U * (dp.abs() + delta.abs())
        e_ds = ds.abs() * (H + rel) * (1 + H) + p * e_dp * (1 + H + rel)
        e_p = p * (H + rel) * (1 + H)
        shared = lambda t: t.reshape(b, hk, self.times, nk, d).sum(2)
        dq, dk, dv = self.scale * ds @ self.k, shared(self.scale * ds.transpose(2, 3) @ self.q), shared(p.transpose(2, 3) @ do)
        sums = 4 * (nk + nq * self.times) * U                   # of the accumulations
        t_q = self.scale * ((e_ds + sums * ds.abs()) @ self.k.abs())
        t_k = shared(self.scale * ((e_ds + sums * ds.abs()).transpose(2, 3) @ self.q.abs()))
        t_v = shared((e_p + sums * p).transpose(2, 3) @ do.abs())
        # (what underflows in fp32 is below 1e-30 here)
        return [(x, t * (1 + H) + H * x.abs() + 1e-30) for x, t in ((dq, t_q), (dk, t_k), (dv, t_v))]


def run(q, k, v, causal=False, ql=None, kl=None, scale=None, grad=True, layout_grad=None):
    b, nq, h, d = q.shape
    nk, hk = k.shape[1:3]
    desc = B.attention_desc(b, h, nq, nk, d, kv_heads=hk, causal=causal, scale=scale)
    need, need_g = B.surgeon_attention_workspace(desc), B.surgeon_attention_grad_workspace(desc)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")            # NaNs where nothing is written
    pad = torch.full((b * nq * h * d + 64,), 7.0, dtype=BF16, device="cuda")         # canaries behind the output
    out, lse = pad[:b * nq * h * d].view(b, nq, h, d), torch.full((b, h, nq), 9.0, device="cuda")
    got = B.surgeon_attention(desc, q, k, v, q_lengths=ql, kv_lengths=kl, out=out, lse=lse, workspace=ws)
    assert got is out and bool((pad[b * nq * h * d:] == 7.0).all()) and bool((ws[need:] == 0xFF).all())
    ref = Reference(q, k, v, causal, desc.scale, ql, kl)
    ref.check(out, lse)
    if not grad:
        return ref, out, lse
    g = torch.Generator(device="cuda").manual_seed(5)
    dout = (0.1 * torch.randn(b, nq, h, d, generator=g, device="cuda")).to(BF16)
    if ql is not None:                                # garbage behind the sequences must not matter
        dout[torch.arange(nq, device="cuda")[None] >= ql[:, None]] = float("nan")
    ws = torch.full((need_g + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    like = lambda t: torch.full_like(t, 3.0) if layout_grad is None else layout_grad(t)
    dq, dk, dv = B.surgeon_attention_grad(desc, q, k, v, out, dout, lse, q_lengths=ql, kv_lengths=kl, dq=like(q), dk=like(k), dv=like(v), workspace=ws)
    assert bool((ws[need_g:] == 0xFF).all())
    for name, got, (want, tol) in zip("qkv", (dq, dk, dv), ref.gradients(out, dout, lse, ql)):
        e = (got.double().transpose(1, 2) - want).abs()
        assert torch.isfinite(got).all() and (e <= tol).all(), ("d" + name, (e / tol).max())
    return ref, out, lse, dq, dk, dv


# tiles and blocks and their edges, one row, one key, odd lengths; heads that share keys; each width of head that is padded otherwise
SHAPES = [(1, 1, 1, 1, 1, 64), (2, 1, 77, 3, 3, 64), (1, 5, 3, 2, 1, 8), (2, 63, 64, 2, 2, 64), (1, 64, 65, 1, 1, 16), (2, 127, 129, 2, 1, 128),
          (1, 128, 128, 2, 2, 64), (1, 129, 192, 3, 3, 72), (3, 197, 197, 4, 4, 64), (1, 256, 257, 2, 2, 32), (1, 257, 511, 1, 1, 128), (1, 300, 40, 4, 2, 120),
          (2, 513, 640, 2, 2, 64), (1, 700, 1025, 2, 1, 56), (1, 1, 3000, 8, 2, 128), (2, 7, 1500, 8, 2, 64), (1, 100, 2100, 2, 2, 80), (20, 40, 50, 8, 8, 64),
          (1, 2000, 1, 2, 2, 64), (1, 1300, 1300, 8, 4, 64),
          # few rows: spread over a tile's warps, with items for every SM and without; too many rows for that; heads in one tile, keys not shared out
          (200, 1, 600, 2, 2, 64), (80, 20, 520, 2, 2, 64), (160, 9, 600, 4, 1, 128), (1, 32, 545, 1, 1, 128), (3, 8, 1025, 4, 1, 40)]


@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
@pytest.mark.parametrize("b,nq,nk,h,hk,d", SHAPES)
def test_matches_the_formulas(b, nq, nk, h, hk, d, causal):
    q, k, v, _ = make(b, nq, nk, h, hk, d)
    run(q, k, v, causal)


@pytest.mark.parametrize("layout", ["packed", "heads"])
@pytest.mark.parametrize("n,h,d,causal", [(197, 3, 64, False), (70, 2, 128, True), (300, 5, 24, True)])
def test_layouts(layout, n, h, d, causal):
    q, k, v, _ = make(2, n, n, h, h, d, layout)
    if layout == "packed":                            # the gradients as the qkv layer's backward pass reads them
        whole = torch.full((2, n, 3, h, d), 3.0, dtype=BF16, device="cuda")
        parts = iter(whole.unbind(2))
        run(q, k, v, causal, layout_grad=lambda t: next(parts))
    else:
        run(q, k, v, causal)


def lengths(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


RAGGED = [((100, 100), (130, 130)), ((0, 200), (17, 200)), ((200, 1), (0, 128)), ((64, 65), (127, 129)), ((500, -3), (1000, 5))]


@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
@pytest.mark.parametrize("ql,kl", RAGGED)
@pytest.mark.parametrize("d,h,hk", [(64, 2, 2), (128, 4, 1)])
def test_padded_batches(ql, kl, d, h, hk, causal):
    """Rows behind the sequences hold NaN and infinities, which reach nothing."""
    q, k, v, _ = make(2, 200, 200, h, hk, d, seed=3)
    clip = lambda n: max(0, min(200, n))
    for n in range(2):
        q[n, clip(ql[n]):] = float("nan")
        k[n, clip(kl[n]):] = float("inf")
        v[n, clip(kl[n]):] = float("nan")
    run(q, k, v, causal, lengths(*(clip(n) for n in ql)), lengths(*(clip(n) for n in kl)))


@pytest.mark.parametrize("kl", [(5, 1500), (0, 0), (1281, 640)])
def test_few_queries_of_a_padded_batch(kl):
    q, k, v, _ = make(2, 2, 1500, 8, 2, 64, seed=4)
    for n in range(2):
        k[n, kl[n]:] = float("nan")
        v[n, kl[n]:] = float("inf")
    run(q, k, v, False, lengths(2, 1), lengths(*kl))
    run(q[:, :1], k, v, True, None, lengths(*kl))


@pytest.mark.parametrize("b,causal", [(7, False), (7, True), (300, False)])
def test_sequences_of_any_order(b, causal):
    """The backward pass takes the longest first, as far as a CTA can sort them; ends of blocks, equal lengths and empty ones among them."""
    n = 150
    g = torch.Generator().manual_seed(b)
    ql, kl = (torch.randint(0, n + 1, (b,), generator=g, dtype=torch.int32).cuda() for _ in range(2))
    ql[:5], kl[:5] = lengths(64, 64, 0, 128, n), lengths(64, 64, n, 1, n)
    q, k, v, _ = make(b, n, n, 2, 1, 64, seed=b)
    run(q, k, v, causal, ql, kl)


def test_rows_without_a_key():
    """Causal with fewer keys than queries: the first rows see nothing."""
    q, k, v, _ = make(1, 300, 100, 2, 2, 64)
    ref, out, lse, dq, dk, dv = run(q, k, v, causal=True)
    assert bool((out[:, :200] == 0).all()) and bool((lse[:, :, :200] == -math.inf).all()) and bool((dq[:, :200] == 0).all())
    q, k, v, _ = make(2, 10, 0, 2, 2, 64)             # no key at all
    desc = B.attention_desc(2, 2, 10, 0, 64)
    lse = torch.zeros(2, 2, 10, device="cuda")
    out = B.surgeon_attention(desc, q, k, v, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv = B.surgeon_attention_grad(desc, q, k, v, out, torch.ones_like(out), lse)
    assert bool((dq == 0).all()) and dk.numel() == 0
    q, k, v, _ = make(2, 0, 10, 2, 2, 64)             # no query: the keys' gradients are 0
    desc = B.attention_desc(2, 2, 0, 10, 64)
    out, lse = B.surgeon_attention(desc, q, k, v), torch.zeros(2, 2, 0, device="cuda")
    dq, dk, dv = B.surgeon_attention_grad(desc, q, k, v, out, out, lse)
    assert dq.numel() == 0 and bool((dk == 0).all()) and bool((dv == 0).all())


@pytest.mark.parametrize("d,nq,nk", [(64, 200, 900), (128, 130, 700), (64, 3, 2000)])
def test_scores_that_grow_along_the_keys(d, nq, nk):
    """The maximum of the first block is far below the last one's, and far above: o and l are scaled, or the rest vanishes."""
    q, k, v, _ = make(1, nq, nk, 2, 2, d, seed=7)
    q[..., 0] = 8.0
    ramp = torch.linspace(0, 200, nk, device="cuda")
    for sign in (1.0, -1.0):
        k[..., 0] = (sign * ramp).to(BF16)[None, :, None]
        run(q, k, v, scale=0.5)
    k[..., 0] = torch.where(torch.arange(nk, device="cuda") % 2 == 0, 300.0, -300.0).to(BF16)[None, :, None]
    run(q, k, v, scale=1.0)


def test_a_nan_stays_in_its_row():
    q, k, v, _ = make(1, 200, 300, 1, 1, 64)
    q[0, 77] = float("nan")
    desc = B.attention_desc(1, 1, 200, 300, 64)
    lse = torch.empty(1, 1, 200, device="cuda")
    out = B.surgeon_attention(desc, q, k, v, lse=lse)
    bad = torch.isnan(out).any(3)[0, :, 0]
    assert bad[77] and int(bad.sum()) == 1 and bool(torch.isnan(lse[0, 0, 77])) and bool(torch.isnan(out[0, 77]).all())
    k[0, 250, 0, 3] = float("nan")                       # a key that every query sees
    assert bool(torch.isnan(B.surgeon_attention(desc, q, k, v)).all())


def test_gradients_that_are_not_wanted_and_repeats():
    q, k, v, _ = make(2, 300, 520, 4, 2, 64)
    _, out, lse, dq, dk, dv = run(q, k, v, causal=True)
    desc = B.attention_desc(2, 4, 300, 520, 64, kv_heads=2, causal=True)
    dout = (0.1 * torch.randn(2, 300, 4, 64, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")).to(BF16)
    a, none, none2 = B.surgeon_attention_grad(desc, q, k, v, out, dout, lse, want_dkv=False)
    assert torch.equal(a, dq) and none is None and none2 is None
    none, b, c = B.surgeon_attention_grad(desc, q, k, v, out, dout, lse, want_dq=False)
    assert none is None and torch.equal(b, dk) and torch.equal(c, dv)
    for _ in range(3):                                # bit for bit
        again = B.surgeon_attention(desc, q, k, v)
        assert torch.equal(again, out)
        for x, y in zip(B.surgeon_attention_grad(desc, q, k, v, out, dout, lse), (dq, dk, dv)):
            assert torch.equal(x, y)


def test_keys_far_apart():
    """Strides whose products pass 32 bits."""
    far = (1 << 31) + 64
    store = torch.empty(2 * far + 4096 * 64, dtype=BF16, device="cuda")
    q, k0, v0, _ = make(2, 40, 50, 2, 2, 64)
    k = store.as_strided((2, 50, 2, 64), (far, 128, 64, 1))
    v = store.as_strided((2, 50, 2, 64), (far, 128, 64, 1), storage_offset=8192)
    k.copy_(k0)
    v.copy_(v0)
    run(q, k, v)


def test_against_differences():
    """The gradients of sum(o w), of forward passes in 64 bits at points either side."""
    q, k, v, g = make(1, 33, 47, 2, 1, 32)
    w = torch.randn(1, 33, 2, 32, generator=g, device="cuda").to(BF16)
    desc = B.attention_desc(1, 2, 33, 47, 32, kv_heads=1, causal=True)
    lse = torch.empty(1, 2, 33, device="cuda")
    out = B.surgeon_attention(desc, q, k, v, lse=lse)
    grads = B.surgeon_attention_grad(desc, q, k, v, out, w, lse)
    for at in range(3):
        way = torch.randn(*(q, k, v)[at].shape, generator=g, device="cuda").double()

        def value(h):
            t = [x.double() for x in (q, k, v)]
            t[at] = t[at] + h * way
            return (Reference(*t, True, desc.scale).o.transpose(1, 2) * w.double()).sum()

        slope = ((value(1e-4) - value(-1e-4)) / 2e-4).item()
        got = (grads[at].double() * way).sum().item()
        # each element of a gradient is off by some 3 roundings to bf16; their errors are independent
        assert abs(got - slope) <= 6 * H * (grads[at].double() * way).norm().item() + 1e-3 * abs(slope)
