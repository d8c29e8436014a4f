"""CPU-side checks of attention, group norm and dropout: scratch sizes, refusals that are decided on the host, places that overlap.  No kernel is
launched: every call below is refused before anything reaches the device (the addresses are never touched)."""
import ctypes as C
import math

import pytest
import torch

from paper_2503_20354_b200 import binding as B
from paper_2503_20354_b200 import build as lib_build

OK, INVALID, SMALL, UNSUPPORTED = B.SURGEON_OK, B.SURGEON_ERR_INVALID_ARG, B.SURGEON_ERR_BUFFER_TOO_SMALL, B.SURGEON_ERR_UNSUPPORTED
F32, BF16 = B.SURGEON_F32, B.SURGEON_BF16
P = 1 << 24                                       # aligned addresses that are not looked at, far enough apart
BATCH, HEADS, ROWS, DIM = 2, 3, 10, 16


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


def rows(at, batch=None, row=HEADS * DIM, head=DIM):
    return B.Heads(at, ROWS * HEADS * DIM if batch is None else batch, row, head)


def desc(**k):
    return B.attention_desc(**{**dict(batch=BATCH, heads=HEADS, q_len=ROWS, kv_len=ROWS, head_dim=DIM), **k})


def attention(d=None, q=None, k=None, v=None, o=None, ql=None, kl=None, lse=5 * P, ws=6 * P, size=1 << 30, **skip):
    q, k, v, o = q or rows(P), k or rows(2 * P), v or rows(3 * P), o or rows(4 * P)
    return B.lib().surgeon_attention(d or desc(), None if "q" in skip else q, k, v, ql, kl, o, lse, ws, size, None)


def attention_grad(d=None, lse=6 * P, ql=None, kl=None, dq=0, dk=0, dv=0, ws=10 * P, size=1 << 30, **given):
    t = {n: given.get(n, rows((i + 1) * P)) for i, n in enumerate(("q", "k", "v", "o", "dout"))}
    g = [rows((7 + i) * P) if x == 0 else x for i, x in enumerate((dq, dk, dv))]
    return B.lib().surgeon_attention_grad(d or desc(), t["q"], t["k"], t["v"], t["o"], t["dout"], lse, ql, kl, *g, ws, size, None)


def test_attention_descriptors():
    for bad in (dict(batch=0), dict(heads=0), dict(kv_heads=2), dict(kv_heads=-1), dict(q_len=-1), dict(kv_len=-1), dict(head_dim=0), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-60)):
        assert attention(desc(**bad)) == INVALID and attention_grad(desc(**bad)) == INVALID, bad
        assert B.surgeon_attention_workspace(desc(**bad)) == 0 and B.surgeon_attention_grad_workspace(desc(**bad)) == 0
    for bad in (dict(head_dim=12), dict(head_dim=136), dict(q_len=1 << 30), dict(kv_len=1 << 30), dict(batch=1 << 20, q_len=1 << 12)):
        assert attention(desc(**bad)) == UNSUPPORTED and attention_grad(desc(**bad)) == UNSUPPORTED, bad
    d = desc()
    d.reserved = 1
    assert attention(d) == INVALID
    assert attention(desc(q_len=0)) == OK                                       # nothing to do
    assert B.lib().surgeon_attention(None, rows(P), rows(P), rows(P), None, None, rows(P), None, None, 0, None) == INVALID


def test_attention_operands():
    for bad in (B.Heads(None, 480, 48, 16), rows(P + 8), rows(P, row=44), rows(P, head=20), rows(P, row=0), rows(P, head=-16), rows(P, batch=1 << 38)):
        assert attention(q=bad) == INVALID and attention(k=bad) == INVALID and attention_grad(q=bad) == INVALID and attention_grad(dout=bad) == INVALID
        assert attention(o=bad) == INVALID and attention_grad(dq=bad) == INVALID
    # outputs whose elements share places: rows closer than their heads, sequences closer than their rows
    for bad in (rows(7 * P, row=DIM), rows(7 * P, batch=HEADS * DIM), rows(7 * P, head=8)):
        assert attention(o=bad) == INVALID and attention_grad(dq=bad) == INVALID and attention_grad(dk=bad) == INVALID
    assert attention(lse=P + 4) == INVALID and attention(ql=P + 2) == INVALID and attention(ws=P + 8) == INVALID
    assert attention_grad(lse=None) == INVALID and attention_grad(ws=None) == INVALID and attention_grad(kl=P + 1) == INVALID
    assert attention_grad(dk=None) == INVALID and attention_grad(dv=None) == INVALID           # together or not at all
    need = B.surgeon_attention_grad_workspace(desc())
    assert need > 0 and attention_grad(size=need - 1) == SMALL
    d = desc(q_len=1, kv_len=4096)                                              # few queries: the keys' parts need scratch
    need = B.surgeon_attention_workspace(d)
    one = lambda at: B.Heads(at, HEADS * DIM, HEADS * DIM, DIM)
    far = lambda at: B.Heads(at, 4096 * HEADS * DIM, HEADS * DIM, DIM)
    call = lambda ws, size: B.lib().surgeon_attention(d, one(P), far(2 * P), far(3 * P), None, None, one(4 * P), None, ws, size, None)
    assert need > 0 and call(5 * P, need - 1) == SMALL and call(None, 0) == INVALID


def test_attention_places():
    n = BATCH * ROWS * HEADS * DIM * 2
    for at in (P, P + 16, P + n - 16, P - n + 16):                              # the output over an operand, as little as 16 bytes
        assert attention(o=rows(at)) == INVALID and attention_grad(dq=rows(at)) == INVALID and attention_grad(dv=rows(at)) == INVALID
    assert attention(lse=4 * P) == INVALID and attention(lse=P) == INVALID and attention(ql=4 * P) == INVALID and attention(kl=5 * P) == INVALID
    assert attention_grad(dk=rows(7 * P)) == INVALID and attention_grad(dv=rows(8 * P + 32)) == INVALID
    for at in (P, 6 * P, 7 * P, 9 * P):
        assert attention_grad(ws=at) == INVALID
    # slices of one buffer [batch, row, 3, head, dim] lie apart; shifted by a head they do not
    packed = lambda at, i: B.Heads(at + i * HEADS * DIM * 2, ROWS * 3 * HEADS * DIM, 3 * HEADS * DIM, DIM)
    small = B.surgeon_attention_grad_workspace(desc()) - 1
    qkv = dict(q=packed(P, 0), k=packed(P, 1), v=packed(P, 2))
    assert attention_grad(**qkv, dq=packed(7 * P, 0), dk=packed(7 * P, 1), dv=packed(7 * P, 2), size=small) == SMALL     # (only the scratch is refused)
    shifted = B.Heads(7 * P + (HEADS + 1) * DIM * 2, ROWS * 3 * HEADS * DIM, 3 * HEADS * DIM, DIM)
    assert attention_grad(**qkv, dq=packed(7 * P, 0), dk=packed(7 * P, 1), dv=shifted) == INVALID
    assert attention_grad(**qkv, dq=packed(P, 0)) == INVALID                    # over the queries
    # heads-first slices [batch, 3, head, row, dim]
    first = lambda at, i: B.Heads(at + i * HEADS * ROWS * DIM * 2, 3 * HEADS * ROWS * DIM, DIM, ROWS * DIM)
    assert attention_grad(dq=first(7 * P, 0), dk=first(7 * P, 1), dv=first(7 * P, 0)) == INVALID


def norm(x=P, b=2, p=5, c=24, groups=3, dt=F32, gamma=2 * P, beta=3 * P, eps=1e-5, act=0, y=4 * P, stats=5 * P, ws=6 * P, size=1 << 30):
    return B.lib().surgeon_group_norm(x, b, p, c, groups, dt, gamma, beta, eps, act, y, stats, ws, size, None)


def norm_grad(x=P, dy=2 * P, b=2, p=5, c=24, groups=3, dt=F32, gdt=F32, gamma=3 * P, beta=4 * P, stats=5 * P, act=0, dx=6 * P, dg=7 * P, db=8 * P, ws=9 * P,
              size=1 << 30):
    return B.lib().surgeon_group_norm_grad(x, dy, b, p, c, groups, dt, gdt, gamma, beta, stats, act, dx, dg, db, 0, ws, size, None)


def test_group_norm_refusals():
    for bad in (dict(x=None), dict(y=None), dict(ws=None), dict(b=-1), dict(p=-1), dict(c=0), dict(groups=0), dict(groups=5), dict(groups=48), dict(dt=2),
                dict(eps=0.0), dict(eps=math.nan), dict(eps=math.inf), dict(act=4), dict(act=-1), dict(x=P + 4), dict(gamma=P + 4), dict(stats=P + 8),
                dict(y=P + 16), dict(stats=P), dict(ws=P + 32), dict(y=2 * P), dict(ws=5 * P)):
        assert norm(**bad) == INVALID, bad
    assert norm(b=1 << 20, p=1 << 20) == UNSUPPORTED and norm(c=1 << 21, groups=1) == UNSUPPORTED and norm(b=1 << 62, p=1 << 62) == UNSUPPORTED
    assert norm(b=0, x=None, y=None, ws=None) == OK and norm(p=0) == OK
    need = B.surgeon_group_norm_workspace(2, 5, 24, 3)
    assert need > 0 and norm(size=need - 1) == SMALL and B.surgeon_group_norm_workspace(2, 5, 24, 5) == 0
    assert B.surgeon_group_norm_workspace(1 << 40, 5, 24, 3) == 0


def test_group_norm_grad_refusals():
    for bad in (dict(x=None), dict(dy=None), dict(stats=None), dict(ws=None), dict(c=25), dict(groups=7), dict(gdt=3), dict(act=7), dict(dy=P + 4),
                dict(dg=P + 8), dict(dx=P), dict(dx=2 * P + 16), dict(dg=6 * P), dict(db=7 * P), dict(ws=2 * P), dict(dg=5 * P)):
        assert norm_grad(**bad) == INVALID, bad
    assert norm_grad(gdt=BF16) == UNSUPPORTED
    need = B.surgeon_group_norm_grad_workspace(2, 5, 24, 3)
    assert need > 0 and norm_grad(size=need - 1) == SMALL
    # the linear layer takes no SiLU
    assert B.lib().surgeon_linear(B.linear_desc(8, 16, 24), P, 2 * P, None, B.SURGEON_ACT_SILU, None, BF16, 3 * P, None, 4 * P, 1 << 30, None) == INVALID


def test_dropout_refusals():
    def call(x=P, n=100, dt=F32, p=0.5, later=None, res=2 * P, y=3 * P):
        return B.lib().surgeon_dropout(x, n, dt, p, 1, 2, later, res, y, None)

    for bad in (dict(x=None), dict(y=None), dict(n=-1), dict(dt=2), dict(p=-0.1), dict(p=1.1), dict(p=math.nan), dict(x=P + 4), dict(y=3 * P + 8), dict(res=P + 2),
                dict(later=P + 4), dict(y=P + 16), dict(y=2 * P + 384), dict(later=3 * P)):
        assert call(**bad) == INVALID, bad
    assert call(n=1 << 31) == UNSUPPORTED and call(n=0, x=None, y=None, res=None) == OK


def test_binding_refuses_before_the_library():
    """Tensors that are on no GPU, of other shapes or types; what the marshalling in C++ leaves goes through the same checks."""
    t = torch.zeros(BATCH, ROWS, HEADS, DIM, dtype=torch.bfloat16)
    x = torch.zeros(2, 5, 24)
    try:
        with pytest.raises((ValueError, RuntimeError)):
            B.surgeon_attention(desc(), t, t, t, out=t, workspace=torch.zeros(1, dtype=torch.uint8))
        with pytest.raises((ValueError, RuntimeError)):
            B.surgeon_group_norm(x, 3, out=x, workspace=torch.zeros(1, dtype=torch.uint8))
        with pytest.raises((ValueError, RuntimeError)):
            B.surgeon_dropout(x, 0.5, 1, out=x)
    except AssertionError:
        if torch.cuda.is_available():
            raise
    with pytest.raises(ValueError):
        B.surgeon_group_norm(torch.zeros(5), 1)
    with pytest.raises((TypeError, ValueError, RuntimeError, AssertionError)):
        B.surgeon_dropout(x.half(), 0.5, 1)


def test_structures_match_the_header():
    assert C.sizeof(B.Heads) == 32 and C.sizeof(B.AttentionDesc) == 40
    d = B.attention_desc(2, 4, 8, 16, 64)
    assert d.kv_heads == 4 and d.causal == 0 and d.scale == 0.125
