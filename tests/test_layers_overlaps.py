"""CPU: outputs that overlap operands, scratch or one another, by as little as 16 bytes at either end, are refused by the layers around
the store.  No kernel is launched: every call below is refused on the host (the addresses are never touched)."""
import itertools

import pytest

from paper_2503_20354_b200 import binding as B
from paper_2503_20354_b200 import build as lib_build

INVALID = B.SURGEON_ERR_INVALID_ARG
F32, BF16 = B.SURGEON_F32, B.SURGEON_BF16
ROWS, C_IN, C_OUT = 40, 64, 24
STEP = 1 << 24                                        # places that do not touch


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


class Call:
    """A call whose buffers lie apart; `sizes` are their bytes, `writes` the names of those that it writes."""

    def __init__(self, sizes, writes, call, may=()):
        self.sizes, self.writes, self.call, self.may = sizes, writes, call, may
        self.at = {name: (i + 1) * STEP for i, name in enumerate(sizes)}

    def overlapping(self):
        """(written, other, place of the written one) of all pairs: at the same address (unless it may), behind it, before it."""
        for w, o in itertools.product(self.writes, self.sizes):
            if w == o:
                continue
            at, n_w, n_o = self.at[o], self.sizes[w], self.sizes[o]
            last = (n_o - 1) // 16 * 16               # the last aligned place inside the other
            before = (n_w - 1) // 16 * 16
            for place in {at, at + last, at - before, at + 16 if n_o > 16 else at}:
                if not (place == at and (w, o) in self.may):
                    yield w, o, place

    def check(self):
        n = 0
        for w, o, place in self.overlapping():
            assert self.call(**{**self.at, w: place}) == INVALID, (w, o, place - self.at[o])
            n += 1
        assert n


def norm_call(dt):
    size = 4 if dt == F32 else 2
    sizes = dict(x=ROWS * C_IN * size, gamma=C_IN * 4, beta=C_IN * 4, y=ROWS * C_IN * size, stats=ROWS * 8)

    def call(x, gamma, beta, y, stats):
        return B.lib().surgeon_layer_norm(x, ROWS, C_IN, dt, gamma, beta, 1e-5, y, stats, None)

    return Call(sizes, ["y", "stats"], call, may=[("y", "x")])


def norm_grad_call(dt, gdt):
    size, gsize = (4 if t == F32 else 2 for t in (dt, gdt))
    need = B.surgeon_layer_norm_grad_workspace(ROWS, C_IN)
    n = ROWS * C_IN
    sizes = dict(x=n * size, dy=n * gsize, gamma=C_IN * 4, stats=ROWS * 8, res=n * gsize, dx=n * gsize, dg=C_IN * 4, db=C_IN * 4, ws=need)

    def call(x, dy, gamma, stats, res, dx, dg, db, ws):
        return B.lib().surgeon_layer_norm_grad(x, dy, ROWS, C_IN, dt, gdt, gamma, stats, res, dx, dg, db, 0, ws, need, None)

    return Call(sizes, ["dx", "dg", "db", "ws"], call, may=[("dx", "dy"), ("dx", "res")])


def linear_call(dt):
    d = B.linear_desc(ROWS, C_IN, C_OUT)
    need, size, n = B.surgeon_linear_workspace(d), 4 if dt == F32 else 2, ROWS * C_OUT
    sizes = dict(x=ROWS * C_IN * 2, w=C_OUT * C_IN * 2, bias=C_OUT * 4, res=n * size, y=n * size, pre=n * 2, ws=need)

    def call(x, w, bias, res, y, pre, ws):
        return B.lib().surgeon_linear(d, x, w, bias, B.SURGEON_ACT_GELU, res, dt, y, pre, ws, need, None)

    return Call(sizes, ["y", "pre", "ws"], call, may=[("y", "res")])


def linear_grad_call(gdt, xdt):
    d = B.linear_desc(ROWS, C_IN, C_OUT)
    need, n = B.surgeon_linear_grad_workspace(d), ROWS * C_OUT
    gsize, xsize = (4 if t == F32 else 2 for t in (gdt, xdt))
    sizes = dict(dy=n * gsize, w=C_OUT * C_IN * 2, pre=n * 2, dx=ROWS * C_IN * xsize, dz=n * 4, db=C_OUT * 4, ws=need)

    def call(dy, w, pre, dx, dz, db, ws):
        return B.lib().surgeon_linear_grad(d, dy, gdt, w, pre, B.SURGEON_ACT_RELU, xdt, dx, dz, db, 0, ws, need, None)

    return Call(sizes, ["dx", "dz", "db", "ws"], call)


@pytest.mark.parametrize("make", [lambda: norm_call(F32), lambda: norm_call(BF16), lambda: norm_grad_call(F32, F32),
                                  lambda: norm_grad_call(BF16, F32), lambda: norm_grad_call(BF16, BF16), lambda: linear_call(F32),
                                  lambda: linear_call(BF16), lambda: linear_grad_call(F32, F32), lambda: linear_grad_call(BF16, BF16),
                                  lambda: linear_grad_call(BF16, F32)],
                         ids=["norm_fp32", "norm_bf16", "norm_grad_fp32", "norm_grad_bf16_fp32", "norm_grad_bf16", "linear_fp32",
                              "linear_bf16", "linear_grad_fp32", "linear_grad_bf16", "linear_grad_bf16_fp32"])
def test_overlaps_are_refused(make):
    make().check()
