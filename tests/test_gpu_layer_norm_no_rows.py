"""GPU: the backward layer norm of no rows, with the scratch that its query asks for: none."""
import ctypes as C

import pytest
import torch

from paper_2503_20354_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("accumulate", [0, 1])
def test_no_rows_need_no_scratch(accumulate):
    """The scratch that is asked for is of 0 bytes; the sums over no rows are zeros all the same."""
    c = 100
    assert B.surgeon_layer_norm_grad_workspace(0, c) == 0
    dg, db = torch.full((c,), 4.0, device="cuda"), torch.full((c,), 5.0, device="cuda")
    for which in ((dg, db), (dg, None), (None, db)):
        dg.fill_(4.0)
        db.fill_(5.0)
        at = [None if t is None else C.c_void_p(t.data_ptr()) for t in which]
        st = B.lib().surgeon_layer_norm_grad(None, None, 0, c, B.SURGEON_F32, B.SURGEON_F32, None, None, None, None, *at, accumulate, None, 0,
                                             C.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == B.SURGEON_OK
        for t, old in ((dg, 4.0), (db, 5.0)):
            written = any(t is w for w in which)
            assert bool((t == (old if accumulate or not written else 0.0)).all())
