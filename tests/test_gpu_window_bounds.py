"""Window calls whose device arrays name more than the call has."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import i32
from window_ref import ALL, Rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,rows,n", [([2600, 1500, 300], [30, 90, 40], 100),
                                         ([2600, 1500, 300], [12, 9, 7], 15),
                                         ([1200], [800], 300), ([40, 700, 30], [20, 30, 25], 20)])
@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_rows_that_are_not_the_calls_are_left_as_they_are(dtype, hq, hkv, hd, lens, rows, n):
    """seq_starts names rows past the call's: they are no sequence's, and the sequences
    before are as they would be alone."""
    r = Rows(dtype, hq, hkv, hd, lens, rows, ALL, 0, seed=24, poison=False, reserve=False)
    whole = [s for s in range(len(rows)) if r.first[s + 1] <= n]
    at = int(r.first[len(whole)])
    coco.coco_window_reserve(r.c.h, n, len(lens), True)
    table, ctx = i32(r.table), i32(lens)
    o = torch.full_like(r.o, 7.0)
    w = r.weights.clone()
    coco.coco_window_attention(r.c.h, 0, r.q[:n], o[:n], r.starts, table, ctx, ALL, 0, w)
    torch.cuda.synchronize()
    assert (o[n:] == 7.0).all()
    assert torch.equal(w[len(whole) + 1:], r.weights[len(whole) + 1:])
    if whole:
        ref, w_ref = torch.full_like(o[:n], 7.0), r.weights.clone()
        starts = np.minimum(r.first, at)
        coco.coco_window_attention(r.c.h, 0, r.q[:n], ref, i32(starts), table, ctx, ALL, 0, w_ref)
        torch.cuda.synchronize()
        assert torch.equal(o[:at], ref[:at]) and torch.equal(w[:len(whole)], w_ref[:len(whole)])


@pytest.mark.parametrize("window,sinks", [(ALL, 0), (ALL, ALL), (ALL - 7, 3), (1, ALL)])
@pytest.mark.parametrize("rows", [[700, 300, 40], [5, 30, 9]])
@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 4, 2, 128), ("f32", 4, 2, 64)])
def test_rows_before_the_context_with_the_widest_windows(dtype, hq, hkv, hd, rows, window, sinks):
    r = Rows(dtype, hq, hkv, hd, [3, 20, 0], rows, window, sinks, seed=25, poison=False)
    r.run()
    r.check()
    assert (r.o[:max(rows[0] - 3, 0)] == 0).all()
