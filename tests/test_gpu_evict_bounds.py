"""An eviction that names a row twice, which no call may: nothing but that row and the
call's lists is written."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("budgets", [[900, 100, 400, 30], [2000, 1, 2000, 64], [300, 300, 300, 300]])
@pytest.mark.parametrize("length", [1000, 6000])
def test_a_row_that_is_named_twice(length, budgets):
    width = 400
    c = Cache("f32", 2, 1, 32, 8, width, max_seqs=4, max_rows=4)
    rng = np.random.default_rng(length)
    w = torch.from_numpy(rng.exponential(size=(4, width * B)).astype(np.float32)).cuda()
    before = w.clone()
    rows = [1, 1, 1, 3]
    lens = [50, length, 60, length]
    n_kept = sum(budgets)
    kept = i32(np.full(n_kept + 4096, -9))
    new, base, starts = i32(np.full(4, -9)), i32(np.full(4, -9)), i32(np.full(5, -9))
    coco.coco_kv_evict(c.h, i32(rows), i32(budgets), 2, 9, i32(lens), w, new, base, kept[:n_kept],
                       starts)
    torch.cuda.synchronize()
    at, kept = starts.cpu().numpy(), kept.cpu().numpy()
    assert at[0] == 0 and (np.diff(at) >= 0).all() and at[-1] <= n_kept
    assert (kept[at[-1]:] == -9).all()
    assert torch.equal(w[[0, 2]], before[[0, 2]])
    assert torch.equal(w[:, length:], before[:, length:])
    # The row that is named once is as it would be alone.
    alone = [i32(np.full(m, -9)) for m in (1, 1, n_kept, 2)]
    w1 = before.clone()
    coco.coco_kv_evict(c.h, i32([3]), i32(budgets[3:]), 2, 9, i32(lens), w1, *alone)
    torch.cuda.synchronize()
    count = int(alone[3][1])
    assert torch.equal(w[3], w1[3]) and new[3] == alone[0][0] and base[3] == alone[1][0]
    assert at[4] - at[3] == count and (kept[at[3]:at[4]] == alone[2][:count].cpu().numpy()).all()
