"""Validation mode reads no array past its end where the starts of its parts are not in
order."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import Cache, i32, tables
from harness import Replica, ragged_prefill_batch, small_bf16_shape
from workloads import device as WD

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("starts", [[0, 9, 3], [0, 2 ** 30, 3], [0, -5, 3], [0, 3, 2]])
def test_compaction_names_starts_out_of_order(starts):
    c = Cache("f32", 2, 1, 32, 8, 4, max_seqs=2)
    table = i32(tables(np.random.default_rng(0), [40, 20], 4, 8))
    coco.coco_layer_set_validate(c.h, True)
    before = [p.clone() for p in c.pools[0]]
    with pytest.raises(coco.CocoError, match="kept_starts not monotone"):
        coco.coco_kv_compact(c.h, 0, 1, i32([0, 1]), i32([0, 0]), i32([1, 2, 3]), i32(starts), table)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(before, c.pools[0]))


@pytest.mark.parametrize("starts", [[0, 90, 12], [0, 2 ** 30, 12], [0, -3, 12]])
def test_layers_name_starts_out_of_order(starts):
    b = ragged_prefill_batch(31, [20, 3], [5, 7], 64)
    rep = Replica.for_batch(small_bf16_shape(), "vs", 1, b)
    hidden = WD.hidden_tensor(rep.shape, "vs", b.hidden_rows)
    before = hidden.clone()
    coco.coco_layer_set_validate(rep.h, True)
    with pytest.raises(coco.CocoError, match="seq_starts not monotone"):
        rep.forward(0, hidden, dict(WD.batch_tensors(b), seq_starts=i32(starts)))
    torch.cuda.synchronize()
    assert torch.equal(hidden, before)
