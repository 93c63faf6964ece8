"""Calls of more rows than their sequences have (one graph for several batch
sizes): the rows past the last sequence are left as they are."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, i32, pack_masks, tables
from test_gpu_missing_pages import SHAPES, Layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_validation_takes_rows_past_the_last_sequence(dtype, hq, hkv, hd):
    """Attention and choice with validation on, the padding's arrays arbitrary: as
    the call of the sequences' rows alone. Sequences past the rows are refused."""
    rng = np.random.default_rng(1)
    lens, nodes, more, top = np.array([300, 40, 16]), np.array([3, 20, 2]), 6, 5
    n, width, num_blocks = int(nodes.sum()), 20, 30
    c = Cache(dtype, hq, hkv, hd, num_blocks, width, seed=1)
    table, ctx = i32(tables(rng, lens, width, num_blocks)), i32(lens)
    starts = i32(np.concatenate([[0], np.cumsum(nodes)]))
    q = c.normal(n + more, hq, hd)
    mask = torch.full((n + more, 1), -1, dtype=torch.int64, device="cuda")
    pos = i32(np.concatenate([np.repeat(lens - 1, nodes), [10 ** 9, -7, 3, 2 ** 31 - 1, 0, -1]]))
    summary = torch.zeros(num_blocks, hkv, 2, hd, dtype=torch.int8, device="cuda")
    scales = torch.zeros(num_blocks, hkv, device="cuda")
    coco.coco_tree_reserve(c.h, n + more, 3)
    coco.coco_sparse_reserve(c.h, n + more, top)
    coco.coco_kv_summarize(c.h, 0, summary, scales, None, ctx, table)

    def calls(rows):
        tree, o = (torch.full_like(q[:rows], 7.0) for _ in "to")
        sel = torch.full((rows, hkv, top), 66, dtype=torch.int32, device="cuda")
        coco.coco_tree_attention(c.h, 0, q[:rows], tree, starts, table, ctx, mask[:rows])
        coco.coco_block_select(c.h, summary, scales, q[:rows], pos[:rows], starts, table, ctx, 1, 1,
                               sel)
        coco.coco_sparse_attention(c.h, 0, q[:rows], o, pos[:rows], starts, table, ctx, sel)
        torch.cuda.synchronize()
        return tree, sel, o

    want = calls(n)
    coco.coco_layer_set_validate(c.h, True)
    for got, ref, fill in zip(calls(n + more), want, (7.0, 66, 7.0)):
        assert torch.equal(got[:n], ref) and (got[n:] == fill).all()
    with pytest.raises(coco.CocoError, match="seq_starts"):
        calls(n - 1)


@pytest.mark.parametrize("dtype", sorted(SHAPES))
def test_tree_layers_cache_no_row_of_no_sequence(dtype):
    """Outside the contract of the layer call: the pages of the sequences, the slots
    behind their tokens among them, and their rows are as without such rows."""
    rng = np.random.default_rng(2)
    lens, news, more = np.array([70, 20, 37]), np.array([9, 3, 30]), 7
    width, num_blocks, n = 6, 14, int(news.sum())
    x = Layers(dtype, num_blocks, width)
    table = tables(rng, lens, width, num_blocks)
    ref_hidden, ref_pools = x.run("tree", table, lens, news)
    for layer, was in zip(x.whole, x.start):
        for p, w in zip(layer, was):
            p.copy_(w)
    starts = np.concatenate([[0], np.cumsum(news)])
    seq = np.repeat(np.arange(3), news)
    pos = (lens - news)[seq] + np.arange(n) - starts[seq]
    seen = np.zeros((n + more, 64), bool)
    seen[np.arange(n), np.arange(n) - starts[seq]] = True
    seen[:, 0] = True
    hidden = x.hidden0.clone()
    coco.coco_layer_tree_forward(x.h, 0, 2, hidden, i32(np.arange(n + more)),
                                 i32(np.append(pos, np.arange(more))), i32(starts), i32(table),
                                 i32(lens), pack_masks(seen, 1))
    torch.cuda.synchronize()
    assert torch.equal(hidden[:n], ref_hidden[:n])
    assert torch.equal(hidden[n + more:], x.hidden0[n + more:])
    for got, ref in zip(x.whole, ref_pools):
        assert all(torch.equal(g, r) for g, r in zip(got, ref))


@pytest.mark.parametrize("dtype", sorted(SHAPES))
def test_validation_of_more_hidden_rows_than_host_memory_is_an_error(dtype):
    """hidden_rows that no host could mark as taken: an error code, no abort."""
    x = Layers(dtype, 4, 2)
    coco.coco_layer_set_validate(x.h, True)
    zero, one, starts, table = i32([0]), i32([1]), i32([0, 1]), i32([[2, -1]])
    mask = torch.ones(1, 1, dtype=torch.int64, device="cuda")
    at = [t.data_ptr() for t in (x.hidden0, zero, starts, table, one, mask)]
    hidden, row, ss, bt, ctx, bits = at
    for name, args in (("coco_layer_tree_forward", (0, 1, hidden, 1 << 60, row, 1, row, ss, 1, bt, ctx,
                                                    bits, 1, None)),
                       ("coco_layer_forward", (0, hidden, 1 << 60, row, 1, row, None, 1, bt, ctx,
                                               None))):
        assert coco._lib.raw_call(name, x.h.raw, *args) == coco._lib.COCO_ENOMEM
        assert "host memory" in coco.coco_last_error()
