"""The cache operators one after another, as a serving step uses them: pages
for drafts, append, tree attention, the accepted path moved up, the rest let go,
a fork, and attention over selected blocks of the result."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, attend, i32, pack_masks, tables, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 6, 2, 96)])
def test_speculative_step_then_fork_then_sparse_decode(dtype, hq, hkv, hd):
    rng = np.random.default_rng(1)
    prior, nodes = np.array([31, 0, 160, 500]), np.array([9, 4, 20, 1])
    n_seqs, width, num_blocks, layers = 4, 40, 90, 2
    c = Cache(dtype, hq, hkv, hd, num_blocks, width, n_layers=layers, seed=1)
    table = tables(rng, list(prior) + [0, 0], width, num_blocks)
    refs = np.zeros(num_blocks, np.int64)
    np.add.at(refs, table[table >= 0], 1)
    dt, dr = i32(table), i32(refs)
    rows = np.arange(n_seqs)
    status = i32(np.zeros(n_seqs))
    # Pages, and the drafts' keys and values.
    coco.coco_kv_alloc(c.h, i32(rows), i32(prior + nodes), dt, dr, status)
    seq = np.repeat(rows, nodes)
    starts = np.concatenate([[0], np.cumsum(nodes)])
    pos = prior[seq] + np.arange(len(seq)) - starts[seq]
    kv = [[c.normal(len(seq), hkv, hd) for _ in "kv"] for _ in range(layers)]
    for layer in range(layers):
        coco.coco_kv_append(c.h, layer, *kv[layer], i32(seq), i32(pos), dt)
    # Trees: node j's parent is j // 2 - 1 or so; the accepted path of each.
    seen = []
    for n in nodes:
        m = np.zeros((n, 64), bool)
        for j in range(n):
            if j:
                m[j] = m[(j - 1) // 2]
            m[j, j] = True
        seen.append(m)
    q, o = c.normal(len(seq), hq, hd, sigma=1.5), c.normal(len(seq), hq, hd)
    coco.coco_tree_reserve(c.h, len(seq), n_seqs)
    coco.coco_tree_attention(c.h, 1, q, o, i32(starts), dt, i32(prior + nodes),
                             pack_masks(np.concatenate(seen), 1))
    torch.cuda.synchronize()
    assert status.cpu().tolist() == [1] * n_seqs
    table, refs = dt.cpu().numpy().astype(np.int64), dr.cpu().numpy()
    assert np.array_equal(refs, np.bincount(table[table >= 0], minlength=num_blocks))
    k, v = c.tokens(1)

    def check(got, qrow, tab, n, mask):
        at = np.arange(n)
        blk = tab[at // B]
        ro, mean, size = attend(qrow, k[blk, at % B], v[blk, at % B], mask, hkv)
        tol = tolerance(dtype, ro, mean, size, n, hd)
        assert (np.abs(got - ro) <= tol).all()

    q64, o64 = q.cpu().double().numpy(), o.cpu().double().numpy()
    for s in rows:
        for j in range(nodes[s]):
            mask = np.concatenate([np.ones(prior[s], bool), seen[s][j, :nodes[s]]])
            check(o64[starts[s] + j], q64[starts[s] + j], table[s], len(mask), mask[None])
    # The last node's path is accepted, moved up, the other blocks let go.
    paths = [np.nonzero(m[-1, :n])[0] for m, n in zip(seen, nodes)]
    base, acc = prior, np.array([len(p) for p in paths])
    kept_starts = np.concatenate([[0], np.cumsum(acc)])
    coco.coco_kv_compact(c.h, 0, layers, i32(rows), i32(base),
                         i32(np.concatenate([b + p for b, p in zip(base, paths)])),
                         i32(kept_starts), dt)
    now = base + acc
    coco.coco_kv_free(c.h, i32(rows), i32(now), dt, dr)
    # A fork of the longest one, two tokens back, and of a whole one.
    cut = np.array([int(now[3]) - 2, int(now[0])])
    coco.coco_kv_fork(c.h, 0, layers, i32([3, 0]), i32([4, 5]), i32(cut), dt, dr, status[:2])
    torch.cuda.synchronize()
    table = dt.cpu().numpy().astype(np.int64)
    assert status[:2].cpu().tolist() == [1, 1]
    for layer in range(layers):
        k, v = c.tokens(layer)
        for s in rows:
            for i, j in enumerate(paths[s]):
                at = base[s] + i
                for got, x in ((k, kv[layer][0]), (v, kv[layer][1])):
                    assert np.array_equal(got[table[s, at // B], at % B],
                                          x[starts[s] + j].cpu().double().numpy())
        for child, parent, n in ((4, 3, cut[0]), (5, 0, cut[1])):
            at = np.arange(n)
            for x in (k, v):
                assert np.array_equal(x[table[child, at // B], at % B],
                                      x[table[parent, at // B], at % B])
    # Sparse decode of all six, layer 1: with room for every block it is dense.
    lens = np.concatenate([now, cut])
    q, o = c.normal(6, hq, hd, sigma=1.5), c.normal(6, hq, hd)
    summary = torch.zeros(num_blocks, hkv, 2, hd, dtype=torch.int8, device="cuda")
    scales = torch.zeros(num_blocks, hkv, device="cuda")
    coco.coco_kv_summarize(c.h, 1, summary, scales, None, i32(lens), dt)
    q64 = q.cpu().double().numpy()
    for top in (40, 6):
        coco.coco_sparse_reserve(c.h, 6, top)
        sel = torch.empty(6, hkv, top, dtype=torch.int32, device="cuda")
        args = (i32(lens - 1), None, dt, i32(lens))
        coco.coco_block_select(c.h, summary, scales, q, *args, 1, 1, sel)
        coco.coco_sparse_attention(c.h, 1, q, o, *args, sel)
        got, chosen = o.cpu().double().numpy(), sel.cpu().numpy()
        for s, n in enumerate(lens):
            mask = np.stack([np.isin(np.arange(n) // B, chosen[s, g]) for g in range(hkv)])
            assert mask.all() == (top * B >= n)
            check(got[s], q64[s], table[s], n, mask)
