"""Attention over long contexts, where an average over random values would hide a
lost block: every key is counted."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, i32, offsets, pack_masks, tables

pytestmark = pytest.mark.gpu


class Counted:
    """Queries of zero, so that all keys weigh the same, and values that count: in
    pass `slot` the key in that slot of a sequence's block b has a 1 in dimension
    b % hd, all else is 0. A row's sums are whole numbers below 2^24, exact in every
    order; its result is off by the division and one rounding to its type (four
    and one fp32 half steps, and a half step of bf16). A key that is lost or
    counted twice moves its dimension by a part in (blocks / hd + 1): over 40000
    keys 1/20, ten times the tolerance."""

    def __init__(self, dtype, hq, hkv, hd, lens, rows):
        rng = np.random.default_rng(31)
        self.lens, self.hd = np.asarray(lens), hd
        blocks = -(-self.lens // B)
        self.c = Cache(dtype, hq, hkv, hd, int(blocks.sum()) + 3, int(blocks.max()), seed=31)
        self.table = tables(rng, lens, int(blocks.max()), self.c.num_blocks)
        self.q = torch.zeros(rows, hq, hd, dtype=self.c.pools[0][0].dtype, device="cuda")
        self.o = torch.empty_like(self.q)
        s = np.repeat(np.arange(len(lens)), blocks)
        b = np.concatenate([np.arange(n) for n in blocks])
        self.phys, self.dim = (torch.from_numpy(x).cuda() for x in (self.table[s, b], b % hd))
        self.vo = torch.from_numpy(offsets(hd)[1]).cuda()

    def fill(self, slot):
        v = self.c.pools[0][1].zero_()
        v[self.phys, :, self.vo[slot, self.dim]] = 1

    def check(self, slot, row, keys):
        at = np.arange(slot, keys, B) // B % self.hd
        want = np.bincount(at, minlength=self.hd) / keys
        step = 5 * 2.0 ** -24 + (2.0 ** -8 if self.c.dtype == "bf16" else 0.0)
        off = np.abs(self.got[row] - want[None])
        assert (off <= want * step).all(), (slot, row, keys, (off - want * step).max())


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 1, 128), ("f32", 2, 1, 32)])
def test_every_key_of_long_contexts_counts_once(dtype, hq, hkv, hd):
    """Trees of 1, 7 and 30 nodes (few columns, and a part rule each side of 128)."""
    trees = [(40000, 7), (20011, 30), (33000, 1), (3, 2), (16391, 2)]
    nodes = [n for _, n in trees]
    x = Counted(dtype, hq, hkv, hd, [p + n for p, n in trees], sum(nodes))
    starts = np.concatenate([[0], np.cumsum(nodes)])
    seen = np.zeros((sum(nodes), 64), bool)
    for s, n in enumerate(nodes):
        seen[starts[s]:starts[s + 1], :n] = np.tri(n, dtype=bool)
    args = [i32(starts), i32(x.table), i32(x.lens), pack_masks(seen, 1)]
    coco.coco_tree_reserve(x.c.h, sum(nodes), len(trees))
    for slot in range(B):
        x.fill(slot)
        coco.coco_tree_attention(x.c.h, 0, x.q, x.o, *args)
        x.got = x.o.cpu().double().numpy()
        for s, (prefix, n) in enumerate(trees):
            for j in range(n):
                x.check(slot, starts[s] + j, prefix + j + 1)


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 1, 128), ("f32", 2, 1, 32)])
def test_every_key_of_long_lists_counts_once(dtype, hq, hkv, hd):
    lens = [40000, 20011, 17, 8200]
    x = Counted(dtype, hq, hkv, hd, lens, len(lens))
    top = x.table.shape[1]
    rng = np.random.default_rng(32)
    sel = np.stack([rng.permutation(np.where(np.arange(top) < -(-n // B), np.arange(top), -1))
                    for n in lens])
    coco.coco_sparse_reserve(x.c.h, len(lens), top)
    args = [i32(x.lens - 1), None, i32(x.table), i32(x.lens),
            i32(np.broadcast_to(sel[:, None], (len(lens), hkv, top)))]
    for slot in range(B):
        x.fill(slot)
        coco.coco_sparse_attention(x.c.h, 0, x.q, x.o, *args)
        x.got = x.o.cpu().double().numpy()
        for s, n in enumerate(lens):
            x.check(slot, s, n)
