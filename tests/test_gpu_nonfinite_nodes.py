"""Trees with non-finite values in single dimensions of single nodes: those come out
in the rows that see them, every other dimension and row as without."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, attend, i32, pack_masks, tables, tolerance

pytestmark = pytest.mark.gpu

# One part and several, few columns and many, prefixes that end inside a stage.
TREES = [(3000, 9), (21, 20), (700, 40), (1045, 1), (5003, 3), (0, 4), (33000, 2)]


class Case:
    def __init__(self, dtype, hq, hkv, hd):
        rng = np.random.default_rng(41)
        self.lens = [p + n for p, n in TREES]
        blocks = sum(-(-n // B) for n in self.lens)
        self.c = Cache(dtype, hq, hkv, hd, blocks + 1, -(-max(self.lens) // B), seed=41)
        self.table = tables(rng, self.lens, self.c.max_blocks, blocks + 1)
        self.starts = np.concatenate([[0], np.cumsum([n for _, n in TREES])])
        rows = int(self.starts[-1])
        self.seen = [np.tri(n, dtype=bool) & (rng.random((n, n)) < 0.7) | np.eye(n, dtype=bool)
                     for _, n in TREES]
        bits = np.zeros((rows, 64), bool)
        for s, m in enumerate(self.seen):
            bits[self.starts[s]:self.starts[s + 1], :len(m)] = m
        self.q = self.c.normal(rows, hq, hd)
        self.q[:, :, 0] = 1.0
        self.k, self.v = self.c.tokens()
        self.args = [i32(self.starts), i32(self.table), i32(self.lens), pack_masks(bits, 1)]
        coco.coco_tree_reserve(self.c.h, rows, len(TREES))

    def at(self, s, t):
        return self.table[s, t // B], t % B

    def run(self):
        self.c.put(0, self.k, self.v)
        o = torch.full_like(self.q, 7.0)
        coco.coco_tree_attention(self.c.h, 0, self.q, o, *self.args)
        torch.cuda.synchronize()
        return o.cpu().double().numpy()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("bf16", 16, 1, 128),
                                             ("f32", 4, 2, 64)])
def test_single_dimensions(dtype, hq, hkv, hd):
    x = Case(dtype, hq, hkv, hd)
    rng = np.random.default_rng(42)
    want_odd = {}  # (row, dim) -> value
    for s, (prefix, n) in enumerate(TREES):
        for j in range(0, n, 3):
            for dim, value in ((5 + j % 7, np.inf), (20 + j % 3, rng.choice([np.inf, -np.inf])),
                               (31, np.nan)):
                x.v[x.at(s, prefix + j) + (slice(None), dim)] = value
                for i in np.nonzero(x.seen[s][:, j])[0]:
                    key = (int(x.starts[s] + i), dim)
                    want_odd[key] = want_odd.get(key, 0.0) + float(value)  # (inf - inf: NaN)
    # A key of score -inf: its weight is 0, and 0 times an infinite value NaN.
    s, j = 2, 7
    x.k[x.at(s, TREES[s][0] + j) + (slice(None), 0)] = -np.inf
    x.v[x.at(s, TREES[s][0] + j) + (slice(None), 30)] = np.inf
    for i in np.nonzero(x.seen[s][:, j])[0]:
        want_odd[int(x.starts[s] + i), 30] = np.nan
    got = x.run()
    assert np.array_equal(got, x.run(), equal_nan=True)  # (the flags are as they were found)
    q = x.q.cpu().double().numpy()
    odd = np.zeros(got.shape, bool)
    for (row, dim), value in want_odd.items():
        odd[row, :, dim] = True
        g = got[row, :, dim]
        assert (np.isnan(g) if np.isnan(value) else g == value).all(), (row, dim, value)
    for s, (prefix, n) in enumerate(TREES):
        at = np.arange(prefix + n)
        k, v = x.k[x.table[s, at // B], at % B], x.v[x.table[s, at // B], at % B]
        weightless = np.isneginf(k).any((1, 2))  # (its score is -inf for every head: q[0] > 0)
        k, v = np.where(np.isfinite(k), k, 0.0), np.where(np.isfinite(v), v, 0.0)
        for i in range(n):
            row = int(x.starts[s] + i)
            seen = np.concatenate([np.ones(prefix, bool), x.seen[s][i]]) & ~weightless
            o, mean, size = attend(q[row], k, v, seen[None], hkv)
            tol = tolerance(dtype, o, mean, size, len(at), hd)
            fine = ~odd[row]
            assert (np.abs(got[row] - o)[fine] <= tol[fine]).all(), (s, i)
    # Without them: the rows and dimensions that saw none have the same bits.
    x.v = np.where(np.isfinite(x.v), x.v, 0.0)
    clean = x.run()
    assert np.array_equal(clean[~odd], got[~odd]) and np.isfinite(clean).all()
