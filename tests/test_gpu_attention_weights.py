"""The weights of sparse attention, and of trees of few columns, where their
differences are the result."""
import math

import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("bf16", 16, 1, 128),
                                             ("f32", 4, 2, 64)])
@pytest.mark.parametrize("keys", [2, 200, 600])
@pytest.mark.parametrize("tree", [False, True])
def test_opposite_values(dtype, hq, hkv, hd, keys, tree):
    """Values +1 and -1 in turn: a row's result is the difference of two halves of
    the weights. A score is off by at most (hd + 4) fp32 half steps of the sum of its
    terms' sizes, a weight by twice that, four half steps of its exponential and, in
    bf16 handles, 2^-16 (two parts of 8 bits: the second's half step of what the
    first's leaves), the sums by keys + 32 half steps, the result by its rounding.
    Weights rounded to bf16 once fail it where there are two keys (of N such errors
    1 / sqrt(N) is left)."""
    rng = np.random.default_rng(keys)
    rows, nb = 24, -(-keys // B)
    c = Cache(dtype, hq, hkv, hd, rows * nb, nb, max_rows=rows, max_seqs=rows, seed=keys)
    table = rng.permutation(rows * nb).reshape(rows, nb)
    _, v = c.tokens()
    v[:] = np.where(np.arange(B) % 2 == 0, 1.0, -1.0)[None, :, None, None]
    k, _ = c.tokens()
    c.put(0, k, v)
    q = c.normal(rows, hq, hd, sigma=0.7)
    o = torch.empty_like(q)
    ctx = i32(np.full(rows, keys))
    if tree:  # one node of its own each
        coco.coco_tree_reserve(c.h, rows, rows)
        coco.coco_tree_attention(c.h, 0, q, o, i32(np.arange(rows + 1)), i32(table), ctx,
                                 torch.ones(rows, 1, dtype=torch.int64, device="cuda"))
    else:
        sel = i32(np.broadcast_to(np.arange(nb), (rows, hkv, nb)))
        coco.coco_sparse_reserve(c.h, rows, nb)
        coco.coco_sparse_attention(c.h, 0, q, o, ctx - 1, None, i32(table), ctx, sel)
    got, q = o.cpu().double().numpy(), q.cpu().double().numpy()
    f, worst = 2.0 ** -24, 0.0
    for r in range(rows):
        at = np.arange(keys)
        kk = k[table[r, at // B], at % B]
        for h in range(hq):
            kh = kk[:, h // (hq // hkv)]
            z = kh @ q[r, h] / math.sqrt(hd)
            size = (np.abs(kh) @ np.abs(q[r, h])).max() / math.sqrt(hd)
            p = np.exp(z - z.max())
            want = (p / p.sum()) @ np.where(at % 2 == 0, 1.0, -1.0)
            w = 2 * (hd + 4) * f * size + 4 * f + (2.0 ** -16 if dtype == "bf16" else 0.0)
            tol = (2 * w + 2 * (keys + 32) * f) * 1.01 + abs(want) * (2.0 ** -8 if dtype == "bf16" else f)
            off = np.abs(got[r, h] - want).max()
            assert off <= tol, (r, h, want, off / tol)
            if dtype == "bf16":  # the weights rounded once, by the formula
                cut = torch.from_numpy(p).bfloat16().double().numpy()
                once = (cut / p.sum()) @ np.where(at % 2 == 0, 1.0, -1.0)
                worst = max(worst, abs(once - want) / tol)
    assert dtype != "bf16" or keys > 2 or worst > 2


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("bf16", 16, 1, 128),
                                             ("f32", 4, 2, 64)])
@pytest.mark.parametrize("tree", [False, True])
def test_infinite_values_come_out(dtype, hq, hkv, hd, tree):
    """A seen value that is infinite is the result in its sign, whatever the key's
    weight (also the largest, an exact power of two); NaN is NaN; the other
    dimensions, and keys that a row does not see, are as without."""
    rng = np.random.default_rng(51)
    lens = [40, 700, 16, 33, 1100]
    nb = [-(-n // B) for n in lens]
    c = Cache(dtype, hq, hkv, hd, sum(nb) + 1, max(nb), max_rows=5, max_seqs=5, seed=51)
    at = np.concatenate([[0], np.cumsum(nb)])
    perm = rng.permutation(sum(nb) + 1)
    table = np.full((5, max(nb)), -1, np.int64)
    for s in range(5):
        table[s, :nb[s]] = perm[at[s]:at[s + 1]]
    k, v = c.tokens()
    q = c.normal(5, hq, hd)
    ctx = i32(lens)
    if tree:
        coco.coco_tree_reserve(c.h, 5, 5)
    else:
        sel = np.full((5, hkv, max(nb)), -1)
        for s in range(5):
            sel[s, :, :nb[s]] = np.arange(nb[s])
        coco.coco_sparse_reserve(c.h, 5, max(nb))

    def run(values):
        c.put(0, k, values)
        o = torch.empty_like(q)
        if tree:
            coco.coco_tree_attention(c.h, 0, q, o, i32(np.arange(6)), i32(table), ctx,
                                     torch.ones(5, 1, dtype=torch.int64, device="cuda"))
        else:
            coco.coco_sparse_attention(c.h, 0, q, o, ctx - 1, None, i32(table), ctx, i32(sel))
        return o.cpu().double().numpy()

    clean = run(v)
    q64 = q.cpu().double().numpy()
    bad, want = v.copy(), {}
    for s, n in enumerate(lens):
        first = k[table[s, np.arange(n) // B], np.arange(n) % B]
        top = int((first[:, 0] @ q64[s, 0]).argmax())  # the largest weight of head 0
        for dim, t, x in ((3, top, np.inf), (4, 0, -np.inf), (5, n - 1, np.inf), (6, n // 2, np.nan),
                          (7, top, -np.inf), (17, min(15, n - 1), np.inf), (30, n - 1, -np.inf)):
            bad[table[s, t // B], t % B, :, dim] = x
            want[s, dim] = x
        if n % B:  # a slot behind the row's keys
            bad[table[s, n // B], n % B] = np.inf
    got = run(bad)
    for (s, dim), x in want.items():
        g = got[s, :, dim]
        assert (np.isnan(g) if x != x else g == x).all(), (s, dim, x, g)
    odd = np.zeros(got.shape, bool)
    for s, dim in want:
        odd[s, :, dim] = True
    assert np.array_equal(got[~odd], clean[~odd])
