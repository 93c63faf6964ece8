"""Calls whose block tables lack pages, as after an allocation that a short pool
did not serve: the tokens without a page are not cached, nothing else is touched,
and the other requests of the call come out as without them. The pools lie inside
larger tensors whose blocks on both sides are compared too."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, DT, Cache, i32, pack_masks, tables

pytestmark = pytest.mark.gpu

GUARD = 4  # blocks before and behind a pool


def guarded_pools(dtype, hkv, hd, num_blocks, n_layers, seed):
    """Whole tensors, and the pools inside them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    whole = [tuple(torch.empty(num_blocks + 2 * GUARD, hkv, B * hd, dtype=DT[dtype],
                               device="cuda").normal_(0.0, 1.0, generator=gen) for _ in "kv")
             for _ in range(n_layers)]
    return whole, [tuple(p[GUARD:GUARD + num_blocks] for p in layer) for layer in whole]


def clones(whole):
    return [[p.clone() for p in layer] for layer in whole]


@pytest.mark.parametrize("dtype,hkv,hd", [("bf16", 2, 128), ("f32", 3, 96), ("f32", 1, 128)])
def test_append(dtype, hkv, hd):
    rng = np.random.default_rng(1)
    lens, width, num_blocks = [60, 45, 33, 70, 16], 6, 25
    whole, pools = guarded_pools(dtype, hkv, hd, num_blocks, 1, 1)
    c = Cache(dtype, hkv, hkv, hd, num_blocks, width, pools=pools)
    table = tables(rng, lens, width, num_blocks)
    table[1, 1], table[1, 2], table[3, 0], table[4, 0] = -1, num_blocks, num_blocks + 1, -2
    # Tokens of a request in order (runs of four, over workgroups), and shuffled.
    seq = np.repeat(np.arange(5), lens)
    pos = np.concatenate([np.arange(n) for n in lens])
    for order in (np.arange(len(seq)), rng.permutation(len(seq))):
        s, p = seq[order], pos[order]
        k, v = c.normal(len(s), hkv, hd), c.normal(len(s), hkv, hd)
        want_k, want_v = (x.copy() for x in c.tokens())
        guard = [torch.cat([w[:GUARD], w[-GUARD:]]).clone() for w in whole[0]]
        blk = table[s, p // B]
        ok = (blk >= 0) & (blk < num_blocks)
        want_k[blk[ok], p[ok] % B] = k.cpu().double().numpy()[ok]
        want_v[blk[ok], p[ok] % B] = v.cpu().double().numpy()[ok]
        coco.coco_kv_append(c.h, 0, k, v, i32(s), i32(p), i32(table))
        torch.cuda.synchronize()
        got_k, got_v = c.tokens()
        assert np.array_equal(got_k, want_k) and np.array_equal(got_v, want_v)
        for w, g in zip(whole[0], guard):
            assert torch.equal(torch.cat([w[:GUARD], w[-GUARD:]]), g)


SHAPES = {"bf16": (512, 8, 2, 128, 768), "f32": (260, 4, 2, 64, 684)}  # d, Hq, Hkv, hd, F


class Layers:
    """Two layers of random weights over guarded pools."""

    def __init__(self, dtype, num_blocks, width, max_rows=128):
        d, hq, hkv, hd, f = SHAPES[dtype]
        self.dtype, self.num_blocks, self.hkv, self.hd = dtype, num_blocks, hkv, hd
        self.whole, pools = guarded_pools(dtype, hkv, hd, num_blocks, 2, 3)
        gen = torch.Generator(device="cuda").manual_seed(4)
        shapes = {"w_qkv": ((hq + 2 * hkv) * hd, d), "w_o": (d, hq * hd), "w_gate_up": (2 * f, d),
                  "w_down": (d, f), "gamma_attn": (d,), "gamma_mlp": (d,)}
        layers = [dict({n: torch.empty(s, dtype=DT[dtype], device="cuda").normal_(
            0.0, 0.1, generator=gen) for n, s in shapes.items()}, k_cache=k, v_cache=v)
            for k, v in pools]
        self.h = coco.coco_layer_init(
            coco.make_config(d, hq, hkv, hd, f, 2, dtype, max_rows, 8, width, 1e4, 1e-5), layers)
        self.hidden0 = torch.empty(max_rows, d, dtype=DT[dtype], device="cuda").normal_(
            0.0, 1.0, generator=gen)
        self.start = clones(self.whole)
        coco.coco_tree_reserve(self.h, max_rows, 8)
        coco.coco_sparse_reserve(self.h, max_rows, 3)

    def run(self, kind, table, lens, news):
        """The call from the initial pools; hidden rows and pools after it."""
        for layer, was in zip(self.whole, self.start):
            for p, w in zip(layer, was):
                p.copy_(w)
        hidden, n = self.hidden0.clone(), int(news.sum())
        starts = np.concatenate([[0], np.cumsum(news)])
        seq = np.repeat(np.arange(len(news)), news)
        pos = (lens - news)[seq] + np.arange(n) - starts[seq]
        rows, pos, table, ctx = i32(np.arange(n)), i32(pos), i32(table), i32(lens)
        if kind in ("decode", "prefill"):
            coco.coco_layer_span_forward(self.h, 0, 2, hidden, rows, pos,
                                         None if kind == "decode" else i32(starts), table, ctx)
        elif kind == "tree":
            seen = np.zeros((n, 64), bool)
            seen[np.arange(n), np.arange(n) - starts[seq]] = True
            seen[:, 0] = True
            coco.coco_layer_tree_forward(self.h, 0, 2, hidden, rows, pos, i32(starts), table, ctx,
                                         pack_masks(seen, 1))
        else:
            summary = torch.zeros(self.num_blocks, self.hkv, 2, self.hd, dtype=torch.int8,
                                  device="cuda")
            scales = torch.zeros(self.num_blocks, self.hkv, device="cuda")
            selected = torch.zeros(n, self.hkv, 3, dtype=torch.int32, device="cuda")
            for layer in (0, 1):
                coco.coco_kv_summarize(self.h, layer, summary, scales, None, i32(lens - 1), table)
                coco.coco_layer_sparse_forward(self.h, layer, hidden, rows, pos, table, ctx, summary,
                                               scales, 1, 1, selected)
        torch.cuda.synchronize()
        return hidden, clones(self.whole)


@pytest.mark.parametrize("dtype", sorted(SHAPES))
@pytest.mark.parametrize("kind", ["decode", "prefill", "tree", "sparse"])
def test_layers_write_nothing_without_a_page(kind, dtype):
    """Request 1 did not get its last page, 2 has one id past the pool, 4 has
    none at all; 0, 3 and 5 are served."""
    rng = np.random.default_rng(2)
    lens = np.array([70, 49, 33, 20, 9, 97])
    news = np.ones(6, np.int64) if kind in ("decode", "sparse") else np.array([9, 20, 6, 1, 9, 30])
    width, num_blocks = 8, 26
    x = Layers(dtype, num_blocks, width)
    full = tables(rng, lens, width, num_blocks)
    short = full.copy()
    short[1, 3], short[2, 2], short[4, 0] = -1, num_blocks + 1, -1
    ref_hidden, ref_pools = x.run(kind, full, lens, news)
    hidden, pools = x.run(kind, short, lens, news)
    starts = np.concatenate([[0], np.cumsum(news)])
    for s in (0, 3, 5):
        rows = slice(int(starts[s]), int(starts[s + 1]))
        assert torch.equal(hidden[rows], ref_hidden[rows]), s
    assert torch.equal(hidden[int(starts[-1]):], x.hidden0[int(starts[-1]):])
    # Layer 0's keys and values depend on the call's rows alone; the unserved
    # requests' in layer 1 on what they attended: there, their blocks are left out.
    for layer in (0, 1):
        loose = [] if layer == 0 else [b for s in (1, 2, 4) for b in short[s] if 0 <= b < num_blocks]
        for got, ref, was in zip(pools[layer], ref_pools[layer], x.start[layer]):
            want = was.clone()
            for s in range(6):
                for b in short[s]:
                    if 0 <= b < num_blocks:
                        want[GUARD + b] = ref[GUARD + b]
            keep = [i for i in range(len(want)) if i - GUARD not in loose]
            assert torch.equal(got[keep], want[keep]), layer


@pytest.mark.parametrize("dtype", sorted(SHAPES))
def test_a_step_after_a_short_allocation(dtype):
    """Pages from a pool too small for all, then the drafts' layers, all on the
    device: the served requests' bits are those of a pool with room."""
    rng = np.random.default_rng(5)
    lens, news = np.array([30, 64, 17, 5]), np.array([15, 10, 20, 4])
    width, num_blocks = 8, 14
    x = Layers(dtype, num_blocks, width)
    table = tables(rng, lens, width, num_blocks)
    held = np.zeros(num_blocks, np.int64)
    held[table[table >= 0]] = 1
    free = np.nonzero(held == 0)[0]
    held[free[2:]] = 1  # two left, for requests 0 and 1
    dt, dr, status = i32(table), i32(held), i32(np.zeros(4))
    coco.coco_kv_alloc(x.h, i32(np.arange(4)), i32(lens + news), dt, dr, status)
    assert status.cpu().tolist() == [1, 1, 0, 1]  # (3 needs no more than it has)
    table = dt.cpu().numpy().astype(np.int64)
    hidden, pools = x.run("tree", table, lens + news, news)
    assert table[2, 1] >= 0 and table[2, 2] < 0
    full = table.copy()
    spare = Layers(dtype, num_blocks + 1, width)  # request 2's page is one more block
    full[2, 2] = num_blocks
    spare.hidden0 = x.hidden0
    for layer, was in zip(spare.start, x.start):
        for p, w in zip(layer, was):
            p[:GUARD + num_blocks] = w[:GUARD + num_blocks]
    ref_hidden, ref_pools = spare.run("tree", full, lens + news, news)
    starts = np.concatenate([[0], np.cumsum(news)])
    for s in (0, 1, 3):
        rows = slice(int(starts[s]), int(starts[s + 1]))
        assert torch.equal(hidden[rows], ref_hidden[rows]), s
        for layer in (0, 1):
            for got, ref in zip(pools[layer], ref_pools[layer]):
                blocks = [GUARD + b for b in table[s] if b >= 0]
                assert torch.equal(got[blocks], ref[blocks]), (s, layer)
    for layer in (0, 1):
        for got, was in zip(pools[layer], x.start[layer]):
            rest = sorted(set(range(len(got))) - {GUARD + b for b in table[table >= 0]})
            assert torch.equal(got[rest], was[rest])


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64),
                                             ("f32", 3, 1, 160)])
def test_attention_reads_inside_the_pool(dtype, hq, hkv, hd):
    """With NaN on both sides of the pools, every row of the call is finite, and
    the served requests' rows are as with all pages."""
    rng = np.random.default_rng(6)
    lens, nodes = np.array([70, 900, 33, 20, 9]), np.array([5, 9, 3, 20, 9])
    width, num_blocks = 60, 80
    whole, pools = guarded_pools(dtype, hkv, hd, num_blocks, 1, 6)
    for w in whole[0]:
        w[:GUARD], w[-GUARD:] = float("nan"), float("nan")
    c = Cache(dtype, hq, hkv, hd, num_blocks, width, pools=pools)
    full = tables(rng, lens, width, num_blocks)
    short = full.copy()
    short[1, [3, 40, 56]], short[2, 2], short[4, 0] = -1, num_blocks + 2, -GUARD
    rows = int(nodes.sum())
    starts, ctx = i32(np.concatenate([[0], np.cumsum(nodes)])), i32(lens)
    q, out = c.normal(rows, hq, hd), [torch.empty(rows, hq, hd, dtype=DT[dtype], device="cuda")
                                      for _ in range(2)]
    mask = torch.full((rows, 1), -1, dtype=torch.int64, device="cuda")
    coco.coco_tree_reserve(c.h, rows, 5)
    coco.coco_sparse_reserve(c.h, rows, 60)
    selected = i32(np.broadcast_to(np.arange(60), (rows, hkv, 60)))
    positions = i32(np.repeat(lens - 1, nodes))

    def tree(table, o):
        coco.coco_tree_attention(c.h, 0, q, o, starts, i32(table), ctx, mask)

    def sparse(table, o):
        coco.coco_sparse_attention(c.h, 0, q, o, positions, starts, i32(table), ctx, selected)

    served = np.isin(np.repeat(np.arange(5), nodes), [0, 3])
    for call in (tree, sparse):
        for table, o in zip((full, short), out):
            call(table, o)
        torch.cuda.synchronize()
        assert torch.isfinite(out[1]).all()
        assert torch.equal(out[0][served], out[1][served])


@pytest.mark.parametrize("dtype", sorted(SHAPES))
@pytest.mark.parametrize("kind", ["decode", "prefill", "tree", "sparse"])
def test_layers_read_inside_the_pool(kind, dtype):
    rng = np.random.default_rng(7)
    lens = np.array([70, 49, 33, 20, 9, 97])
    news = np.ones(6, np.int64) if kind in ("decode", "sparse") else np.array([9, 20, 6, 1, 9, 30])
    width, num_blocks = 8, 26
    x = Layers(dtype, num_blocks, width)
    for layer in x.start:
        for p in layer:
            p[:GUARD], p[-GUARD:] = float("nan"), float("nan")
    table = tables(rng, lens, width, num_blocks)
    table[1, 3], table[1, 0], table[2, 2], table[4, 0] = -1, -2, num_blocks + 1, -1
    hidden, _ = x.run(kind, table, lens, news)
    assert torch.isfinite(hidden).all()
