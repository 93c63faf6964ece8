"""Attention for trees of drafted tokens, against the 64-bit definition."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, attend, i32, pack_masks, tables, tolerance

pytestmark = pytest.mark.gpu


def path_masks(rng, n, words, spread=4):
    """Ancestors and self of a random tree's nodes."""
    seen = np.zeros((n, 64 * words), bool)
    for j in range(n):
        parent = j - int(rng.integers(1, spread + 1))
        if parent >= 0:
            seen[j] = seen[parent]
        seen[j, j] = True
    return seen


class Call:
    """Trees of (prefix, nodes) over one cache; masks as wide as `words`."""

    def __init__(self, dtype, hq, hkv, hd, trees, words=None, seed=0, masks=path_masks,
                 num_blocks=None, spoil=True):
        rng = np.random.default_rng(seed)
        self.trees = trees
        lens = [p + n for p, n in trees]
        used = sum(-(-x // B) for x in lens)
        width = max(1, -(-max(lens) // B) + 2)
        self.starts = np.concatenate([[0], np.cumsum([n for _, n in trees])]).astype(np.int64)
        rows = int(self.starts[-1])
        self.c = Cache(dtype, hq, hkv, hd, num_blocks or used + 3, width, seed=seed,
                       max_seqs=max(len(trees), 1))
        self.table = tables(rng, lens, width, self.c.num_blocks)
        self.words = words or max(1, -(-max(n for _, n in trees) // 64))
        self.seen = [masks(rng, n, self.words) for _, n in trees]
        # Bits from a tree's size on are ignored.
        noise = [s | ((np.arange(64 * self.words) >= len(s))[None] &
                      (rng.random(s.shape) < 0.5)) for s in self.seen]
        if spoil:  # slots past the tokens, and free blocks, hold anything
            k, v = self.c.tokens()
            for i, (a, x) in enumerate(((k, np.nan), (v, np.inf))):
                held = np.zeros((self.c.num_blocks, B), bool)
                for s, n in enumerate(lens):
                    at = np.arange(n)
                    held[self.table[s, at // B], at % B] = True
                a[~held] = x
            self.c.put(0, k, v)
        self.q = self.c.normal(rows, hq, hd, sigma=1.5)
        self.o = torch.full_like(self.q, 7.0)
        self.mask = pack_masks(np.concatenate(noise), self.words)
        self.args = [i32(self.starts), i32(self.table), i32(lens), self.mask]
        coco.coco_tree_reserve(self.c.h, rows, len(trees))

    def run(self, stream=None):
        coco.coco_tree_attention(self.c.h, 0, self.q, self.o, *self.args, stream=stream)

    def check(self):
        torch.cuda.synchronize()
        c = self.c
        k, v = c.tokens()
        got, q = self.o.cpu().double().numpy(), self.q.cpu().double().numpy()
        for s, (prefix, nodes) in enumerate(self.trees):
            at = np.arange(prefix + nodes)
            ks, vs = k[self.table[s, at // B], at % B], v[self.table[s, at // B], at % B]
            for j in range(nodes):
                seen = np.concatenate([np.ones(prefix, bool), self.seen[s][j, :nodes]])
                o, mean, size = attend(q[self.starts[s] + j], ks, vs, seen[None], c.hkv)
                off = np.abs(got[self.starts[s] + j] - o)
                tol = tolerance(c.dtype, o, mean, size, len(at), c.hd)
                assert (off <= tol).all(), (s, j, prefix, nodes, (off / tol).max())


HEADS = [("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("bf16", 4, 4, 128), ("bf16", 16, 1, 128),
         ("bf16", 16, 2, 128), ("f32", 4, 2, 64), ("f32", 3, 1, 32), ("f32", 8, 1, 96),
         ("f32", 2, 2, 256), ("f32", 20, 1, 64)]
TREES = {
    "one": [(0, 1)],
    "token": [(1000, 1)],
    "edges": [(15, 1), (16, 1), (0, 16), (1, 15), (17, 33), (31, 2), (255, 1), (256, 1)],
    "ragged": [(0, 5), (300, 26), (77, 1), (513, 17), (1, 64), (129, 3)],
    "wide": [(40, 65), (700, 130), (0, 64), (5, 128)],
    "empty": [(0, 0), (50, 0), (20, 4), (0, 0)],
}


@pytest.mark.parametrize("trees", sorted(TREES))
@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS)
def test_matches_the_definition(dtype, hq, hkv, hd, trees):
    call = Call(dtype, hq, hkv, hd, TREES[trees], seed=len(trees))
    call.run()
    call.check()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_masks_of_any_kind(dtype, hq, hkv, hd):
    """Random sets (rows without a bit among them, with and without a prefix),
    masks wider than the trees."""
    def any_set(rng, n, words):
        seen = (rng.random((n, 64 * words)) < rng.choice([0.02, 0.3, 1.0], size=(n, 1)))
        seen[rng.random(n) < 0.3] = False
        return seen & (np.arange(64 * words) < n)[None]
    call = Call(dtype, hq, hkv, hd, [(0, 40), (9, 70), (0, 3), (200, 100)], words=4, seed=3,
                masks=any_set)
    call.run()
    call.check()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_unseen_nodes_may_hold_anything(dtype, hq, hkv, hd):
    """NaN and infinities in the keys and values of nodes: rows that do not see
    them are as without, rows that see a NaN or infinite value have it."""
    call = Call(dtype, hq, hkv, hd, [(21, 20), (0, 40), (530, 9)], seed=5)
    k, v = call.c.tokens()
    bad = [(0, 3), (1, 17), (2, 2)]
    for (s, j), x in zip(bad, (np.nan, np.inf, -np.inf)):
        at = call.trees[s][0] + j
        v[call.table[s, at // B], at % B] = x
        if x != x:
            k[call.table[s, at // B], at % B] = x
    call.c.put(0, k, v)
    call.run()
    torch.cuda.synchronize()
    got = call.o.cpu().double().numpy()
    clean_k, clean_v = np.nan_to_num(k, nan=0, posinf=0, neginf=0), \
        np.nan_to_num(v, nan=0, posinf=0, neginf=0)
    hit = np.zeros(len(got), bool)
    for (s, j), x in zip(bad, (np.nan, np.inf, -np.inf)):
        rows = call.starts[s] + np.nonzero(call.seen[s][:, j])[0]
        hit[rows] = True
        assert (np.isnan(got[rows]) if x != x else got[rows] == x).all()
    assert np.isfinite(got[~hit]).all()
    call.c.put(0, clean_k, clean_v)
    call.run()
    torch.cuda.synchronize()
    again = call.o.cpu().double().numpy()
    assert np.array_equal(again[~hit], got[~hit])
    call.check()


# Up to 16 columns (nodes times heads of a group) and just above, in one call.
FEW = [(8, 2, [(0, 1), (20, 4), (530, 3), (1100, 2), (40, 5), (5000, 4), (3, 4)]),
       (16, 1, [(0, 1), (15, 1), (700, 1), (31, 2)]),
       (4, 4, [(0, 16), (9, 15), (640, 12), (50, 17), (2047, 1), (7, 3)]),
       (5, 1, [(511, 1), (512, 3), (513, 2), (100, 4), (16400, 1)])]


@pytest.mark.parametrize("hq,hkv,trees", FEW)
def test_few_columns_with_masks_of_any_kind(hq, hkv, trees):
    def any_set(rng, n, words):
        seen = rng.random((n, 64 * words)) < 0.6
        seen[rng.random(n) < 0.2] = False
        return seen & (np.arange(64 * words) < n)[None]
    for masks in (path_masks, any_set):
        call = Call("bf16", hq, hkv, 128, trees, words=2, seed=21, masks=masks)
        call.run()
        call.check()


@pytest.mark.parametrize("hq,hkv,trees", FEW)
def test_few_columns_among_nodes_that_hold_anything(hq, hkv, trees):
    call = Call("bf16", hq, hkv, 128, trees, seed=22)
    k, v = call.c.tokens()
    hit = np.zeros(int(call.starts[-1]), bool)
    for s, (prefix, nodes) in enumerate(trees):
        if nodes < 2:
            continue
        j = nodes // 2
        k[call.table[s, (prefix + j) // B], (prefix + j) % B] = np.nan
        v[call.table[s, (prefix + j) // B], (prefix + j) % B] = np.nan
        hit[call.starts[s] + np.nonzero(call.seen[s][:, j])[0]] = True
    call.c.put(0, k, v)
    call.run()
    torch.cuda.synchronize()
    got = call.o.cpu().double().numpy()
    assert np.isnan(got[hit]).all() and np.isfinite(got[~hit]).all()
    call.c.put(0, np.nan_to_num(k), np.nan_to_num(v))
    call.run()
    torch.cuda.synchronize()
    assert np.array_equal(call.o.cpu().double().numpy()[~hit], got[~hit])
    # A value that is seen but infinite comes out, in its sign.
    s = max(range(len(trees)), key=lambda i: trees[i][1])
    at = trees[s][0]  # the first node
    v[call.table[s, at // B], at % B] = -np.inf
    call.c.put(0, np.nan_to_num(k), np.where(np.isnan(v), 0, v))
    call.run()
    torch.cuda.synchronize()
    got = call.o.cpu().double().numpy()
    rows = call.starts[s] + np.nonzero(call.seen[s][:, 0])[0]
    assert (got[rows] == -np.inf).all()
    rest = np.setdiff1d(np.arange(len(got)), rows)
    assert np.isfinite(got[rest]).all()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 1, 128), ("f32", 2, 1, 32)])
def test_long_contexts(dtype, hq, hkv, hd):
    call = Call(dtype, hq, hkv, hd, [(40000, 7), (3, 2), (20011, 30), (9000, 1)], seed=7)
    call.run()
    call.check()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_rows_do_not_depend_on_the_rest_of_the_call(dtype, hq, hkv, hd):
    trees = [(0, 5), (3000, 26), (77, 1), (513, 40), (1, 64), (9000, 3)]
    call = Call(dtype, hq, hkv, hd, trees, seed=9)
    call.run()
    whole = call.o.clone()
    starts, table, lens, mask = call.args
    for pick in ([3], [5, 1], [0, 2, 4]):
        rows = np.concatenate([np.arange(call.starts[s], call.starts[s + 1]) for s in pick])
        rows = torch.from_numpy(rows).cuda()
        n = [trees[s][1] for s in pick]
        o = torch.empty(len(rows), hq, hd, dtype=call.q.dtype, device="cuda")
        coco.coco_tree_attention(call.c.h, 0, call.q[rows], o,
                                 i32(np.concatenate([[0], np.cumsum(n)])), table[pick],
                                 lens[pick], mask[rows])
        assert torch.equal(o, whole[rows]), pick


@pytest.mark.parametrize("hq,hkv,hd", [(16, 4, 64), (8, 1, 128), (12, 2, 32)])
def test_fp32_rows_of_a_full_chip_and_alone(hq, hkv, hd):
    """The number of heads per workgroup follows the call's rows; the bits do not."""
    call = Call("f32", hq, hkv, hd, [(500, 60), (30, 50)], seed=19)
    call.run()
    call.check()
    starts, table, lens, mask = call.args
    # A tree's first nodes (which see none behind them) in calls of few rows.
    for s, (prefix, nodes) in enumerate(call.trees):
        r0 = int(call.starts[s])
        for n in (1, 7):
            few = torch.empty_like(call.o[:n])
            coco.coco_tree_attention(call.c.h, 0, call.q[r0:r0 + n], few, i32([0, n]),
                                     table[s:s + 1], i32([prefix + n]), mask[r0:r0 + n])
            assert torch.equal(few, call.o[r0:r0 + n]), (s, n)


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_more_sequences_than_a_launch_takes(dtype, hq, hkv, hd):
    rng = np.random.default_rng(5)
    trees = [(int(p), int(n)) for p, n in zip(rng.integers(0, 40, 2100), rng.integers(0, 3, 2100))]
    trees[1023], trees[1024], trees[2099] = (500, 30), (400, 2), (700, 20)
    call = Call(dtype, hq, hkv, hd, trees, seed=18)
    for _ in range(2):  # the counters of every launch are left as they were found
        call.o.fill_(7.0)
        call.run()
        call.check()


def test_blocks_past_32_bit_offsets():
    """Pools of more than 2^31 elements, the sequence in their last blocks."""
    hkv, n = 8, (1 << 31) // (8 * B * 128) + 64
    call = Call("bf16", 8, hkv, 128, [(70, 9)], seed=11, spoil=False, num_blocks=16)
    small = call.c
    pools = [tuple(torch.zeros(n, hkv, B * 128, dtype=torch.bfloat16, device="cuda") for _ in "kv")]
    big = Cache("bf16", 8, hkv, 128, n, call.table.shape[1], pools=pools)
    for p, src in zip(pools[0], small.pools[0]):
        p[-16:] = src
    coco.coco_tree_reserve(big.h, 9, 1)
    call.run()
    call.check()
    o = torch.empty_like(call.o)
    shifted = torch.where(call.args[1] < 0, -1, call.args[1] + (n - 16)).to(torch.int32)
    coco.coco_tree_attention(big.h, 0, call.q, o, call.args[0], shifted, *call.args[2:])
    assert torch.equal(o, call.o)


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_streams_and_graph_replay(dtype, hq, hkv, hd):
    call = Call(dtype, hq, hkv, hd, [(600, 9), (0, 3), (2500, 33)], seed=13)
    call.run()
    torch.cuda.synchronize()
    want = call.o.clone()
    side = torch.cuda.Stream()
    call.o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    call.run(stream=side)
    side.synchronize()
    assert torch.equal(call.o, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    other = Call(dtype, hq, hkv, hd, [(100, 5)], seed=14)
    for _ in range(3):
        call.o.zero_()
        other.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(call.o, want)


def test_reserve_that_grows_keeps_captured_graphs():
    call = Call("bf16", 8, 2, 128, [(6000, 9)], seed=15)
    call.run()
    torch.cuda.synchronize()
    want = call.o.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    coco.coco_tree_reserve(call.c.h, 4096, 64)
    call.run()
    torch.cuda.synchronize()
    assert torch.equal(call.o, want)
    call.o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(call.o, want)


def test_refusals():
    call = Call("bf16", 8, 2, 128, [(20, 3), (5, 2)], seed=17)
    c = call.c
    starts, table, lens, mask = call.args
    fresh = Cache("bf16", 8, 2, 128, 4, 2)
    with pytest.raises(coco.CocoError, match="coco_tree_reserve") as e:
        coco.coco_tree_attention(fresh.h, 0, call.q, call.o, starts, table[:, :2].contiguous(),
                                 lens, mask)
    assert e.value.code == -4
    with pytest.raises(coco.CocoError, match="layer 1"):
        coco.coco_tree_attention(c.h, 1, call.q, call.o, starts, table, lens, mask)
    with pytest.raises(coco.CocoError, match="positive"):
        coco.coco_tree_reserve(c.h, 0, 1)
    with pytest.raises(ValueError, match="seq_starts"):
        coco.coco_tree_attention(c.h, 0, call.q, call.o, starts[:-1], table, lens, mask)
    with pytest.raises(ValueError, match="tree_mask"):
        coco.coco_tree_attention(c.h, 0, call.q, call.o, starts, table, lens, mask[:-1])
    with pytest.raises(TypeError, match="q must be"):
        coco.coco_tree_attention(c.h, 0, call.q.float(), call.o, starts, table, lens, mask)
    odd = torch.empty(call.q.numel() + 1, dtype=call.q.dtype, device="cuda")[1:].view_as(call.q)
    with pytest.raises(coco.CocoError, match="aligned"):
        coco.coco_tree_attention(c.h, 0, odd, call.o, starts, table, lens, mask)
    empty = call.q[:0]
    coco.coco_tree_attention(c.h, 0, empty, empty, starts[:1], table[:0], lens[:0], mask[:0])
    # Contents are checked in validation mode, before anything is launched.
    coco.coco_layer_set_validate(c.h, True)
    call.o.fill_(7.0)
    for args, text in (((starts, table, i32([2, 7]), mask), "3 nodes in 2"),
                       ((i32([0, 4, 3]), table, lens, mask), "seq_starts"),
                       ((starts, torch.where(table >= 0, 99, table).to(torch.int32), lens, mask),
                        "out of range"),
                       ((starts, table, i32([23, 1 << 20]), mask), "ctx_lens")):
        with pytest.raises(coco.CocoError, match=text):
            coco.coco_tree_attention(c.h, 0, call.q, call.o, *args)
    torch.cuda.synchronize()
    assert (call.o == 7.0).all()
    call.run()
    call.check()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_rows_past_the_last_sequence_are_left_as_they_are(dtype, hq, hkv, hd):
    call = Call(dtype, hq, hkv, hd, [(600, 3), (40, 30), (0, 2)], seed=23)
    call.run()
    torch.cuda.synchronize()
    n, more = len(call.o), 6
    starts, table, lens, mask = call.args
    q = torch.cat([call.q, torch.full_like(call.q[:more], float("nan"))])
    o = torch.full_like(q, 7.0)
    masks = torch.cat([mask, torch.full_like(mask[:more], -1)])
    coco.coco_tree_reserve(call.c.h, n + more, 3)
    coco.coco_tree_attention(call.c.h, 0, q, o, starts, table, lens, masks)
    torch.cuda.synchronize()
    assert torch.equal(o[:n], call.o) and (o[n:] == 7.0).all()


def test_tensors_of_another_device_are_refused():
    call = Call("bf16", 8, 2, 128, [(20, 3)], seed=20)
    here, call.c.h.device = call.c.h.device, call.c.h.device + 1
    with pytest.raises(ValueError, match="q must be on the handle's GPU"):
        call.run()
    call.c.h.device = here
    call.run()
    call.check()
