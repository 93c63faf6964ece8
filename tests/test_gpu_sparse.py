"""Block summaries, the choice of blocks, and attention over chosen blocks,
against the definition (whole numbers, and 64 bits)."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, attend, choose, i32, summary_of, tables, tolerance

pytestmark = pytest.mark.gpu

HEADS = [("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("bf16", 16, 1, 128), ("f32", 4, 2, 64),
         ("f32", 3, 1, 32), ("f32", 20, 1, 96), ("f32", 70, 1, 160), ("f32", 2, 2, 256)]


class Rows:
    """Rows at positions of sequences with the given lengths; rows None: each
    sequence's newest token (decode)."""

    def __init__(self, dtype, hq, hkv, hd, lens, rows=None, top=5, seed=0, extra_width=1):
        rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens)
        width = max(1, int(-(-self.lens.max() // B)) + extra_width)
        self.c = Cache(dtype, hq, hkv, hd, int((-(-self.lens // B)).sum()) + 2, width, seed=seed,
                       max_seqs=len(lens))
        self.table = tables(rng, lens, width, self.c.num_blocks)
        if rows is None:
            self.seq, self.pos, self.starts = np.arange(len(lens)), self.lens - 1, None
        else:
            self.seq = np.repeat(np.arange(len(lens)), [len(r) for r in rows])
            self.pos = np.concatenate([np.asarray(r, np.int64) for r in rows])
            self.starts = i32(np.concatenate([[0], np.cumsum([len(r) for r in rows])]))
        self.n, self.top = len(self.seq), top
        self.keys = np.maximum(0, np.minimum(self.lens[self.seq], self.pos + 1))
        self.q = self.c.normal(self.n, hq, hd, sigma=1.5)
        self.o = torch.full_like(self.q, 7.0)
        self.summary = torch.full((self.c.num_blocks, hkv, 2, hd), 99, dtype=torch.int8, device="cuda")
        self.scales = torch.full((self.c.num_blocks, hkv), 3.0, device="cuda")
        self.selected = torch.full((self.n, hkv, top), 77, dtype=torch.int32, device="cuda")
        self.rest = (i32(self.pos), self.starts, i32(self.table), i32(self.lens))
        coco.coco_sparse_reserve(self.c.h, self.n, top)

    def summarize(self, first=None):
        coco.coco_kv_summarize(self.c.h, 0, self.summary, self.scales, first, self.rest[3],
                               self.rest[2])

    def select(self, first=0, last=0):
        coco.coco_block_select(self.c.h, self.summary, self.scales, self.q, *self.rest, first, last,
                               self.selected)

    def attention(self):
        coco.coco_sparse_attention(self.c.h, 0, self.q, self.o, *self.rest, self.selected)

    def check_summary(self, first=None):
        k, _ = self.c.tokens()
        want, scales = self.before[0].copy(), self.before[1].copy()
        for s, n in enumerate(self.lens):
            for b in range(0 if first is None else first[s] // B, -(-int(n) // B)):
                blk = self.table[s, b]
                for g in range(self.c.hkv):
                    want[blk, g], scales[blk, g] = summary_of(k[blk, :min(B, n - b * B), g])
        assert np.array_equal(self.summary.cpu().numpy(), want)
        assert np.array_equal(self.scales.cpu().numpy(), scales)

    def snapshot(self):
        self.before = self.summary.cpu().numpy(), self.scales.cpu().numpy()

    def check_select(self, first=0, last=0):
        sm, sc = self.summary.cpu().numpy(), self.scales.cpu().numpy()
        q = self.q.cpu().double().numpy().reshape(self.n, self.c.hkv, -1, self.c.hd)
        got = self.selected.cpu().numpy()
        for i in range(self.n):
            blk = self.table[self.seq[i], :-(-int(self.keys[i]) // B)]
            for g in range(self.c.hkv):
                want = choose(q[i, g], sm[blk, g], sc[blk, g], self.top, first, last) \
                    if len(blk) else np.full(self.top, -1)
                assert np.array_equal(got[i, g], want), (i, g)

    def check_attention(self):
        k, v = self.c.tokens()
        c = self.c
        got, q, sel = (t.cpu().double().numpy() for t in (self.o, self.q, self.selected))
        for i in range(self.n):
            n = int(self.keys[i])
            at = np.arange(n)
            blk = self.table[self.seq[i], at // B]
            seen = np.stack([np.isin(at // B, sel[i, g]) for g in range(c.hkv)]) if n else \
                np.zeros((c.hkv, 0), bool)
            o, mean, size = attend(q[i], k[blk, at % B], v[blk, at % B],
                                   seen if c.hkv > 1 else seen[:1], c.hkv)
            off = np.abs(got[i] - o)
            tol = tolerance(c.dtype, o, mean, size, min(n, self.top * B), c.hd)
            assert (off <= tol).all(), (i, (off / tol).max())


@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS)
def test_summaries(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [1, 16, 17, 300, 47], seed=1)
    k, v = r.c.tokens()
    k[r.table[3, 2]] = 0.0                     # a block of zeros
    k[r.table[3, 3], 5, :, 4] = np.nan         # elements that count as 0
    k[r.table[3, 4], 0, :, 7] = np.inf
    k[r.table[3, 5]] *= 2.0 ** -30
    k[r.table[3, 6]] *= 2.0 ** 110             # held within the exponents
    k[r.table[2, 1], 1:] = np.nan              # slots past the tokens
    r.c.put(0, k, v)
    r.snapshot()
    r.summarize()
    r.check_summary()
    # New tokens: only their blocks change.
    r.snapshot()
    k[r.table[3, 18], 3] = 50.0
    k[r.table[3, 17], 3] = 50.0
    k[r.table[4, 2], 14] = -9.0
    r.c.put(0, k, v)
    first = np.array([0, 15, 16, 16 * 18 + 2, 47])
    r.summarize(i32(first))
    r.check_summary([0, 15, 16, 16 * 18 + 2, 47])


@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS)
@pytest.mark.parametrize("top,first,last", [(1, 0, 0), (5, 1, 2), (8, 0, 8), (3, 1, 2), (40, 2, 1)])
def test_choice_and_attention(dtype, hq, hkv, hd, top, first, last):
    r = Rows(dtype, hq, hkv, hd, [1, 700, 33, 16 * 40, 16 * 41 + 1, 2000, 80], top=top, seed=2)
    r.summarize()
    r.select(first, last)
    torch.cuda.synchronize()
    r.check_select(first, last)
    r.attention()
    r.check_attention()


def test_rows_of_a_prompt_and_rows_without_keys():
    rows = [[0, 15, 16, 299], [], [-1, 5, 120], [31]]
    for dtype, hq, hkv, hd in (("bf16", 8, 2, 128), ("f32", 4, 2, 64)):
        r = Rows(dtype, hq, hkv, hd, [300, 40, 100, 0], rows=rows, top=4, seed=3)
        r.summarize()
        r.select(1, 1)
        torch.cuda.synchronize()
        r.check_select(1, 1)
        r.attention()
        r.check_attention()
        assert (r.o[4] == 0).all() and (r.o[-1] == 0).all()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_positions_past_the_cache_attend_all_of_it(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [200, 33], rows=[[150, 199, 10 ** 6, 2 ** 31 - 1], [2 ** 31 - 2]],
             top=5, seed=11)
    r.summarize()
    r.select(1, 1)
    torch.cuda.synchronize()
    r.check_select(1, 1)
    r.attention()
    r.check_attention()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("top", [4, 40])
def test_rows_past_the_last_sequence_are_left_as_they_are(dtype, hq, hkv, hd, top):
    rows = [[0, 15, 1299], [5, 39], [99]]
    r = Rows(dtype, hq, hkv, hd, [1300, 40, 100], rows=rows, top=top, seed=10)
    r.summarize()
    r.select(1, 1)
    r.attention()
    torch.cuda.synchronize()
    want = r.selected.clone(), r.o.clone()
    # The same sequences in a call of more rows, whose arrays hold anything.
    pos, starts, table, lens = r.rest
    more = 5
    q = torch.cat([r.q, torch.full_like(r.q[:more], float("nan"))])
    pos = torch.cat([pos, i32([10 ** 9, -7, 3, 2 ** 31 - 1, 0])])
    sel = torch.cat([torch.full_like(r.selected, 55), torch.full_like(r.selected[:more], 66)])
    o = torch.full_like(q, 7.0)
    coco.coco_sparse_reserve(r.c.h, r.n + more, top)
    coco.coco_block_select(r.c.h, r.summary, r.scales, q, pos, starts, table, lens, 1, 1, sel)
    coco.coco_sparse_attention(r.c.h, 0, q, o, pos, starts, table, lens, sel)
    torch.cuda.synchronize()
    assert torch.equal(sel[:r.n], want[0]) and torch.equal(o[:r.n], want[1])
    assert (sel[r.n:] == 66).all() and (o[r.n:] == 7.0).all()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_ties_go_to_the_lowest_block(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [16 * 90, 16 * 700], top=30, seed=4)
    r.summarize()
    r.summary.copy_(torch.randint(-1, 2, (r.c.num_blocks, hkv, 1, 1), device="cuda",
                                  generator=r.c.gen).expand_as(r.summary))
    r.scales.fill_(0.5)
    for first, last in ((0, 0), (2, 3)):
        r.select(first, last)
        torch.cuda.synchronize()
        r.check_select(first, last)


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_long_context_and_odd_queries(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [30011, 16 * 1024, 60000], top=64, seed=5)
    r.q[0] = 0
    r.q[1, 0, 3], r.q[1, 1, 9] = float("inf"), float("nan")
    r.q[2] *= 1e-3
    r.summarize()
    r.select(1, 4)
    torch.cuda.synchronize()
    r.check_select(1, 4)
    r.q[1, 0, 3] = r.q[1, 1, 9] = 1.0
    r.attention()
    r.check_attention()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 4, 1, 128), ("f32", 3, 1, 32)])
def test_contexts_of_more_than_8192_blocks(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [16 * 8192, 70, 16 * 8192 + 33, 16 * 10000], top=33, seed=9)
    r.summarize()
    for first, last in ((1, 4), (0, 0), (20, 13)):
        r.select(first, last)
        torch.cuda.synchronize()
        r.check_select(first, last)
    r.select(1, 4)
    r.attention()
    r.check_attention()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_lists_of_the_callers_own(dtype, hq, hkv, hd):
    """Any order, gaps, entries outside the row's blocks, an empty list; keys
    and values behind the row's position and in other blocks hold NaN."""
    r = Rows(dtype, hq, hkv, hd, [200, 150, 90], top=9, seed=6)
    lists = np.full((3, hkv, 9), -1)
    lists[0] = [3, -1, 12, 0, 999, 7, -5, 1, 11]
    lists[1, 0] = [9, 8, -1, -1, -1, -1, -1, -1, 2]
    lists[1, 1:] = [0, 1, 2, 3, 4, 5, 6, 7, 10]
    lists[2, :, 4] = 5
    lists[2, 0] = -1
    r.selected.copy_(i32(lists))
    k, v = r.c.tokens()
    used = np.zeros((r.c.num_blocks, B, hkv), bool)
    for s in range(3):
        for g in range(hkv):
            for b in lists[s, g]:
                if 0 <= b < -(-int(r.lens[s]) // B):
                    used[r.table[s, b], :min(B, int(r.lens[s]) - b * B), g] = True
    k[~used], v[~used] = np.nan, np.nan
    r.c.put(0, k, v)
    r.attention()
    got = r.o.cpu().double().numpy()
    assert np.isfinite(got).all() and (got[2, :hq // hkv] == 0).all()
    r.c.put(0, np.nan_to_num(k), np.nan_to_num(v))
    r.check_attention()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_streams_graphs_and_other_rows(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [3000, 77, 900, 16], top=12, seed=7)

    def step():
        r.summarize()
        r.select(1, 1)
        r.attention()

    step()
    torch.cuda.synchronize()
    want = r.o.clone(), r.selected.clone(), r.summary.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for t in (r.o, r.selected):
            t.zero_()
        r.summary.fill_(99)  # as the blocks without tokens have been
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((r.o, r.selected, r.summary), want))
    side = torch.cuda.Stream()
    r.o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(r.o, want[0])
    # Each row alone: the same bits.
    pos, _, table, lens = r.rest
    for i in range(r.n):
        sel, o = torch.empty_like(r.selected[:1]), torch.empty_like(r.o[:1])
        one = slice(i, i + 1)
        coco.coco_block_select(r.c.h, r.summary, r.scales, r.q[one], pos[one], None, table[one],
                               lens[one], 1, 1, sel)
        coco.coco_sparse_attention(r.c.h, 0, r.q[one], o, pos[one], None, table[one], lens[one], sel)
        assert torch.equal(sel, want[1][one]) and torch.equal(o, want[0][one])


def test_refusals():
    r = Rows("bf16", 8, 2, 128, [40, 50], top=3, seed=8)
    h, (pos, _, table, lens) = r.c.h, r.rest
    r.summarize()
    with pytest.raises(coco.CocoError, match="keep_first"):
        r.select(2, 2)
    with pytest.raises(coco.CocoError, match="keep_first"):
        r.select(-1, 2)
    for rows, blocks in ((0, 3), (65536, 3), (2, 0), (2, (1 << 24) + 1)):
        with pytest.raises(coco.CocoError, match="outside"):
            coco.coco_sparse_reserve(h, rows, blocks)
    more = torch.empty(2, 2, 4, dtype=torch.int32, device="cuda")
    with pytest.raises(coco.CocoError, match="coco_sparse_reserve") as e:
        coco.coco_block_select(h, r.summary, r.scales, r.q, pos, None, table, lens, 0, 0, more)
    assert e.value.code == -4
    with pytest.raises(coco.CocoError, match="coco_sparse_reserve"):
        coco.coco_sparse_attention(h, 0, r.q, r.o, pos, None, table, lens, more)
    with pytest.raises(ValueError, match="selected"):
        coco.coco_sparse_attention(h, 0, r.q, r.o, pos, None, table, lens, more[:1])
    with pytest.raises(ValueError, match="summary"):
        coco.coco_kv_summarize(h, 0, r.summary[:-1], r.scales[:-1], None, lens, table)
    with pytest.raises(ValueError, match="summary must be"):
        coco.coco_block_select(h, r.summary[..., :64], r.scales, r.q, pos, None, table, lens, 0, 0,
                               r.selected)
    with pytest.raises(coco.CocoError, match="layer 3"):
        coco.coco_sparse_attention(h, 3, r.q, r.o, pos, None, table, lens, r.selected)
    coco.coco_layer_set_validate(h, True)
    r.select()
    for sel, text in (([[0, 0, 1]], "ascending"), ([[0, 1, 3]], "past the row"), ([[2, 1, -1]], "ascending")):
        bad = i32([[sel[0], sel[0]], [sel[0], sel[0]]])
        with pytest.raises(coco.CocoError, match=text):
            coco.coco_sparse_attention(h, 0, r.q, r.o, pos, None, table, lens, bad)
    with pytest.raises(coco.CocoError, match="ctx_lens"):
        coco.coco_kv_summarize(h, 0, r.summary, r.scales, None, i32([40, 1000]), table)
    with pytest.raises(coco.CocoError, match="positions"):
        coco.coco_block_select(h, r.summary, r.scales, r.q, i32([3, -2]), None, table, lens, 0, 0,
                               r.selected)
    r.attention()
    r.check_attention()
