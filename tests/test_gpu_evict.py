"""Eviction by accumulated weight: the choice, the moved weights, and with it the
compaction of the cache and its pages, against plain lists."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, attend, i32, tables, tolerance

pytestmark = pytest.mark.gpu


def keep(w, n, budget, first, last):
    """Slots that a row of n tokens keeps, ascending."""
    if n <= budget:
        return list(range(n))
    first = min(first, budget)
    last = min(last, budget - first)
    middle = list(range(first, n - last))
    key = [-np.inf if np.isnan(w[t]) else w[t] for t in middle]
    best = sorted(range(len(middle)), key=lambda i: (-key[i], i))
    # (NaN below -inf)
    best.sort(key=lambda i: (np.isnan(w[middle[i]]), -key[i], i))
    return sorted(list(range(first)) + [middle[i] for i in best[:budget - first - last]] +
                  list(range(n - last, n)))


class Evict:
    def __init__(self, lens, budgets, first=0, last=0, weights=None, rows=None, n_kept=None, width=None,
                 handle=None):
        self.lens = np.asarray(lens)
        self.rows = np.arange(len(lens)) if rows is None else np.asarray(rows)
        self.budgets, self.first, self.last = np.asarray(budgets), first, last
        self.width = width or max(1, int(-(-self.lens.max() // B)) + 1)
        self.c = handle or Cache("f32", 2, 1, 32, 8, self.width, max_seqs=max(len(lens), 1), max_rows=4)
        w = np.zeros((len(lens), self.width * B), np.float32) if weights is None else weights
        self.w = torch.from_numpy(w).cuda()
        n = len(self.rows)
        self.n_kept = int(np.minimum(self.budgets, 1 << 20).clip(0).sum()) if n_kept is None else n_kept
        self.new, self.base = i32(np.full(n, -9)), i32(np.full(n, -9))
        self.kept, self.starts = i32(np.full(self.n_kept + 3, -9))[:self.n_kept], i32(np.full(n + 1, -9))
        self.none = weights is None

    def run(self):
        self.before = self.w.cpu().numpy().copy()
        coco.coco_kv_evict(self.c.h, i32(self.rows), i32(self.budgets), self.first, self.last,
                           i32(self.lens), None if self.none else self.w, self.new, self.base,
                           self.kept, self.starts)
        torch.cuda.synchronize()

    def check(self):
        new, base, kept, starts = (t.cpu().numpy() for t in (self.new, self.base, self.kept, self.starts))
        want_w = self.before.copy()
        at, full = 0, False
        lists = []
        for i, s in enumerate(self.rows):
            n, b = int(self.lens[s]), max(int(self.budgets[i]), 0)
            ids = keep(self.before[s], n, b, self.first, self.last)
            lo = next((d for d, t in enumerate(ids) if t != d), len(ids))
            tail = ids[lo:] if n > b else []
            full = full or at + len(tail) > self.n_kept
            if n <= b or (full and tail):
                tail, lo, b = [], n, n
                ids = list(range(n))
            assert (new[i], base[i]) == (len(ids), lo), i
            assert starts[i] == at, i
            assert kept[at:at + len(tail)].tolist() == tail, i
            at += len(tail)
            want_w[s, :len(ids)] = self.before[s, ids]
            want_w[s, len(ids):n] = 0.0
            lists.append(ids)
        assert starts[-1] == at and (kept[at:] == -9).all()
        if not self.none:
            assert np.array_equal(self.w.cpu().numpy(), want_w, equal_nan=True)
        return lists


def heavy(rng, lens, width, kind):
    w = rng.exponential(size=(len(lens), width * B)).astype(np.float32) ** 3
    if kind == "ties":
        w = np.floor(w)
    elif kind == "zeros":
        w[:] = 0.0
    elif kind == "odd":
        w[rng.random(w.shape) < 0.1] = np.nan
        w[rng.random(w.shape) < 0.1] = np.inf
        w[rng.random(w.shape) < 0.1] = -np.inf
        w[rng.random(w.shape) < 0.1] *= -1
        w[rng.random(w.shape) < 0.05] = -0.0
        w[rng.random(w.shape) < 0.05] = 0.0
        w[rng.random(w.shape) < 0.05] = np.float32(1e-42)
    return w


LENS = [0, 1, 2, 16, 17, 100, 1000, 4095, 4096, 4097, 5000, 8200]


@pytest.mark.parametrize("kind", ["heavy", "ties", "zeros", "odd"])
@pytest.mark.parametrize("first,last", [(0, 0), (1, 0), (4, 30), (0, 200), (70, 3), (5000, 7)])
def test_choice(kind, first, last):
    rng = np.random.default_rng(1)
    budgets = [0, 0, 1, 16, 3, 64, 900, 4000, 4000, 33, 4999, 4200]
    e = Evict(LENS, budgets, first, last, heavy(rng, LENS, 514, kind), width=514)
    e.run()
    e.check()


@pytest.mark.parametrize("kind", ["heavy", "ties", "zeros", "odd"])
@pytest.mark.parametrize("width", [64, 65])
def test_choice_in_narrow_tables(kind, width):
    rng = np.random.default_rng(4)
    lens = [0, 1, 2, 255, 256, 257, 900, 1000, 1023, 1024]
    for first, last in ((0, 0), (4, 30), (0, 200), (700, 3)):
        e = Evict(lens, [0, 0, 1, 100, 255, 3, 64, 999, 512, 1000], first, last,
                  heavy(rng, lens, width, kind), width=width)
        e.run()
        e.check()


def test_choice_of_long_rows():
    # More slots than a workgroup keeps in registers.
    rng = np.random.default_rng(2)
    lens = [33000, 40001, 32768, 70000]
    for kind in ("heavy", "ties"):
        e = Evict(lens, [32000, 5, 32767, 40000], 2, 100, heavy(rng, lens, 4400, kind), width=4400)
        e.run()
        e.check()


def test_without_weights_the_first_and_last_tokens_stay():
    e = Evict([100, 30, 900], [40, 40, 64], 4, 36)
    e.run()
    lists = e.check()
    assert lists[0] == [0, 1, 2, 3] + list(range(64, 100))


def test_some_rows_in_any_order_and_rows_out_of_range():
    rng = np.random.default_rng(3)
    lens = [100, 200, 300, 400]
    e = Evict(lens, [50, 399, 60], 1, 5, heavy(rng, lens, 40, "heavy"), rows=[3, 0, 2], width=40)
    e.run()
    e.check()
    e = Evict(lens, [50, 60, 70], 1, 5, heavy(rng, lens, 40, "heavy"), rows=[2, 1, 3], width=40)
    e.rows = np.array([2, 9, -1])
    e.run()
    assert e.new.tolist() == [50, 0, 0] and e.starts[1:].tolist() == [e.starts[1].item()] * 3


@pytest.mark.parametrize("n_kept", [0, 1, 40, 99, 130, 200])
def test_lists_that_do_not_fit_are_not_written(n_kept):
    rng = np.random.default_rng(4)
    lens = [100, 100, 50, 100, 100, 100]
    e = Evict(lens, [50, 40, 60, 45, 0, 50], 2, 5, heavy(rng, lens, 8, "heavy"), n_kept=n_kept, width=8)
    e.run()
    e.check()


def test_many_requests():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 60, 2500)
    e = Evict(lens, rng.integers(0, 60, 2500), 1, 2, heavy(rng, lens, 4, "ties"), width=4, n_kept=20000)
    e.run()
    e.check()


def test_captured_evictions_replay():
    rng = np.random.default_rng(6)
    lens = [300, 20, 4500]
    e = Evict(lens, [100, 30, 4000], 2, 9, heavy(rng, lens, 290, "heavy"), width=290)
    first = e.w.clone()
    args = (i32(e.rows), i32(e.budgets), 2, 9, i32(e.lens), e.w, e.new, e.base, e.kept, e.starts)
    e.before = first.cpu().numpy()
    coco.coco_kv_evict(e.c.h, *args)
    torch.cuda.synchronize()
    e.check()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            coco.coco_kv_evict(e.c.h, *args)
    for _ in range(3):
        for t in (e.new, e.base, e.kept, e.starts):
            t.fill_(-9)
        e.w.copy_(first)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        e.check()


def test_validation_mode_names_what_is_wrong():
    e = Evict([100, 30], [50, 40], weights=np.zeros((2, 128), np.float32), width=8)
    coco.coco_layer_set_validate(e.c.h, True)
    e.run()
    e.check()
    for change, text in (("rows", "sequence"), ("same", "duplicate"), ("keep", "keep_lens"),
                         ("room", "do not fit n_kept = 49")):
        rows, budgets, kept = np.array([0, 1]), np.array([50, 40]), e.kept
        if change == "rows":
            rows = np.array([0, 2])
        elif change == "same":
            rows = np.array([1, 1])
        elif change == "keep":
            budgets = np.array([-1, 3])
        else:
            kept = e.kept[:49]
        with pytest.raises(coco.CocoError, match=text):
            coco.coco_kv_evict(e.c.h, i32(rows), i32(budgets), 0, 0, i32(e.lens), e.w, e.new, e.base,
                               kept, e.starts)


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_a_bounded_cache_through_its_calls(dtype, hq, hkv, hd):
    """Prompt rows and single tokens add up weights; rows above their budget are cut
    back, their pages go, and the next tokens attend what is left."""
    rng = np.random.default_rng(7)
    lens, budget, first, last = np.array([130, 40, 77]), 48, 2, 12
    width, nb = 12, 30
    c = Cache(dtype, hq, hkv, hd, nb, width, n_layers=2, max_rows=200, max_seqs=3, seed=7)
    table = i32(tables(rng, lens, width, nb))
    refs = np.zeros(nb, np.int64)
    refs[table.cpu().numpy()[table.cpu().numpy() >= 0]] = 1
    refs = i32(refs)
    weights = torch.zeros(3, width * B, device="cuda")
    coco.coco_window_reserve(c.h, 200, 3, True)
    rows = np.array([30, 40, 9])
    q = c.normal(int(rows.sum()), hq, hd, sigma=1.5)
    o = torch.empty_like(q)
    coco.coco_window_attention(c.h, 0, q, o, i32(np.concatenate([[0], np.cumsum(rows)])), table, i32(lens),
                               2 ** 31 - 1, 0, weights)
    torch.cuda.synchronize()
    w0 = weights.cpu().numpy()
    old = [c.tokens(layer) for layer in range(2)]
    t0 = table.cpu().numpy()
    assert np.abs(w0.sum(1) - rows * hq).max() < 1e-2
    n_kept = 3 * budget
    new, base, kept, starts = i32(np.zeros(3)), i32(np.zeros(3)), i32(np.zeros(n_kept)), i32(np.zeros(4))
    every = i32(np.arange(3))
    coco.coco_layer_set_validate(c.h, True)  # lists shorter than their room are taken
    coco.coco_kv_evict(c.h, every, i32(np.full(3, budget)), first, last, i32(lens), weights, new, base, kept,
                       starts)
    coco.coco_kv_compact(c.h, 0, 2, every, base, kept, starts, table)
    coco.coco_kv_free(c.h, every, new, table, refs)
    coco.coco_layer_set_validate(c.h, False)
    torch.cuda.synchronize()
    now = new.cpu().numpy()
    assert now.tolist() == [budget, 40, budget]
    assert int((refs > 0).sum()) == int((-(-now // B)).sum())
    ids = [keep(w0[s], int(lens[s]), budget, first, last) for s in range(3)]
    w1 = weights.cpu().numpy()
    t1 = table.cpu().numpy()
    for layer in range(2):
        k, v = c.tokens(layer)
        for s in range(3):
            to, at = np.arange(now[s]), np.array(ids[s])
            for x, y in ((k, old[layer][0]), (v, old[layer][1])):
                assert np.array_equal(x[t1[s, to // B], to % B], y[t0[s, at // B], at % B])
            assert np.array_equal(w1[s, :now[s]], w0[s, at]) and (w1[s, now[s]:] == 0).all()
    # The next token goes behind what is left, and attends it.
    status = i32(np.zeros(3))
    coco.coco_kv_alloc(c.h, every, i32(now + 1), table, refs, status)
    kn, vn = c.normal(3, hkv, hd), c.normal(3, hkv, hd)
    coco.coco_kv_append(c.h, 0, kn, vn, every, i32(now), table)
    q, o = c.normal(3, hq, hd, sigma=1.5), torch.empty(3, hq, hd, dtype=kn.dtype, device="cuda")
    coco.coco_window_attention(c.h, 0, q, o, None, table, i32(now + 1), 2 ** 31 - 1, 0, weights)
    torch.cuda.synchronize()
    assert status.tolist() == [1, 1, 1]
    t1 = table.cpu().numpy()
    k, v = c.tokens(0)
    for s in range(3):
        at = np.arange(now[s] + 1)
        ref, mean, size = attend(q[s].cpu().double().numpy(), k[t1[s, at // B], at % B],
                                 v[t1[s, at // B], at % B], np.ones((1, len(at)), bool), hkv)
        tol = tolerance(dtype, ref, mean, size, len(at), hd)
        assert (np.abs(o[s].cpu().double().numpy() - ref) <= tol).all()
    assert np.abs((weights.cpu().numpy() - w1).sum(1) - hq).max() < 1e-3


@pytest.mark.parametrize("dtype,hkv,hd", [("bf16", 3, 128), ("f32", 2, 32), ("f32", 1, 96), ("f32", 1, 160),
                                          ("f32", 2, 256)])
def test_lists_move_alike_however_long_the_calls_list_is(dtype, hkv, hd):
    """Short and long lists, from bases anywhere in a block, with places that no block
    holds, in calls with room for little more than them and for many more."""
    rng = np.random.default_rng(hd)
    #        base, candidates, share kept
    cases = [(0, 40, 0.5), (37, 26, 0.3), (5, 1, 1.0), (16, 300, 0.7), (3, 64, 1.0), (8, 9, 0.0),
             (100, 200, 0.1), (15, 17, 0.5), (31, 290, 0.9), (2, 66, 1.0)]
    lens = [b + n for b, n, _ in cases]
    width, nb = 24, sum(-(-n // B) for n in lens) + 2
    c = Cache(dtype, hkv, hkv, hd, nb, width, n_layers=2, seed=9)
    table = tables(rng, lens, width, nb)
    whole = table.copy()
    table[3, 9], table[8, 3], table[8, 12] = -1, nb, -5
    for few in (True, False):
        rows = rng.permutation(len(cases))
        base = np.array([cases[r][0] for r in rows])
        kept = [cases[r][0] + np.nonzero(rng.random(cases[r][1]) < cases[r][2])[0] for r in rows]
        if few:
            kept = [k[:28] for k in kept]
        starts = np.concatenate([[0], np.cumsum([len(k) for k in kept])])
        listed = np.concatenate(kept)
        assert (len(listed) <= 32 * len(rows)) == few
        before = [c.tokens(layer) for layer in range(2)]
        for room in (len(listed), 40 * len(rows)) if few else (len(listed),):
            for layer in range(2):
                c.put(layer, *before[layer])
            coco.coco_kv_compact(c.h, 0, 2, i32(rows), i32(base),
                                 i32(np.concatenate([listed, np.full(max(room - len(listed), 0), 7)])),
                                 i32(starts), i32(table))
            torch.cuda.synchronize()
            for layer in range(2):
                for got, old in zip(c.tokens(layer), before[layer]):
                    want = old.copy()
                    for r, b, k in zip(rows, base, kept):
                        to = b + np.arange(len(k))
                        fine = (table[r, to // B] == whole[r, to // B]) & (table[r, k // B] == whole[r, k // B])
                        to, k = to[fine], k[fine]
                        want[table[r, to // B], to % B] = old[table[r, k // B], k % B]
                    assert np.array_equal(got, want), (few, room, layer)
