"""The cache's pages: allocation, forks, frees, copies and compaction, against
the same steps in Python."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, Cache, i32, tables

pytestmark = pytest.mark.gpu


def ref_take(refs, needs):
    """(ids of each request or None): lowest free blocks, in order until one
    does not fit; needs of None are not served and take nothing."""
    free = [i for i, r in enumerate(refs) if r == 0]
    out, at = [], 0
    for n in needs:
        if n is None:
            out.append(None)
            continue
        out.append([] if n == 0 else free[at:at + n] if at + n <= len(free) else None)
        at += n
    return out


def ref_alloc(table, refs, rows, lens):
    width = table.shape[1]
    ok = [0 <= r < len(table) and 0 <= n <= width * B for r, n in zip(rows, lens)]
    holes = [[b for b in range(-(-n // B)) if table[r, b] < 0] if k else None
             for r, n, k in zip(rows, lens, ok)]
    got = ref_take(refs, [None if h is None else len(h) for h in holes])
    for r, h, ids in zip(rows, holes, got):
        if ids is not None:
            table[r, h] = ids
            refs[ids] = 1
    return np.array([ids is not None for ids in got], np.int64)


def ref_fork(table, refs, src, dst, lens):
    got = ref_take(refs, [int(n % B != 0) for n in lens])
    copies = []
    for a, b, n, ids in zip(src, dst, lens, got):
        table[b] = -1
        if ids is None:
            continue
        full = n // B
        table[b, :full] = table[a, :full]
        np.add.at(refs, table[a, :full], 1)
        if ids:
            table[b, full] = ids[0]
            refs[ids[0]] = 1
            copies.append((table[a, full], ids[0]))
    return np.array([ids is not None for ids in got], np.int64), copies


def ref_free(table, refs, rows, keep):
    for r, n in zip(rows, keep):
        for b in range(-(-n // B), table.shape[1]):
            if table[r, b] >= 0:
                refs[table[r, b]] -= 1
                table[r, b] = -1


def same(dev, want):
    assert np.array_equal(dev.cpu().numpy().astype(np.int64), want)


def state(rng, lens, width, num_blocks, taken=0):
    """Table and counts: rows of the lengths, `taken` other blocks held elsewhere."""
    table = tables(rng, lens, width, num_blocks)
    refs = np.zeros(num_blocks, np.int64)
    np.add.at(refs, table[table >= 0], 1)
    free = np.nonzero(refs == 0)[0]
    refs[rng.permutation(free)[:taken]] = 1
    return table, refs


@pytest.mark.parametrize("seed", range(3))
@pytest.mark.parametrize("num_blocks,taken", [(400, 60), (60, 5), (30000, 29000)])
def test_alloc(num_blocks, taken, seed):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 60, size=24)
    lens[5] = 0
    width = 24
    if num_blocks == 60:
        lens //= 2
    table, refs = state(rng, lens, width, num_blocks, taken)
    table[3, 1:2] = -1  # a hole
    refs = np.zeros(num_blocks, np.int64) + (refs > 0)
    c = Cache("f32", 2, 1, 32, num_blocks, width)
    rows = rng.permutation(24)[:17]
    want = np.minimum(lens[rows] + rng.integers(0, 200, size=17), width * B)
    want[2] = 0
    dt, dr, status = i32(table), i32(refs), i32(np.full(17, 9))
    coco.coco_kv_alloc(c.h, i32(rows), i32(want), dt, dr, status)
    served = ref_alloc(table, refs, rows, want)
    if num_blocks == 60:
        assert 0 < served.sum() < len(served)
    same(status, served)
    same(dt, table)
    same(dr, refs)


def test_alloc_of_many_requests_and_rows_out_of_range():
    n, width, blocks = 1300, 3, 2500
    c = Cache("f32", 2, 1, 32, blocks, width, max_seqs=n)
    rng = np.random.default_rng(0)
    table, refs = state(rng, np.zeros(n, int), width, blocks, 200)
    rows, want = rng.permutation(n), rng.integers(0, 49, size=n)
    rows[7], rows[1200], want[11], want[12] = -1, n, 49, -3  # not served
    dt, dr, status = i32(table), i32(refs), i32(np.zeros(n))
    coco.coco_kv_alloc(c.h, i32(rows), i32(want), dt, dr, status)
    same(status, ref_alloc(table, refs, rows, want))
    same(dt, table)
    same(dr, refs)


def test_alloc_of_more_than_32_bits_of_blocks():
    """139 rows that ask for 2^24 blocks each: none is served, whatever their sum."""
    n, width, blocks = 140, 1 << 24, 40
    c = Cache("f32", 1, 1, 32, blocks, width, max_seqs=n)
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    lens = np.full(n, width * B)
    lens[0], lens[77] = 40, 0
    refs, status = i32(np.arange(blocks) % 2), i32(np.full(n, 9))
    coco.coco_kv_alloc(c.h, i32(np.arange(n)), i32(lens), table, refs, status)
    same(status, (lens <= 40).astype(np.int64))
    assert table[0, :4].tolist() == [0, 2, 4, -1]
    assert (table[1:] == -1).all() and (table[0, 3:] == -1).all()
    same(refs, np.isin(np.arange(blocks), [0, 2, 4]) | (np.arange(blocks) % 2))


@pytest.mark.parametrize("dtype,hkv,hd,layers", [("bf16", 2, 128, 3), ("f32", 1, 32, 1),
                                                 ("f32", 3, 96, 70), ("bf16", 8, 128, 1)])
@pytest.mark.parametrize("short", [False, True])
def test_fork_free_and_fork_again(dtype, hkv, hd, layers, short):
    rng = np.random.default_rng(layers)
    parents = np.array([1, 16, 17, 100, 0, 47, 160])
    width, n_child = 12, 12
    lens_all = np.concatenate([parents, np.zeros(n_child, int)])
    used = int((-(-parents // B)).sum())
    num_blocks = used + (4 if short else 20)
    c = Cache(dtype, 2 * hkv, hkv, hd, num_blocks, width, n_layers=layers, seed=1)
    table, refs = state(rng, lens_all, width, num_blocks)
    src = rng.integers(0, len(parents), size=n_child)
    dst = len(parents) + rng.permutation(n_child)
    lens = np.array([max(0, int(parents[s]) - int(rng.integers(0, 20))) for s in src])
    dt, dr, status = i32(table), i32(refs), i32(np.full(n_child, 9))
    pools = [[p.clone() for p in layer] for layer in c.pools]
    first, count = (1, layers - 1) if layers > 1 else (0, 1)
    for _ in range(2):
        coco.coco_kv_fork(c.h, first, count, i32(src), i32(dst), i32(lens), dt, dr, status)
        served, copies = ref_fork(table, refs, src, dst, lens)
        assert short == (not served.all())
        for layer in pools[first:first + count]:
            for p in layer:
                for a, b in copies:
                    p[b] = p[a]
        same(status, served)
        same(dt, table)
        same(dr, refs)
        for got, want in zip(c.pools, pools):
            assert all(torch.equal(g, w) for g, w in zip(got, want))
        # Some children shrink, the others go; one is named twice.
        keep = np.where(rng.random(n_child) < 0.5, lens // 2, 0)
        keep[0] = 0
        coco.coco_kv_free(c.h, i32(np.append(dst, dst[0])), i32(np.append(keep, 0)), dt, dr)
        ref_free(table, refs, np.append(dst, dst[0]), np.append(keep, 0))
        same(dt, table)
        same(dr, refs)
        coco.coco_kv_free(c.h, i32(dst), None, dt, dr)
        ref_free(table, refs, dst, np.zeros(n_child, int))
        same(dt, table)
        same(dr, refs)


@pytest.mark.parametrize("dtype,hkv,hd", [("bf16", 3, 128), ("f32", 2, 32)])
def test_copy(dtype, hkv, hd):
    c = Cache(dtype, hkv, hkv, hd, 40, 2, n_layers=2, seed=2)
    want = [[p.clone() for p in layer] for layer in c.pools]
    perm = np.random.default_rng(2).permutation(40)
    src, dst = perm[:13].copy(), perm[13:26].copy()
    src[4], src[5], dst[6] = src[3], 400, -1  # a source twice; pairs outside the pools
    coco.coco_kv_copy(c.h, 1, 1, i32(src), i32(dst))
    for p in want[1]:
        for a, b in zip(src, dst):
            if 0 <= a < 40 and 0 <= b < 40:
                p[b] = p[a].clone()
    for got, w in zip(c.pools, want):
        assert all(torch.equal(x, y) for x, y in zip(got, w))


@pytest.mark.parametrize("dtype,hkv,hd,layers", [("bf16", 2, 128, 2), ("f32", 1, 32, 1),
                                                 ("f32", 2, 160, 1), ("f32", 1, 256, 1),
                                                 ("bf16", 1, 128, 65)])
def test_compact(dtype, hkv, hd, layers):
    rng = np.random.default_rng(hd)
    #        base, candidates, share kept
    cases = [(0, 40, 0.5), (37, 26, 0.3), (5, 1, 1.0), (16, 300, 0.7), (3, 64, 1.0), (8, 9, 0.0),
             (100, 200, 0.1), (15, 17, 0.5)]
    lens = [b + n for b, n, _ in cases]
    width, num_blocks = 24, sum(-(-n // B) for n in lens) + 2
    c = Cache(dtype, hkv, hkv, hd, num_blocks, width, n_layers=layers, seed=3)
    table = tables(rng, lens, width, num_blocks)
    rows = rng.permutation(len(cases))
    base = np.array([cases[r][0] for r in rows])
    kept = [cases[r][0] + np.nonzero(rng.random(cases[r][1]) < cases[r][2])[0] for r in rows]
    starts = np.concatenate([[0], np.cumsum([len(k) for k in kept])])
    before = [c.tokens(l) for l in range(layers)]
    coco.coco_kv_compact(c.h, 0, layers, i32(rows), i32(base), i32(np.concatenate(kept)),
                         i32(starts), i32(table))
    torch.cuda.synchronize()
    for l in range(layers):
        for got, old in zip(c.tokens(l), before[l]):
            want = old.copy()
            for r, b, k in zip(rows, base, kept):
                to = b + np.arange(len(k))
                want[table[r, to // B], to % B] = old[table[r, k // B], k % B]
            assert np.array_equal(got, want), l


def test_a_fork_of_a_row_into_itself_is_not_served():
    """Its row and counts are as if it had not been made, the others' served."""
    rng = np.random.default_rng(8)
    width, num_blocks = 6, 30
    c = Cache("f32", 2, 1, 32, num_blocks, width, seed=8)
    table, refs = state(rng, np.array([40, 33, 0, 0]), width, num_blocks)
    dt, dr, status = i32(table), i32(refs), i32(np.full(3, 9))
    pools = [p.clone() for p in c.pools[0]]
    src, dst, lens = [0, 1, 1], [2, 1, 3], [37, 20, 33]
    coco.coco_kv_fork(c.h, 0, 1, i32(src), i32(dst), i32(lens), dt, dr, status)
    served, copies = ref_fork(table, refs, [0, 1], [2, 3], [37, 33])
    same(status, np.array([served[0], 0, served[1]]))
    same(dt, table)
    same(dr, refs)
    for got, want in zip(c.pools[0], pools):
        for a, b in copies:
            want[b] = want[a]
        assert torch.equal(got, want)


def test_graph_replay_of_a_speculative_step():
    """Trim, alloc and fork captured once and replayed: integers and pools as
    the eager run's every time."""
    rng = np.random.default_rng(4)
    lens = np.array([30, 77, 5, 0, 0, 0])
    width, num_blocks = 10, 60
    c = Cache("bf16", 4, 2, 128, num_blocks, width, n_layers=2, seed=4)
    table, refs = state(rng, lens, width, num_blocks, 11)
    dt, dr = i32(table), i32(refs)
    status, status2 = i32(np.zeros(3)), i32(np.zeros(3))
    src, dst, cut, grown = i32([0, 1, 1]), i32([3, 4, 5]), i32([29, 64, 70]), i32([50, 100, 90])

    def step():
        coco.coco_kv_free(c.h, dst, None, dt, dr)
        coco.coco_kv_fork(c.h, 0, 2, src, dst, cut, dt, dr, status)
        coco.coco_kv_alloc(c.h, dst, grown, dt, dr, status2)

    step()
    torch.cuda.synchronize()
    ref_fork(table, refs, [0, 1, 1], [3, 4, 5], [29, 64, 70])
    ref_alloc(table, refs, [3, 4, 5], [50, 100, 90])
    same(dt, table)
    want = [t.clone() for t in (dt, dr, status, status2)] + [p.clone() for l in c.pools for p in l]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    scratch = torch.empty(1 << 20, device="cuda")
    for _ in range(3):
        scratch.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [dt, dr, status, status2] + [p for l in c.pools for p in l]
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_validation_of_arrays_that_fit_no_memory_is_an_error():
    """n_seqs of a table that no host could copy: an error code, no abort."""
    c = Cache("f32", 1, 1, 32, 4, 1 << 22)
    coco.coco_layer_set_validate(c.h, True)
    one, table, refs = i32([0]), i32(np.full(64, -1)), i32(np.zeros(4))
    rc = coco._lib.raw_call("coco_kv_free", c.h.raw, one.data_ptr(), None, 1, table.data_ptr(),
                            2 ** 31 - 1, refs.data_ptr(), None)
    assert rc == coco._lib.COCO_ENOMEM and "host memory" in coco.coco_last_error()


def test_refusals():
    c = Cache("bf16", 4, 2, 128, 20, 4, n_layers=2, max_seqs=3)
    table, refs = i32(np.full((5, 4), -1)), i32(np.zeros(20))
    table[0, 0], refs[0] = 7, 0
    refs[7] = 1
    one, status = i32([1]), i32([9])
    h = c.h
    with pytest.raises(coco.CocoError, match="max_seqs"):
        coco.coco_kv_alloc(h, i32([0, 1, 2, 3]), i32([1] * 4), table, refs, i32([0] * 4))
    with pytest.raises(coco.CocoError, match="layers"):
        coco.coco_kv_fork(h, 1, 2, i32([0]), one, i32([4]), table, refs, status)
    with pytest.raises(coco.CocoError, match="layers"):
        coco.coco_kv_copy(h, 0, 0, one, i32([2]))
    with pytest.raises(ValueError, match="ref_counts"):
        coco.coco_kv_free(h, one, None, table, refs[:19])
    with pytest.raises(ValueError, match="kept_starts"):
        coco.coco_kv_compact(h, 0, 1, one, one, one, one, table)
    nothing = i32([])
    coco.coco_kv_alloc(h, nothing, nothing, table, refs, nothing)
    coco.coco_kv_free(h, nothing, None, table, refs)
    coco.coco_kv_copy(h, 0, 2, nothing, nothing)
    coco.coco_kv_compact(h, 0, 2, nothing, nothing, nothing, i32([0]), table)
    coco.coco_kv_compact(h, 0, 2, one, one, nothing, i32([0, 0]), table)
    coco.coco_layer_set_validate(h, True)
    before = [t.clone() for t in (table, refs)]
    for call, text in (
            (lambda: coco.coco_kv_alloc(h, i32([1, 1]), i32([1, 1]), table, refs, i32([0, 0])),
             "duplicate"),
            (lambda: coco.coco_kv_alloc(h, one, i32([65]), table, refs, status), "length"),
            (lambda: coco.coco_kv_fork(h, 0, 2, i32([0]), i32([0]), i32([4]), table, refs, status),
             "parent and a child"),
            (lambda: coco.coco_kv_fork(h, 0, 2, i32([2]), i32([1]), i32([4]), table, refs, status),
             "block_table"),
            (lambda: coco.coco_kv_fork(h, 0, 2, i32([2]), i32([0]), i32([0]), table, refs, status),
             "still holds"),
            (lambda: coco.coco_kv_copy(h, 0, 2, i32([1, 2]), i32([2, 3])), "from and to"),
            (lambda: coco.coco_kv_copy(h, 0, 2, i32([1]), i32([20])), "dst_blocks"),
            (lambda: coco.coco_kv_free(h, i32([5]), None, table, refs), "sequence"),
            (lambda: coco.coco_kv_free(h, i32([0]), None, table, i32(np.zeros(20))), "reference"),
            (lambda: coco.coco_kv_compact(h, 0, 2, i32([0]), i32([3]), i32([2]), i32([0, 1]),
                                          table), "ascending"),
            (lambda: coco.coco_kv_compact(h, 0, 2, i32([0]), i32([3]), i32([17]), i32([0, 1]),
                                          table), "block_table")):
        with pytest.raises(coco.CocoError, match=text):
            call()
    assert torch.equal(table, before[0]) and torch.equal(refs, before[1])
    coco.coco_kv_fork(h, 0, 2, i32([0]), one, i32([4]), table, refs, status)
    assert int(status[0]) == 1 and int(table[1, 0]) == 0
