"""Attention through a window and a context's first tokens, with and without the
sums of its weights, against 64 bits: single tokens and prompts."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, i32
from window_ref import ALL, Rows

pytestmark = pytest.mark.gpu

HEADS = [("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("bf16", 16, 1, 128), ("bf16", 3, 3, 128),
         ("f32", 4, 2, 64), ("f32", 3, 1, 32), ("f32", 20, 1, 96), ("f32", 9, 9, 160),
         ("f32", 2, 2, 256)]
SHOWN = [(1, 0), (1, 3), (16, 1), (17, 16), (100, 20), (512, 5), (200, 5000), (ALL, 0), (ALL, 7)]
LENS = [0, 1, 15, 16, 17, 33, 300, 511, 513, 700]


@pytest.mark.parametrize("window,sinks", SHOWN)
@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS[:3] + HEADS[4:6])
def test_single_tokens(dtype, hq, hkv, hd, window, sinks):
    r = Rows(dtype, hq, hkv, hd, LENS, None, window, sinks, seed=1)
    r.run()
    r.check()


@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS)
def test_single_tokens_of_every_head_layout(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [40, 1, 1700], None, 600, 18, seed=2)
    r.run()
    r.check()


def test_single_tokens_without_weights_give_the_same_output():
    r = Rows("bf16", 8, 2, 128, [1300, 40, 9], None, 1000, 4, seed=3)
    r.run()
    ref = r.o.clone()
    weights, r.weights = r.weights, None
    before = weights.clone()
    r.o.fill_(7.0)
    r.run()
    torch.cuda.synchronize()
    assert torch.equal(r.o, ref) and torch.equal(weights, before)


# (cached tokens with the call's, the call's)
PROMPTS = [(1, 1), (17, 17), (45, 40), (333, 33), (0, 0), (700, 1), (170, 130), (16, 2), (259, 3)]


@pytest.mark.parametrize("window,sinks", SHOWN)
@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS[:3] + HEADS[4:5])
def test_prompts(dtype, hq, hkv, hd, window, sinks):
    r = Rows(dtype, hq, hkv, hd, *zip(*PROMPTS), window, sinks, seed=4, pad=3)
    r.run()
    r.check()


@pytest.mark.parametrize("dtype,hq,hkv,hd", HEADS)
def test_prompts_of_every_head_layout(dtype, hq, hkv, hd):
    r = Rows(dtype, hq, hkv, hd, [200, 90, 20], [150, 31, 20], 75, 18, seed=5)
    r.run()
    r.check()


@pytest.mark.parametrize("window,sinks,lens,rows", [
    (ALL, 0, [2600, 1100, 1030], [3, 64, 1]),      # lists in parts
    (1500, 40, [2600, 300], [70, 300]),
    (ALL, 0, [1400], [1400]),                      # many tiles, in one part
    (130, 1, [1400, 5], [1300, 5]),
    (40, 700, [1500, 640], [900, 640]),            # first tokens wider than the window
    (300, 0, [2100], [2100]),
])
def test_long_prompts(window, sinks, lens, rows):
    r = Rows("bf16", 4, 1, 128, lens, rows, window, sinks, seed=6)
    r.run()
    r.check()


@pytest.mark.parametrize("window,sinks,lens,rows", [
    (ALL, 0, [1400, 9], [1400, 9]),
    (130, 1, [1100, 5], [1000, 5]),
    (40, 300, [700], [650]),
])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 1, 64), (5, 1, 32)])
def test_long_prompts_of_f32(hq, hkv, hd, window, sinks, lens, rows):
    r = Rows("f32", hq, hkv, hd, lens, rows, window, sinks, seed=17)
    r.run()
    r.check()


FEW = [(2000, 16), (700, 17), (1100, 1), (33, 5), (520, 12), (9, 9), (3, 2)]


@pytest.mark.parametrize("window,sinks", [(ALL, 0), (100, 20), (17, 0), (600, 3)])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 2), (5, 1), (16, 1)])
def test_sequences_of_few_rows(hq, hkv, window, sinks):
    """Up to 64 columns and just above, in one call and each in its own, padded."""
    r = Rows("bf16", hq, hkv, 128, *zip(*FEW), window, sinks, seed=18, pad=2)
    r.run()
    r.check()
    ref, tol = r.expect()[:2]
    for s, (n, rows) in enumerate(FEW):
        at = slice(int(r.first[s]), int(r.first[s + 1]))
        for pad in (0, 1, 40):
            q = torch.cat([r.q[at], r.q[:1].expand(pad, -1, -1)])
            o = torch.full_like(q, 5.0)
            w = torch.from_numpy(r.before[s:s + 1]).float().cuda()
            coco.coco_window_reserve(r.c.h, rows + pad, 1, True)
            coco.coco_window_attention(r.c.h, 0, q, o, i32([0, rows]), i32(r.table[s:s + 1]),
                                       i32(r.lens[s:s + 1]), window, sinks, w)
            torch.cuda.synchronize()
            assert (o[rows:] == 5.0).all()
            if (rows + pad) * (hq // hkv) <= 64 or rows * (hq // hkv) > 64:
                assert torch.equal(o[:rows], r.o[at]) and torch.equal(w[0], r.weights[s])
            else:  # of one kind by the call's rows: within the bound of the exact result too
                assert (np.abs(o[:rows].cpu().double().numpy() - ref[at]) <= tol[at]).all()


def test_rows_before_the_context_see_nothing():
    # More rows than cached tokens: those without a slot.
    for dtype, hd in (("bf16", 128), ("f32", 64)):
        r = Rows(dtype, 4, 1, hd, [3, 20], [8, 4], 10, 2, seed=7)
        r.run()
        r.check()
        assert (r.o[:5] == 0).all()


@pytest.mark.parametrize("rows", [None, [90], [20]])
@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(dtype, hd, rows):
    r = Rows(dtype, 4, 2, hd, [200], rows, 40, 6, seed=8, weigh=False, poison=False)
    k, v = r.c.tokens()
    places = {120: np.inf, 150: -np.inf, 170: np.nan, 199: np.inf, 3: -np.inf, 60: np.nan, 155: np.inf}
    for t, x in places.items():
        v[r.table[0, t // B], t % B, :, t % 7::9] = x
    v[r.table[0, 155 // B], 155 % B, :, 150 % 7::9] = np.inf  # beside -inf of another key
    r.c.put(0, k, v)
    r.run()
    torch.cuda.synchronize()
    got = r.o.cpu().double().numpy()
    q = r.q.cpu().double().numpy()
    for i, p in enumerate(r.slots):
        t = np.array([x for x in range(p + 1) if x > p - 40 or x < 6])
        kk, vv = k[r.table[0, t // B], t % B], v[r.table[0, t // B], t % B]
        for h in range(4):
            z = kk[:, h // 2] @ q[i, h] / np.sqrt(hd)
            w = np.exp(z - z.max())
            with np.errstate(invalid="ignore"):
                ref = (w[:, None] / w.sum() * vv[:, h // 2]).sum(0)
            fine = np.isfinite(ref)
            assert np.array_equal(np.isfinite(got[i, h]), fine), (i, h)
            odd = ~fine
            assert np.array_equal(got[i, h][odd], ref[odd], equal_nan=True), (i, h)
            assert np.abs(got[i, h][fine] - ref[fine]).max() < 0.05


def test_scores_that_are_not_finite():
    # A key of -inf scores is left out (0 weight); a row of nothing but such gives zeros.
    r = Rows("f32", 2, 1, 32, [5, 40], None, 3, 0, seed=9, poison=False)
    k, v = r.c.tokens()
    r.q.fill_(1.0)
    k[r.table[0, 0], 2:5] = -np.inf
    k[r.table[1, 39 // B], 39 % B] = -np.inf
    r.c.put(0, k, v)
    r.run()
    torch.cuda.synchronize()
    assert (r.o[0] == 0).all() and torch.isfinite(r.o).all()
    w = r.weights.cpu().double().numpy() - r.before
    assert np.abs(w[0]).max() < 1e-6 and np.abs(w[1].sum() - 2) < 1e-5 and abs(w[1, 39]) < 1e-6


@pytest.mark.parametrize("dtype,hq,hkv,hd", [HEADS[0], HEADS[4]])
@pytest.mark.parametrize("rows", [None, [100, 3, 40, 17]])
def test_any_split_of_the_sequences_gives_the_same_bits(dtype, hq, hkv, hd, rows):
    r = Rows(dtype, hq, hkv, hd, [1300, 20, 600, 70], rows, 900, 10, seed=10)
    r.run()
    torch.cuda.synchronize()
    weights = torch.from_numpy(r.before).float().cuda()
    for part in ([2], [0, 3], [1]):
        at = np.concatenate([np.arange(r.first[s], r.first[s + 1]) for s in part])
        q, o = r.q[at].contiguous(), torch.empty(len(at), hq, hd, dtype=r.q.dtype, device="cuda")
        starts = None if rows is None else i32(np.concatenate([[0], np.cumsum(r.news[part])]))
        w = weights[part].contiguous()
        coco.coco_window_attention(r.c.h, 0, q, o, starts, i32(r.table[part]), i32(r.lens[part]),
                                   900, 10, w)
        torch.cuda.synchronize()
        assert torch.equal(o, r.o[at]) and torch.equal(w, r.weights[part])


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("rows", [None, [60, 5]])
def test_captured_calls_replay_as_they_ran(dtype, hd, rows):
    r = Rows(dtype, 8, 2, hd, [1200, 77], rows, 700, 4, seed=11)
    table, lens = i32(r.table), i32(r.lens)

    def call():
        coco.coco_window_attention(r.c.h, 0, r.q, r.o, r.starts, table, lens, 700, 4, r.weights)

    first = torch.from_numpy(r.before).float().cuda()
    call()
    torch.cuda.synchronize()
    o, w = r.o.clone(), r.weights.clone()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
    for _ in range(4):
        r.o.fill_(3.0)
        r.weights.copy_(first)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(r.o, o) and torch.equal(r.weights, w)
        call()  # eager between replays
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 32)])
def test_many_sequences(dtype, hd):
    # More than a launch of the prompts' kernel takes.
    lens = [(7 * s) % 40 + 3 for s in range(1500)]
    r = Rows(dtype, 2, 1, hd, lens, [1 + s % 3 for s in range(1500)], 12, 2, seed=12)
    r.run()
    r.check()


def test_rows_of_more_weight_groups_than_reserved_are_refused():
    r = Rows("bf16", 4, 1, 128, [30, 40], None, 10, 0, seed=13, weigh=False)
    w = torch.zeros(2, r.table.shape[1] * B, device="cuda")
    with pytest.raises(coco.CocoError, match="no room for weights") as e:
        coco.coco_window_attention(r.c.h, 0, r.q, r.o, None, i32(r.table), i32(r.lens), 10, 0, w)
    assert e.value.code == -4
    coco.coco_window_reserve(r.c.h, 2, 2, True)
    coco.coco_window_attention(r.c.h, 0, r.q, r.o, None, i32(r.table), i32(r.lens), 10, 0, w)
    torch.cuda.synchronize()
    assert abs(float(w.sum()) - 2 * 4) < 1e-4


def test_validation_mode_names_what_is_wrong():
    r = Rows("bf16", 4, 1, 128, [100, 40], [5, 3], 20, 4, seed=14, weigh=False)
    coco.coco_layer_set_validate(r.c.h, True)
    r.run()
    r.check()  # table entries that nobody reaches are not looked at
    for change, text in (({"table": (0, 5, -1)}, "block_table"), ({"lens": (1, 2)}, "3 rows in 2"),
                         ({"starts": [0, 6, 5]}, "monotone"), ({"starts": [1, 5, 8]}, "run from 0")):
        table, lens, starts = r.full.copy(), r.lens.copy(), r.first.copy()
        if "table" in change:
            s, b, x = change["table"]
            table[s, b] = x
        if "lens" in change:
            lens[change["lens"][0]] = change["lens"][1]
        if "starts" in change:
            starts = np.array(change["starts"])
        with pytest.raises(coco.CocoError, match=text):
            coco.coco_window_attention(r.c.h, 0, r.q, r.o, i32(starts), i32(table), i32(lens), 20, 4)


def test_pools_past_4_gib():
    # Blocks whose offsets pass 32 bits (elements and bytes).
    nb = 2 ** 31 // (8 * B * 128) + 64
    k, v = (torch.empty(nb, 8, B * 128, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    r = Rows("bf16", 8, 8, 128, [100], [20], 50, 4, seed=15, poison=False)
    used = np.arange(nb - 8, nb)
    for big, small in zip((k, v), r.c.pools[0]):
        big[torch.from_numpy(used[:7])] = small[torch.from_numpy(r.table[0, :7])]
    from cache_ref import Cache
    c = Cache("bf16", 8, 8, 128, nb, r.c.max_blocks, max_rows=20, pools=[(k, v)])
    coco.coco_window_reserve(c.h, 20, 1, True)
    table = np.full((1, r.c.max_blocks), -1)
    table[0, :7] = used[:7]
    r.run()
    for starts, rows in ((r.starts, slice(0, 20)), (None, slice(19, 20))):
        o = torch.empty_like(r.o[rows])
        w = torch.from_numpy(r.before).float().cuda()
        coco.coco_window_attention(c.h, 0, r.q[rows].contiguous(), o, starts, i32(table), i32([100]),
                                   50, 4, w)
        torch.cuda.synchronize()
        if starts is not None:
            assert torch.equal(o, r.o) and torch.equal(w, r.weights)
        else:
            assert (o - r.o[rows]).abs().max() < 0.05
