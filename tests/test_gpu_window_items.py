"""Window calls with more work than the card takes at once, and over long contexts: the
kernels' workgroups take several items, and lists pass what a wave holds of them."""
import numpy as np
import pytest
import torch

import paper_2607_04181_amd as coco
from cache_ref import B, i32, offsets
from window_ref import ALL, Rows, sees

pytestmark = pytest.mark.gpu


def poison(r, sequences):
    """NaN and infinities where no row of these sequences sees them."""
    ko, vo = offsets(r.c.hd)
    for s in sequences:
        t = np.arange(-(-int(r.lens[s]) // B) * B)
        seen = np.zeros(len(t), bool)
        for p in r.slots[r.seq == s]:
            seen |= sees(p, t, r.window, r.sinks)
        t = t[~seen]
        blocks = torch.from_numpy(r.table[s, t // B])[:, None, None].cuda()
        heads = torch.arange(r.c.hkv, device="cuda")[None, :, None]
        for pool, off, x in zip(r.c.pools[0], (ko, vo), (np.nan, (np.nan, np.inf)[s % 2])):
            pool[blocks, heads, torch.from_numpy(off[t % B])[:, None].cuda()] = x


def a_few_at_a_time(r, step):
    """The call's results from calls of `step` sequences."""
    o, w = torch.full_like(r.o, 7.0), torch.from_numpy(r.before).float().cuda()
    for s0 in range(0, len(r.lens), step):
        s1 = min(s0 + step, len(r.lens))
        at = slice(int(r.first[s0]), int(r.first[s1]))
        coco.coco_window_attention(r.c.h, 0, r.q[at], o[at], i32(r.first[s0:s1 + 1] - r.first[s0]),
                                   i32(r.table[s0:s1]), i32(r.lens[s0:s1]), r.window, r.sinks,
                                   w[s0:s1])
    torch.cuda.synchronize()
    return o, w


# 256 columns to an item of prompts and 16 of few rows, times eight key/value heads and parts:
# 912 items or more of prompts on 256 workgroups, 2400 of few rows on 512, and 2400 of the
# weights on 768.
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (300, 20)])
@pytest.mark.parametrize("kind", ["prompts", "few", "both"])
def test_many_items(kind, window, sinks):
    rng = np.random.default_rng(41)
    rows, lens = [], []
    if kind != "few":
        rows += [int(x) for x in rng.choice([70, 130, 257, 300, 515], 60)]
    if kind != "prompts":
        rows += [int(x) for x in rng.integers(1, 17, 300 if kind == "few" else 60)]
    rows = [rows[i] for i in rng.permutation(len(rows))]
    lens = [n + int(rng.integers(0, 700 if n > 16 else 200)) for n in rows]
    lens[1] = max(lens[1], 1900)
    r = Rows("bf16", 8, 8, 128, lens, rows, window, sinks, seed=26, poison=False)
    poison(r, range(0, len(lens), 3))
    o, w = a_few_at_a_time(r, 2)
    table, ctx = i32(r.table), i32(r.lens)
    first = torch.from_numpy(r.before).float().cuda()

    def call():
        coco.coco_window_attention(r.c.h, 0, r.q, r.o, r.starts, table, ctx, window, sinks, r.weights)

    def check():
        torch.cuda.synchronize()
        assert torch.isfinite(r.o).all() and torch.isfinite(r.weights).all()
        assert torch.equal(r.o, o) and torch.equal(r.weights, w)
        r.o.fill_(3.0)
        r.weights.copy_(first)

    call()
    check()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call()
    for _ in range(3):
        torch.cuda.synchronize()
        g.replay()
        check()
        call()
        check()


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 4, 1, 128), ("f32", 2, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (18000, 300)])
def test_single_tokens_of_long_contexts(dtype, hq, hkv, hd, window, sinks):
    r = Rows(dtype, hq, hkv, hd, [20005, 40, 17003], None, window, sinks, seed=27)
    r.run()
    r.check()


@pytest.mark.parametrize("dtype,hq,lens,rows", [
    ("bf16", 4, [9005, 20003], [8, 3]),        # few rows, in 16 parts
    ("bf16", 2, [20003, 9001], [40, 33]),      # up to 512 columns, in 16 parts
    ("bf16", 4, [9005], [135]),                # whole lists of more than 64 stages
    ("bf16", 4, [5003, 4499], [150, 140]),
    ("f32", 2, [9005, 17001], [4, 2]),
])
def test_prompts_of_long_contexts(dtype, hq, lens, rows):
    r = Rows(dtype, hq, 1, 128 if dtype == "bf16" else 64, lens, rows, ALL, 0, seed=28)
    r.run()
    r.check()
    o, w = r.o.clone(), r.weights.clone()
    # The same bits without the NaN behind the contexts, which makes items be done again.
    v = r.c.tokens()[1]
    k = np.nan_to_num(r.c.tokens()[0], nan=2.0)
    r.c.put(0, k, np.nan_to_num(v, nan=1.0, posinf=1.0, neginf=1.0))
    r.weights.copy_(torch.from_numpy(r.before))
    r.run()
    torch.cuda.synchronize()
    assert torch.equal(r.o, o) and torch.equal(r.weights, w)
