"""Operators for contexts that outgrow their cache as performance cases: attention
over a sliding window and a context's first tokens, of single tokens and of
prompts; the same with each key's softmax weights added up; and eviction of the
tokens with the least of them.

Where `own` is false, `run` computes a case from elementary torch operations in
32 bits, rounded once at the end; where it is true, it makes the calls that a
serving program makes of the library. Both work on the same state: the pools in
the library's tile layout, block tables, index arrays, and the handle.

Case fields (all plain values):
  kind    "window" or "evict"
  heads   a key of HEADS
  seqs    requests in the call
  median, sigma, top   lognormal distribution of the cached context lengths
          (clipped to top)
  lens    seed of the length draws (lengths belong to the case, values to the seed)
  rows    window: most new tokens of a request; 0: one token of each, as decode rows
  window, sinks   window: newest and first tokens that a row sees
  weigh   window: whether the keys' weights are added up
  layers  evict: layers of the handle
  budget  evict: tokens that a longer request keeps
  first, last   evict: how many of those are its first and last
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 16
ALL = 2 ** 31 - 1  # a window that no context fills

# (query heads, key/value heads, head_dim, dtype, longest context): the head
# layouts and context limits of the layer shapes in cases.py.
HEADS = {
    "tiny": (4, 2, 64, "f32", 1024),
    "small_f32": (16, 4, 64, "f32", 4096),
    "8b": (32, 8, 128, "bf16", 16400),
    "32b": (40, 8, 128, "bf16", 8208),
    "70b": (64, 8, 128, "bf16", 32784),
}


def listed():
    return [
        # One request, one token: the latency of the call.
        dict(name="window_8b_1", kind="window", heads="8b", seqs=1, rows=0, window=1024, sinks=4,
             weigh=False, median=2500, sigma=0.1, top=8192, lens=1),
        # fp32 reference runs of a small model, token by token.
        dict(name="window_f32_5", kind="window", heads="small_f32", seqs=5, rows=0, window=300,
             sinks=2, weigh=False, median=800, sigma=0.7, top=4000, lens=2),
        # The ordinary decode batch of a model with a window, uneven contexts,
        # some of them shorter than the window.
        dict(name="window_8b_64", kind="window", heads="8b", seqs=64, rows=0, window=4096, sinks=4,
             weigh=False, median=6000, sigma=0.6, top=16000, lens=3),
        # Few requests with long contexts and a window that takes in half of them.
        dict(name="window_70b_4_long", kind="window", heads="70b", seqs=4, rows=0, window=16000,
             sinks=16, weigh=False, median=30000, sigma=0.05, top=32000, lens=4),
        # fp32 prompts, odd lengths.
        dict(name="window_f32_3x77", kind="window", heads="small_f32", seqs=3, rows=77, window=130,
             sinks=1, weigh=False, median=400, sigma=0.6, top=2000, lens=5),
        # Chunks of four prompts over what is cached of them, window shorter than both.
        dict(name="window_32b_4x512", kind="window", heads="32b", seqs=4, rows=512, window=1000,
             sinks=4, weigh=False, median=2000, sigma=0.8, top=7000, lens=6),
        # One long prompt from its start.
        dict(name="window_8b_1x8000", kind="window", heads="8b", seqs=1, rows=8000, window=4096,
             sinks=4, weigh=False, median=1, sigma=0.1, top=2, lens=7),
        # fp32 decode that keeps count of its weights.
        dict(name="weigh_f32_3", kind="window", heads="small_f32", seqs=3, rows=0, window=ALL,
             sinks=0, weigh=True, median=500, sigma=0.7, top=3000, lens=8),
        # The ordinary decode batch that keeps count.
        dict(name="weigh_8b_64", kind="window", heads="8b", seqs=64, rows=0, window=ALL, sinks=0,
             weigh=True, median=2000, sigma=0.7, top=8000, lens=9),
        # The last tokens of prompts, whose weights say what of the prompt to keep.
        dict(name="weigh_8b_16x64", kind="window", heads="8b", seqs=16, rows=64, window=ALL,
             sinks=0, weigh=True, median=4000, sigma=0.6, top=14000, lens=10),
        # A few fp32 requests cut back: the latency of the calls.
        dict(name="evict_f32_4", kind="evict", heads="small_f32", seqs=4, layers=2, budget=200,
             first=2, last=40, median=280, sigma=0.3, top=1000, lens=11),
        # A batch whose contexts grew past their budget since the last time.
        dict(name="evict_8b_64", kind="evict", heads="8b", seqs=64, layers=4, budget=2000, first=4,
             last=500, median=2200, sigma=0.15, top=4000, lens=12),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    what = rng.choice(["decode", "decode", "decode", "prompt", "prompt", "prompt", "evict"])
    heads = rng.choice(["8b", "8b", "32b", "70b", "small_f32", "tiny"])
    hq, _, _, dtype, longest = HEADS[heads]
    f32 = dtype == "f32"
    c = dict(kind="window", heads=heads, lens=rng.randrange(1 << 30),
             sigma=round(rng.uniform(0.05, 0.8), 3))
    if what == "evict":
        c.update(kind="evict", seqs=log_int(1, 64), layers=rng.randrange(1, 5))
        top = min(longest - 2 * BLOCK, 300_000 // (c["seqs"] * c["layers"]), 8000)
        c.update(median=log_int(20, max(21, top // 2)))
        c.update(top=max(c["median"] + 1, top))
        c.update(budget=max(4, int(c["median"] * rng.uniform(0.5, 1.1))))
        c.update(first=rng.randrange(0, min(8, c["budget"] // 4) + 1))
        c.update(last=rng.randrange(0, c["budget"] // 2 + 1))
        return c
    c.update(weigh=rng.random() < 0.4)
    if what == "decode":
        c.update(seqs=log_int(1, 16 if f32 else 64), rows=0)
        top = min(longest - 2 * BLOCK, 350_000 // c["seqs"])
    else:
        c.update(seqs=log_int(1, 16), rows=log_int(2, 256 if f32 else 4000))
        # New tokens times query heads times keys of a request, over the call.
        most = (20_000_000 if f32 else 700_000_000) // (c["seqs"] * hq)
        c.update(rows=max(2, min(c["rows"], int(math.sqrt(most)) // 2)))
        top = max(1, min(longest - 2 * BLOCK, most // c["rows"]) - c["rows"])
    c.update(median=log_int(1, max(2, top // 2)))
    c.update(top=max(c["median"] + 1, top))
    c.update(window=ALL if rng.random() < 0.25 else log_int(1, max(2, min(8192, top))),
             sinks=rng.choice([0, 1, 4, rng.randrange(0, 100)]))
    return c


# ----------------------------------------------------------------------------
# Lengths of a case (from the case alone)
# ----------------------------------------------------------------------------


def _lengths(c):
    """(cached tokens of each request with the call's, how many of them are the call's)."""
    rng = np.random.default_rng(c["lens"])
    x = rng.lognormal(math.log(c["median"]), c["sigma"], size=c["seqs"])
    ctx = np.clip(np.floor(x), 1, c["top"]).astype(np.int64)
    if not c.get("rows"):
        return ctx, np.ones(c["seqs"], np.int64)
    news = rng.integers(max(1, c["rows"] // 2), c["rows"] + 1, size=c["seqs"])
    news[0] = c["rows"]
    return ctx + news, news


def _seen_counts(c, ctx, news):
    """(sum over rows of the keys they see, keys that any row of a request sees)."""
    pairs, union = 0, 0
    for n, new in zip(ctx.tolist(), news.tolist()):
        p = np.arange(n - new, n)
        lo = np.maximum(0, p + 1 - min(c["window"], n))
        pairs += int((p + 1 - lo + np.minimum(c["sinks"], lo)).sum())
        union += n - int(lo[0]) + min(c["sinks"], int(lo[0]))
    return pairs, union


def _evicted(c, ctx):
    """Per request: tokens above its budget."""
    return np.maximum(ctx - c["budget"], 0)


def prepare(case, seed):
    c = case
    hq, hkv, hd, dtype, longest = HEADS[c["heads"]]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)

    def normal(*shape, sigma=1.0):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, sigma, generator=gen)

    def i32(a):
        return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()

    ctx, news = _lengths(c)
    n_layers, width = c.get("layers", 1), -(-longest // BLOCK)
    need = -(-ctx // BLOCK)
    # evict: the rows hold pages up to their budgets, the call gets those behind.
    held = np.minimum(need, -(-c["budget"] // BLOCK)) if c["kind"] == "evict" else need
    used, extra = int(held.sum()), int((need - held).sum())
    # Blocks of other requests lie between: a seventh more than are used.
    n_blocks = used + extra + (used + extra) // 7 + 1
    perm = rng.permutation(n_blocks)
    table = np.full((c["seqs"], width), -1, np.int64)
    at = np.concatenate([[0], np.cumsum(held)])
    for s in range(c["seqs"]):
        table[s, :held[s]] = perm[at[s]:at[s + 1]]
    layers = [{"k_cache": normal(n_blocks, hkv, BLOCK * hd), "v_cache": normal(n_blocks, hkv, BLOCK * hd)}
              for _ in range(n_layers)]
    st = {"case": c, "layers": layers, "longest": int(ctx.max()), "block_table": i32(table),
          "ctx_lens": i32(ctx), "news": int(news.max())}
    n_rows = int(news.sum())
    if c["kind"] == "evict" or c["weigh"]:
        # What earlier steps added up: a few heavy tokens, many light ones.
        w = torch.empty(c["seqs"], width * BLOCK, device="cuda").exponential_(generator=gen) ** 3
        st["weights"] = torch.where(torch.arange(width * BLOCK, device="cuda")[None] <
                                    st["ctx_lens"][:, None], w, 0.0)
    if c["kind"] == "evict":
        refs = np.zeros(n_blocks, np.int64)
        refs[perm[:used]] = 1
        refs[perm[used + extra:]] = 1
        n = c["seqs"]
        st.update(ref_counts=i32(refs), status=i32(np.zeros(n)), seqs=i32(np.arange(n)),
                  keep_lens=i32(np.full(n, c["budget"])), new_lens=i32(np.zeros(n)),
                  base_lens=i32(np.zeros(n)), kept_starts=i32(np.zeros(n + 1)),
                  kept=i32(np.full(n * c["budget"], -1)))
    else:
        if c["rows"]:
            st["seq_starts"] = i32(np.concatenate([[0], np.cumsum(news)]))
        # Queries that prefer some keys: logits of a few units.
        st["q"] = normal(n_rows, hq, hd, sigma=1.5)
        st["o"] = torch.empty(n_rows, hq, hd, dtype=dt, device="cuda")
    if own:
        st["handle"] = _handle(st, n_rows, c["seqs"], width)
    return st


# ----------------------------------------------------------------------------
# The library's calls
# ----------------------------------------------------------------------------


def _handle(st, n_rows, n_seqs, width):
    """A replica's handle over the pools. The operators read no weights of the
    layers, so the projections are as narrow as a handle takes."""
    import paper_2607_04181_amd as coco
    c = st["case"]
    hq, hkv, hd, dtype, _ = HEADS[c["heads"]]
    d = 128
    dt = st["layers"][0]["k_cache"].dtype

    def zeros(*shape):
        return torch.zeros(shape, dtype=dt, device="cuda")

    layers = [dict(w, w_qkv=zeros((hq + 2 * hkv) * hd, d), w_o=zeros(d, hq * hd),
                   w_gate_up=zeros(2 * d, d), w_down=zeros(d, d), gamma_attn=zeros(d),
                   gamma_mlp=zeros(d)) for w in st["layers"]]
    cfg = coco.make_config(d, hq, hkv, hd, d, len(layers), dtype, n_rows, n_seqs, width, 1.0e4, 1e-6)
    h = coco.coco_layer_init(cfg, layers)
    if c["kind"] == "window":
        coco.coco_window_reserve(h, n_rows, n_seqs, c["weigh"])
    return h


def _run_own(st):
    import paper_2607_04181_amd as coco
    c, h, table = st["case"], st["handle"], st["block_table"]
    if c["kind"] == "window":
        coco.coco_window_attention(h, 0, st["q"], st["o"], st.get("seq_starts"), table,
                                   st["ctx_lens"], c["window"], c["sinks"], st.get("weights"))
        return
    seqs, refs = st["seqs"], st["ref_counts"]
    coco.coco_kv_alloc(h, seqs, st["ctx_lens"], table, refs, st["status"])
    coco.coco_kv_evict(h, seqs, st["keep_lens"], c["first"], c["last"], st["ctx_lens"], st["weights"],
                       st["new_lens"], st["base_lens"], st["kept"], st["kept_starts"])
    coco.coco_kv_compact(h, 0, len(st["layers"]), seqs, st["base_lens"], st["kept"],
                         st["kept_starts"], table)
    coco.coco_kv_free(h, seqs, st["new_lens"], table, refs)


# ----------------------------------------------------------------------------
# The plain forms
# ----------------------------------------------------------------------------


def _k_view(pool, hkv, hd):  # [block, head, dim / 32, dim % 32 / 8, slot, dim % 8]
    return pool.view(-1, hkv, hd // 32, 4, BLOCK, 8)


def _v_view(pool, hkv, hd):  # [block, head, dim / 32, slot / 4, dim % 16, dim % 32 / 16, slot % 4]
    return pool.view(-1, hkv, hd // 32, 4, 16, 2, 4)


def _window_plain(st):
    c = st["case"]
    hq, hkv, hd, _, _ = HEADS[c["heads"]]
    w, n, nb = st["layers"][0], st["news"], -(-st["longest"] // BLOCK)
    ctx, dev = st["ctx_lens"].long(), st["q"].device
    s, g, keys = len(ctx), hq // hkv, nb * BLOCK
    starts = st["seq_starts"].long() if c["rows"] else torch.arange(s + 1, device=dev)
    blk = st["block_table"][:, :nb].long().clamp(min=0)
    k = _k_view(w["k_cache"], hkv, hd)[blk]  # [request, block, head, ...]
    k = k.permute(0, 2, 1, 5, 3, 4, 6).reshape(s, hkv, keys, hd).float()
    v = _v_view(w["v_cache"], hkv, hd)[blk]
    v = v.permute(0, 2, 1, 4, 7, 3, 6, 5).reshape(s, hkv, keys, hd).float()
    row = starts[:-1, None] + torch.arange(n, device=dev)[None]
    live = row < starts[1:, None]
    # [request, head, new token, query head of the group, key]
    q = st["q"][row.clamp(max=len(st["q"]) - 1)].float().view(s, n, hkv, g, hd).transpose(1, 2)
    z = torch.matmul(q.reshape(s, hkv, n * g, hd), k.transpose(-1, -2)).div_(math.sqrt(hd))
    slot = (ctx - (starts[1:] - starts[:-1]))[:, None] + torch.arange(n, device=dev)[None]
    t = torch.arange(keys, device=dev)
    seen = (t <= slot[..., None]) & ((t > slot[..., None] - c["window"]) | (t < c["sinks"]))
    seen = (seen & live[..., None])[:, None, :, None]
    z = z.view(s, hkv, n, g, keys).masked_fill_(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = z.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total == 0, 1.0, total))
    o = torch.matmul(p.view(s, hkv, n * g, keys), v).view(s, hkv, n, g, hd).transpose(1, 2)
    out = torch.cat([st["o"], st["o"][:1]])  # a row past the end takes the padding
    out[torch.where(live, row, len(st["o"]))] = o.reshape(s, n, hq, hd).to(out.dtype)
    st["o"].copy_(out[:-1])
    if c["weigh"]:
        st["weights"][:, :keys] += p.sum((1, 2, 3))


def _evict_plain(st):
    c = st["case"]
    hq, hkv, hd, _, _ = HEADS[c["heads"]]
    table, refs, weights = st["block_table"], st["ref_counts"], st["weights"]
    ctx, keep, dev = st["ctx_lens"].long(), st["keep_lens"].long(), weights.device
    # Pages of the new tokens: the lowest free blocks in order, for the requests
    # that come before the first that does not fit.
    entry = torch.arange(table.shape[1], device=dev)[None]
    want = (table < 0) & (entry < ((ctx + BLOCK - 1) // BLOCK)[:, None])
    free = torch.argsort((refs != 0).to(torch.int8), stable=True)
    rank = torch.cumsum(want.view(-1).long(), 0).view(want.shape)
    served = (rank[:, -1] <= (refs == 0).sum()) | ~want.any(1)
    ids = free[(rank - 1).clamp(0, len(refs) - 1)]
    taken = want & served[:, None]
    refs.index_add_(0, ids.view(-1), taken.view(-1).to(refs.dtype))
    table.copy_(torch.where(taken, ids.to(torch.int32), table))
    st["status"].copy_(served)
    # What each request keeps.
    t = torch.arange(weights.shape[1], device=dev)[None]
    live = t < ctx[:, None]
    always = (t < c["first"]) | (t >= (ctx - c["last"])[:, None])
    score = torch.where(live, torch.where(always, math.inf, weights), -math.inf)
    order = torch.sort(score, dim=1, descending=True, stable=True)[1]
    place = torch.empty_like(order).scatter_(1, order, t.expand_as(order).contiguous())
    cut = (ctx > keep)[:, None]
    stays = live & ((place < keep[:, None]) | ~cut)
    new = torch.minimum(ctx, keep)
    base = torch.where(stays, weights.shape[1], t.expand_as(stays)).amin(1)
    base = torch.where(cut[:, 0], base, ctx)
    moves = stays & (t >= base[:, None])
    count = moves.sum(1)
    starts = torch.cumsum(count, 0) - count
    to = torch.cumsum(moves.long(), 1) - 1  # place behind base
    listed = torch.where(moves, starts[:, None] + to, st["kept"].numel())
    kept = torch.cat([st["kept"], st["kept"].new_zeros(1)])
    kept[listed.view(-1)] = t.expand_as(listed).reshape(-1).to(torch.int32)
    st["kept"].copy_(kept[:-1])
    st["kept_starts"].copy_(torch.cat([starts, starts[-1:] + count[-1:]]))
    st["new_lens"].copy_(new)
    st["base_lens"].copy_(base)
    # Their weights, keys and values move up behind the base.
    spare = weights.shape[1]
    dest = torch.where(moves, base[:, None] + to, spare)
    moved = torch.where(t < base[:, None], weights, 0.0)
    moved = torch.cat([torch.where(cut, moved, weights), weights.new_zeros(len(ctx), 1)], 1)
    moved.scatter_(1, dest, weights)
    weights.copy_(moved[:, :-1])
    # Each place takes the token that moves there, or its own; places past the
    # context repeat what the first one takes.
    src = torch.cat([t.expand_as(dest), dest[:, :1]], 1).scatter(1, dest, t.expand_as(dest))
    dst = torch.where(live, t, 0)[:, :st["longest"]]
    src = torch.where(live, src[:, :-1], src[:, :1])[:, :st["longest"]]
    rows = torch.arange(len(ctx), device=dev)[:, None].expand_as(dst)
    b0, s0 = table[rows, src // BLOCK].long(), src % BLOCK
    b1, s1 = table[rows, dst // BLOCK].long(), dst % BLOCK
    for w in st["layers"]:
        kp, vp = _k_view(w["k_cache"], hkv, hd), _v_view(w["v_cache"], hkv, hd)
        kp[b1, :, :, :, s1] = kp[b0, :, :, :, s0]
        vp[b1, :, :, s1 // 4, :, :, s1 % 4] = vp[b0, :, :, s0 // 4, :, :, s0 % 4]
    # Pages behind the budgets.
    drop = (table >= 0) & (entry >= ((new + BLOCK - 1) // BLOCK)[:, None])
    refs.index_add_(0, table.clamp(min=0).view(-1).long(), -drop.view(-1).to(refs.dtype))
    table.copy_(torch.where(drop, -1, table))


def run(st):
    c = st["case"]
    if own:
        _run_own(st)
    else:
        {"window": _window_plain, "evict": _evict_plain}[c["kind"]](st)
    if c["kind"] == "window":
        return {"o": st["o"], "weights": st["weights"]} if c["weigh"] else {"o": st["o"]}
    out = {x: st[x] for x in ("block_table", "ref_counts", "status", "new_lens", "base_lens",
                              "kept", "kept_starts", "weights")}
    return dict(out, k_cache=[w["k_cache"] for w in st["layers"]],
                v_cache=[w["v_cache"] for w in st["layers"]])


# ----------------------------------------------------------------------------
# Work, and the results in 64 bits
# ----------------------------------------------------------------------------


def work(case):
    c = case
    hq, hkv, hd, dtype, _ = HEADS[c["heads"]]
    eb = 2 if dtype == "bf16" else 4
    ctx, news = _lengths(c)
    token = 2 * hkv * hd * eb
    if c["kind"] == "window":
        pairs, union = _seen_counts(c, ctx, news)
        return {"bytes": union * (token + (8 if c["weigh"] else 0)) + int(news.sum()) * 2 * hq * hd * eb +
                4 * int((-(-ctx // BLOCK)).sum()),
                "flops": 4 * hq * hd * pairs}
    # At most every kept token moves; those before the first evicted one do not. A
    # token among the rest is evicted about evenly: one in a few is the first.
    cut = _evicted(c, ctx)
    kept = int(np.where(cut > 0, np.minimum(ctx, c["budget"]) - c["first"], 0).sum())
    pages = int((-(-ctx // BLOCK)).sum() - (-(-np.minimum(ctx, c["budget"]) // BLOCK)).sum())
    return {"bytes": kept * (2 * token * c["layers"] + 8) + 8 * int(np.where(cut > 0, ctx, 0).sum()) +
            16 * pages, "flops": 0}


def _offsets(hd):
    """Where dimension h of slot t lies in a key tile and in a value tile, [16, hd]."""
    t, h = torch.arange(BLOCK)[:, None], torch.arange(hd)[None]
    k = ((h // 32) * 64 + (h % 32) // 8 * 16 + t) * 8 + h % 8
    v = (((h // 32) * 64 + t // 4 * 16 + h % 16) * 2 + (h // 16) % 2) * 4 + t % 4
    return k.cuda(), v.cuda()


def _tokens64(pool, blocks, offsets, n):
    """A request's first n tokens in 64 bits, [head, token, dim]."""
    x = pool[blocks].double()
    x = x[:, :, offsets.reshape(-1)].view(x.shape[0], x.shape[1], *offsets.shape)
    return x.transpose(0, 1).reshape(x.shape[1], -1, offsets.shape[1])[:, :n].contiguous()


def exact(case, seed):
    c = case
    if c["kind"] == "evict":
        return None  # bytes are moved, or whole numbers computed
    hq, hkv, hd, _, _ = HEADS[c["heads"]]
    st = prepare(c, seed)
    ctx, news = _lengths(c)
    ko, vo = _offsets(hd)
    first = np.concatenate([[0], np.cumsum(news)])
    o = torch.zeros(st["o"].shape, dtype=torch.float64, device="cuda")
    weights = st["weights"].double() if c["weigh"] else None
    for s in range(c["seqs"]):
        n, new = int(ctx[s]), int(news[s])
        blocks = st["block_table"].long()[s, :-(-n // BLOCK)]
        k, v = (_tokens64(st["layers"][0][x], blocks, off, n)
                for x, off in (("k_cache", ko), ("v_cache", vo)))
        q = st["q"][int(first[s]):int(first[s]) + new].double()
        for r0 in range(0, new, 1024):  # (a square of long prompts in pieces)
            p = torch.arange(n - new + r0, n - new + min(new, r0 + 1024), device="cuda")[:, None]
            t = torch.arange(n, device="cuda")[None]
            hidden = (t > p) | ((t <= p - c["window"]) & (t >= c["sinks"]))
            for h in range(hq):
                z = (q[r0:r0 + 1024, h] @ k[h * hkv // hq].T) * hd ** -0.5
                a = torch.nan_to_num(torch.softmax(z.masked_fill(hidden, -math.inf), -1), 0.0)
                o[int(first[s]) + r0:int(first[s]) + r0 + len(p), h] = a @ v[h * hkv // hq]
                if c["weigh"]:
                    weights[s, :n] += a.sum(0)
    return {"o": o, "weights": weights} if c["weigh"] else {"o": o}
