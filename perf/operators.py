"""The operators on a replica's paged cache as performance cases: attention for
trees of drafted tokens, the cache's pages (allocate, fork, free, compact), and
attention over the blocks that a cheap score selects.

Where `own` is false, `run` computes a case from elementary torch operations in
32 bits, rounded once at the end; where it is true, it makes the calls that a
serving program makes of the library. Both work on the same state: the pools in
the library's tile layout, block tables, index arrays, and the handle.

Case fields (all plain values):
  kind    "tree", "fork", "verify", "summarize" or "sparse"
  heads   a key of HEADS
  seqs    requests in the call (fork: parents)
  median, sigma, top   lognormal distribution of the cached context lengths
          (clipped to top)
  lens    seed of the length draws (lengths belong to the case, values to the seed)
  nodes   tree, verify: most drafted tokens of a request
  layers  fork, verify: layers of the handle
  forks   fork: children
  blocks, first, last  sparse: blocks a row attends, and how many of them are
          always the context's first and last
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 16

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
        # One request, one token, no draft: the latency of the call.
        dict(name="tree_8b_1x1", kind="tree", heads="8b", seqs=1, nodes=1, median=1024, sigma=0.1,
             top=8192, lens=1),
        # fp32 reference runs of a small model with short drafts.
        dict(name="tree_f32_3x13", kind="tree", heads="small_f32", seqs=3, nodes=13, median=300,
             sigma=0.6, top=2000, lens=2),
        # One request over a long document, a full tree each step.
        dict(name="tree_70b_1x61_long", kind="tree", heads="70b", seqs=1, nodes=61, median=30000,
             sigma=0.05, top=32000, lens=3),
        # The ordinary speculative batch: small ragged trees, uneven contexts.
        dict(name="tree_8b_64x26", kind="tree", heads="8b", seqs=64, nodes=26, median=2048,
             sigma=0.8, top=12000, lens=4),
        # Wide trees on the largest heads: the products are the work.
        dict(name="tree_70b_32x64", kind="tree", heads="70b", seqs=32, nodes=64, median=4096,
             sigma=0.5, top=16000, lens=5),
        # A few beams of one small model branch: launches and the block search.
        dict(name="fork_f32_4", kind="fork", heads="small_f32", layers=2, seqs=2, forks=4,
             median=200, sigma=0.7, top=1000, lens=6),
        # Parallel samples of many prompts: children replace the last step's.
        dict(name="fork_8b_256", kind="fork", heads="8b", layers=4, seqs=32, forks=256,
             median=1024, sigma=0.8, top=8192, lens=7),
        # The cache side of a speculative step: pages for the drafts, append,
        # and the accepted path moved up.
        dict(name="verify_8b_64x26", kind="verify", heads="8b", layers=4, seqs=64, nodes=26,
             median=1024, sigma=0.8, top=8192, lens=8),
        # The summaries of prompts just prefilled.
        dict(name="summarize_8b_16", kind="summarize", heads="8b", seqs=16, median=3000, sigma=0.6,
             top=12000, lens=9),
        # fp32 with few blocks.
        dict(name="sparse_f32_5", kind="sparse", heads="small_f32", seqs=5, median=1500, sigma=0.7,
             top=4000, blocks=24, first=1, last=2, lens=10),
        # One request over a long document.
        dict(name="sparse_70b_1_long", kind="sparse", heads="70b", seqs=1, median=30000, sigma=0.05,
             top=32000, blocks=128, first=1, last=4, lens=11),
        # A decode batch over long contexts.
        dict(name="sparse_8b_96_long", kind="sparse", heads="8b", seqs=96, median=10000, sigma=0.4,
             top=16000, blocks=128, first=1, last=4, lens=12),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["tree", "tree", "tree", "fork", "verify", "summarize", "sparse", "sparse"])
    heads = rng.choice(["8b", "8b", "32b", "70b", "small_f32", "tiny"])
    hq, _, _, dtype, longest = HEADS[heads]
    c = dict(kind=kind, heads=heads, lens=rng.randrange(1 << 30), sigma=round(rng.uniform(0.1, 0.8), 3))
    f32 = dtype == "f32"
    if kind == "tree":
        c.update(seqs=log_int(1, 16 if f32 else 64), nodes=log_int(1, 32 if f32 else 64))
        most = 300_000 * 32 // (hq * c["nodes"]) if f32 else 8_000_000 * 32 // (hq * c["nodes"])
    elif kind == "fork":
        c.update(seqs=log_int(1, 32), layers=rng.randrange(1, 5))
        c.update(forks=c["seqs"] * log_int(1, 8))
        most = 80_000
    elif kind == "verify":
        c.update(seqs=log_int(1, 64), nodes=log_int(1, 64), layers=rng.randrange(1, 5))
        most = 80_000
    elif kind == "summarize":
        c.update(seqs=log_int(1, 16))
        most = 80_000
    else:
        c.update(seqs=log_int(1, 96), blocks=log_int(4, 128))
        c.update(first=rng.randrange(0, 3), last=rng.randrange(0, min(8, c["blocks"] - 2)))
        most = 1_000_000
    top = min(longest - 2 * BLOCK - c.get("nodes", 0), 16000 if heads != "70b" else 32000)
    c.update(median=log_int(16, max(17, min(top // 2, most // c["seqs"] // 2))))
    c.update(top=max(c["median"] + 1, min(top, most // c["seqs"])))
    return c


# ----------------------------------------------------------------------------
# Lengths and shapes of a case (from the case alone)
# ----------------------------------------------------------------------------


def _lengths(c):
    """(cached tokens of each request before the call, its drafted tokens)."""
    rng = np.random.default_rng(c["lens"])
    x = rng.lognormal(math.log(c["median"]), c["sigma"], size=c["seqs"])
    ctx = np.clip(np.floor(x), 1, c["top"]).astype(np.int64)
    if "nodes" not in c:
        return ctx, np.zeros(c["seqs"], np.int64)
    news = rng.integers(max(1, c["nodes"] // 2), c["nodes"] + 1, size=c["seqs"])
    news[0] = c["nodes"]
    return ctx, news


def _trees(c, news):
    """[request, node, node]: whether a node sees another (its path up to the
    root, and itself); parents are drawn among the eight nodes before."""
    rng = np.random.default_rng(c["lens"] + 1)
    n = int(news.max())
    back = rng.integers(1, 9, size=(len(news), n))
    sees = np.zeros((len(news), n, n), bool)
    every = np.arange(len(news))
    for j in range(n):
        parent = j - back[:, j]
        has = parent >= 0
        sees[has, j] = sees[every[has], parent[has]]
        sees[:, j, j] = True
    return sees & (np.arange(n)[None, None] < news[:, None, None])


def _kept(c, news):
    """Accepted nodes of each request: an ascending path of its nodes."""
    rng = np.random.default_rng(c["lens"] + 2)
    take = rng.random((len(news), int(news.max()))) < 0.3
    return take & (np.arange(take.shape[1])[None] < news[:, None])


def _forks(c, ctx):
    """(parent, child row, shared length) of each fork."""
    rng = np.random.default_rng(c["lens"] + 3)
    src = np.arange(c["forks"]) % c["seqs"]
    # Most children branch at the end of their parent, some further back.
    cut = np.where(rng.random(c["forks"]) < 0.75, 0, rng.integers(0, 48, size=c["forks"]))
    return src, c["seqs"] + np.arange(c["forks"]), np.maximum(1, ctx[src] - cut)


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
    # The tree's drafted tokens are in the cache; verify gets their pages in the call.
    cached = ctx + news if c["kind"] == "tree" else ctx
    need = -(-cached // BLOCK)
    used = int(need.sum())
    extra = c.get("forks", 0) + (int((-(-(ctx + news) // BLOCK) - need).sum())
                                 if c["kind"] == "verify" else 0)
    # Blocks of other requests lie between: a seventh more than are used.
    n_blocks = used + extra + (used + extra) // 7 + 1
    perm = rng.permutation(n_blocks)
    rows = c["seqs"] + c.get("forks", 0)
    table = np.full((rows, width), -1, np.int64)
    at = np.concatenate([[0], np.cumsum(need)])
    for s in range(c["seqs"]):
        table[s, :need[s]] = perm[at[s]:at[s + 1]]
    refs = np.zeros(n_blocks, np.int64)
    refs[perm[:used]] = 1
    refs[perm[used + extra:]] = 1
    layers = [{"k_cache": normal(n_blocks, hkv, BLOCK * hd), "v_cache": normal(n_blocks, hkv, BLOCK * hd)}
              for _ in range(n_layers)]
    st = {"case": c, "layers": layers, "longest": int(cached.max()), "block_table": i32(table),
          "ref_counts": i32(refs), "ctx_lens": i32(cached), "news": int(news.max())}
    n_rows = c["seqs"]
    if c["kind"] == "tree":
        n_rows = int(news.sum())
        sees = _trees(c, news)
        words = -(-sees.shape[1] // 64)
        bits = np.zeros((c["seqs"], sees.shape[1], words * 64), bool)
        bits[:, :, :sees.shape[1]] = sees
        packed = np.packbits(bits, axis=-1, bitorder="little").view(np.int64)
        packed = packed[np.arange(sees.shape[1])[None] < news[:, None]]
        st["tree_mask"] = torch.from_numpy(packed).cuda()
        st["seq_starts"] = i32(np.concatenate([[0], np.cumsum(news)]))
    elif c["kind"] == "fork":
        src, dst, lens = _forks(c, ctx)
        st.update(src_seq=i32(src), dst_seq=i32(dst), lens=i32(lens), status=i32(np.zeros(len(src))))
    elif c["kind"] == "verify":
        n_rows = int(news.sum())
        seq = np.repeat(np.arange(c["seqs"]), news)
        first = np.concatenate([[0], np.cumsum(news)])
        kept = _kept(c, news)
        s, j = np.nonzero(kept)
        st.update(seqs=i32(np.arange(c["seqs"])), base_lens=i32(ctx), draft_lens=i32(ctx + news),
                  seq_idx=i32(seq), positions=i32(ctx[seq] + np.arange(n_rows) - first[seq]),
                  kept=i32(ctx[s] + j), status=i32(np.zeros(c["seqs"])),
                  kept_starts=i32(np.concatenate([[0], np.cumsum(kept.sum(1))])),
                  k=[normal(n_rows, hkv, hd) for _ in range(n_layers)],
                  v=[normal(n_rows, hkv, hd) for _ in range(n_layers)])
    else:
        # The pages' summaries; the sparse cases' are those of all keys but the
        # newest, whose block they bring up to date.
        st["summary"] = torch.zeros(n_blocks, hkv, 2, hd, dtype=torch.int8, device="cuda")
        st["scales"] = torch.zeros(n_blocks, hkv, device="cuda")
        if c["kind"] == "sparse":
            _summarize_plain(st, torch.zeros_like(st["ctx_lens"]), st["ctx_lens"].clamp(min=2) - 1,
                             -(-int(ctx.max()) // BLOCK))
            st["positions"] = i32(ctx - 1)
            st["selected"] = torch.empty(c["seqs"], hkv, c["blocks"], dtype=torch.int32, device="cuda")
    if c["kind"] in ("tree", "sparse"):
        # Queries that prefer some keys: logits of a few units.
        st["q"] = normal(n_rows, hq, hd, sigma=1.5)
        st["o"] = torch.empty(n_rows, hq, hd, dtype=dt, device="cuda")
    if own:
        st["handle"] = _handle(st, n_rows, rows, width)
    return st


# ----------------------------------------------------------------------------
# The library's calls
# ----------------------------------------------------------------------------


def _handle(st, n_rows, n_seqs, width):
    """A replica's handle over the pools. The operators read no weights, so
    the layers' projections are as narrow as a handle takes."""
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
    if c["kind"] == "tree":
        coco.coco_tree_reserve(h, n_rows, n_seqs)
    elif c["kind"] == "sparse":
        coco.coco_sparse_reserve(h, n_rows, c["blocks"])
    return h


def _run_own(st):
    import paper_2607_04181_amd as coco
    c, h, table, refs = st["case"], st["handle"], st["block_table"], st["ref_counts"]
    n_layers = len(st["layers"])
    if c["kind"] == "tree":
        coco.coco_tree_attention(h, 0, st["q"], st["o"], st["seq_starts"], table, st["ctx_lens"],
                                 st["tree_mask"])
    elif c["kind"] == "fork":
        coco.coco_kv_free(h, st["dst_seq"], None, table, refs)
        coco.coco_kv_fork(h, 0, n_layers, st["src_seq"], st["dst_seq"], st["lens"], table, refs,
                          st["status"])
    elif c["kind"] == "verify":
        coco.coco_kv_free(h, st["seqs"], st["base_lens"], table, refs)
        coco.coco_kv_alloc(h, st["seqs"], st["draft_lens"], table, refs, st["status"])
        for layer in range(n_layers):
            coco.coco_kv_append(h, layer, st["k"][layer], st["v"][layer], st["seq_idx"],
                                st["positions"], table)
        coco.coco_kv_compact(h, 0, n_layers, st["seqs"], st["base_lens"], st["kept"],
                             st["kept_starts"], table)
    elif c["kind"] == "summarize":
        coco.coco_kv_summarize(h, 0, st["summary"], st["scales"], None, st["ctx_lens"], table)
    else:
        coco.coco_kv_summarize(h, 0, st["summary"], st["scales"], st["positions"], st["ctx_lens"],
                               table)
        coco.coco_block_select(h, st["summary"], st["scales"], st["q"], st["positions"], None,
                               table, st["ctx_lens"], c["first"], c["last"], st["selected"])
        coco.coco_sparse_attention(h, 0, st["q"], st["o"], st["positions"], None, table,
                                   st["ctx_lens"], st["selected"])


# ----------------------------------------------------------------------------
# The plain forms
# ----------------------------------------------------------------------------


def _k_view(pool, hkv, hd):  # [block, head, dim / 32, dim % 32 / 8, slot, dim % 8]
    return pool.view(-1, hkv, hd // 32, 4, BLOCK, 8)


def _v_view(pool, hkv, hd):  # [block, head, dim / 32, slot / 4, dim % 16, dim % 32 / 16, slot % 4]
    return pool.view(-1, hkv, hd // 32, 4, 16, 2, 4)


def _k_blocks(pool, hkv, hd, blk, heads):
    """Keys of blocks blk at heads, [*blk.shape, slot, dim] in 32 bits."""
    x = _k_view(pool, hkv, hd)[blk, heads]
    n = x.dim()
    return x.permute(*range(n - 4), n - 2, n - 4, n - 3, n - 1).reshape(*x.shape[:-4], BLOCK, hd).float()


def _v_blocks(pool, hkv, hd, blk, heads):
    x = _v_view(pool, hkv, hd)[blk, heads]
    n = x.dim()
    return x.permute(*range(n - 5), n - 4, n - 1, n - 5, n - 2, n - 3) \
            .reshape(*x.shape[:-5], BLOCK, hd).float()


def _softmax_product(z, seen, v):
    """softmax of z over the keys that are seen, times v; 0 where there are none."""
    z = torch.where(seen, z, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    return torch.where(total == 0, 0.0, torch.matmul(p, v) / total)


def _tree_plain(st):
    hq, hkv, hd, _, _ = HEADS[st["case"]["heads"]]
    w, n, nb = st["layers"][0], st["news"], -(-st["longest"] // BLOCK)
    starts, ctx = st["seq_starts"].long(), st["ctx_lens"].long()
    s, dev = len(ctx), ctx.device
    blk = st["block_table"][:, :nb].long().clamp(min=0)[:, None].expand(s, hkv, nb)
    heads = torch.arange(hkv, device=dev)[None, :, None].expand(s, hkv, nb)
    k = _k_blocks(w["k_cache"], hkv, hd, blk, heads).view(s, hkv, nb * BLOCK, hd)
    v = _v_blocks(w["v_cache"], hkv, hd, blk, heads).view(s, hkv, nb * BLOCK, hd)
    row = (starts[:-1, None] + torch.arange(n, device=dev)[None])
    live = row < starts[1:, None]
    at = row.clamp(max=len(st["q"]) - 1)
    # [request, head, node, query head of the group, key]
    q = st["q"][at].float().view(s, n, hkv, hq // hkv, hd).transpose(1, 2)
    z = torch.matmul(q.reshape(s, hkv, -1, hd), k.transpose(-1, -2)) / math.sqrt(hd)
    prefix = ctx - (starts[1:] - starts[:-1])
    node = torch.arange(nb * BLOCK, device=dev)[None] - prefix[:, None]
    inside = (node >= 0) & (node < (ctx - prefix)[:, None])
    node = node.clamp(0, 64 * st["tree_mask"].shape[1] - 1)[:, None].expand(s, n, nb * BLOCK)
    words = torch.gather(st["tree_mask"][at], 2, node >> 6)
    seen = ((words >> (node & 63)) & 1).bool() & inside[:, None]
    seen = seen | (torch.arange(nb * BLOCK, device=dev)[None] < prefix[:, None])[:, None]
    seen = seen[:, None, :, None].expand(s, hkv, n, hq // hkv, nb * BLOCK).reshape(z.shape)
    o = _softmax_product(z, seen, v).view(s, hkv, n, hq // hkv, hd).transpose(1, 2)
    out = torch.cat([st["o"], st["o"][:1]])  # a row past the end takes the padding
    out[torch.where(live, row, len(st["o"]))] = o.reshape(s, n, hq, hd).to(out.dtype)
    st["o"].copy_(out[:-1])


def _free_plain(table, refs, rows, keep):
    part = table[rows]
    drop = (part >= 0) & (torch.arange(part.shape[1], device=part.device)[None] >=
                          ((keep + BLOCK - 1) // BLOCK)[:, None])
    refs.index_add_(0, part.clamp(min=0).view(-1).long(), -drop.view(-1).to(refs.dtype))
    table[rows] = torch.where(drop, -1, part)


def _lowest_free(refs, want, n):
    """For each wanted place (row-major) the lowest free blocks in order, and
    whether its request (a row) is served: in order, until one does not fit."""
    order = torch.argsort((refs != 0).to(torch.int8), stable=True)
    rank = torch.cumsum(want.view(-1).long(), 0).view(want.shape)
    served = (rank[:, -1] <= (refs == 0).sum()) | ~want.any(1)
    ids = order[(rank - 1).clamp(0, n - 1)]
    return ids, served


def _fork_plain(st):
    hq, hkv, hd, _, _ = HEADS[st["case"]["heads"]]
    table, refs = st["block_table"], st["ref_counts"]
    src, dst, lens = st["src_seq"].long(), st["dst_seq"].long(), st["lens"].long()
    _free_plain(table, refs, dst, torch.zeros_like(lens))
    entry = torch.arange(table.shape[1], device=table.device)[None]
    tail = (lens % BLOCK != 0)[:, None]
    ids, served = _lowest_free(refs, tail, len(refs))
    shared = (entry < (lens // BLOCK)[:, None]) & served[:, None]
    is_tail = (entry == (lens // BLOCK)[:, None]) & tail & served[:, None]
    part = table[src]
    refs.index_add_(0, part.clamp(min=0).view(-1).long(), shared.view(-1).to(refs.dtype))
    copied = tail[:, 0] & served
    spare = len(refs)  # a place past the pool takes what is not served
    more = torch.cat([refs, refs.new_zeros(1)])
    more[torch.where(copied, ids[:, 0], spare)] = 1
    refs.copy_(more[:spare])
    table[dst] = torch.where(shared, part, torch.where(is_tail, ids.to(torch.int32), -1))
    st["status"].copy_(served)
    # Forks that are not served copy the first parent's block to itself.
    old = torch.gather(part, 1, (lens // BLOCK).clamp(max=table.shape[1] - 1)[:, None])[:, 0].long()
    old = torch.where(copied, old, part[0, 0].long())
    new = torch.where(copied, ids[:, 0], part[0, 0].long())
    for w in st["layers"]:
        w["k_cache"][new] = w["k_cache"][old]
        w["v_cache"][new] = w["v_cache"][old]


def _verify_plain(st):
    hq, hkv, hd, _, _ = HEADS[st["case"]["heads"]]
    table, refs = st["block_table"], st["ref_counts"]
    rows, base, lens = st["seqs"].long(), st["base_lens"].long(), st["draft_lens"].long()
    _free_plain(table, refs, rows, base)
    entry = torch.arange(table.shape[1], device=table.device)[None]
    want = (table[rows] < 0) & (entry < ((lens + BLOCK - 1) // BLOCK)[:, None])
    ids, served = _lowest_free(refs, want, len(refs))
    taken = want & served[:, None]
    refs.index_add_(0, ids.view(-1), taken.view(-1).to(refs.dtype))
    table[rows] = torch.where(taken, ids.to(torch.int32), table[rows])
    st["status"].copy_(served)
    seq, pos = st["seq_idx"].long(), st["positions"].long()
    blk, slot = table[seq, pos // BLOCK].long(), pos % BLOCK
    kept, starts = st["kept"].long(), st["kept_starts"].long()
    of = torch.searchsorted(starts, torch.arange(len(kept), device=kept.device), right=True) - 1
    to = base[of] + torch.arange(len(kept), device=kept.device) - starts[of]
    b0, s0 = table[rows[of], kept // BLOCK].long(), kept % BLOCK
    b1, s1 = table[rows[of], to // BLOCK].long(), to % BLOCK
    for w, k, v in zip(st["layers"], st["k"], st["v"]):
        kp, vp = _k_view(w["k_cache"], hkv, hd), _v_view(w["v_cache"], hkv, hd)
        kp[blk, :, :, :, slot] = k.view(len(seq), hkv, hd // 32, 4, 8)
        vp[blk, :, :, slot // 4, :, :, slot % 4] = v.view(len(seq), hkv, hd // 32, 2, 16).transpose(-1, -2)
        kp[b1, :, :, :, s1] = kp[b0, :, :, :, s0]
        vp[b1, :, :, s1 // 4, :, :, s1 % 4] = vp[b0, :, :, s0 // 4, :, :, s0 % 4]


def _exponent(amax):
    """x with amax < 2^x, within [-100, 100]."""
    return torch.frexp(amax)[1].clamp(-100, 100)


def _summarize_plain(st, first, ctx, n):
    """The summaries of the blocks that hold tokens first .. ctx - 1, at most n of a request."""
    _, hkv, hd, _, _ = HEADS[st["case"]["heads"]]
    dev = ctx.device
    entry = (first // BLOCK).long()[:, None] + torch.arange(n, device=dev)[None]
    entry = torch.where(BLOCK * entry < ctx[:, None], entry, entry[:, :1])  # past the end: the first again
    left = ctx[:, None] - BLOCK * entry
    blk = torch.gather(st["block_table"], 1, entry).long()
    k = _k_blocks(st["layers"][0]["k_cache"], hkv, hd, blk[:, :, None].expand(-1, -1, hkv),
                  torch.arange(hkv, device=dev)[None, None].expand(*blk.shape, hkv))
    k = torch.where(torch.isfinite(k), k, 0.0)
    filled = (torch.arange(BLOCK, device=dev) < left[:, :, None])[:, :, None, :, None]
    hi = torch.where(filled, k, -math.inf).amax(-2)
    lo = torch.where(filled, k, math.inf).amin(-2)
    x = _exponent(torch.maximum(hi.abs(), lo.abs()).amax(-1))
    up = torch.ldexp(torch.ones((), device=dev), 7 - x)[..., None]
    both = torch.stack([torch.ceil(hi * up), torch.floor(lo * up)], -2).clamp(-127, 127)
    st["summary"][blk] = both.to(torch.int8)
    st["scales"][blk] = torch.ldexp(torch.ones((), device=dev), x - 7)


def _prompts_plain(st):
    _summarize_plain(st, torch.zeros_like(st["ctx_lens"]), st["ctx_lens"], -(-st["longest"] // BLOCK))


def _sparse_plain(st):
    c = st["case"]
    hq, hkv, hd, _, _ = HEADS[c["heads"]]
    w, top = st["layers"][0], c["blocks"]
    _summarize_plain(st, st["positions"], st["ctx_lens"], 1)
    ctx, pos = st["ctx_lens"].long(), st["positions"].long()
    keys = torch.minimum(ctx, pos + 1)
    nb = -(-st["longest"] // BLOCK)
    s, dev = len(ctx), ctx.device
    q = st["q"].float().view(s, hkv, hq // hkv, hd)
    fine = torch.where(torch.isfinite(q), q, 0.0)
    x = _exponent(fine.abs().amax((-1, -2), keepdim=True))
    q8 = torch.round(fine * torch.ldexp(torch.ones((), device=dev), 7 - x)).clamp(-127, 127)
    blk = st["block_table"][:, :nb].long().clamp(min=0)
    both = st["summary"][blk].permute(0, 2, 1, 3, 4).float()  # [row, head, block, hi / lo, dim]
    # Sums of at most 256 products of bytes: whole numbers below 2^23, exact.
    dots = torch.matmul(q8.clamp(min=0), both[:, :, :, 0].transpose(-1, -2)) + \
        torch.matmul(q8.clamp(max=0), both[:, :, :, 1].transpose(-1, -2))
    score = dots.amax(2) * st["scales"][blk].transpose(1, 2)
    entry = torch.arange(max(nb, top), device=dev)
    have = ((keys + BLOCK - 1) // BLOCK)[:, None, None]
    score = torch.nn.functional.pad(score, (0, len(entry) - nb), value=-math.inf)
    always = (entry < c["first"]) | (entry >= have - c["last"])
    score = torch.where(entry < have, torch.where(always, math.inf, score), -math.inf)
    ids = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :top]
    ids = torch.where(ids < have, ids, 1 << 30).sort(-1)[0]
    ids = torch.where(ids < have, ids, -1)
    st["selected"].copy_(ids)
    phys = torch.gather(blk[:, None].expand(s, hkv, nb), 2, ids.clamp(0, nb - 1))
    heads = torch.arange(hkv, device=dev)[None, :, None].expand(s, hkv, top)
    k = _k_blocks(w["k_cache"], hkv, hd, phys, heads).view(s, hkv, top * BLOCK, hd)
    v = _v_blocks(w["v_cache"], hkv, hd, phys, heads).view(s, hkv, top * BLOCK, hd)
    at = (ids[..., None] * BLOCK + torch.arange(BLOCK, device=dev)).view(s, hkv, 1, -1)
    seen = (ids >= 0)[..., None].expand(s, hkv, top, BLOCK).reshape(s, hkv, 1, -1) & \
        (at < keys[:, None, None, None])
    z = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(hd)
    st["o"].copy_(_softmax_product(z, seen, v).view(s, hq, hd))


def run(st):
    kind = st["case"]["kind"]
    if own:
        _run_own(st)
    else:
        {"tree": _tree_plain, "fork": _fork_plain, "verify": _verify_plain,
         "summarize": _prompts_plain, "sparse": _sparse_plain}[kind](st)
    if kind == "tree":
        return {"o": st["o"]}
    if kind in ("summarize", "sparse"):
        out = {"summary": st["summary"], "scales": st["scales"]}
        return out if kind == "summarize" else dict(out, o=st["o"], selected=st["selected"])
    return {"block_table": st["block_table"], "ref_counts": st["ref_counts"], "status": st["status"],
            "k_cache": [w["k_cache"] for w in st["layers"]],
            "v_cache": [w["v_cache"] for w in st["layers"]]}


# ----------------------------------------------------------------------------
# Work, and the results in 64 bits
# ----------------------------------------------------------------------------


def work(case):
    c = case
    hq, hkv, hd, dtype, _ = HEADS[c["heads"]]
    eb = 2 if dtype == "bf16" else 4
    ctx, news = _lengths(c)
    token = 2 * hkv * hd * eb
    if c["kind"] == "tree":
        pairs = int((ctx * news).sum()) + int(_trees(c, news).sum())
        rows = int(news.sum())
        return {"bytes": int((ctx + news).sum()) * token + rows * (2 * hq * hd * eb + 8),
                "flops": 4 * hq * hd * pairs}
    if c["kind"] == "fork":
        _, _, lens = _forks(c, ctx)
        # A child's entries are dropped, its parent's read, its own written, counts
        # moved both ways; a partial last block is copied in every layer.
        copied = int((lens % BLOCK != 0).sum())
        return {"bytes": copied * BLOCK * token * 2 * c["layers"] +
                7 * 4 * int((-(-lens // BLOCK)).sum()), "flops": 0}
    if c["kind"] == "verify":
        moved = int(_kept(c, news).sum())
        return {"bytes": 2 * token * c["layers"] * (int(news.sum()) + moved) +
                12 * (int(news.sum()) + moved), "flops": 0}
    blocks = -(-ctx // BLOCK)
    summary = hkv * (2 * hd + 4)
    if c["kind"] == "summarize":
        return {"bytes": int(ctx.sum()) * token // 2 + int(blocks.sum()) * (summary + 4), "flops": 0}
    chosen = np.minimum(blocks, c["blocks"])
    tokens = np.where(chosen < blocks, chosen * BLOCK, ctx)
    # The newest block's keys and summary, every summary, the chosen keys and values.
    newest = int(((ctx - 1) % BLOCK + 1).sum()) * token // 2 + c["seqs"] * summary
    return {"bytes": newest + int(blocks.sum()) * (summary + 4) + int(tokens.sum()) * token +
            c["seqs"] * (2 * hq * hd * eb + 4 * hkv * c["blocks"]),
            "flops": 4 * hq * hd * int(tokens.sum()) + 2 * hq * 2 * hd * int(blocks.sum())}


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


def _attend64(q, k, v, seen):
    """softmax(q k / sqrt(hd)) v over the keys seen, one head."""
    z = (q @ k.T) / math.sqrt(q.shape[-1])
    z = z.masked_fill(~seen, -math.inf)
    return torch.nan_to_num(z.softmax(-1), 0.0) @ v


def exact(case, seed):
    c = case
    if c["kind"] in ("fork", "verify", "summarize"):
        return None  # bytes are moved, or whole numbers and powers of two computed
    hq, hkv, hd, _, _ = HEADS[c["heads"]]
    g = hq // hkv
    st = prepare(c, seed)
    ctx, news = _lengths(c)
    table = st["block_table"].long()
    ko, vo = _offsets(hd)
    w = st["layers"][0]
    o = torch.zeros(st["o"].shape, dtype=torch.float64, device="cuda")
    if c["kind"] == "tree":
        sees = torch.from_numpy(_trees(c, news)).cuda()
        first = np.concatenate([[0], np.cumsum(news)])
        for s in range(c["seqs"]):
            n, total = int(news[s]), int(ctx[s] + news[s])
            blocks = table[s, :-(-total // BLOCK)]
            k, v = _tokens64(w["k_cache"], blocks, ko, total), _tokens64(w["v_cache"], blocks, vo, total)
            seen = torch.ones(n, total, dtype=torch.bool, device="cuda")
            seen[:, int(ctx[s]):] = sees[s, :n, :n]
            rows = slice(int(first[s]), int(first[s + 1]))
            for h in range(hq):
                o[rows, h] = _attend64(st["q"][rows, h].double(), k[h // g], v[h // g], seen)
        return {"o": o}
    _summarize_plain(st, st["positions"], st["ctx_lens"], 1)
    selected = np.full(st["selected"].shape, -1, np.int32)
    q = st["q"].double()
    for s in range(c["seqs"]):
        n = int(ctx[s])
        nb = -(-n // BLOCK)
        blocks = table[s, :nb]
        k, v = _tokens64(w["k_cache"], blocks, ko, n), _tokens64(w["v_cache"], blocks, vo, n)
        for head in range(hkv):
            qh = q[s, head * g:(head + 1) * g]
            x = min(100, max(-100, math.frexp(float(qh.abs().max()))[1]))
            q8 = (qh * 2.0 ** (7 - x)).round().clamp(-127, 127)
            hi, lo = (st["summary"][blocks, head, i].double() for i in (0, 1))
            bound = torch.where(q8[:, None] > 0, q8[:, None] * hi[None], q8[:, None] * lo[None]).sum(-1)
            score = (bound.amax(0) * st["scales"][blocks, head].double()).cpu().numpy()
            score[:c["first"]] = math.inf
            score[max(0, nb - c["last"]):] = math.inf
            ids = np.sort(np.lexsort((np.arange(nb), -score))[:c["blocks"]])
            selected[s, head, :len(ids)] = ids
            at = (torch.from_numpy(ids).cuda()[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")).view(-1)
            at = at[at < n]
            seen = torch.ones(1, len(at), dtype=torch.bool, device="cuda")
            o[s, head * g:(head + 1) * g] = _attend64(qh, k[head][at], v[head][at], seen)
    return {"summary": None, "scales": None, "o": o, "selected": torch.from_numpy(selected).cuda()}
