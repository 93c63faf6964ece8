"""Layers whose rows attend a tree of drafts or selected blocks: the tree layers
against the oracle run on every path as a prompt, through acceptance and the next
decode step; the sparse layer against its parts in 64 bits."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
import paper_2607_04181_amd as coco
import workloads as W
from cache_ref import B, attend, choose, i32, offsets, pack_masks, summary_of, tolerance
from harness import (TOL, Replica, gpu_cache_tokens, normwise_err, oracle_cache,
                     oracle_decode_rows, oracle_weights, ragged_decode_batch,
                     ragged_prefill_batch, small_bf16_shape, to64)
from workloads import device as WD

pytestmark = pytest.mark.gpu

# fp32 dot products of up to 700 terms: at most 700 * 2^-24 = 4e-5 of the sum
# of the products' magnitudes, and a few such in a row.
TOL32 = 1e-4

SHAPES = {"bf16": small_bf16_shape(), "bf16_group16": small_bf16_shape(d=512, hq=16, hkv=1),
          "f32": W.LayerShape(260, 4, 2, 64, 684, 1.0e4, 1e-6, "f32")}


def bound(shape):
    return TOL if shape.dtype == "bf16" else TOL32


def assert_close(shape, got, ref, h0, layers, times=1):
    """What the layers add, within the bound of a layer's output, and the stored
    rows' roundings: each layer rounds x + its own part once, half a step of the
    stored value (2^-8 of it for bf16), which is what a small part added to
    a large row loses, and the next layer carries that on."""
    half = 2.0 ** -8 if shape.dtype == "bf16" else 2.0 ** -24
    limit = bound(shape) * np.abs(ref - h0).max() + layers * half * np.abs(ref).max()
    off = np.abs(got - ref).max()
    assert off <= times * limit, (off, limit)


def parents_of(rng, nodes):
    return [np.array([-1] + [rng.integers(max(-1, j - 5), j) for j in range(1, n)]) for n in nodes]


def paths(parents):
    out = []
    for j in range(len(parents)):
        p = [j]
        while parents[p[0]] >= 0:
            p.insert(0, int(parents[p[0]]))
        out.append(p)
    return out


class Trees:
    def __init__(self, shape, tag, priors, nodes, seed, words=1, n_layers=2):
        rng = np.random.default_rng(seed)
        self.shape, self.tag, self.n_layers = shape, tag, n_layers
        b = ragged_prefill_batch(seed, priors, nodes, max_ctx=int(max(np.add(priors, nodes))) + 20,
                                 hidden_rows=sum(nodes) + 3)
        self.paths = [paths(p) for p in parents_of(rng, nodes)]
        depth = np.concatenate([[len(p) - 1 for p in ps] for ps in self.paths])
        seq = np.repeat(np.arange(len(nodes)), nodes)
        self.b = dataclasses.replace(b, positions=(np.asarray(priors)[seq] + depth).astype(np.int32))
        seen = np.zeros((sum(nodes), 64 * words), bool)
        for s, ps in enumerate(self.paths):
            for j, p in enumerate(ps):
                seen[self.b.seq_starts[s] + j, p] = True
        self.mask = pack_masks(seen, words)
        self.rep = Replica.for_batch(shape, tag, n_layers, self.b)
        coco.coco_tree_reserve(self.rep.h, self.b.n_rows, self.b.n_seqs)
        self.hidden = WD.hidden_tensor(shape, tag, self.b.hidden_rows)
        self.t = WD.batch_tensors(self.b)

    def forward(self, hidden, stream=None):
        t = self.t
        coco.coco_layer_tree_forward(self.rep.h, 0, self.n_layers, hidden, t["row_idx"],
                                     t["positions"], t["seq_starts"], t["block_table"],
                                     t["ctx_lens"], self.mask, stream)

    def path_oracle(self, s, path, h0, weights):
        """Hidden rows and caches of each layer after the path as a prompt."""
        n = len(path)
        rows = self.b.seq_starts[s] + np.asarray(path)
        prior = int(self.b.prior_lens[s])
        sub = dataclasses.replace(
            self.b, row_idx=self.b.row_idx[rows], positions=np.arange(prior, prior + n, dtype=np.int32),
            seq_starts=np.array([0, n]), prior_lens=self.b.prior_lens[s:s + 1],
            ctx_lens=np.array([prior + n]), block_table=self.b.block_table[s:s + 1])
        hid, caches = h0, []
        for layer in range(self.n_layers):
            cache = oracle_cache(self.shape, self.tag, layer, sub, [0], self.b.num_blocks)
            hid, _ = oracle.layer_forward(weights[layer], self.shape, hid, sub.row_idx,
                                          sub.positions, sub.seq_starts, sub.ctx_lens, cache)
            caches.append(cache)
        return hid[sub.row_idx], caches


@pytest.mark.parametrize("name", list(SHAPES))
def test_tree_layers_match_every_path_as_a_prompt_and_an_accepted_path_stays(name):
    shape = SHAPES[name]
    priors, nodes = [0, 31, 150, 16], [3, 18, 9, 1]
    x = Trees(shape, f"tl_{name}", priors, nodes, seed=71)
    h0 = to64(x.hidden)
    x.forward(x.hidden)
    torch.cuda.synchronize()
    got = to64(x.hidden)
    weights = [oracle_weights(shape, x.tag, layer) for layer in range(2)]
    others = sorted(set(range(x.b.hidden_rows)) - set(x.b.row_idx.tolist()))
    assert np.array_equal(got[others], h0[others])
    leaves = [max(ps, key=len) for ps in x.paths]
    accepted = []
    for s, ps in enumerate(x.paths):
        kv = [gpu_cache_tokens(t, x.b, s, priors[s], priors[s] + nodes[s]) for t in x.rep.layers]
        for p in ps:
            if any(len(q) > len(p) and q[:len(p)] == p for q in ps):
                continue  # a longer path holds it
            ref, caches = x.path_oracle(s, p, h0, weights)
            rows = x.b.row_idx[x.b.seq_starts[s] + np.asarray(p)]
            assert_close(shape, got[rows], ref, h0[rows], 2)
            for (k, v), c in zip(kv, caches):
                assert normwise_err(k[p], c.K[0][priors[s]:]) < bound(shape)
                assert normwise_err(v[p], c.V[0][priors[s]:]) < bound(shape)
            if p == leaves[s]:
                accepted.append(caches)
    # The longest paths are accepted: moved up, and decoded on.
    lens = np.array([len(p) for p in leaves])
    coco.coco_kv_compact(x.rep.h, 0, 2, i32(np.arange(4)), i32(priors),
                         i32(np.concatenate([pr + np.asarray(p) for pr, p in zip(priors, leaves)])),
                         i32(np.concatenate([[0], np.cumsum(lens)])), x.t["block_table"])
    now = np.asarray(priors) + lens
    row_idx = np.array([0, 3, 1, 2], np.int32)
    before = to64(x.hidden)
    coco.coco_layer_span_forward(x.rep.h, 0, 2, x.hidden, i32(row_idx), i32(now), None,
                                 x.t["block_table"], i32(now + 1))
    torch.cuda.synchronize()
    got = to64(x.hidden)
    for s in range(4):
        hid = before
        for layer in range(2):
            c = accepted[s][layer]
            cache = oracle.KVCache([np.concatenate([c.K[0], np.zeros_like(c.K[0][:1])])],
                                   [np.concatenate([c.V[0], np.zeros_like(c.V[0][:1])])])
            hid, _ = oracle.layer_forward(weights[layer], shape, hid, row_idx[s:s + 1],
                                          now[s:s + 1], None, now[s:s + 1] + 1, cache)
        r = row_idx[s]
        assert_close(shape, got[r], hid[r], before[r], 2)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_a_chain_is_a_prompt_and_wide_trees_fill_row_tiles(name):
    """One path per tree, longer than a mask word and a row tile: the prompt's result."""
    shape = SHAPES[name]
    priors, nodes = [5, 64], [150, 70]
    x = Trees(shape, f"tc_{name}", priors, nodes, seed=72, words=3, n_layers=1)
    seen = np.zeros((sum(nodes), 192), bool)
    for s, n in enumerate(nodes):
        seen[x.b.seq_starts[s]:x.b.seq_starts[s + 1], :n] = np.tri(n, dtype=bool)
    x.mask = pack_masks(seen, 3)
    pos = np.concatenate([p + np.arange(n) for p, n in zip(priors, nodes)])
    x.t["positions"] = i32(pos)
    whole = x.hidden.clone()
    coco.coco_layer_forward(x.rep.h, 0, whole, x.t["row_idx"], x.t["positions"],
                            x.t["seq_starts"], x.t["block_table"], x.t["ctx_lens"])
    torch.cuda.synchronize()
    kv = [gpu_cache_tokens(x.rep.layers[0], x.b, s, priors[s], priors[s] + nodes[s]) for s in (0, 1)]
    h0 = to64(x.hidden)
    x.forward(x.hidden)
    torch.cuda.synchronize()
    # Two results of the same row, each within the bound of the exact one.
    assert_close(shape, to64(x.hidden), to64(whole), h0, 1, times=2)
    for s in (0, 1):  # written by the same projection
        for a, b in zip(kv[s], gpu_cache_tokens(x.rep.layers[0], x.b, s, priors[s],
                                                priors[s] + nodes[s])):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_tree_layers_on_a_stream_in_a_graph_and_alone(name):
    shape = SHAPES[name]
    x = Trees(shape, f"tg_{name}", [40, 3, 600], [12, 20, 7], seed=73)
    want = x.hidden.clone()
    x.forward(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = x.hidden.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.forward(out)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.forward(out)
    for _ in range(3):
        out.copy_(x.hidden)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    out.copy_(x.hidden)
    for s in range(3):  # one request at a time: the same bits
        r0, r1 = int(x.b.seq_starts[s]), int(x.b.seq_starts[s + 1])
        t, one = x.t, slice(s, s + 1)
        coco.coco_layer_tree_forward(x.rep.h, 0, 2, out, t["row_idx"][r0:r1], t["positions"][r0:r1],
                                     i32([0, r1 - r0]), t["block_table"][one], t["ctx_lens"][one],
                                     x.mask[r0:r1])
    torch.cuda.synchronize()
    assert torch.equal(out, want)


class Sparse:
    def __init__(self, shape, tag, priors, top, seed):
        self.shape, self.top = shape, top
        self.b = ragged_decode_batch(seed, priors, max_ctx=max(priors) + 40,
                                     hidden_rows=len(priors) + 2)
        self.rep = Replica.for_batch(shape, tag, 1, self.b)
        self.hidden = WD.hidden_tensor(shape, tag, self.b.hidden_rows)
        self.t = WD.batch_tensors(self.b)
        hkv, hd, n = shape.n_kv_heads, shape.head_dim, self.b.n_rows
        self.summary = torch.full((self.b.num_blocks, hkv, 2, hd), 99, dtype=torch.int8,
                                  device="cuda")
        self.scales = torch.full((self.b.num_blocks, hkv), 3.0, device="cuda")
        self.selected = torch.full((n, hkv, top), 77, dtype=torch.int32, device="cuda")
        coco.coco_sparse_reserve(self.rep.h, n, top)
        coco.coco_kv_summarize(self.rep.h, 0, self.summary, self.scales, None,
                               i32(self.b.prior_lens), self.t["block_table"])

    def forward(self, hidden, first=1, last=2, rows=slice(None), selected=None):
        t = self.t
        coco.coco_layer_sparse_forward(
            self.rep.h, 0, hidden, t["row_idx"][rows], t["positions"][rows], t["block_table"][rows],
            t["ctx_lens"][rows], self.summary, self.scales, first, last,
            self.selected[rows] if selected is None else selected)


PRIORS = [700, 33, 0, 16 * 20, 15, 1500, 16 * 21 + 1, 4, 90]


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("rows,top", [(9, 6), (140, 40)])
def test_sparse_layer_matches_its_parts(name, rows, top):
    shape = SHAPES[name]
    priors = (PRIORS * 20)[:rows]
    x = Sparse(shape, f"sl_{name}", priors, top, seed=74)
    h0 = to64(x.hidden)
    x.forward(x.hidden)
    torch.cuda.synchronize()
    b, n, hq, hkv, hd = x.b, x.b.n_rows, shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    dt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
    q = to64(x.rep.workspace(coco.COCO_WS_Q, n, hq * hd, dt)).reshape(n, hq, hd)
    o = to64(x.rep.workspace(coco.COCO_WS_O, n, hq * hd, dt)).reshape(n, hq, hd)
    sm, sc, sel = x.summary.cpu().numpy(), x.scales.cpu().numpy(), x.selected.cpu().numpy()
    ref, rec, cache = oracle_decode_rows(shape, f"sl_{name}", 0, b, range(n), h0, record=True)
    ko, vo = offsets(hd)
    for i in range(0, n, 1 if n < 20 else 7):
        ctx = int(b.ctx_lens[i])
        k, v = gpu_cache_tokens(x.rep.layers[0], b, i, 0, ctx)
        assert normwise_err(k[-1], cache.K[i][ctx - 1]) < bound(shape)
        blk = b.block_table[i, :-(-ctx // B)]
        at = np.arange(ctx)
        for g in range(hkv):
            last = (ctx - 1) // B
            s8, scale = summary_of(k[B * last:, g])
            assert np.array_equal(sm[blk[last], g], s8) and sc[blk[last], g] == scale
            want = choose(q[i].reshape(hkv, -1, hd)[g], sm[blk, g], sc[blk, g], top, 1, 2)
            assert np.array_equal(sel[i, g], want), (i, g)
        seen = np.stack([np.isin(at // B, sel[i, g]) for g in range(hkv)])
        want, mean, size = attend(q[i], k, v, seen, hkv)
        tol = tolerance(shape.dtype, want, mean, size, min(ctx, top * B), hd)
        assert (np.abs(o[i] - want) <= tol).all(), i
        if len(blk) <= top:  # every block: the layer as it is
            r = b.row_idx[i]
            assert_close(shape, to64(x.hidden)[r], ref[i], h0[r], 1)
    # What follows the attention, in 64 bits from the layer's own attention rows.
    w = oracle_weights(shape, f"sl_{name}", 0)
    x0 = h0[b.row_idx]
    x1 = x0 + o.reshape(n, -1) @ w["w_o"].T
    h2 = oracle.layer.rms_norm(x1, w["gamma_mlp"], shape.rms_eps) @ w["w_gate_up"].T
    y = x1 + (oracle.layer.silu(h2[:, :shape.d_ffn]) * h2[:, shape.d_ffn:]) @ w["w_down"].T
    assert_close(shape, to64(x.hidden)[b.row_idx], y, x0, 1)
    others = sorted(set(range(b.hidden_rows)) - set(b.row_idx.tolist()))
    assert np.array_equal(to64(x.hidden)[others], h0[others])


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_sparse_layer_in_a_graph_and_row_by_row(name):
    x = Sparse(SHAPES[name], f"sg_{name}", PRIORS, 5, seed=75)
    want = x.hidden.clone()
    x.forward(want)
    torch.cuda.synchronize()
    selected = x.selected.clone()
    out = x.hidden.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.forward(out)
    for _ in range(3):
        out.copy_(x.hidden)
        x.selected.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(x.selected, selected)
    out.copy_(x.hidden)
    for i in range(x.b.n_rows):
        x.forward(out, rows=slice(i, i + 1))
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_timing_counts_the_attention_of_a_layer_once():
    x = Sparse(SHAPES["bf16"], "tm", PRIORS, 5, seed=76)
    y = Trees(SHAPES["bf16"], "tm", [40, 300], [12, 20], seed=76)
    for rep, call, layers in ((x.rep, lambda: x.forward(x.hidden), 1),
                              (y.rep, lambda: y.forward(y.hidden), 2)):
        coco.coco_layer_set_timing(rep.h, True)
        call()
        got = coco.coco_layer_read_timing(rep.h)
        coco.coco_layer_set_timing(rep.h, False)
        ms, launches = got["attention"]
        assert launches == layers and 0 < ms < 50


def test_refusals():
    y = Trees(SHAPES["bf16"], "rf", [40, 30], [12, 20], seed=77, n_layers=1)
    t, h = y.t, y.rep.h
    args = [y.hidden, t["row_idx"], t["positions"], t["seq_starts"], t["block_table"], t["ctx_lens"],
            y.mask]

    def refused(code, text, at=None, value=None, layers=(0, 1)):
        a = list(args)
        if at is not None:
            a[at] = value
        with pytest.raises(coco.CocoError, match=text) as e:
            coco.coco_layer_tree_forward(h, *layers, *a)
        assert e.value.code == code

    refused(-1, "layers", layers=(0, 2))
    refused(-1, "layers", layers=(1, 1))
    fresh = Replica.for_batch(y.shape, "rf", 1, y.b)
    with pytest.raises(coco.CocoError, match="coco_tree_reserve"):
        coco.coco_layer_tree_forward(fresh.h, 0, 1, *args)
    coco.coco_layer_set_validate(h, True)
    refused(-1, "positions", 2, i32(np.where(np.arange(32) == 5, 10 ** 6, y.b.positions)))
    refused(-1, "nodes in 11 cached", 5, i32([11, 50]))
    refused(-1, "seq_starts", 3, i32([0, 12, 31]))
    refused(-1, "duplicate", 1, i32(np.zeros(32)))
    refused(-1, "block_table", 4, torch.full_like(t["block_table"], -1))
    many = Trees(SHAPES["bf16"], "rf", [40], [70], seed=78, words=2, n_layers=1)
    coco.coco_layer_set_validate(many.rep.h, True)
    m = many.t
    with pytest.raises(coco.CocoError, match="70 nodes for 1 mask"):
        coco.coco_layer_tree_forward(many.rep.h, 0, 1, many.hidden, m["row_idx"], m["positions"],
                                     m["seq_starts"], m["block_table"], m["ctx_lens"],
                                     many.mask[:, :1].contiguous())
    x = Sparse(SHAPES["bf16"], "rf", [40, 70], 5, seed=79)
    with pytest.raises(coco.CocoError, match="keep_first"):
        x.forward(x.hidden, 3, 3)
    with pytest.raises(coco.CocoError, match="coco_sparse_reserve"):
        x.forward(x.hidden, selected=torch.zeros(2, 2, 6, dtype=torch.int32, device="cuda"))
    x.forward(x.hidden)
    y.forward(y.hidden)
    torch.cuda.synchronize()
