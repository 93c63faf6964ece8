"""Layers whose rows attend a window and a context's first tokens, from slots apart
from their positions: against the layer in 64 bits, against the layers as they are
where the window covers everything, and through an eviction."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle
import paper_2607_04181_amd as coco
import workloads as W
from cache_ref import B, attend, i32, tolerance
from harness import (TOL, Replica, gpu_cache_tokens, normwise_err, oracle_cache, oracle_weights,
                     ragged_decode_batch, ragged_prefill_batch, small_bf16_shape, to64)
from window_ref import ALL, sees
from workloads import device as WD

pytestmark = pytest.mark.gpu

SHAPES = {"bf16": small_bf16_shape(), "bf16_group16": small_bf16_shape(d=512, hq=16, hkv=1),
          "f32": W.LayerShape(260, 4, 2, 64, 684, 1.0e4, 1e-6, "f32")}
# fp32 dot products of up to 700 terms: at most 700 * 2^-24 = 4e-5 of the sum
# of the products' magnitudes, and a few such in a row.
TOL32 = 1e-4


def bound(shape):
    return TOL if shape.dtype == "bf16" else TOL32


def assert_close(shape, got, ref, h0, layers, times=1):
    """What the layers add, within the bound of a layer's output, and the stored
    rows' roundings: half a step of the stored value for each layer."""
    half = 2.0 ** -8 if shape.dtype == "bf16" else 2.0 ** -24
    limit = bound(shape) * np.abs(ref - h0).max() + layers * half * np.abs(ref).max()
    off = np.abs(got - ref).max()
    assert off <= times * limit, (off, limit)


def layer64(w, shape, x, positions, seq, slots, cache, window, sinks):
    """One layer on rows x in 64 bits; cache: K and V of each sequence by slot."""
    hq, hkv, hd, f = shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn
    n = len(x)
    qkv = oracle.layer.rms_norm(x, w["gamma_attn"], shape.rms_eps) @ w["w_qkv"].T
    q, k, v = np.split(qkv, [hq * hd, (hq + hkv) * hd], axis=1)
    q, k, v = q.reshape(n, hq, hd), k.reshape(n, hkv, hd), v.reshape(n, hkv, hd)
    for i in range(n):
        cache.K[seq[i]][slots[i]] = oracle.layer.rope(k[i], positions[i], shape.rope_theta)
        cache.V[seq[i]][slots[i]] = v[i]
    o = np.zeros((n, hq, hd))
    for i in range(n):
        t = np.arange(slots[i] + 1)
        t = t[sees(slots[i], t, window, sinks)]
        o[i] = attend(oracle.layer.rope(q[i], positions[i], shape.rope_theta), cache.K[seq[i]][t],
                      cache.V[seq[i]][t], np.ones((1, len(t)), bool), hkv)[0]
    x1 = x + o.reshape(n, -1) @ w["w_o"].T
    gu = oracle.layer.rms_norm(x1, w["gamma_mlp"], shape.rms_eps) @ w["w_gate_up"].T
    return x1 + (oracle.layer.silu(gu[:, :f]) * gu[:, f:]) @ w["w_down"].T


class Layers:
    """priors: cached tokens before the call; rows: the call's of each sequence (None:
    one each, without seq_starts); ahead: by how much a sequence's positions are
    ahead of its slots."""

    def __init__(self, shape, tag, priors, rows, window, sinks, seed, ahead=0, n_layers=2,
                 weigh=True):
        self.shape, self.tag, self.n_layers = shape, tag, n_layers
        self.window, self.sinks = window, sinks
        n = len(priors)
        news = [1] * n if rows is None else rows
        longest = int(max(np.add(priors, news))) + 20 + int(np.max(ahead))
        spare = sum(news) + 2
        b = (ragged_decode_batch(seed, priors, max_ctx=longest, hidden_rows=spare) if rows is None
             else ragged_prefill_batch(seed, priors, rows, max_ctx=longest, hidden_rows=spare))
        self.seq = np.repeat(np.arange(n), news)
        self.slots = b.positions.astype(np.int64)
        self.b = dataclasses.replace(
            b, positions=(b.positions + np.broadcast_to(ahead, n)[self.seq]).astype(np.int32))
        self.rep = Replica.for_batch(shape, tag, n_layers, self.b)
        coco.coco_window_reserve(self.rep.h, b.n_rows, n, weigh)
        self.hidden = WD.hidden_tensor(shape, tag, b.hidden_rows)
        self.t = WD.batch_tensors(self.b)
        width = b.block_table.shape[1] * B
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.weights = (torch.rand(n, width, device="cuda", generator=gen) if weigh else None)

    def forward(self, hidden, weights, first=0, n=None, stream=None, rows=slice(None),
                seqs=slice(None), starts=None):
        t = self.t
        coco.coco_layer_window_forward(
            self.rep.h, first, n or self.n_layers, hidden, t["row_idx"][rows], t["positions"][rows],
            t["seq_starts"] if starts is None else starts, t["block_table"][seqs],
            t["ctx_lens"][seqs], self.window, self.sinks, weights, stream)

    def expect(self, h0):
        rows, caches = h0[self.b.row_idx], []
        for layer in range(self.n_layers):
            cache = oracle_cache(self.shape, self.tag, layer, self.b, range(self.b.n_seqs),
                                 self.b.num_blocks)
            rows = layer64(oracle_weights(self.shape, self.tag, layer), self.shape, rows,
                           self.b.positions, self.seq, self.slots, cache, self.window, self.sinks)
            caches.append(cache)
        return rows, caches


PROMPTS = ([0, 31, 150, 16, 300], [40, 18, 9, 1, 150])
SINGLE = ([700, 33, 0, 320, 15, 4, 90] * 3, None)


@pytest.mark.parametrize("window,sinks", [(25, 4), (1, 0), (ALL, 0)])
@pytest.mark.parametrize("priors,rows", [PROMPTS, SINGLE], ids=["prompts", "single"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_layers_match_64_bits(name, priors, rows, window, sinks):
    shape = SHAPES[name]
    x = Layers(shape, f"wl_{name}", priors, rows, window, sinks, seed=81,
               ahead=np.arange(len(priors)) * 7)
    h0 = to64(x.hidden)
    x.forward(x.hidden, x.weights)
    torch.cuda.synchronize()
    got, (ref, caches) = to64(x.hidden), x.expect(h0)
    assert_close(shape, got[x.b.row_idx], ref, h0[x.b.row_idx], 2)
    others = sorted(set(range(x.b.hidden_rows)) - set(x.b.row_idx.tolist()))
    assert np.array_equal(got[others], h0[others])
    for s in range(x.b.n_seqs):
        p0, p1 = int(x.b.prior_lens[s]), int(x.b.ctx_lens[s])
        for layer, cache in enumerate(caches):
            k, v = gpu_cache_tokens(x.rep.layers[layer], x.b, s, 0, p1)
            assert np.array_equal(k[:p0], cache.K[s][:p0]) and np.array_equal(v[:p0], cache.V[s][:p0])
            assert normwise_err(k[p0:], cache.K[s][p0:]) < bound(shape)
            assert normwise_err(v[p0:], cache.V[s][p0:]) < bound(shape)


@pytest.mark.parametrize("priors,rows", [PROMPTS, SINGLE], ids=["prompts", "single"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_attention_rows_and_weights_from_the_layers_own_queries(name, priors, rows):
    shape = SHAPES[name]
    x = Layers(shape, f"wq_{name}", priors, rows, 60, 5, seed=82, n_layers=1)
    before = x.weights.cpu().double().numpy()
    x.forward(x.hidden, x.weights)
    torch.cuda.synchronize()
    n, hq, hkv, hd = x.b.n_rows, shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    dt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
    q = to64(x.rep.workspace(coco.COCO_WS_Q, n, hq * hd, dt)).reshape(n, hq, hd)
    o = to64(x.rep.workspace(coco.COCO_WS_O, n, hq * hd, dt)).reshape(n, hq, hd)
    f = 2.0 ** -24
    grow, off = np.zeros_like(before), np.zeros_like(before)
    for s in range(x.b.n_seqs):
        k, v = gpu_cache_tokens(x.rep.layers[0], x.b, s, 0, int(x.b.ctx_lens[s]))
        for i in np.nonzero(x.seq == s)[0]:
            t = np.arange(x.slots[i] + 1)
            t = t[sees(x.slots[i], t, 60, 5)]
            want, mean, size = attend(q[i], k[t], v[t], np.ones((1, len(t)), bool), hkv)
            tol = tolerance(shape.dtype, want, mean, size, len(t), hd)
            assert (np.abs(o[i] - want) <= tol).all(), i
            for h in range(hq):
                z = k[t, h * hkv // hq] @ q[i, h] / np.sqrt(hd)
                w = np.exp(z - z.max())
                w /= w.sum()
                grow[s, t] += w
                # As in the operator's own tests: the score's fp32 steps twice, the
                # exponentials' and the sum's own.
                off[s, t] += w * (2 * (2 * (hd + 4) * f * size[h, 0] + 4 * f) +
                                  2 * (len(t) + 32) * f)
    terms = max(np.bincount(x.seq)) * hq + 8
    tol = (off + terms * f * grow) * 1.01 + 1e-30 + f * (before + grow) * 2
    got = x.weights.cpu().double().numpy()
    assert (np.abs(got - before - grow) <= tol).all()
    assert np.array_equal(got[grow == 0], before[grow == 0])


@pytest.mark.parametrize("priors,rows", [PROMPTS, SINGLE], ids=["prompts", "single"])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_a_window_over_everything_is_the_layer_as_it_is(name, priors, rows):
    shape = SHAPES[name]
    x = Layers(shape, f"wa_{name}", priors, rows, ALL, 0, seed=83, weigh=False)
    h0, whole = to64(x.hidden), x.hidden.clone()
    x.rep.span(0, 2, whole, x.t)
    torch.cuda.synchronize()
    pools = [{k: t[k].clone() for k in ("k_cache", "v_cache")} for t in x.rep.layers]
    x.forward(x.hidden, None)
    torch.cuda.synchronize()
    # Two results of the same row, each within the bound of the exact one.
    assert_close(shape, to64(x.hidden), to64(whole), h0, 2, times=2)
    for k in ("k_cache", "v_cache"):  # written by the same projection
        assert torch.equal(pools[0][k], x.rep.layers[0][k])


@pytest.mark.parametrize("priors,rows", [PROMPTS, SINGLE], ids=["prompts", "single"])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_layer_by_layer_on_a_stream_in_a_graph_and_alone(name, priors, rows):
    x = Layers(SHAPES[name], f"wg_{name}", priors, rows, 70, 3, seed=84, ahead=5)
    want, w_want = x.hidden.clone(), x.weights.clone()
    x.forward(want, w_want)
    out, w = x.hidden.clone(), x.weights.clone()
    x.forward(out, w, 0, 1)
    x.forward(out, w, 1, 1)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(w, w_want)
    none = x.hidden.clone()
    x.forward(none, None)
    torch.cuda.synchronize()
    assert torch.equal(none, want)
    side = torch.cuda.Stream()
    out.copy_(x.hidden)
    w.copy_(x.weights)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x.forward(out, w)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(w, w_want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.forward(out, w)
    for i in range(3):
        out.copy_(x.hidden)
        w.copy_(x.weights)
        graph.replay()
        if i == 1:  # an eager call of the same handle between the replays
            torch.cuda.synchronize()
            x.forward(none, None)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(w, w_want)
    out.copy_(x.hidden)
    w.copy_(x.weights)
    first = np.concatenate([[0], np.cumsum(np.bincount(x.seq))])
    for s in range(x.b.n_seqs):  # one sequence at a time: the same bits
        r = slice(int(first[s]), int(first[s + 1]))
        x.forward(out, w[s:s + 1], rows=r, seqs=slice(s, s + 1),
                  starts=None if rows is None else i32([0, r.stop - r.start]))
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(w, w_want)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_generation_goes_on_over_what_an_eviction_kept(name):
    """A prompt with its weights counted, an eviction by them, and two decode steps
    whose slots are behind what was kept and whose positions go on."""
    shape, budget = SHAPES[name], [50, 200, 33]
    priors, rows = [0, 90, 30], [120, 60, 30]
    x = Layers(shape, f"we_{name}", priors, rows, ALL, 0, seed=85, n_layers=2)
    n, nb, h = 3, x.b.num_blocks, x.rep.h
    x.weights.zero_()
    x.forward(x.hidden, x.weights)
    ctx = x.b.ctx_lens.astype(np.int64)
    table = x.t["block_table"]
    ref_counts = torch.zeros(nb, dtype=torch.int32, device="cuda")
    for s in range(n):
        ref_counts[table[s, :-(-int(ctx[s]) // B)].long()] = 1
    new, base, starts = (i32(np.zeros(k)) for k in (n, n, n + 1))
    kept, status = i32(np.full(sum(budget), -1)), i32(np.zeros(n))
    weights = x.weights.cpu().double().numpy()
    coco.coco_kv_evict(h, i32(np.arange(n)), i32(budget), 2, 10, i32(ctx), x.weights, new, base,
                       kept, starts)
    # What stays, by the definition: in slot order.
    stays = []
    for s in range(n):
        keep = min(budget[s], ctx[s])
        order = np.arange(ctx[s])
        if keep < ctx[s]:
            always = (order < 2) | (order >= ctx[s] - 10)
            rank = np.lexsort((order, -np.where(always, np.inf, weights[s, :ctx[s]])))
            order = np.sort(rank[:keep])
        stays.append(order)
    assert new.cpu().tolist() == [len(o) for o in stays]
    old = [[gpu_cache_tokens(x.rep.layers[layer], x.b, s, 0, int(ctx[s])) for s in range(n)]
           for layer in range(2)]
    coco.coco_kv_compact(h, 0, 2, i32(np.arange(n)), base, kept, starts, table)
    coco.coco_kv_free(h, i32(np.arange(n)), new, table, ref_counts)
    lens = np.array([len(o) for o in stays])
    pos = ctx.copy()
    caches = [oracle.KVCache([np.concatenate([kv[s][0][stays[s]], np.zeros((2,) + kv[s][0].shape[1:])])
                              for s in range(n)],
                             [np.concatenate([kv[s][1][stays[s]], np.zeros((2,) + kv[s][1].shape[1:])])
                              for s in range(n)]) for kv in old]
    row_idx = np.array([4, 0, 2], np.int32)
    w64 = [oracle_weights(shape, x.tag, layer) for layer in range(2)]
    for step in range(2):
        coco.coco_kv_alloc(h, i32(np.arange(n)), i32(lens + 1), table, ref_counts, status)
        assert (status == 1).all()
        before, w_before = to64(x.hidden), x.weights.clone()
        coco.coco_layer_window_forward(h, 0, 2, x.hidden, i32(row_idx), i32(pos), None, table,
                                       i32(lens + 1), 40, 3, x.weights)
        torch.cuda.synchronize()
        rows64 = before[row_idx]
        for layer in range(2):
            rows64 = layer64(w64[layer], shape, rows64, pos, np.arange(n), lens, caches[layer], 40, 3)
        assert_close(shape, to64(x.hidden)[row_idx], rows64, before[row_idx], 2)
        # Every row and head gives 1, each layer.
        grown = (x.weights - w_before).double().sum(1).cpu().numpy()
        assert np.abs(grown - 2 * shape.n_q_heads).max() < 1e-3
        lens, pos = lens + 1, pos + 1


@pytest.mark.parametrize("priors,rows", [PROMPTS, SINGLE], ids=["prompts", "single"])
@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_timing_counts_the_attention_of_a_layer_once(name, priors, rows):
    x = Layers(SHAPES[name], f"wt_{name}", priors, rows, 70, 3, seed=87)
    coco.coco_layer_set_timing(x.rep.h, True)
    x.forward(x.hidden, x.weights)
    got = coco.coco_layer_read_timing(x.rep.h)
    coco.coco_layer_set_timing(x.rep.h, False)
    ms, launches = got["attention"]
    assert launches == 2 and 0 < ms < 50


def test_refusals():
    x = Layers(SHAPES["bf16"], "rf", [40, 30], [12, 20], 16, 2, seed=86, n_layers=1)
    t, h = x.t, x.rep.h
    args = [x.hidden, t["row_idx"], t["positions"], t["seq_starts"], t["block_table"], t["ctx_lens"],
            16, 2, x.weights]

    def refused(code, text, at=None, value=None, layers=(0, 1)):
        a = list(args)
        if at is not None:
            a[at] = value
        with pytest.raises(coco.CocoError, match=text) as e:
            coco.coco_layer_window_forward(h, *layers, *a)
        assert e.value.code == code

    refused(-1, "layers", layers=(0, 2))
    refused(-1, "layers", layers=(1, 1))
    refused(-1, "window = 0", 6, 0)
    refused(-1, "n_sinks", 7, -1)
    fresh = Replica.for_batch(x.shape, "rf", 1, x.b)
    with pytest.raises(coco.CocoError, match="coco_window_reserve"):
        coco.coco_layer_window_forward(fresh.h, 0, 1, *args)
    coco.coco_window_reserve(fresh.h, x.b.n_rows, 2, False)
    with pytest.raises(coco.CocoError, match="weights"):
        coco.coco_layer_window_forward(fresh.h, 0, 1, *args)
    coco.coco_layer_set_validate(h, True)
    refused(-1, "positions", 2, i32(np.where(np.arange(32) == 5, 10 ** 6, x.b.positions)))
    refused(-1, "12 rows in 11 cached", 5, i32([11, 50]))
    refused(-1, "seq_starts", 3, i32([0, 12, 31]))
    refused(-1, "duplicate", 1, i32(np.zeros(32)))
    refused(-1, "block_table", 4, torch.full_like(t["block_table"], -1))
    # Blocks that no row reaches may name anything: slots 40 - 8 < t, and the first two.
    table = t["block_table"].clone()
    table[0, 1] = -1
    refused(-1, "block_table", 4, table)  # (a window of 16 reaches it)
    args[4], args[6] = table, 8
    coco.coco_layer_window_forward(h, 0, 1, *args)
    torch.cuda.synchronize()
