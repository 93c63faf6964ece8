"""Small replicas around a paged cache, and plain 64-bit forms of the cache
operators, for their tests. Pools are filled whole (free blocks and unfilled
slots hold NaN where a test asks for it), tables are shuffled."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2607_04181_amd as coco

B = 16
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Cache:
    """A handle of thin layers over pools of its own."""

    def __init__(self, dtype, hq, hkv, hd, num_blocks, max_blocks, n_layers=1, max_rows=64,
                 max_seqs=64, seed=0, pools=None):
        self.dtype, self.hq, self.hkv, self.hd = dtype, hq, hkv, hd
        self.num_blocks, self.max_blocks = num_blocks, max_blocks
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.pools = pools or [tuple(self.normal(num_blocks, hkv, B * hd) for _ in "kv")
                               for _ in range(n_layers)]
        d = 128
        shapes = {"w_qkv": ((hq + 2 * hkv) * hd, d), "w_o": (d, hq * hd), "w_gate_up": (2 * d, d),
                  "w_down": (d, d), "gamma_attn": (d,), "gamma_mlp": (d,)}
        layers = [dict({k: torch.zeros(s, dtype=DT[dtype], device="cuda")
                        for k, s in shapes.items()}, k_cache=k, v_cache=v) for k, v in self.pools]
        self.h = coco.coco_layer_init(
            coco.make_config(d, hq, hkv, hd, d, len(layers), dtype, max_rows, max_seqs, max_blocks,
                             1e4, 1e-5), layers)

    def normal(self, *shape, sigma=1.0):
        return torch.empty(shape, dtype=DT[self.dtype], device="cuda").normal_(
            0.0, sigma, generator=self.gen)

    def tokens(self, layer=0):
        """Keys and values by place, [block, slot, head, dim], 64 bits on the CPU."""
        ko, vo = offsets(self.hd)
        k, v = (p.detach().cpu().double().numpy() for p in self.pools[layer])
        return k[:, :, ko].transpose(0, 2, 1, 3), v[:, :, vo].transpose(0, 2, 1, 3)

    def put(self, layer, k, v):
        """Sets the pools from values by place (float arrays of stored values)."""
        ko, vo = offsets(self.hd)
        for pool, x, off in zip(self.pools[layer], (k, v), (ko, vo)):
            t = np.empty((self.num_blocks, self.hkv, B * self.hd))
            t[:, :, off.reshape(-1)] = x.transpose(0, 2, 1, 3).reshape(self.num_blocks, self.hkv, -1)
            pool.copy_(torch.from_numpy(t).to(pool.dtype))


def offsets(hd):
    """Where dimension h of slot t lies in a key and a value tile, [16, hd]."""
    t, h = np.arange(B)[:, None], np.arange(hd)[None]
    return (((h // 32) * 64 + (h % 32) // 8 * 16 + t) * 8 + h % 8,
            (((h // 32) * 64 + t // 4 * 16 + h % 16) * 2 + (h // 16) % 2) * 4 + t % 4)


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def tables(rng, lens, max_blocks, num_blocks):
    """Rows of shuffled blocks for the lengths, -1 behind."""
    perm = rng.permutation(num_blocks)
    table = np.full((len(lens), max_blocks), -1, np.int64)
    at = 0
    for s, n in enumerate(lens):
        nb = -(-int(n) // B)
        table[s, :nb] = perm[at:at + nb]
        at += nb
    assert at <= num_blocks
    return table


def pack_masks(seen, words):
    """Rows of truth values (64 * words each) as int64 words."""
    return torch.from_numpy(np.packbits(seen, axis=-1, bitorder="little").view(np.int64)
                            .reshape(len(seen), words)).cuda()


def attend(q, k, v, seen, hkv):
    """One row: q [Hq, hd], k and v [keys, Hkv, hd], seen [Hkv or 1, keys].
    Returns o and, for the tolerance, the weighted mean of |v| and the largest
    sum of |q k| / sqrt(hd), each per head."""
    hq, hd = q.shape
    g = hq // hkv
    o, mean, size = np.zeros((hq, hd)), np.zeros((hq, hd)), np.zeros((hq, 1))
    for h in range(hq):
        use = np.nonzero(seen[h // g if len(seen) > 1 else 0])[0]
        if not len(use):
            continue
        kk, vv = k[use, h // g], v[use, h // g]
        z = kk @ q[h] / math.sqrt(hd)
        p = np.exp(z - z.max())
        p /= p.sum()
        o[h], mean[h] = p @ vv, p @ np.abs(vv)
        size[h] = (np.abs(kk) @ np.abs(q[h])).max() / math.sqrt(hd)
    return o, mean, size


def tolerance(dtype, o, mean, size, keys, hd):
    """Bound of the kernels' error. A score is off by at most (hd + 4) fp32 half
    steps of the sum of its terms' sizes; a probability by twice that, four half
    steps of its exponential and, for bf16 handles, one bf16 rounding (2^-8); a
    weighted sum divided by the sum of its weights by twice what each
    probability is off (numerator and denominator), plus their sums' own fp32
    steps (at most keys + 32); the result by one rounding to its type."""
    f = 2.0 ** -24
    p = 2 * (hd + 4) * f * size + 4 * f + (2.0 ** -8 if dtype == "bf16" else 0.0)
    step = 2.0 ** -8 if dtype == "bf16" else f
    return mean * (2 * p + 2 * (keys + 32) * f) * 1.01 + np.abs(o) * step + 1e-30


def exponent(a):
    """x with a < 2^x, held within +-100."""
    return min(100, max(-100, math.frexp(a)[1])) if a else 0


def summary_of(keys):
    """Bytes and scale of one block's cached keys at one head, [tokens, hd]."""
    keys = np.where(np.isfinite(keys), keys, 0.0)
    hi, lo = keys.max(0), keys.min(0)
    x = exponent(float(max(np.abs(hi).max(), np.abs(lo).max())))
    up = 2.0 ** (7 - x)
    return (np.stack([np.ceil(hi * up), np.floor(lo * up)]).clip(-127, 127).astype(np.int8),
            2.0 ** (x - 7))


def choose(q, summary, scales, top, first, last):
    """Blocks for one (row, kv head): q [G, hd], summary [nb, 2, hd], scales [nb]."""
    nb = len(scales)
    q = np.where(np.isfinite(q), q, 0.0)
    q8 = np.rint(q * 2.0 ** (7 - exponent(float(np.abs(q).max())))).clip(-127, 127).astype(np.int64)
    s = summary.astype(np.int64)
    dots = np.where(q8[:, None] > 0, q8[:, None] * s[None, :, 0], q8[:, None] * s[None, :, 1]).sum(-1)
    score = dots.max(0) * scales.astype(np.float64)
    always = (np.arange(nb) < first) | (np.arange(nb) >= nb - last)
    order = np.lexsort((np.arange(nb), -np.where(always, np.inf, score)))
    ids = np.full(top, -1)
    take = np.sort(order[:top])
    ids[:len(take)] = take
    return ids
