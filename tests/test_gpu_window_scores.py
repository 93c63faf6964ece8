"""Scores that are not finite in a window call: they reach the rows that see their keys,
and the weights of the slots that those rows see, and nothing else."""
import numpy as np
import pytest
import torch

from cache_ref import B, attend, tolerance
from window_ref import ALL, Rows, sees

pytestmark = pytest.mark.gpu


def expect(r):
    """o with its tolerance, and what the weights grow by with theirs (NaN where a row that
    sees the slot has a sum that is NaN). A score of -inf has no weight."""
    c, f = r.c, 2.0 ** -24
    k, v = c.tokens()
    q = r.q.cpu().double().numpy()
    o, tol = np.zeros((r.n, c.hq, c.hd)), np.zeros((r.n, c.hq, c.hd))
    width = r.table.shape[1] * B
    grow, off = np.zeros((len(r.lens), width)), np.zeros((len(r.lens), width))
    for i, (s, p) in enumerate(zip(r.seq, r.slots)):
        t = np.nonzero(sees(p, np.arange(p + 1), r.window, r.sinks))[0]
        blk = r.table[s, t // B]
        for h in range(c.hq):
            kk, vv = (x[blk, t % B, h * c.hkv // c.hq] for x in (k, v))
            with np.errstate(invalid="ignore"):
                z = kk @ q[i, h] / np.sqrt(c.hd)
            if np.isnan(z).any() or (z == np.inf).any():
                o[i, h] = np.nan
                grow[s, t] = np.nan
                continue
            u = np.nonzero(z > -np.inf)[0]
            ref, mean, size = attend(q[i, h][None], kk[u][:, None], vv[u][:, None],
                                     np.ones((1, len(u)), bool), 1)
            o[i, h], tol[i, h] = ref[0], tolerance(c.dtype, ref, mean, size, len(u), c.hd)[0]
            w = np.exp(z[u] - z[u].max())
            w /= w.sum()
            grow[s, t[u]] += w
            # As window_ref's: scores twice, exponentials, the sum.
            off[s, t[u]] += w * (2 * (2 * (c.hd + 4) * f * size[0, 0] + 4 * f) +
                                 2 * (len(u) + 32) * f)
    terms = r.news.max() * c.hq + 8
    w_tol = (off + terms * f * np.nan_to_num(grow)) * 1.01 + 1e-30
    return o, tol, grow, w_tol + f * (r.before + np.nan_to_num(grow)) * 2


@pytest.mark.parametrize("window,sinks", [(40, 6), (ALL, 0), (17, 0)])
@pytest.mark.parametrize("rows", [[90, 60], [12, 7], None])
@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 4, 2, 128), ("bf16", 8, 1, 128),
                                             ("f32", 4, 2, 64), ("f32", 6, 2, 96)])
def test_scores_that_are_not_finite_stay_with_the_rows_that_see_them(dtype, hq, hkv, hd, rows,
                                                                    window, sinks):
    r = Rows(dtype, hq, hkv, hd, [200, 60], rows, window, sinks, seed=21, poison=False)
    k, v = r.c.tokens()
    for t, d, x in ((150, 3, np.nan), (120, 5, np.inf), (192, 1, np.inf), (90, 2, -np.inf)):
        k[r.table[0, t // B], t % B, 0, d] = x
    r.c.put(0, k, v)
    if rows is not None:
        r.q[5, 1, 7] = float("nan")
    r.run()
    torch.cuda.synchronize()
    o, tol, grow, w_tol = expect(r)
    got = r.o.cpu().double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(o))
    fine = ~np.isnan(o)
    assert (np.abs(got - o)[fine] <= tol[fine]).all()
    w = r.weights.cpu().double().numpy()
    assert np.array_equal(np.isnan(w), np.isnan(grow)), np.argwhere(np.isnan(w) != np.isnan(grow))[:5]
    fine = ~np.isnan(grow)
    assert (np.abs(w - r.before - grow)[fine] <= w_tol[fine]).all()
    assert np.array_equal(w[grow == 0], r.before[grow == 0])
