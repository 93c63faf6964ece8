"""What a window call's rows do not see changes no bit of their results."""
import numpy as np
import pytest
import torch

from cache_ref import B
from window_ref import ALL, Rows, sees

pytestmark = pytest.mark.gpu

FORMS = [("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("f32", 4, 2, 64)]


def run_with(r, k, v):
    """o and the weights with these keys and values, from the weights before."""
    r.c.put(0, k, v)
    r.o.fill_(7.0)
    r.weights.copy_(torch.from_numpy(r.before))
    r.run()
    torch.cuda.synchronize()
    return r.o.clone(), r.weights.clone()


def hidden(r, s):
    """Places of sequence s that none of its rows sees, in blocks of its table."""
    t = np.arange(-(-int(r.lens[s]) // B) * B)
    seen = np.zeros(len(t), bool)
    for p in r.slots[r.seq == s]:
        seen |= sees(p, t, r.window, r.sinks)
    return t[~seen]


@pytest.mark.parametrize("window,sinks", [(75, 18), (ALL, 0), (200, 1)])
@pytest.mark.parametrize("lens,rows", [([300, 701, 45], [150, 290, 45]), ([300, 701, 45], [3, 7, 12]),
                                       ([300, 701, 45], None), ([1100], [600])])
@pytest.mark.parametrize("dtype,hq,hkv,hd", FORMS)
def test_hidden_places_change_no_bits(dtype, hq, hkv, hd, lens, rows, window, sinks):
    r = Rows(dtype, hq, hkv, hd, lens, rows, window, sinks, seed=22, poison=False)
    k, v = r.c.tokens()
    ref = None
    for x, y in ((0.5, 1.0), (np.nan, np.nan), (np.inf, -np.inf)):
        for s in range(len(lens)):
            t = hidden(r, s)
            k[r.table[s, t // B], t % B], v[r.table[s, t // B], t % B] = x, y
        o, w = run_with(r, k, v)
        ref = ref or (o, w)
        assert torch.equal(o, ref[0]) and torch.equal(w, ref[1]), (x, y)


@pytest.mark.parametrize("rows", [[150, 40], [12, 7]])
@pytest.mark.parametrize("dtype,hq,hkv,hd", FORMS)
def test_a_value_that_is_not_finite_changes_no_bits_of_other_rows(dtype, hq, hkv, hd, rows):
    r = Rows(dtype, hq, hkv, hd, [300, 45], rows, 75, 18, seed=23, poison=False)
    k, v = r.c.tokens()
    o, w = run_with(r, k, v)
    v[r.table[0, 299 // B], 299 % B] = np.nan  # of the first sequence's last row alone
    o2, w2 = run_with(r, k, v)
    last = rows[0] - 1
    assert torch.isnan(o2[last]).all()
    o2[last] = o[last]
    assert torch.equal(o, o2) and torch.equal(w, w2)
