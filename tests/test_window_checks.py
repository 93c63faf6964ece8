"""What the binding and the library refuse of window and eviction calls before any
kernel, on the CPU."""
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2607_04181_amd", "libcoco.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libcoco.so not built")

I32 = torch.int32


def handle(dtype="bf16"):
    from paper_2607_04181_amd import _lib
    cfg = _lib.make_config(512, 8, 2, 128, 768, 2, dtype, 16, 16, 8, 1e4, 1e-5)
    return _lib.Handle(None, cfg, [], [20, 30])


def ints(n):
    return torch.zeros(n, dtype=I32)


def window_args(n=5, seqs=2):
    q = torch.zeros(n, 8, 128, dtype=torch.bfloat16)
    return [q, q.clone(), ints(seqs + 1), torch.zeros(seqs, 8, dtype=I32), ints(seqs), 4, 1,
            torch.zeros(seqs, 128)]


@pytest.mark.parametrize("at,value,exc,text", [
    (0, torch.zeros(5, 8, 128), TypeError, "q must be"),
    (0, torch.zeros(5, 8, 64, dtype=torch.bfloat16), ValueError, "q must be"),
    (1, torch.zeros(4, 8, 128, dtype=torch.bfloat16), ValueError, "o must have 5"),
    (2, ints(2), ValueError, "seq_starts must have 3"),
    (2, None, ValueError, "ctx_lens has 2 entries for 5 rows"),
    (3, torch.zeros(1, 8, dtype=I32), ValueError, "block_table has 1"),
    (3, torch.zeros(2, 9, dtype=I32), ValueError, "block_table must be"),
    (7, torch.zeros(1, 128), ValueError, "weights must be"),
    (7, torch.zeros(2, 127), ValueError, "weights must be"),
])
def test_window_attention_refuses_mismatched_shapes(at, value, exc, text):
    import paper_2607_04181_amd as coco
    args = window_args()
    args[at] = value
    with pytest.raises(exc, match=text):
        coco.coco_window_attention(handle(), 0, *args)
    with pytest.raises(ValueError, match="on the GPU"):
        coco.coco_window_attention(handle(), 0, *window_args())


def test_window_layers_refuse_mismatched_shapes():
    import paper_2607_04181_amd as coco
    b = [torch.zeros(8, 512, dtype=torch.bfloat16), ints(4), ints(4), None,
         torch.zeros(4, 8, dtype=I32), ints(4), 4, 1]
    with pytest.raises(ValueError, match="weights must be"):
        coco.coco_layer_window_forward(handle(), 0, 1, *b, torch.zeros(3, 128))
    b[2] = ints(3)
    with pytest.raises(ValueError, match="positions has"):
        coco.coco_layer_window_forward(handle(), 0, 1, *b)


EVICT = dict(seq_idx=ints(3), keep_lens=ints(3), keep_first=1, keep_last=1, ctx_lens=ints(4),
             weights=torch.zeros(4, 128), new_lens=ints(3), base_lens=ints(3), kept=ints(9),
             kept_starts=ints(4))


@pytest.mark.parametrize("name,value,text", [
    ("keep_lens", ints(2), "keep_lens must have 3"), ("new_lens", ints(4), "new_lens must have 3"),
    ("base_lens", ints(2), "base_lens must have 3"), ("kept_starts", ints(3), "kept_starts must have 4"),
    ("weights", torch.zeros(3, 128), "weights must be"), ("weights", torch.zeros(4, 64), "weights must be"),
    ("seq_idx", ints(3), "on the GPU"),
])
def test_evict_refuses_mismatched_shapes(name, value, text):
    import paper_2607_04181_amd as coco
    with pytest.raises(ValueError, match=text):
        coco.coco_kv_evict(handle(), **dict(EVICT, **{name: value}))


def test_library_refuses_calls_without_a_handle():
    from paper_2607_04181_amd import _lib
    for name, args in (("coco_window_reserve", (None, 1, 1, 0)),
                       ("coco_window_attention", (None, 0, None, None, 1, None, 1, None, None, 4, 0,
                                                  None, None)),
                       ("coco_layer_window_forward", (None, 0, 1, None, 1, None, 1, None, None, 1,
                                                      None, None, 4, 0, None, None)),
                       ("coco_kv_evict", (None, None, None, 1, 0, 0, None, None, 1, None, None, None,
                                          0, None, None))):
        assert _lib.raw_call(name, *args) == _lib.COCO_EINVAL
        assert "handle is NULL" in _lib.coco_last_error()
