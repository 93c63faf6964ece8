"""What the binding and the library refuse of the cache operators before any
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


def pages():
    return dict(table=torch.zeros(4, 8, dtype=I32), refs=ints(20))


def test_pages_refuse_mismatched_shapes():
    import paper_2607_04181_amd as coco
    h, p = handle(), pages()
    with pytest.raises(ValueError, match="lens must have 3"):
        coco.coco_kv_alloc(h, ints(3), ints(2), p["table"], p["refs"], ints(3))
    with pytest.raises(ValueError, match="status must have 3"):
        coco.coco_kv_alloc(h, ints(3), ints(3), p["table"], p["refs"], ints(2))
    with pytest.raises(ValueError, match="block_table must be"):
        coco.coco_kv_alloc(h, ints(3), ints(3), p["table"][:, :7], p["refs"], ints(3))
    with pytest.raises(ValueError, match="ref_counts must have 20"):
        coco.coco_kv_free(h, ints(3), None, p["table"], ints(19))
    with pytest.raises(ValueError, match="src_seq must have 3"):
        coco.coco_kv_fork(h, 0, 1, ints(2), ints(3), ints(3), p["table"], p["refs"], ints(3))
    with pytest.raises(ValueError, match="keep_lens must have 3"):
        coco.coco_kv_free(h, ints(3), ints(2), p["table"], p["refs"])
    with pytest.raises(ValueError, match="dst_blocks must have 3"):
        coco.coco_kv_copy(h, 0, 1, ints(3), ints(4))
    with pytest.raises(ValueError, match="kept_starts must have 4"):
        coco.coco_kv_compact(h, 0, 1, ints(3), ints(3), ints(9), ints(3), p["table"])
    with pytest.raises(ValueError, match="on the GPU"):
        coco.coco_kv_alloc(h, ints(3), ints(3), p["table"], p["refs"], ints(3))


def tree(n=5, seqs=2):
    q = torch.zeros(n, 8, 128, dtype=torch.bfloat16)
    return [q, q.clone(), ints(seqs + 1), torch.zeros(seqs, 8, dtype=I32), ints(seqs),
            torch.zeros(n, 1, dtype=torch.int64)]


@pytest.mark.parametrize("at,value,exc,text", [
    (0, torch.zeros(5, 8, 128), TypeError, "q must be"),
    (0, torch.zeros(5, 8, 64, dtype=torch.bfloat16), ValueError, "q must be"),
    (1, torch.zeros(4, 8, 128, dtype=torch.bfloat16), ValueError, "o must have 5"),
    (2, ints(2), ValueError, "seq_starts must have 3"),
    (3, torch.zeros(1, 8, dtype=I32), ValueError, "block_table has 1"),
    (5, torch.zeros(4, 1, dtype=torch.int64), ValueError, "tree_mask must be"),
    (5, torch.zeros(5, dtype=torch.int64), ValueError, "tree_mask must be"),
])
def test_tree_attention_refuses_mismatched_shapes(at, value, exc, text):
    import paper_2607_04181_amd as coco
    args = tree()
    args[at] = value
    with pytest.raises(exc, match=text):
        coco.coco_tree_attention(handle(), 0, *args)
    with pytest.raises(ValueError, match="on the GPU"):
        coco.coco_tree_attention(handle(), 0, *tree())


def test_sparse_calls_refuse_mismatched_shapes():
    import paper_2607_04181_amd as coco
    h = handle()
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    summary, scales = torch.zeros(20, 2, 2, 128, dtype=torch.int8), torch.zeros(20, 2)
    table, sel = torch.zeros(3, 8, dtype=I32), torch.zeros(3, 2, 4, dtype=I32)
    with pytest.raises(ValueError, match="layer's 30 blocks"):
        coco.coco_kv_summarize(h, 1, summary, scales, None, ints(3), table)
    with pytest.raises(ValueError, match="scales must have 40"):
        coco.coco_kv_summarize(h, 0, summary, scales[:19], None, ints(3), table)
    with pytest.raises(ValueError, match="first_lens must have 3"):
        coco.coco_kv_summarize(h, 0, summary, scales, ints(2), ints(3), table)
    with pytest.raises(ValueError, match="summary must be"):
        coco.coco_block_select(h, summary[:, :, :1], scales, q, ints(3), None, table, ints(3), 0, 0,
                               sel)
    with pytest.raises(ValueError, match="ctx_lens has 2 entries for 3 rows"):
        coco.coco_block_select(h, summary, scales, q, ints(3), None, table, ints(2), 0, 0, sel)
    with pytest.raises(ValueError, match="positions must have 3"):
        coco.coco_sparse_attention(h, 0, q, q, ints(4), None, table, ints(3), sel)
    with pytest.raises(ValueError, match="selected must be"):
        coco.coco_sparse_attention(h, 0, q, q, ints(3), None, table, ints(3), sel[:, :1])
    with pytest.raises(ValueError, match="on the GPU"):
        coco.coco_sparse_attention(h, 0, q, q, ints(3), None, table, ints(3), sel)


def test_layers_refuse_mismatched_shapes():
    import paper_2607_04181_amd as coco
    h, rows = handle(), torch.zeros(6, 512, dtype=torch.bfloat16)
    table, mask = torch.zeros(2, 8, dtype=I32), torch.zeros(5, 1, dtype=torch.int64)
    batch = [rows, ints(5), ints(5), ints(3), table, ints(2)]
    with pytest.raises(ValueError, match="seq_starts must be given"):
        coco.coco_layer_tree_forward(h, 0, 1, *batch[:3], None, *batch[4:], mask)
    with pytest.raises(ValueError, match="tree_mask must be"):
        coco.coco_layer_tree_forward(h, 0, 1, *batch, mask[:4])
    with pytest.raises(ValueError, match="seq_starts must have"):
        coco.coco_layer_tree_forward(h, 0, 1, *batch[:3], ints(2), *batch[4:], mask)
    with pytest.raises(ValueError, match="on the GPU"):
        coco.coco_layer_tree_forward(h, 0, 1, *batch, mask)
    summary, scales = torch.zeros(30, 2, 2, 128, dtype=torch.int8), torch.zeros(30, 2)
    sel = torch.zeros(2, 2, 4, dtype=I32)
    step = [rows, ints(2), ints(2), table, ints(2)]
    with pytest.raises(ValueError, match="layer's 30 blocks"):
        coco.coco_layer_sparse_forward(h, 1, *step, summary[:20], scales[:20], 0, 0, sel)
    with pytest.raises(ValueError, match="selected must be"):
        coco.coco_layer_sparse_forward(h, 1, *step, summary, scales, 0, 0, sel[:1])
    with pytest.raises(ValueError, match="ctx_lens has 3"):
        coco.coco_layer_sparse_forward(h, 1, *step[:4], ints(3), summary, scales, 0, 0, sel)
    with pytest.raises(ValueError, match="on the GPU"):
        coco.coco_layer_sparse_forward(h, 1, *step, summary, scales, 0, 0, sel)


def test_calls_without_a_handle_are_errors():
    from paper_2607_04181_amd import _lib
    for name in ("coco_kv_alloc", "coco_kv_fork", "coco_kv_free", "coco_kv_copy",
                 "coco_kv_compact", "coco_tree_attention", "coco_kv_summarize",
                 "coco_block_select", "coco_sparse_attention", "coco_layer_tree_forward",
                 "coco_layer_sparse_forward"):
        args = [0 if t in (_lib.ctypes.c_int32, _lib.ctypes.c_int64) else None
                for t in getattr(_lib._lib, name).argtypes]
        assert _lib.raw_call(name, *args) == _lib.COCO_EINVAL
        assert "handle is NULL" in _lib.coco_last_error()
    for name in ("coco_tree_reserve", "coco_sparse_reserve"):
        assert _lib.raw_call(name, None, 1, 1) == _lib.COCO_EINVAL
