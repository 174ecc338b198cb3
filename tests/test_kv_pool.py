"""Pool.empty: zeroed pages of the documented shapes, with the parts that were asked for."""
import pytest
import torch


@pytest.mark.parametrize("dtype", [None, torch.float16])
@pytest.mark.parametrize("weight,pos,box", [(True, True, False), (False, False, False), (True, True, True), (False, True, True)])
def test_empty_pools(dtype, weight, pos, box):
    from paper_2609_09643_amd import kv
    p = kv.Pool.empty(5, 3, 32, 64, dtype=dtype, device="cpu", weight=weight, pos=pos, box=box)
    want = {"k": ((5, 3, 32, 64), dtype or torch.bfloat16), "v": ((5, 3, 64, 32), dtype or torch.bfloat16),
            "weight": ((5, 3, 32), torch.float32) if weight else None, "pos": ((5, 3, 32), torch.int32) if pos else None,
            "box": ((5, 3, 2, 64), torch.int8) if box else None, "box_scale": ((5, 3), torch.float32) if box else None}
    for name, is_ in want.items():
        t = getattr(p, name)
        if is_ is None:
            assert t is None, name
        else:
            assert (tuple(t.shape), t.dtype) == is_ and not t.any(), name
    a = p._args
    assert (a.dtype, a.head_dim, a.n_kv, a.page, a.n_pages) == (kv.BF16 if dtype is None else kv.FP16, 64, 3, 32, 5)
    for name in want:
        t = getattr(p, name)
        assert getattr(a, name) == (None if t is None else t.data_ptr()), name
