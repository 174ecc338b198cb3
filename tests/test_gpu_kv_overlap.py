"""Attention that writes its results over its queries: the same values where it is allowed, an error where the
weights' product reads the queries again."""
import pytest

import kv_cases as K

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,group,lens,new", [(64, 4, (300, 70), (1, 2)), (128, 8, (5000,), (2,)), (256, 3, (90,), (2,)),
                                                (128, 4, (700, 300), (400, 1)), (64, 2, (3000,), (100,))])
def test_results_over_their_queries(dim, group, lens, new):
    import torch
    from paper_2609_09643_amd import kv
    from paper_2609_09643_amd.unison import UnisonError
    c = K.Case("bf16", dim, 64, 2, group, lens, new, seed=dim)
    pool, seqs = K.device(c, max_len=max(lens))
    q = K.rows(c.q, "bf16")
    want, lse = kv.attend(pool, seqs, q, lse=True)
    weight = pool.weight.clone()
    with pytest.raises(UnisonError):
        kv.attend(pool, seqs, q, decay=1.0, out=q)
    assert torch.equal(pool.weight.view(torch.int32), weight.view(torch.int32))
    got, e = kv.attend(pool, seqs, q, out=q, lse=True)
    assert got is q and torch.equal(q, want) and torch.equal(e, lse)
