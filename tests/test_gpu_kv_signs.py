"""Sparse attention with a negative scale: the pages that it selects are those of the largest scale * q.k."""
import copy

import numpy as np
import pytest

import kv_cases as K

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim,page,n_kv,group,lens,new", [
    ("bf16", 128, 64, 2, 4, (1, 700, 64), (1, 1, 1)), ("fp16", 64, 16, 3, 1, (33, 0, 500, 16), (2, 0, 3, 16)),
    ("bf16", 256, 32, 1, 6, (350, 2), (2, 4)), ("fp16", 128, 16, 1, 17, (300,), (3,))])
@pytest.mark.parametrize("n_sel,first,last", [(3, 1, 1), (6, 0, 2)])
def test_negative_scales(dtype, dim, page, n_kv, group, lens, new, n_sel, first, last):
    import torch
    from paper_2609_09643_amd import kv
    c = K.Case(dtype, dim, page, n_kv, group, lens, new, seed=n_sel + dim)
    turned = copy.deepcopy(c)
    turned.q = -c.q
    sel = turned.choose(n_sel, first, last)
    scale = -dim ** -0.5
    want, lse, _, tol, tol_lse, _ = c.attend(scale, chosen=sel)
    pool, seqs = K.device(c)
    q = K.rows(c.q, dtype)
    out, got, e = kv.attend_blocks(pool, seqs, q, n_sel, first, last, scale, lse=True)
    assert np.array_equal(got.cpu().numpy(), sel)
    K.near(out, want, tol, "out")
    K.near(e, lse, tol_lse, "lse")
    other, same, _ = kv.attend_blocks(pool, seqs, -q, n_sel, first, last, -scale, lse=True)
    # the products' signs are all turned and turned back; the matrix cores need not round both alike
    assert torch.equal(same, got)
    K.near(other, want, tol, "out of the turned queries")
