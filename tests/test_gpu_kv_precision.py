"""What attention's second product keeps of small probabilities, on the GPU against 64 bits."""
import numpy as np
import pytest

import kv_cases as K

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_amd import kv
    return kv


def sink(dtype, dim, nats, n, new, group, max_pages):
    """One entry with all the weight and next to no values, the others `nats` to nats + 1 below it with values of
    about 1: their sum is what the output consists of."""
    c = K.Case(dtype, dim, 64, 1, group, (n,), (new,), max_pages=max_pages, seed=int(nats))
    r = np.random.Generator(np.random.PCG64(int(nats)))
    below, at = r.random(n), np.arange(n)
    page, slot = c.pages[0, at // 64], at % 64
    k = np.zeros((n, dim))
    k[:, 0] = -below
    k[7, 0] = nats
    c.k[page, 0, slot] = K.to_type(k, dtype)
    v = 0.5 + r.random((n, dim))
    v[7] = 2.0 ** -20 * r.standard_normal(dim)
    c.v[page, 0, :, slot] = K.to_type(v, dtype)
    c.q[:] = 0.0
    c.q[:, :, 0] = 1.0
    return c


@pytest.mark.parametrize("nats", [15, 17, 18])
@pytest.mark.parametrize("dim,n,new,group,max_pages", [
    (64, 1000, 1, 2, None), (128, 600, 1, 4, None), (128, 4000, 1, 4, 1 << 18), (256, 600, 4, 7, None),
    (128, 600, 64, 4, None), (256, 4000, 20, 2, 1 << 18)])
def test_long_weak_tails(kv, dim, n, new, group, max_pages, nats):
    """fp16 in the second product.  With the largest p of a row at 2^7 or more there, a smaller one is rounded to
    within the larger of 2^-11 of itself and 2^-25, that is 2^-32 of the largest."""
    c = sink("fp16", dim, nats, n, new, group, max_pages)
    want, lse, _, _, tol_lse, _ = c.attend(1.0)
    pool, seqs = K.device(c, parts=())
    out, e = kv.attend(pool, seqs, K.rows(c.q, c.dtype), 1.0, lse=True)
    _, k, v = c.entries(0, 0, n)
    tol = np.zeros_like(want)
    for t, limit in c.rows(0):
        s = k[:limit] @ c.q[t, 0]
        p = np.exp(s - lse[t, 0])
        # a score's error (one product that is not zero, a few roundings of the score's and the lse's size), exp and the sums
        dp = 8 * STEP * (np.abs(s).max() + abs(lse[t, 0])) + (16 + limit) * STEP
        tol[t] = 2.0 ** -11 * np.abs(want[t]) + 2.0 ** -25 \
            + (np.maximum(2.0 ** -11 * p, 2.0 ** -32 * p.max()) + dp * p) @ np.abs(v[:limit])
    K.near(out, want, tol, "out")
    K.near(e, lse, tol_lse, "lse")
