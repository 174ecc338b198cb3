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


def bounds(c, out, lse, scale, chosen=None):
    """What the few-rows kernel's result may be off by: the result's own rounding, the scores', the exponentials' and
    the sums' in 32 bits, and of p what its two parts leave: a rounding's half step of a half step."""
    half = K.HALF[c.dtype]
    tol = np.zeros_like(out)
    for i in range(len(c.lens)):
        for h in range(c.n_kv):
            all_e, all_k, all_v = c.entries(i, h, c.lens[i])
            for t, limit in c.rows(i):
                use = all_e < limit
                if chosen is not None:
                    use &= np.isin(all_e // c.page, chosen[t, h])
                k, v = all_k[use], np.abs(all_v[use])
                if not len(k):
                    continue
                for x in range(h * c.group, (h + 1) * c.group):
                    s = scale * (k @ c.q[t, x])
                    p = np.exp(s - lse[t, x])
                    ds = (c.dim + 2) * STEP * abs(scale) * (np.abs(k) @ np.abs(c.q[t, x])).max() \
                        + 8 * STEP * (np.abs(s).max() + abs(lse[t, x]))
                    dp = 2 * ds + (16 + len(k)) * STEP
                    low = 2.0 ** -32 * p.max() if c.dtype == "fp16" else 0.0   # a part below the normal range
                    tol[t, x] = half * np.abs(out[t, x]) + ((1.01 * half * half + dp) * p + low) @ v + 2.0 ** -25
    return tol


@pytest.mark.parametrize("dtype,dim,page,n_kv,group", [
    ("bf16", 64, 16, 2, 3), ("bf16", 128, 64, 2, 4), ("fp16", 128, 32, 1, 5), ("bf16", 256, 32, 1, 6),
    ("fp16", 256, 16, 1, 7), ("bf16", 64, 64, 1, 20), ("bf16", 256, 64, 1, 18)])
@pytest.mark.parametrize("lens,new", [((9, 40), (1, 1)), ((300, 31, 700), (4, 1, 2))])
def test_few_rows_keep_their_probabilities(kv, dtype, dim, page, n_kv, group, lens, new):
    """Up to 32 rows a sequence and kv head: p is not rounded to the inputs' type."""
    c = K.Case(dtype, dim, page, n_kv, group, lens, [min(n, 32 // group) for n in new], seed=dim + group)
    scale = dim ** -0.5
    want, lse, _, _, _, _ = c.attend(scale)
    tol = bounds(c, want, lse, scale)
    pool, seqs = K.device(c, max_len=max(lens))
    q = K.rows(c.q, dtype)
    K.near(kv.attend(pool, seqs, q, scale), want, tol, "out")
    K.near(kv.attend(pool, seqs, q, scale, decay=1.0), want, tol, "out with weights")
    sel = c.choose(4, 1, 2)
    want, lse, _, _, _, _ = c.attend(scale, chosen=sel)
    out, got = kv.attend_blocks(pool, seqs, q, 4, 1, 2, scale)
    assert np.array_equal(got.cpu().numpy(), sel)
    K.near(out, want, bounds(c, want, lse, scale, sel), "sparse out")
