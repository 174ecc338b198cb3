"""Tensors that the paged-KV operators change in place pass autograd's version counters: a backward pass that saved
their old values fails instead of using the new ones."""
import pytest

import kv_cases as K

pytestmark = pytest.mark.gpu
NAMES = ("k", "v", "weight", "pos", "box", "box_scale")


def test_what_each_call_changes():
    import torch
    from paper_2609_09643_amd import kv
    c = K.Case("bf16", 64, 16, 2, 2, (60, 20), (1, 2), seed=1)
    pool, seqs = K.device(c)
    q, new = K.rows(c.q, "bf16"), (K.rows(c.new_k, "bf16"), K.rows(c.new_v, "bf16"))
    pos = torch.zeros(c.n_tok, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)

    def changed(call):
        before = {n: getattr(pool, n)._version for n in NAMES}
        before["out"] = out._version
        got = call()
        after = {n: getattr(pool, n)._version for n in NAMES}
        after["out"] = out._version
        return {n for n in after if after[n] != before[n]}, got

    assert changed(lambda: kv.append(pool, seqs, *new, pos))[0] == set(NAMES)
    assert changed(lambda: kv.attend(pool, seqs, q))[0] == set()
    assert changed(lambda: kv.attend(pool, seqs, q, out=out))[0] == {"out"}
    assert changed(lambda: kv.attend(pool, seqs, q, decay=0.5))[0] == {"weight"}
    assert changed(lambda: kv.attend_blocks(pool, seqs, q, 2))[0] == set()
    names, gone = changed(lambda: kv.victims(pool, seqs, 15, max_evict=50))
    assert names == set()
    assert changed(lambda: kv.compact(pool, seqs, *gone))[0] == set(NAMES)


def test_a_backward_pass_of_old_values_fails():
    import torch
    from paper_2609_09643_amd import kv
    c = K.Case("bf16", 64, 16, 1, 2, (60,), (1,), seed=1)
    pool, seqs = K.device(c, parts=("weight",))
    leaf = torch.ones_like(pool.weight, requires_grad=True)
    loss = (leaf * pool.weight).sum()
    kv.attend(pool, seqs, K.rows(c.q, "bf16"), decay=1.0)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


def test_pools_of_inference_tensors():
    """They have no version to count."""
    import torch
    from paper_2609_09643_amd import kv
    c = K.Case("bf16", 64, 16, 1, 2, (60,), (1,), seed=1)
    with torch.inference_mode():
        pool, seqs = K.device(c)
        q = K.rows(c.q, "bf16")
    outside = kv.attend(pool, seqs, q, decay=1.0)
    with torch.inference_mode():
        kv.append(pool, seqs, K.rows(c.new_k, "bf16"), K.rows(c.new_v, "bf16"),
                  torch.zeros(c.n_tok, dtype=torch.int32, device="cuda"))
        kv.compact(pool, seqs, *kv.victims(pool, seqs, 30, max_evict=50))
    assert outside.shape == q.shape
