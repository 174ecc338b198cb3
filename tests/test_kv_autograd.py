"""The paged-KV operators have no backward pass: the binding refuses what autograd follows."""
import pytest
import torch

from paper_2609_09643_amd.unison import UnisonError


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_amd import kv
    kv._kv()
    return kv


def tensors():
    z = torch.zeros
    return dict(k=z(3, 2, 16, 64, dtype=torch.bfloat16), v=z(3, 2, 64, 16, dtype=torch.bfloat16), weight=z(3, 2, 16),
                pos=z(3, 2, 16, dtype=torch.int32))


def batch(kv):
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return kv.Seqs(i32(2, 1), i32(2), i32(3), n_tok=2, max_new=1)


def test_rows_that_require_a_gradient(kv):
    pool = kv.Pool(**tensors())
    leaf = torch.zeros(2, 4, 64, dtype=torch.bfloat16, requires_grad=True)
    for q in (leaf, leaf * 2, leaf[:, ::2]):
        with pytest.raises(UnisonError, match="gradient"):
            kv._rows(q, "q", pool, 2, None)
        kv._rows(q.detach(), "q", pool, 2, None)
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                kv._rows(q, "q", pool, 2, None)


def test_rows_with_a_tangent(kv):
    import torch.autograd.forward_ad as fw
    pool = kv.Pool(**tensors())
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with fw.dual_level():
        dual = fw.make_dual(q, torch.ones_like(q))
        with pytest.raises(UnisonError, match="tangent"):
            kv._rows(dual, "q", pool, 2, None)
        with torch.no_grad(), pytest.raises(UnisonError, match="tangent"):
            kv._rows(dual, "q", pool, 2, None)
        kv._rows(q, "q", pool, 2, None)
        with pytest.raises(UnisonError, match="tangent"):
            kv.Pool(**dict(tensors(), k=fw.make_dual(tensors()["k"], torch.ones_like(tensors()["k"]))))


@pytest.mark.parametrize("name", ["k", "v", "weight"])
@pytest.mark.parametrize("before", [False, True])
def test_pools_that_require_a_gradient(kv, name, before):
    """From the start (the parameters of a module that runs without gradients) or later on: the calls refuse."""
    t, seqs = tensors(), batch(kv)
    if before:
        t[name].requires_grad_()
    pool = kv.Pool(**t)
    if not before:
        kv._On(pool, seqs)
        t[name].requires_grad_()
    for call in (lambda: kv.attend(pool, seqs, torch.zeros(2, 4, 64, dtype=torch.bfloat16)),
                 lambda: kv.attend_blocks(pool, seqs, torch.zeros(2, 4, 64, dtype=torch.bfloat16), 1),
                 lambda: kv.append(pool, seqs, t["k"], t["v"]), lambda: kv.compact(pool, seqs, None, None, None)):
        with pytest.raises(UnisonError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(UnisonError, match="GPU"):
            call()
    with pytest.raises(UnisonError, match="GPU"):                       # whole numbers have no gradient
        kv.victims(pool, seqs, 4)
