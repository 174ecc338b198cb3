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
def test_pools_that_require_a_gradient(kv, name):
    t = tensors()
    t[name].requires_grad_()
    with pytest.raises(UnisonError, match="gradient"):
        kv.Pool(**t)
    with torch.no_grad():
        kv.Pool(**t)


@pytest.mark.parametrize("name", ["k", "v", "weight"])
def test_pools_that_come_to_require_a_gradient(kv, name):
    pool, seqs = kv.Pool(**tensors()), batch(kv)
    kv._On(pool, seqs)
    getattr(pool, name).requires_grad_()
    with pytest.raises(UnisonError, match="gradient"):
        kv._On(pool, seqs)
    with torch.no_grad():
        kv._On(pool, seqs)
