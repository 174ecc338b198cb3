"""The paged-KV operators refuse bad arguments on the host, before anything reaches a GPU."""
import ctypes as C
import os

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, CAPACITY = 0, -1, -3
P = 0x10000                                # an aligned address that nothing reads


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_amd import kv
    kv._kv()
    return kv


def pool(kv, **change):
    f = dict(dtype=0, head_dim=128, n_kv=2, page=64, n_pages=10, pad0=0, k=P, v=P, weight=P, pos=P, box=P, box_scale=P)
    f.update(change)
    return kv.PoolArgs(**f)


def seqs(kv, **change):
    f = dict(n_seq=3, max_pages=4, n_tok=5, max_new=2, max_len=0, pad0=0, pages=P, len=P, tok=P)
    f.update(change)
    return kv.SeqsArgs(**f)


def rows(kv, p=P, tok=256, head=128):
    return kv.RowsArgs(p, tok, head)


ALL = ("append", "attend", "blocks", "victims", "compact")
TOKENS, ATTENTION = ALL[:3], ALL[1:3]


def calls(kv, p, s, r=None, only=ALL, n_q=4, ws=P, ws_bytes=1 << 40, out=P, lse=None, scale=0.1, weights=1, decay=1.0):
    """The result of each call in `only`; the arguments under test are wrong for all of them."""
    L, r = kv._kv(), r or rows(kv)
    a, b, x = C.byref(p), C.byref(s), C.byref(r)
    call = {
        "append": lambda: L.unison_kv_append(None, a, b, x, x, P),
        "attend": lambda: L.unison_kv_attend(None, ws, ws_bytes, a, b, n_q, x, scale, weights, decay, out, lse),
        "blocks": lambda: L.unison_kv_attend_blocks(None, ws, ws_bytes, a, b, n_q, x, scale, 2, 0, 1, out, lse, P),
        "victims": lambda: L.unison_kv_victims(None, a, b, 8, 0, 0, 1, P, P, P),
        "compact": lambda: L.unison_kv_compact(None, a, b, 1, P, P, P),
    }
    return {name: call[name]() for name in only}


def test_struct_layouts(kv):
    assert (C.sizeof(kv.PoolArgs), C.sizeof(kv.SeqsArgs), C.sizeof(kv.RowsArgs)) == (72, 48, 24)


@pytest.mark.parametrize("change", [
    dict(dtype=2), dict(head_dim=96), dict(head_dim=0), dict(head_dim=512), dict(n_kv=0), dict(n_kv=1025),
    dict(page=8), dict(page=48), dict(page=512), dict(page=0), dict(n_pages=0), dict(n_pages=1 << 31),
    dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(weight=P + 4), dict(pos=P + 4),
    dict(box=None), dict(box_scale=None), dict(box=P + 1), dict(box_scale=P + 4)])
def test_pools(kv, change):
    got = calls(kv, pool(kv, **change), seqs(kv))
    assert set(got.values()) == {INVALID}, (change, got)


@pytest.mark.parametrize("change,code", [
    (dict(max_pages=0), INVALID), (dict(max_pages=(1 << 24) + 1), CAPACITY), (dict(n_seq=65536), CAPACITY),
    (dict(max_len=257), INVALID), (dict(max_new=0), INVALID), (dict(n_tok=1 << 31), INVALID),
    (dict(pages=None), INVALID), (dict(len=None), INVALID), (dict(len=P + 2), INVALID)])
def test_batches(kv, change, code):
    got = calls(kv, pool(kv), seqs(kv, **change))
    assert set(got.values()) == {code}, (change, got)


def test_tokens_are_needed_where_they_are_read(kv):
    assert set(calls(kv, pool(kv), seqs(kv, tok=None, n_seq=2), only=TOKENS).values()) == {INVALID}


def test_nothing_to_do(kv):
    got = calls(kv, pool(kv, k=None, v=None, weight=P, box=None, box_scale=None),
                seqs(kv, n_seq=0, pages=None, len=None, tok=None), ws=None, ws_bytes=0, out=None)
    assert set(got.values()) == {OK}, got
    got = calls(kv, pool(kv), seqs(kv, n_tok=0, max_new=0, tok=None, n_seq=0))
    assert set(got.values()) == {OK}, got


@pytest.mark.parametrize("r", [dict(p=None), dict(p=P + 8), dict(tok=255), dict(head=4), dict(tok=1 << 41)])
def test_rows(kv, r):
    assert set(calls(kv, pool(kv), seqs(kv), rows(kv, **r), only=TOKENS).values()) == {INVALID}


@pytest.mark.parametrize("more", [
    dict(n_q=0), dict(n_q=3), dict(n_q=2 * 129), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(ws=None), dict(ws=P + 128), dict(out=None), dict(out=P + 8), dict(lse=P + 2), dict(ws_bytes=1)])
def test_attention(kv, more):
    assert set(calls(kv, pool(kv), seqs(kv), only=ATTENTION, **more).values()) == {INVALID}



def test_weights(kv):
    L = kv._kv()
    x = C.byref(rows(kv))
    for decay in (-0.1, 1.1, float("nan")):
        assert L.unison_kv_attend(None, P, 1 << 40, C.byref(pool(kv)), C.byref(seqs(kv)), 4, x, 0.1, 1, decay, P,
                                  None) == INVALID
    assert L.unison_kv_attend(None, P, 1 << 40, C.byref(pool(kv, weight=None)), C.byref(seqs(kv)), 4, x, 0.1, 1, 1.0,
                              P, None) == INVALID


def test_too_many_rows(kv):
    assert set(calls(kv, pool(kv), seqs(kv, n_tok=(1 << 31) - 1), only=ATTENTION).values()) == {CAPACITY}


def test_workspace_sizes(kv):
    L, n = kv._kv(), C.c_size_t()
    p = pool(kv, k=None, v=None)
    assert L.unison_kv_attend_size(C.byref(p), C.byref(seqs(kv)), 4, 1, 0, C.byref(n)) == OK
    assert L.unison_kv_attend_size(C.byref(p), C.byref(seqs(kv)), 4, 1, 0, None) == INVALID
    assert L.unison_kv_attend_size(C.byref(p), C.byref(seqs(kv)), 3, 1, 0, C.byref(n)) == INVALID
    assert L.unison_kv_attend_size(None, C.byref(seqs(kv)), 4, 1, 0, C.byref(n)) == INVALID
    assert L.unison_kv_attend_size(C.byref(p), C.byref(seqs(kv, max_pages=32769)), 4, 0, 4, C.byref(n)) == CAPACITY
    assert L.unison_kv_attend_size(C.byref(p), C.byref(seqs(kv, n_seq=0)), 4, 0, 0, C.byref(n)) == OK
    assert n.value == 0


@pytest.mark.parametrize("weights", [0, 1])
def test_workspaces_go_by_the_tokens_that_sequences_can_have(kv, weights):
    """One sequence of 64 new tokens among a million rows: its partial results, and a word a row and head."""
    L, n = kv._kv(), C.c_size_t()
    p = pool(kv, n_pages=5000, k=None, v=None)
    s = seqs(kv, n_seq=1, max_pages=4000, max_new=64, n_tok=1 << 20, max_len=60000)
    assert L.unison_kv_attend_size(C.byref(p), C.byref(s), 4, weights, 0, C.byref(n)) == OK
    rows, splits, dim = 64 * 4, 60000 // 128, 256
    assert n.value <= splits * rows * (dim + 2) * 4 + ((1 << 20) * 4 * 4 + 60256 * 4 * 64) * weights + 4096


@pytest.mark.parametrize("n_sel,first,last", [(0, 0, 0), (4097, 0, 1), (2, 0, 0), (2, 1, 2), (4, 1 << 31, 1 << 31)])
def test_block_counts(kv, n_sel, first, last):
    L = kv._kv()
    x = C.byref(rows(kv))
    assert L.unison_kv_attend_blocks(None, P, 1 << 40, C.byref(pool(kv)), C.byref(seqs(kv)), 4, x, 0.1, n_sel, first,
                                     last, P, None, P) == INVALID


def test_blocks_need_boxes_and_a_place_for_the_choice(kv):
    L = kv._kv()
    x = C.byref(rows(kv))
    for p, s, sel, code in ((pool(kv, box=None, box_scale=None), seqs(kv), P, INVALID), (pool(kv), seqs(kv), None, INVALID),
                            (pool(kv), seqs(kv, max_pages=32769), P, CAPACITY)):
        assert L.unison_kv_attend_blocks(None, P, 1 << 40, C.byref(p), C.byref(s), 4, x, 0.1, 2, 0, 1, P, None,
                                         sel) == code


@pytest.mark.parametrize("budget,first,recent,most", [(0, 0, 0, 1), (8, 4, 5, 1), (8, 0, 0, 0), (8, 0, 0, (1 << 30) + 1)])
def test_eviction_counts(kv, budget, first, recent, most):
    assert kv._kv().unison_kv_victims(None, C.byref(pool(kv)), C.byref(seqs(kv)), budget, first, recent, most, P, P,
                                      P) == INVALID


def test_eviction_needs(kv):
    L, s = kv._kv(), seqs(kv)
    for p in (pool(kv, weight=None), pool(kv, pos=None)):
        assert L.unison_kv_victims(None, C.byref(p), C.byref(s), 8, 0, 0, 1, P, P, P) == INVALID
    for lists in ((None, P, P), (P, None, P), (P, P, None), (P + 2, P, P)):
        assert L.unison_kv_victims(None, C.byref(pool(kv)), C.byref(s), 8, 0, 0, 1, *lists) == INVALID
        assert L.unison_kv_compact(None, C.byref(pool(kv)), C.byref(s), 1, *lists) == INVALID
    assert L.unison_kv_compact(None, C.byref(pool(kv)), C.byref(s), 0, P, P, P) == INVALID


def test_append_needs_positions_exactly_where_the_pool_has_them(kv):
    L, x = kv._kv(), C.byref(rows(kv))
    assert L.unison_kv_append(None, C.byref(pool(kv)), C.byref(seqs(kv)), x, x, None) == INVALID
    assert L.unison_kv_append(None, C.byref(pool(kv, pos=None)), C.byref(seqs(kv)), x, x, P) == INVALID


def test_tensors(kv):
    """The binding's own checks, on host tensors."""
    import torch
    from paper_2609_09643_amd.unison import UnisonError
    z = torch.zeros
    k, v = z(3, 2, 16, 64, dtype=torch.bfloat16), z(3, 2, 64, 16, dtype=torch.bfloat16)
    i32 = lambda *s: z(*s, dtype=torch.int32)
    for bad in ((k.float(), v.float()), (k, v.half()), (k, v.transpose(2, 3)), (k[0], v), (k[:, :1], v)):
        with pytest.raises(UnisonError):
            kv.Pool(*bad)
    for more in (dict(weight=z(3, 2, 8)), dict(pos=z(3, 2, 16)), dict(box=z(3, 2, 2, 64, dtype=torch.int8)),
                 dict(box=z(3, 2, 2, 64), box_scale=z(3, 2))):
        with pytest.raises(UnisonError):
            kv.Pool(k, v, **more)
    pool = kv.Pool(k, v, weight=z(3, 2, 16), pos=i32(3, 2, 16))
    for bad in ((i32(2, 1).long(), i32(2)), (i32(2), i32(2)), (i32(2, 1), i32(3)), (i32(2, 1), i32(2), i32(2)),
                (i32(2, 1), i32(2), None, 3)):
        with pytest.raises(UnisonError):
            kv.Seqs(*bad)
    for more in (dict(n_tok=-1), dict(max_new=1 << 31), dict(max_len=-2)):
        with pytest.raises(UnisonError):
            kv.Seqs(i32(2, 1), i32(2), i32(3), **more)
    seqs = kv.Seqs(i32(2, 1), i32(2), i32(3), n_tok=2, max_new=1)
    q = z(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(UnisonError, match="GPU"):
        kv.attend(pool, seqs, q)
    with pytest.raises(UnisonError, match="GPU"):
        kv.victims(pool, seqs, 4)
    for bad in (q.half(), q[:1], q[0], z(2, 4, 32, dtype=torch.bfloat16), z(2, 64, 4, dtype=torch.bfloat16).transpose(1, 2)):
        with pytest.raises(UnisonError):
            kv._rows(bad, "q", pool, 2, None)
    assert np.array_equal([kv._rows(q[:, ::2], "q", pool, 2, 2).head_stride], [128])
