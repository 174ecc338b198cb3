"""The paged-KV operators on the GPU against the plain implementation in 64 bits."""
import numpy as np
import pytest

import kv_cases as K

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    from paper_2609_09643_amd import kv
    return kv


def check_attend(kv, c, scale=None, decay=0.5, **more):
    scale = c.dim ** -0.5 if scale is None else scale
    want, lse, got, tol, tol_lse, tol_got = c.attend(scale)
    pool, seqs = K.device(c, **more)
    q = K.rows(c.q, c.dtype)
    out, e = kv.attend(pool, seqs, q, scale, lse=True)
    K.near(out, want, tol, "out")
    K.near(e, lse, tol_lse, "lse")
    again, e = kv.attend(pool, seqs, q, scale, decay=decay, lse=True)
    K.near(again, want, tol, "out with weights")
    K.near(e, lse, tol_lse, "lse with weights")
    weight = pool.weight.cpu().numpy()
    for i, n in enumerate(c.lens):
        for o in range(-(-n // c.page)):
            if not c.there(i, o):
                continue
            p, m = c.pages[i, o], min(c.page, n - o * c.page)
            old, add = c.weight[p, :, :m].astype(np.float64), got[i][:, o * c.page:o * c.page + m]
            w = old if not c.new[i] else decay * old + add
            # the terms' own bounds, and a step for each addition
            t = 0 * w if not c.new[i] else tol_got[i][:, o * c.page:o * c.page + m] \
                + 2.0 ** -24 * (c.new[i] * c.group + 4) * w
            d = np.abs(weight[p, :, :m] - w) - t
            assert (d <= 0).all(), "weight of sequence %d page %d: %g over" % (i, o, d.max())
            assert np.isnan(weight[p, :, m:]).all()
    if c.weight.size:
        owned = {int(p) for i, n in enumerate(c.lens) for p in c.pages[i, :-(-n // c.page)]}
        for p in set(range(c.n_pages)) - owned:
            assert np.array_equal(weight[p], c.weight[p], equal_nan=True), "a page of no sequence"


LENS = [
    ((1,), (1,)), ((16,), (1,)), ((17,), (1,)), ((777,), (1,)),
    ((0, 1, 33, 300), (0, 1, 1, 1)),              # an empty sequence
    ((40, 0, 7, 129), (3, 2, 7, 0)),              # tokens without entries, a whole new one, none new
    ((5, 2), (9, 4)),                             # more tokens than entries: the first see nothing
    ((258, 130, 65), (5, 64, 17)),
]


@pytest.mark.parametrize("lens,new", LENS)
@pytest.mark.parametrize("dtype,dim,page,n_kv,group", [
    ("bf16", 128, 64, 2, 4), ("fp16", 64, 16, 3, 1), ("bf16", 256, 32, 1, 6), ("fp16", 128, 256, 1, 5)])
def test_attend(kv, dtype, dim, page, n_kv, group, lens, new):
    check_attend(kv, K.Case(dtype, dim, page, n_kv, group, lens, new, seed=len(lens) + dim))


@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 15, 16, 17, 33, 71, 128])
@pytest.mark.parametrize("new", [1, 2, 5])
def test_attend_groups(kv, group, new):
    check_attend(kv, K.Case("bf16", 64, 16, 1, group, (90, 33), (new, 1), seed=group))


@pytest.mark.parametrize("dtype,dim,page,n_kv,group", [
    ("bf16", 128, 64, 1, 4), ("fp16", 64, 16, 2, 1), ("bf16", 256, 128, 1, 2), ("fp16", 128, 32, 1, 3)])
@pytest.mark.parametrize("lens,new", [((200, 131), (200, 131)), ((511,), (127,)), ((300, 40, 1), (140, 1, 1)),
                                      ((128, 256), (128, 129)), ((1100,), (65,))])
def test_attend_many_tokens(kv, dtype, dim, page, n_kv, group, lens, new):
    check_attend(kv, K.Case(dtype, dim, page, n_kv, group, lens, new, seed=7))


@pytest.mark.parametrize("dtype,dim,page,group", [("bf16", 128, 16, 4), ("fp16", 64, 64, 7), ("bf16", 256, 32, 3)])
@pytest.mark.parametrize("lens,new", [((600,), (600,)), ((700, 30, 260, 0), (300, 1, 257, 2)), ((90,), (700,))])
def test_weights_of_split_rows(kv, dtype, dim, page, group, lens, new):
    """So few blocks of entries that their rows are split: some splits see nothing, some sequences have one row,
    or tokens that see nothing, or a page that is not there."""
    check_attend(kv, K.Case(dtype, dim, page, 1, group, lens, new, missing=[(0, 1)], seed=dim), decay=0.9)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens,new", [((5000, 3), (1, 1)), ((4099, 700), (4, 2)), ((2500,), (40,))])
def test_attend_long(kv, dtype, lens, new):
    check_attend(kv, K.Case(dtype, 128, 64, 1, 8, lens, new, seed=3), max_len=max(lens))


def test_many_tokens_over_more_pages_than_a_block_keeps(kv):
    """17,000 entries in pages of 16: the page ids of a long chunk come in windows."""
    check_attend(kv, K.Case("bf16", 64, 16, 1, 2, (17000, 16500), (40, 1), seed=3))


@pytest.mark.parametrize("n_kv,seqs", [(2, 1), (2, 40)])
def test_splits_of_loose_bounds(kv, n_kv, seqs):
    """A page table and a bound far beyond the lengths: most pieces of the walk are empty."""
    lens = [1 + (i * 37) % 300 for i in range(seqs)]
    c = K.Case("fp16", 64, 32, n_kv, 2, lens, [1] * seqs, max_pages=4000, seed=1)
    check_attend(kv, c)
    check_attend(kv, c, max_len=100000)
    check_blocks(kv, c, 4, 1, 1)


@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("group,new", [(4, (1, 1)), (4, (8, 1)), (5, (4, 7)), (16, (1, 2))])
def test_few_rows_of_much_to_read(kv, dim, group, new):
    """Bounds of 320,000 entries send few rows to the kernel of many."""
    c = K.Case("bf16", dim, 16, 1, group, (1300, 90), new, max_pages=20000, seed=dim + group)
    want, lse, _, tol, tol_lse, _ = c.attend(0.1)
    check_attend(kv, c, scale=0.1)
    pool, seqs = K.device(c)
    out, e = kv.attend(pool, seqs, K.rows(c.q, c.dtype), 0.1, decay=1.0, lse=True)
    K.near(out, want, tol, "out with weights")
    K.near(e, lse, tol_lse, "lse with weights")


@pytest.mark.parametrize("missing", [[(0, 0)], [(0, 1), (0, 2), (1, 0)], [(0, 4), (1, 0), (1, 1), (1, 2)]])
def test_pages_that_are_not_there(kv, missing):
    """Holes at the start, inside, at the end, and a sequence without any page."""
    for new in ((1, 1), (30, 40)):
        c = K.Case("bf16", 64, 32, 2, 2, (150, 70), new, missing=missing, seed=5)
        check_attend(kv, c)


@pytest.mark.parametrize("sharp,scale", [(0.0, None), (1.5, 0.0), (1.5, -0.3), (40.0, None), (200.0, 0.125)])
def test_attend_scores(kv, sharp, scale):
    """Equal scores, a scale of 0, a negative one, and scores of hundreds, where one entry has all."""
    check_attend(kv, K.Case("fp16", 64, 16, 2, 2, (200, 31), (1, 20), sharp=sharp, seed=9), scale=scale)


@pytest.mark.parametrize("new", [1, 70])
def test_rising_scores(kv, new):
    """Keys along the query, each longer than the last: the maximum moves in every tile."""
    c = K.Case("bf16", 64, 16, 1, 2, (400,), (new,), seed=2)
    for e in range(400):
        c.k[c.pages[0, e // 16], 0, e % 16] = K.to_type(np.full(64, e / 25.0), "bf16")
    c.q[:] = K.to_type(np.full_like(c.q, 0.5), "bf16")
    check_attend(kv, c)


@pytest.mark.parametrize("decay", [0.0, 0.7, 1.0])
def test_decay(kv, decay):
    check_attend(kv, K.Case("bf16", 64, 16, 2, 2, (70, 300), (1, 40), seed=4), decay=decay)


def test_strided_queries_and_rows_of_no_sequence(kv):
    """q as a slice of one projection's output; rows behind the last sequence stay."""
    import torch
    c = K.Case("bf16", 128, 64, 2, 3, (100, 50), (2, 1), tail=4, seed=6)
    want, lse, _, tol, tol_lse, _ = c.attend(0.1)
    pool, seqs = K.device(c)
    wide = torch.full((c.n_tok, 10, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 1:7] = K.rows(c.q, c.dtype)
    out = torch.full((c.n_tok, 6, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    got = kv.attend(pool, seqs, wide[:, 1:7], 0.1, out=out)
    assert got is out and (out[3:] == 7.0).all()
    K.near(out[:3], want[:3], tol[:3], "out")
    t = K.rows(c.q, c.dtype).transpose(0, 1).contiguous().transpose(0, 1)   # heads outermost
    K.near(kv.attend(pool, seqs, t, 0.1)[:3], want[:3], tol[:3], "out of transposed rows")


@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("lens,new", [((1500,), (60,)), ((1500, 700), (60, 41))])
def test_many_tokens_among_many_rows(kv, dim, lens, new):
    """Rows of other calls in the same arrays: partial results are kept by sequence, not by row."""
    import torch
    c = K.Case("bf16", dim, 64, 1, 4, lens, new, tail=2000, seed=dim)
    want, lse, _, tol, tol_lse, _ = c.attend(0.1)
    pool, seqs = K.device(c)
    n = sum(new)
    for decay in (None, 0.5):
        out = torch.full((c.n_tok, 4, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        _, e = kv.attend(pool, seqs, K.rows(c.q, c.dtype), 0.1, decay=decay, lse=True, out=out)
        assert (out[n:] == 7.0).all()
        K.near(out[:n], want[:n], tol[:n], "out")
        K.near(e[:n], lse[:n], tol_lse[:n], "lse")


def test_bounds_of_the_device_arrays(kv):
    """Lengths and token ranges beyond the bounds are cut to them."""
    import torch
    c = K.Case("bf16", 64, 16, 1, 2, (100, 60), (1, 2), seed=8)
    want, _, _, tol, _, _ = c.attend(0.125)
    pool, seqs = K.device(c)
    kv.attend(pool, seqs, K.rows(c.q, c.dtype), 0.125)
    wild = kv.Seqs(seqs.pages, torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32, device="cuda"),
                   torch.tensor([-7, 1, 2 ** 30], dtype=torch.int32, device="cuda"), n_tok=3, max_new=2, max_len=100)
    out = kv.attend(pool, wild, K.rows(c.q, c.dtype), 0.125)
    # sequence 0 has 100 entries and token 0; sequence 1 none and tokens 1 and 2
    K.near(out[:1], want[:1], tol[:1], "out")
    assert (out[1:] == 0).all()


def test_shared_pages(kv):
    """Two sequences over the same pages, attention without weights."""
    c = K.Case("bf16", 64, 16, 2, 2, (90, 90), (1, 1), seed=11)
    c.pages[1] = c.pages[0]
    c.q[1] = c.q[0]
    want, _, _, tol, _, _ = c.attend(0.125)
    pool, seqs = K.device(c)
    out = kv.attend(pool, seqs, K.rows(c.q, c.dtype), 0.125)
    K.near(out, want, tol, "out")
    assert (out[0] == out[1]).all()


def test_pages_past_32_bits(kv):
    """Pages whose elements' offsets pass 2^32: every operator as on the same pages of a small pool."""
    import torch
    c = K.Case("bf16", 128, 64, 8, 2, (300, 150), (2, 1), seed=12)
    small, seqs = K.device(c)
    n_pages = (1 << 32) // (8 * 64 * 128) + 100
    shape = (n_pages, 8, 64, 128)
    big = kv.Pool(torch.empty(shape, dtype=torch.bfloat16, device="cuda"),
                  torch.empty((n_pages, 8, 128, 64), dtype=torch.bfloat16, device="cuda"),
                  torch.empty(shape[:3], dtype=torch.float32, device="cuda"),
                  torch.empty(shape[:3], dtype=torch.int32, device="cuda"),
                  torch.empty((n_pages, 8, 2, 128), dtype=torch.int8, device="cuda"),
                  torch.empty((n_pages, 8), dtype=torch.float32, device="cuda"))
    at = torch.arange(n_pages - c.n_pages, n_pages, device="cuda")   # all beyond 2^32 elements
    names = ("k", "v", "weight", "pos", "box", "box_scale")
    for name in names:
        getattr(big, name)[at] = getattr(small, name)
    pages = torch.where(seqs.pages >= 0, seqs.pages + (n_pages - c.n_pages), -1).to(torch.int32)
    far = kv.Seqs(pages, seqs.length, seqs.tok, n_tok=c.n_tok, max_new=2)
    q, pos = K.rows(c.q, "bf16"), torch.arange(c.n_tok, dtype=torch.int32, device="cuda")
    new = K.rows(c.new_k, "bf16"), K.rows(c.new_v, "bf16")
    for a, b in ((small, seqs), (big, far)):
        kv.append(a, b, *new, pos)
    assert torch.equal(kv.attend(small, seqs, q, decay=0.5), kv.attend(big, far, q, decay=0.5))
    for x, y in zip(kv.attend_blocks(small, seqs, q, 3), kv.attend_blocks(big, far, q, 3)):
        assert torch.equal(x, y)
    gone = kv.victims(small, seqs, 120, 4, 16, 200)
    for x, y in zip(gone, kv.victims(big, far, 120, 4, 16, 200)):
        assert torch.equal(x, y)
    kv.compact(small, seqs, *gone)
    kv.compact(big, far, *gone)
    for name in names:
        x, y = getattr(small, name), getattr(big, name)[at]
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype,dim,page,n_kv,lens,new", [
    ("bf16", 128, 64, 2, (1, 64, 65, 300), (1, 1, 1, 100)),
    ("fp16", 64, 16, 3, (40, 0, 7, 33), (40, 0, 9, 2)),          # a sequence with more tokens than entries
    ("bf16", 256, 32, 1, (70, 31), (33, 31)),
    ("fp16", 128, 256, 1, (700,), (513,)),
    ("bf16", 64, 128, 2, (129, 128, 127), (2, 3, 127))])
@pytest.mark.parametrize("strided", [False, True])
def test_append(kv, dtype, dim, page, n_kv, lens, new, strided):
    import torch
    c = K.Case(dtype, dim, page, n_kv, 1, lens, new, seed=dim + page, tail=2)
    pos = np.arange(1000, 1000 + c.n_tok).astype(np.int32)
    want = c.append(pos)
    pool, seqs = K.device(c)
    k, v = K.rows(c.new_k, dtype), K.rows(c.new_v, dtype)
    if strided:
        both = torch.stack((k, v), 1).reshape(c.n_tok, 2 * n_kv, dim)
        k, v = both[:, :n_kv], both[:, n_kv:]
    kv.append(pool, seqs, k, v, torch.from_numpy(pos).cuda())
    same_pool(pool, want)


def same_pool(pool, want):
    for name in ("k", "v", "weight", "pos", "box", "box_scale"):
        got = getattr(pool, name)
        if got is not None:
            got = got.double().cpu().numpy()
            assert np.array_equal(got, np.asarray(getattr(want, name), np.float64), equal_nan=True), name


def test_append_to_a_pool_of_keys_and_values_alone(kv):
    c = K.Case("bf16", 64, 16, 2, 1, (50, 20), (5, 20), missing=[(0, 3)], seed=1)
    want = c.append(np.zeros(c.n_tok, np.int32))
    pool, seqs = K.device(c, parts=())
    kv.append(pool, seqs, K.rows(c.new_k, "bf16"), K.rows(c.new_v, "bf16"))
    same_pool(pool, want)


def test_boxes_of_tiny_and_large_keys(kv):
    import torch
    c = K.Case("bf16", 64, 16, 1, 1, (16, 16, 16, 16), (16, 16, 16, 16), seed=1)
    for i, f in enumerate((0.0, 1e-37, 1e30, 2.0)):
        c.new_k[16 * i:16 * i + 16] = K.to_type(f * np.sign(c.new_k[16 * i:16 * i + 16]), "bf16")
    want = c.append(np.zeros(c.n_tok, np.int32))
    pool, seqs = K.device(c)
    kv.append(pool, seqs, K.rows(c.new_k, "bf16"), K.rows(c.new_v, "bf16"),
              torch.zeros(c.n_tok, dtype=torch.int32, device="cuda"))
    same_pool(pool, want)


# ------------------------------------------------------------------ sparse attention

def check_blocks(kv, c, n_sel, first, last):
    scale = c.dim ** -0.5
    sel = c.choose(n_sel, first, last)
    want, lse, _, tol, tol_lse, _ = c.attend(scale, chosen=sel)
    pool, seqs = K.device(c)
    out, got, e = kv.attend_blocks(pool, seqs, K.rows(c.q, c.dtype), n_sel, first, last, scale, lse=True)
    n = int(c.tok[-1])
    assert np.array_equal(got.cpu().numpy()[:n], sel[:n])
    K.near(out[:n], want[:n], tol[:n], "out")
    K.near(e[:n], lse[:n], tol_lse[:n], "lse")


@pytest.mark.parametrize("n_sel,first,last", [(1, 0, 1), (3, 1, 1), (6, 0, 2), (8, 2, 6), (64, 1, 4)])
@pytest.mark.parametrize("dtype,dim,page,n_kv,group,lens,new", [
    ("bf16", 128, 64, 2, 4, (1, 700, 64), (1, 1, 1)),
    ("fp16", 64, 16, 3, 1, (33, 0, 500, 16), (2, 0, 3, 16)),
    ("bf16", 256, 32, 1, 6, (350, 2), (2, 4)),
    ("fp16", 128, 16, 1, 17, (300,), (3,))])
def test_blocks(kv, dtype, dim, page, n_kv, group, lens, new, n_sel, first, last):
    check_blocks(kv, K.Case(dtype, dim, page, n_kv, group, lens, new, seed=n_sel), n_sel, first, last)


def test_blocks_many_pages_and_ties(kv):
    c = K.Case("bf16", 64, 16, 1, 2, (9000, 2000), (2, 1), seed=4)
    check_blocks(kv, c, 40, 1, 2)
    # the same box everywhere: the lowest pages win
    c.box[:] = c.box[0]
    c.box_scale[:] = 0.25
    check_blocks(kv, c, 33, 0, 1)


@pytest.mark.parametrize("bound", [300, 1500, 6000, 12000, 32768])
def test_blocks_by_the_bound_on_pages(kv, bound):
    """The kernel that chooses goes by the bound on the lengths: each of them, on the same pages."""
    c = K.Case("bf16", 64, 16, 1, 2, (4500, 900), (2, 1), max_pages=bound, seed=5)
    check_blocks(kv, c, 9, 1, 2)


def test_blocks_of_a_very_long_sequence(kv):
    c = K.Case("fp16", 64, 16, 1, 1, (144000,), (1,), seed=6)
    check_blocks(kv, c, 50, 2, 3)


def test_blocks_more_than_a_block_keeps(kv):
    """Over 1,024 chosen pages: a second piece of the walk."""
    check_blocks(kv, K.Case("bf16", 64, 16, 1, 2, (20000, 17000), (2, 1), seed=7), 1100, 0, 1)


def test_blocks_zero_queries_and_missing_pages(kv):
    c = K.Case("fp16", 64, 16, 2, 2, (300, 200), (1, 2), missing=[(0, 3), (0, 18), (1, 0), (1, 12)], seed=4)
    check_blocks(kv, c, 5, 1, 2)
    c.q[0] = 0.0
    check_blocks(kv, c, 5, 0, 1)


def test_blocks_of_all_pages_is_attention(kv):
    c = K.Case("bf16", 128, 32, 2, 4, (400, 90), (1, 2), seed=2)
    pool, seqs = K.device(c)
    q = K.rows(c.q, "bf16")
    out, sel = kv.attend_blocks(pool, seqs, q, 16)
    want, _, _, tol, _, _ = c.attend(128 ** -0.5)
    K.near(out, want, tol, "out")
    assert (sel[0, 0, :13].cpu() == np.arange(13)).all() and (sel[0, :, 13:] == -1).all()


# ------------------------------------------------------------------ eviction

def check_victims(kv, c, budget, first, recent, max_evict):
    want = c.victims(budget, first, recent, max_evict)
    pool, seqs = K.device(c)
    got = kv.victims(pool, seqs, budget, first, recent, max_evict)
    for a, b, name in zip(got, want, ("victims", "src", "new_len")):
        assert np.array_equal(a.cpu().numpy(), b), name
    after = c.compact(*want)
    kv.compact(pool, seqs, *got)
    same_pool(pool, after)
    kv.compact(pool, seqs, *got)                       # the same lists once more change nothing
    same_pool(pool, after)


@pytest.mark.parametrize("dtype,dim,page,n_kv", [("bf16", 64, 16, 3), ("fp16", 128, 64, 1), ("bf16", 256, 256, 2)])
@pytest.mark.parametrize("lens,budget,first,recent,max_evict", [
    ((1, 2, 0), 1, 0, 0, 1), ((65, 64, 63), 64, 4, 16, 1), ((300, 129, 40), 40, 4, 20, 400),
    ((300, 129, 40), 40, 4, 36, 17), ((511,), 200, 0, 0, 311), ((130,), 129, 0, 129, 3)])
@pytest.mark.parametrize("ties", [False, True])
def test_eviction(kv, dtype, dim, page, n_kv, lens, budget, first, recent, max_evict, ties):
    c = K.Case(dtype, dim, page, n_kv, 1, lens, (0,) * len(lens), seed=budget, ties=ties)
    check_victims(kv, c, budget, first, recent, max_evict)


def test_eviction_of_long_sequences(kv):
    for ties in (False, True):
        c = K.Case("bf16", 64, 64, 1, 1, (5000, 2100, 1024), (0, 0, 0), seed=1, ties=ties)
        check_victims(kv, c, 1000, 4, 64, 5000)
        check_victims(kv, c, 4999, 4, 64, 1)


@pytest.mark.parametrize("bound", [1000, 4096, 8000, 16000, 32768, 65536, 65552])
def test_eviction_by_the_bound_on_lengths(kv, bound):
    """The kernel goes by the bound on the lengths: each of them, on the same entries."""
    for ties in (False, True):
        c = K.Case("bf16", 64, 16, 2, 1, (900, 300, 0), (0, 0, 0), max_pages=(bound + 15) // 16, seed=2, ties=ties)
        check_victims(kv, c, 299, 3, 40, 700)
        check_victims(kv, c, 899, 3, 40, 2)
        check_victims(kv, c, 298, 0, 298, 2)


@pytest.mark.parametrize("length", [15000, 31001, 65536, 66001])
def test_eviction_of_very_long_sequences(kv, length):
    c = K.Case("bf16", 64, 256, 1, 1, (length, length - 7), (0, 0), seed=3)
    check_victims(kv, c, length // 3, 4, 100, length)
    check_victims(kv, c, length - 2, 4, 100, 3)


def test_eviction_of_equal_weights(kv):
    """Weights that were never added to: the lowest slots of the unprotected."""
    c = K.Case("bf16", 64, 64, 1, 1, (20000, 3000), (0, 0), seed=3)
    c.weight[:] = 0.0
    check_victims(kv, c, 1000, 4, 100, 20000)


def test_eviction_of_odd_weights(kv):
    """NaN, infinities, signed zeros and negative weights; one position everywhere: all are recent."""
    c = K.Case("bf16", 64, 16, 1, 1, (200,), (0,), seed=1)
    odd = np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, -1.0, 1e-42, 3e38], np.float32)
    for e in range(200):
        c.weight[c.pages[0, e // 16], 0, e % 16] = odd[(e * 5) % 8]
    check_victims(kv, c, 90, 2, 10, 200)
    c.pos[:] = 5
    check_victims(kv, c, 190, 0, 3, 200)
    c.pos[:] = 2 ** 31 - 1
    check_victims(kv, c, 190, 0, 190, 200)


def test_eviction_with_missing_pages(kv):
    c = K.Case("bf16", 64, 16, 2, 1, (100, 90), (0, 0), missing=[(0, 2), (1, 5)], seed=3)
    check_victims(kv, c, 50, 2, 10, 60)


# ------------------------------------------------------------------ together

def test_a_session_grows_attends_and_is_kept_within_its_budget(kv):
    """Turns appended, attended over and evicted, step after step, as a serving loop runs them: every
    step against the plain implementation on the state that the GPU left."""
    import torch
    c = K.Case("bf16", 64, 16, 2, 2, (0, 0), (0, 0), max_pages=8, spare=20, seed=0)
    c.pages[0], c.pages[1] = np.arange(8), np.arange(8, 16)
    c.k[:], c.v[:], c.weight[:] = np.nan, np.nan, np.nan
    pool, _ = K.device(c)
    length = torch.zeros(2, dtype=torch.int32, device="cuda")
    pages = torch.from_numpy(c.pages).cuda()
    r = np.random.Generator(np.random.PCG64(1))
    at = [0, 0]
    for new in ((60, 3), (1, 50), (1, 1), (20, 1), (1, 1), (0, 30)):
        c.new, c.tok = list(new), np.array([0, new[0], sum(new)], np.int32)
        c.n_tok, c.lens = sum(new), [int(x) + n for x, n in zip(length.cpu(), new)]
        c.q, c.new_k, c.new_v = (K.to_type(r.standard_normal((c.n_tok, h, 64)), "bf16") for h in (4, 2, 2))
        pos = np.concatenate([np.arange(a, a + n) for a, n in zip(at, new)]).astype(np.int32)
        at = [a + n for a, n in zip(at, new)]
        tok = torch.from_numpy(c.tok).cuda()
        length.copy_(torch.tensor(c.lens, dtype=torch.int32))
        seqs = kv.Seqs(pages, length, tok, n_tok=c.n_tok, max_new=max(new))
        kv.append(pool, seqs, K.rows(c.new_k, "bf16"), K.rows(c.new_v, "bf16"), torch.from_numpy(pos).cuda())
        c = c.append(pos)
        same_pool(pool, c)
        want, _, got, tol, _, tol_got = c.attend(0.125)
        K.near(kv.attend(pool, seqs, K.rows(c.q, "bf16"), 0.125, decay=1.0), want, tol, "out")
        weight = pool.weight.cpu().numpy()
        for i, n in enumerate(c.lens):
            if not new[i]:
                continue
            for e in range(n):
                p, s = c.pages[i, e // 16], e % 16
                w = c.weight[p, :, s].astype(np.float64) + got[i][:, e]
                assert (np.abs(weight[p, :, s] - w) <= tol_got[i][:, e] + 2.0 ** -24 * (2 * new[i] + 4) * w).all()
        c.weight = weight
        sel = c.choose(3, 1, 1)
        sparse, chosen = kv.attend_blocks(pool, seqs, K.rows(c.q, "bf16"), 3, 1, 1, 0.125)
        assert np.array_equal(chosen.cpu().numpy(), sel)
        want, _, _, tol, _, _ = c.attend(0.125, chosen=sel)
        K.near(sparse, want, tol, "sparse out")
        lists = c.victims(40, 2, 8, 64)
        gone = kv.victims(pool, seqs, 40, 2, 8, 64)
        for a, b in zip(gone, lists):
            assert np.array_equal(a.cpu().numpy(), b)
        kv.compact(pool, seqs, *gone)
        c = c.compact(*lists)
        same_pool(pool, c)
        length.copy_(gone[2])
    assert length.tolist() == [40, 40]


def test_captured_steps_replay_as_eager_ones(kv):
    """A decode step with weights, sparse attention and an eviction, recorded once and replayed among
    eager calls; two graphs of it hold workspaces of their own."""
    import torch
    c = K.Case("bf16", 128, 64, 2, 4, (1000, 300), (1, 1), seed=1)
    pool, seqs = K.device(c)
    other, seqs2 = K.device(c)
    q = K.rows(c.q, "bf16")

    def step(pool, seqs):
        out = kv.attend(pool, seqs, q, decay=1.0)
        sparse, sel = kv.attend_blocks(pool, seqs, q, 4)
        gone = kv.victims(pool, seqs, 250, 4, 16, 800)
        kv.append(pool, seqs, q[:, :2], q[:, 2:4], seqs.tok[:2])
        return [out, sparse, sel, *gone]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(pool, seqs)
    torch.cuda.synchronize()
    pool.weight.copy_(other.weight)
    for name in ("k", "v", "pos", "box", "box_scale"):
        getattr(pool, name).copy_(getattr(other, name))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step(pool, seqs)
        graphs.append((g, got))
    for turn in range(4):
        g, got = graphs[turn % 2]
        g.replay()
        want = step(other, seqs2)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), turn
        for name in ("k", "v", "weight", "pos", "box", "box_scale"):
            assert torch.equal(getattr(pool, name).view(torch.uint8), getattr(other, name).view(torch.uint8)), name


def test_calls_on_another_stream(kv):
    import torch
    c = K.Case("bf16", 64, 16, 1, 2, (500,), (1,), seed=1)
    pool, seqs = K.device(c)
    q = K.rows(c.q, "bf16")
    want = kv.attend(pool, seqs, q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = kv.attend(pool, seqs, q)
    s.synchronize()
    assert torch.equal(got, want)
