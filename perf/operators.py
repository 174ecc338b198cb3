"""The operators on the paged KV of a pool's sessions, as measurable cases.

A session's KV lives in pages of `page` entries: k [n_pages][n_kv][page][dim], v transposed inside
its page [n_pages][n_kv][dim][page], and per entry and kv head the accumulated attention weight, the
token position and, per page and kv head, an int8 box around its keys.  Five operators:

  append   a turn's new tokens into their sessions' pages
  attend   attention of the newest tokens over their session, adding up each entry's weight
  blocks   the same over the pages that a cheap integer score selects for each token
  victims  the entries of least weight that go, and the entries that move into their slots
  compact  those moves

A case is a plain dict.  Lengths follow from it alone: `ragged` spreads them below `length` and `new`.
With own = False, `run` computes the plain form in torch; with own = True it calls the framework.
"""
import torch

own = False


def listed():
    return [
        # a decode step of a serving batch: one new token each for 64 sessions
        {"name": "append_step", "op": "append", "dtype": "bf16", "seqs": 64, "length": 2048, "new": 1, "ragged": 0.9,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64},
        # turns of 200 to 2,000 new tokens over resident prefixes, the growth of a session's prompt
        {"name": "append_turns", "op": "append", "dtype": "bf16", "seqs": 16, "length": 6001, "new": 2000, "ragged": 0.9,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64},
        # the smallest call: one session of a small model decodes a token
        {"name": "decode_one", "op": "attend", "dtype": "fp16", "seqs": 1, "length": 777, "new": 1, "ragged": 0.0,
         "n_q": 8, "n_kv": 2, "dim": 64, "page": 16, "weight": False},
        # a decode step of a large batch whose pool evicts by weight
        {"name": "decode_batch", "op": "attend", "dtype": "bf16", "seqs": 64, "length": 16384, "new": 1, "ragged": 0.8,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "weight": True},
        # a few drafted tokens each, one kv head, an odd group and wide heads
        {"name": "draft_fp16", "op": "attend", "dtype": "fp16", "seqs": 13, "length": 5003, "new": 5, "ragged": 0.7,
         "n_q": 6, "n_kv": 1, "dim": 256, "page": 32, "weight": False},
        # new turns over resident prefixes, weights kept
        {"name": "turns", "op": "attend", "dtype": "bf16", "seqs": 4, "length": 12001, "new": 2000, "ragged": 0.5,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "weight": True},
        # one long session decodes over the selected 64 of its 2,047 pages
        {"name": "blocks_long", "op": "blocks", "dtype": "bf16", "seqs": 1, "length": 131000, "new": 1, "ragged": 0.0,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "select": 64, "first": 1, "last": 2},
        # a batch of long sessions with two tokens each
        {"name": "blocks_batch", "op": "blocks", "dtype": "bf16", "seqs": 24, "length": 32768, "new": 2, "ragged": 0.7,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "select": 40, "first": 1, "last": 4},
        # steady state: every session is one entry over its budget
        {"name": "victims_step", "op": "victims", "dtype": "bf16", "seqs": 64, "length": 4097, "new": 1, "ragged": 0.0,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "budget": 4096, "first": 4, "recent": 256},
        # after long prompts: down to a budget in one go
        {"name": "victims_bulk", "op": "victims", "dtype": "bf16", "seqs": 8, "length": 32768, "new": 1, "ragged": 0.6,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "budget": 8192, "first": 4, "recent": 512},
        # the moves of the two
        {"name": "compact_step", "op": "compact", "dtype": "bf16", "seqs": 64, "length": 4097, "new": 1, "ragged": 0.0,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "budget": 4096, "first": 4, "recent": 256},
        {"name": "compact_bulk", "op": "compact", "dtype": "bf16", "seqs": 8, "length": 32768, "new": 1, "ragged": 0.6,
         "n_q": 32, "n_kv": 8, "dim": 128, "page": 64, "budget": 8192, "first": 4, "recent": 512},
    ]


def _log_int(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return int(min(hi, max(lo, round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "attend", "blocks", "victims", "compact"))
    n_kv = rng.choice((1, 2, 3, 4, 8))
    c = {"op": op, "dtype": rng.choice(("bf16", "fp16")), "seqs": _log_int(rng, 1, 64), "ragged": round(rng.uniform(0, 0.95), 3),
         "n_kv": n_kv, "n_q": n_kv * rng.choice((1, 2, 3, 4, 5, 7, 8, 16)), "dim": rng.choice((64, 128, 128, 256)),
         "page": rng.choice((16, 32, 64, 128, 256))}
    entry = 4 * n_kv * c["dim"]  # bytes of an entry
    if op in ("append", "attend"):
        c["new"] = _log_int(rng, 1, 2500) if rng.random() < 0.5 else rng.randint(1, 8)
        # within the bytes of the largest listed case, and within its products
        most = min(40000, (1 << 31) // (entry * c["seqs"]), 1_500_000_000 // max(1, c["seqs"] * c["new"] * c["n_q"]) * 128 // c["dim"])
        c["length"] = _log_int(rng, 1, max(2, most))
        c["new"] = min(c["new"], c["length"])
        if op == "attend":
            c["weight"] = rng.random() < 0.5
        return c
    if op == "blocks":
        c["new"] = rng.choice((1, 1, 2, 3, 5))
        c["length"] = _log_int(rng, 100, min(200000, (1 << 31) // (entry * c["seqs"])))
        c["new"] = min(c["new"], c["length"])
        c["first"], c["last"] = rng.randint(0, 2), rng.randint(1, 4)
        c["select"] = c["first"] + c["last"] + _log_int(rng, 1, 100)
        return c
    c["new"] = 1
    c["length"] = _log_int(rng, 20, min(60000, (1 << 31) // (entry * c["seqs"])))
    c["budget"] = max(8, c["length"] - 1 if rng.random() < 0.3 else int(c["length"] * rng.uniform(0.1, 0.99)))
    c["first"] = rng.randint(0, 4)
    c["recent"] = rng.randint(0, c["budget"] - 4)
    return c


# ------------------------------------------------------------------ sizes

def _sizes(c):
    """Lengths and new tokens of each sequence: the first one has the largest."""
    length, new = [], []
    for i in range(c["seqs"]):
        n = max(1, int(c["length"] * (1.0 - c["ragged"] * ((i * 0.6180339887) % 1.0))))
        length.append(n)
        new.append(min(n, max(1, int(c["new"] * (1.0 - c["ragged"] * ((i * 0.7548776662) % 1.0))))))
    return length, new


def _seen(length, new):
    """(row, entry) pairs that the new tokens see."""
    return sum(n * ln - n * (n - 1) // 2 for ln, n in zip(length, new))


def work(case):
    c = case
    length, new = _sizes(c)
    toks, entry, row = sum(new), 4 * c["n_kv"] * c["dim"], 2 * c["dim"]
    if c["op"] == "append":
        # the rows in and out with their weights and positions, and the key rows that share their pages for the box
        pages = [(ln - 1) // c["page"] - (ln - n) // c["page"] + 1 for ln, n in zip(length, new)]
        shared = sum((ln - n) % c["page"] for ln, n in zip(length, new))
        return {"bytes": 2 * toks * entry + 8 * toks * c["n_kv"] + shared * entry // 2
                + sum(pages) * c["n_kv"] * (2 * c["dim"] + 4), "flops": 4 * toks * c["n_kv"] * c["dim"]}
    if c["op"] == "attend":
        weights = 8 * c["n_kv"] * sum(length) if c["weight"] else 0
        return {"bytes": sum(length) * entry + 2 * toks * c["n_q"] * row + weights,
                "flops": 4 * c["n_q"] * c["dim"] * _seen(length, new)}
    if c["op"] == "blocks":
        blocks = [-(-ln // c["page"]) for ln in length]
        kept = [min(b, c["select"]) for b in blocks]
        return {"bytes": sum(blocks) * c["n_kv"] * (2 * c["dim"] + 4) + sum(k * n for k, n in zip(kept, new)) * c["page"] * entry
                + 2 * toks * c["n_q"] * row + 4 * toks * c["n_kv"] * c["select"],
                "flops": 4 * c["n_q"] * c["dim"] * c["page"] * sum(k * n for k, n in zip(kept, new))
                + 4 * c["n_kv"] * c["dim"] * sum(b * n for b, n in zip(blocks, new))}
    gone = [max(0, ln - c["budget"]) for ln in length]
    if c["op"] == "victims":
        return {"bytes": c["n_kv"] * sum(8 * ln for ln in length) + 8 * c["n_kv"] * c["seqs"] * max(1, max(gone)),
                "flops": c["n_kv"] * sum(length)}
    # a victim in the kept part is filled by an entry behind it: about budget / length of the victims
    moved = sum(g * min(ln, c["budget"]) // ln for g, ln in zip(gone, length))
    return {"bytes": 2 * moved * (entry + 8 * c["n_kv"]) + 8 * c["n_kv"] * c["seqs"] * max(1, max(gone)), "flops": 0}


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[c["dtype"]]
    n_kv, dim, page = c["n_kv"], c["dim"], c["page"]
    length, new = _sizes(c)
    per = -(-c["length"] // page)
    n_pages = sum(-(-ln // page) for ln in length) + 3

    def rand(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    # keys drift from page to page and share a bias over the channels; queries are sharper than unit ones
    k = torch.randn((n_pages, n_kv, page, dim), generator=g, device="cuda", dtype=dt)
    k += (rand(n_pages, n_kv, 1, dim) * 0.5 + rand(1, n_kv, 1, dim) * 0.5).to(dt)
    v = torch.randn((n_pages, n_kv, dim, page), generator=g, device="cuda", dtype=dt)
    weight = torch.exp(2.0 * rand(n_pages, n_kv, page))
    weight[torch.rand(weight.shape, generator=g, device="cuda") < 0.03] = 0.0  # entries that no token looked at
    pages = torch.full((c["seqs"], per), -1, dtype=torch.int32)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
    at = 0
    for i, ln in enumerate(length):
        n = -(-ln // page)
        pages[i, :n] = order[at:at + n]
        at += n
    pages = pages.cuda()
    s = {"case": c, "k": k, "v": v, "weight": weight, "pages": pages,
         "length": torch.tensor(length, dtype=torch.int32).cuda(),
         "tok": torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda(),
         "n_tok": sum(new), "max_new": max(new), "max_len": max(length), "scale": dim ** -0.5}
    if c["op"] in ("append", "blocks"):
        s["box"] = torch.empty((n_pages, n_kv, 2, dim), device="cuda", dtype=torch.int8)
        s["box_scale"] = torch.empty((n_pages, n_kv), device="cuda", dtype=torch.float32)
        slots = torch.arange(per * page, device="cuda")
        live = (slots < s["length"][:, None]).view(c["seqs"], per, page)
        box, box_scale = _box(k[pages.clamp(min=0).long()].float(), live[:, :, None, :, None])
        there = pages >= 0
        s["box"].zero_()[pages[there].long()] = box[there]
        s["box_scale"].zero_()[pages[there].long()] = box_scale[there]
    if c["op"] != "blocks":
        s["pos"] = torch.zeros((n_pages, n_kv, page), device="cuda", dtype=torch.int32)
    if c["op"] == "append":
        s["new_k"] = rand(s["n_tok"], n_kv, dim).to(dt)
        s["new_v"] = rand(s["n_tok"], n_kv, dim).to(dt)
        s["new_pos"] = torch.cat([torch.arange(ln - n, ln, dtype=torch.int32) for ln, n in zip(length, new)]).cuda()
    elif c["op"] in ("attend", "blocks"):
        weight /= c["length"]  # of the size that one call adds
        s["q"] = (1.5 * rand(s["n_tok"], c["n_q"], dim)).to(dt)
    else:
        # the kept entries of earlier evictions stand in any order, each kv head in its own
        for i, ln in enumerate(length):
            n = -(-ln // page)
            p = torch.argsort(torch.rand((n_kv, n * page), generator=g, device="cuda"), dim=1).to(torch.int32)
            s["pos"][pages[i, :n].long()] = p.view(n_kv, n, page).permute(1, 0, 2)
        s["max_evict"] = max(1, max(length) - c["budget"])
        if c["op"] == "compact":
            s["victims"], s["src"], s["new_len"] = _victims(s)
    return s


# ------------------------------------------------------------------ plain forms

def _box(k, live):
    """int8 boxes of key pages [..., page, dim] with a power-of-two scale: their largest
    magnitude lies in [64, 128) steps; the lower side rounds down, the upper side up."""
    lo = torch.where(live, k, float("inf")).amin(-2)
    hi = torch.where(live, k, float("-inf")).amax(-2)
    top = torch.maximum(lo.abs(), hi.abs()).amax(-1, keepdim=True)
    e = (top.view(torch.int32) >> 23) & 255          # 2^(e - 127) <= top < 2^(e - 126)
    tiny = e < 7
    inv = torch.where(tiny, 0, (260 - e) << 23).view(torch.float32)
    step = torch.where(tiny, 0, (e - 6) << 23).view(torch.float32)
    lo, hi = torch.floor(lo * inv), torch.ceil(hi * inv)
    return torch.stack((lo, hi), -2).clamp(-127, 127).to(torch.int8), step[..., 0]


def _padded(s):
    """(token of each row of [seqs][max_new], whether it is one)."""
    j = torch.arange(s["max_new"], device="cuda")
    t0, t1 = s["tok"][:-1, None].long(), s["tok"][1:, None].long()
    return (t0 + j).clamp(max=s["n_tok"] - 1), t0 + j < t1


def _packed(s, rows):
    """[seqs][max_new][...] back to [n_tok][...]."""
    t = torch.arange(s["n_tok"], device="cuda")
    i = torch.searchsorted(s["tok"][1:].long(), t, right=True)
    return rows[i, t - s["tok"][i].long()]


def _slots(s):
    """Page and slot of each entry [seqs][per * page], and whether the sequence has it."""
    c, per = s["case"], s["pages"].shape[1]
    e = torch.arange(per * c["page"], device="cuda")
    page = s["pages"].repeat_interleave(c["page"], 1).long()
    return page.clamp(min=0), (e % c["page"]).expand(page.shape), (e < s["length"][:, None]) & (page >= 0)


def _of_seqs(x):
    """[seqs][per][n_kv][page] -> [seqs][n_kv][per * page]."""
    return x.permute(0, 2, 1, 3).reshape(x.shape[0], x.shape[2], -1)


def _seq_rows(s):
    """Keys and values [seqs][n_kv][per * page][dim] in 32 bits, zero where there is no entry."""
    p = s["pages"].clamp(min=0).long()
    n, per, n_kv, dim = p.shape[0], p.shape[1], s["case"]["n_kv"], s["case"]["dim"]
    live = _slots(s)[2][:, None, :, None]
    k = s["k"][p].float().permute(0, 2, 1, 3, 4).reshape(n, n_kv, -1, dim)
    v = s["v"][p].float().permute(0, 2, 1, 4, 3).reshape(n, n_kv, -1, dim)
    return torch.where(live, k, 0.0), torch.where(live, v, 0.0)


def _softmax_rows(s, chosen=None):
    """Attention of the new tokens: out [n_tok][n_q][dim] and the probabilities
    [seqs][n_kv][max_new * group][per * page]; `chosen` [seqs][n_kv][max_new][per]: the pages each token reads."""
    c = s["case"]
    n, n_kv, group, m = c["seqs"], c["n_kv"], c["n_q"] // c["n_kv"], s["max_new"]
    k, v = _seq_rows(s)
    tok, is_tok = _padded(s)
    q = s["q"][tok].float().view(n, m, n_kv, group, -1).permute(0, 2, 1, 3, 4).reshape(n, n_kv, m * group, -1)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]).view(n, n_kv, m, group, -1)
    e, new = torch.arange(k.shape[2], device="cuda"), (s["tok"][1:] - s["tok"][:-1]).long()
    limit = s["length"].long()[:, None] - new[:, None] + torch.arange(m, device="cuda") + 1
    see = (e < limit[..., None]) & _slots(s)[2][:, None, :] & is_tok[..., None]      # [n][m][entries]
    see = see[:, None] if chosen is None else see[:, None] & chosen.repeat_interleave(c["page"], -1)
    x.masked_fill_(~see[:, :, :, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(torch.where(top == float("-inf"), 0.0, top)))
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, 1.0, total))
    p = p.view(n, n_kv, m * group, -1)
    out = torch.matmul(p, v).view(n, n_kv, m, group, -1).permute(0, 2, 1, 3, 4).reshape(n, m, c["n_q"], -1)
    return _packed(s, out).to(s["q"].dtype), p


def _append(s):
    c = s["case"]
    t = torch.arange(s["n_tok"], device="cuda")
    i = torch.searchsorted(s["tok"][1:].long(), t, right=True)
    e = s["length"][i].long() - s["tok"][i + 1].long() + t
    page, slot = s["pages"][i, e // c["page"]].long(), e % c["page"]
    s["k"][page, :, slot] = s["new_k"]
    s["v"].transpose(2, 3)[page, :, slot] = s["new_v"]
    s["weight"][page, :, slot] = 0.0
    s["pos"][page, :, slot] = s["new_pos"][:, None]
    # the boxes of the pages that got entries, over every live entry of theirs
    first = (s["length"] - (s["tok"][1:] - s["tok"][:-1])) // c["page"]
    j = torch.arange(s["pages"].shape[1], device="cuda")
    touched = (j >= first[:, None]) & (j * c["page"] < s["length"][:, None])
    seq, at = touched.nonzero(as_tuple=True)
    slots = at[:, None] * c["page"] + torch.arange(c["page"], device="cuda")
    live = slots < s["length"][seq][:, None]
    p = s["pages"][seq, at].long()
    s["box"][p], s["box_scale"][p] = _box(s["k"][p].float(), live[:, None, :, None])
    return [s["k"], s["v"], s["weight"], s["pos"], s["box"], s["box_scale"]]


def _attend(s):
    c = s["case"]
    out, p = _softmax_rows(s)
    if not c["weight"]:
        return [out]
    page, slot, live = _slots(s)
    got = p.sum(2)                                                   # [seqs][n_kv][entries]
    s["weight"][page[live], :, slot[live]] += got.transpose(1, 2)[live]
    return [out, s["weight"]]


def _blocks(s):
    c = s["case"]
    n, n_kv, group, m, per = c["seqs"], c["n_kv"], c["n_q"] // c["n_kv"], s["max_new"], s["pages"].shape[1]
    tok, is_tok = _padded(s)
    q = s["q"].float().view(s["n_tok"], n_kv, -1)
    e = (q.abs().amax(-1).view(torch.int32) >> 23) & 255
    inv = torch.where(e < 7, 0, (260 - e) << 23).view(torch.float32)
    qi = torch.round(q * inv[..., None]).clamp(-127, 127).view(s["n_tok"], n_kv, group, -1)
    both = torch.cat((qi.clamp(max=0).sum(2), qi.clamp(min=0).sum(2)), -1)[tok].permute(0, 2, 1, 3)
    page = s["pages"].clamp(min=0).long()
    box = s["box"][page].permute(0, 2, 3, 4, 1).reshape(n, n_kv, -1, per)
    # whole numbers: exact in 64 bits whatever the order of the sum
    score = torch.matmul(both.double(), box.double()).float() * s["box_scale"][page].transpose(1, 2)[:, :, None]
    new = (s["tok"][1:] - s["tok"][:-1]).long()
    limit = s["length"].long()[:, None] - new[:, None] + torch.arange(m, device="cuda") + 1
    count = ((limit + c["page"] - 1) // c["page"])[:, None, :, None]      # pages that the token sees
    j = torch.arange(per, device="cuda")
    score = torch.where((j < c["first"]) | (j >= count - c["last"]), float("inf"), score)
    there = (j < count) & (s["pages"] >= 0)[:, None, None] & is_tok[:, None, :, None]
    score = torch.where(there, score, float("-inf"))
    best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :c["select"]]
    chosen = torch.zeros_like(there.expand(n, n_kv, m, per)).scatter_(-1, best, True) & there
    sel = torch.sort(torch.where(chosen, j, per), dim=-1)[0][..., :c["select"]]
    sel = torch.nn.functional.pad(torch.where(sel < per, sel, -1), (0, c["select"] - sel.shape[-1]), value=-1)
    out, _ = _softmax_rows(s, chosen)
    return [out, _packed(s, sel.transpose(1, 2)).to(torch.int32)]


def _victims(s):
    c, most = s["case"], s["max_evict"]
    page = s["pages"].clamp(min=0).long()
    live = _slots(s)[2][:, None]
    weight, pos = _of_seqs(s["weight"][page]), _of_seqs(s["pos"][page]).long()
    newest = torch.where(live, pos, -1).amax(-1, keepdim=True)
    kept = (pos < c["first"]) | (pos > newest - c["recent"])
    key = torch.where(live, torch.where(kept, float("inf"), weight), float("inf"))
    n = (s["length"].long() - c["budget"]).clamp(min=0, max=most)
    new_len = s["length"].long() - n
    order = torch.sort(key, dim=-1, stable=True)[1]
    rank = torch.empty_like(order).scatter_(-1, order, torch.arange(key.shape[-1], device="cuda").expand_as(order))
    goes = (rank < n[:, None, None]) & live
    e, none = torch.arange(key.shape[-1], device="cuda"), key.shape[-1]
    fill = torch.nn.functional.pad
    v = torch.sort(torch.where(goes, e, none), dim=-1)[0][..., :most]
    stays = live & ~goes & (e >= new_len[:, None, None])
    src = torch.sort(torch.where(stays, e, none), dim=-1)[0][..., :most]
    v, src = (fill(torch.where(x < none, x, -1), (0, most - x.shape[-1]), value=-1) for x in (v, src))
    src = torch.where((v >= 0) & (v < new_len[:, None, None]), src, -1)
    return v.to(torch.int32), src.to(torch.int32), new_len.to(torch.int32)


def _compact(s):
    c = s["case"]
    i, h, j = (s["src"] >= 0).nonzero(as_tuple=True)
    dst, src = s["victims"][i, h, j].long(), s["src"][i, h, j].long()
    to, at = s["pages"][i, dst // c["page"]].long(), dst % c["page"]
    fr, ft = s["pages"][i, src // c["page"]].long(), src % c["page"]
    s["k"][to, h, at] = s["k"][fr, h, ft]
    s["v"].transpose(2, 3)[to, h, at] = s["v"].transpose(2, 3)[fr, h, ft]
    s["weight"][to, h, at] = s["weight"][fr, h, ft]
    s["pos"][to, h, at] = s["pos"][fr, h, ft]
    return [s["k"], s["v"], s["weight"], s["pos"]]


# ------------------------------------------------------------------ the framework's calls

def _handles(s):
    """The pool and the batch of sequences, as a program makes them once for its tensors."""
    if "pool" not in s:
        from paper_2609_09643_amd import kv
        c = s["case"]
        s["pool"] = kv.Pool(s["k"], s["v"], weight=s["weight"], pos=s.get("pos"), box=s.get("box"),
                            box_scale=s.get("box_scale"))
        s["seqs"] = kv.Seqs(s["pages"], s["length"], s["tok"], n_tok=s["n_tok"], max_new=s["max_new"],
                            max_len=s["max_len"])
        s["call"] = {"append": _own_append, "attend": _own_attend, "blocks": _own_blocks, "victims": _own_victims,
                     "compact": _own_compact}[c["op"]]
        s["kv"] = kv
    return s["kv"], s["pool"], s["seqs"]


def _own_append(s):
    kv, pool, seqs = _handles(s)
    kv.append(pool, seqs, s["new_k"], s["new_v"], s["new_pos"])
    return [s["k"], s["v"], s["weight"], s["pos"], s["box"], s["box_scale"]]


def _own_attend(s):
    kv, pool, seqs = _handles(s)
    if not s["case"]["weight"]:
        return [kv.attend(pool, seqs, s["q"], s["scale"])]
    return [kv.attend(pool, seqs, s["q"], s["scale"], decay=1.0), s["weight"]]


def _own_blocks(s):
    kv, pool, seqs = _handles(s)
    c = s["case"]
    out, sel = kv.attend_blocks(pool, seqs, s["q"], c["select"], first=c["first"], last=c["last"], scale=s["scale"])
    return [out, sel]


def _own_victims(s):
    kv, pool, seqs = _handles(s)
    c = s["case"]
    return list(kv.victims(pool, seqs, c["budget"], first=c["first"], recent=c["recent"], max_evict=s["max_evict"]))


def _own_compact(s):
    kv, pool, seqs = _handles(s)
    kv.compact(pool, seqs, s["victims"], s["src"], s["new_len"])
    return [s["k"], s["v"], s["weight"], s["pos"]]


def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "blocks": _own_blocks, "victims": _own_victims,
                "compact": _own_compact}[op](state)
    return {"append": _append, "attend": _attend, "blocks": _blocks, "victims": _victims, "compact": _compact}[op](state)


# ------------------------------------------------------------------ in 64 bits, sequence by sequence

def exact(case, seed):
    c = case
    if c["op"] == "victims":
        return None  # whole numbers
    length, new = _sizes(c)
    # the products of all heads together: about 20 s at most
    if c["op"] != "append" and c["n_q"] * c["dim"] * sum(n * ln for n, ln in zip(new, length)) > 6e12:
        return None
    s = prepare(case, seed)
    if c["op"] == "compact":
        k, v, weight, where = s["k"].double(), s["v"].double(), s["weight"].double(), s["pages"].cpu()
        for i in range(c["seqs"]):
            for h in range(c["n_kv"]):
                n = int((s["src"][i, h] >= 0).sum())
                d, f = s["victims"][i, h, :n].cpu().long(), s["src"][i, h, :n].cpu().long()
                to, fr = where[i, d // c["page"]].long().cuda(), where[i, f // c["page"]].long().cuda()
                d, f = d.cuda() % c["page"], f.cuda() % c["page"]
                k[to, h, d] = k[fr, h, f]
                v[to, h, :, d] = v[fr, h, :, f]
                weight[to, h, d] = weight[fr, h, f]
        return [k, v, weight, None]
    if c["op"] == "append":
        # copies, and the boxes' steps: 2^(e - 7) where the largest magnitude of a page is in [2^(e - 1), 2^e)
        step, k, v, weight = s["box_scale"].double(), s["k"].double(), s["v"].double(), s["weight"].double()
        at = 0
        for i, (ln, n) in enumerate(zip(length, new)):
            for b in range((ln - n) // c["page"], -(-ln // c["page"])):
                p = int(s["pages"][i, b])
                old = s["k"][p, :, :max(0, ln - n - b * c["page"])].double()
                lo, hi = max(0, b * c["page"] - (ln - n)), min(n, (b + 1) * c["page"] - (ln - n))
                rows = torch.cat((old, s["new_k"][at + lo:at + hi].double().transpose(0, 1)), 1)
                first, n_rows = old.shape[1], hi - lo
                k[p, :, first:first + n_rows] = rows[:, first:]
                v[p, :, :, first:first + n_rows] = s["new_v"][at + lo:at + hi].double().permute(1, 2, 0)
                weight[p, :, first:first + n_rows] = 0.0
                top = rows.abs().amax((1, 2))
                step[p] = torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - 7)
            at += n
        return [k, v, weight, None, None, step]
    group, page = c["n_q"] // c["n_kv"], c["page"]
    weight = s["weight"].double() if c["op"] == "attend" and c["weight"] else None
    outs, at = [], 0
    for i, (ln, n) in enumerate(zip(length, new)):
        p = s["pages"][i, :-(-ln // page)].long()
        got = torch.zeros((c["n_kv"], len(p) * page), dtype=torch.float64, device="cuda")
        out = torch.zeros((n, c["n_q"], c["dim"]), dtype=torch.float64, device="cuda")
        for h in range(c["n_kv"]):
            k = s["k"][p, h].double().reshape(-1, c["dim"])[:ln]
            v = s["v"][p, h].double().transpose(1, 2).reshape(-1, c["dim"])[:ln]
            q = s["q"][at:at + n, h * group:(h + 1) * group].double()
            x = torch.tensordot(q, k, dims=([2], [1])) * s["scale"]              # [n][group][ln]
            see = torch.arange(ln, device="cuda") <= (torch.arange(n, device="cuda") + ln - n)[:, None]
            if c["op"] == "blocks":
                see = see & _exact_pages(s, c, q, p, h, ln, n)[:, torch.arange(ln, device="cuda") // page]
            x = torch.where(see[:, None], x, -float("inf"))
            a = torch.softmax(x, -1)
            out[:, h * group:(h + 1) * group] = torch.tensordot(a, v, dims=([2], [0]))
            got[h, :ln] = a.sum((0, 1))
        if weight is not None:
            weight[p] += got.view(c["n_kv"], len(p), page).transpose(0, 1)
        outs.append(out)
        at += n
    out = torch.cat(outs)
    return [out] if weight is None and c["op"] == "attend" else [out, weight]


def _exact_pages(s, c, q, p, h, ln, n):
    """The pages that each of a sequence's new tokens reads, [n][pages]: the scores summed
    dimension by dimension as the larger product with the box's two sides."""
    e = torch.frexp(q.abs().amax((1, 2)))[1]
    qi = torch.round(torch.ldexp(q, (7 - e)[:, None, None])).clamp(-127, 127)
    box = s["box"][p, h].double()
    score = torch.zeros((n, len(p)), dtype=torch.float64, device="cuda")
    for a in range(q.shape[1]):
        score += torch.maximum(qi[:, a, None] * box[None, :, 0], qi[:, a, None] * box[None, :, 1]).sum(-1)
    score = (score.float() * s["box_scale"][p, h]).cpu()
    use = torch.zeros((n, len(p)), dtype=torch.bool)
    for t in range(n):
        count = -(-(ln - n + t + 1) // c["page"])
        must = set(range(min(c["first"], count))) | set(range(max(0, count - c["last"]), count))
        rest = sorted((j for j in range(count) if j not in must), key=lambda j: (-float(score[t, j]), j))
        use[t, sorted(must) + rest[:max(0, c["select"] - len(must))]] = True
    return use.cuda()
