"""Python binding of the paged-KV operators (argument marshalling only).

A Pool is the pages of the sessions that the residency policy kept, a Seqs the
batch of sequences over it; append, attend, attend_blocks, victims and compact
are the calls of include/unison.h with the same meaning.  Every call runs on
the current stream of the tensors' device and allocates its outputs and its
workspace with torch, so calls on several streams or in several captured
graphs do not share memory.  The tensors behind a Pool and a Seqs stay where
they are: lengths and page tables are updated in place.  There is no backward
pass: tensors that autograd follows are refused.
"""
from __future__ import annotations

import ctypes as C

from .unison import E_INVALID, UnisonError, _check, lib

BF16, FP16 = 0, 1


class PoolArgs(C.Structure):
    _fields_ = [("dtype", C.c_uint32), ("head_dim", C.c_uint32), ("n_kv", C.c_uint32), ("page", C.c_uint32),
                ("n_pages", C.c_uint32), ("pad0", C.c_uint32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("weight", C.c_void_p), ("pos", C.c_void_p), ("box", C.c_void_p), ("box_scale", C.c_void_p)]


class SeqsArgs(C.Structure):
    _fields_ = [("n_seq", C.c_uint32), ("max_pages", C.c_uint32), ("n_tok", C.c_uint32), ("max_new", C.c_uint32),
                ("max_len", C.c_uint32), ("pad0", C.c_uint32), ("pages", C.c_void_p), ("len", C.c_void_p),
                ("tok", C.c_void_p)]


class RowsArgs(C.Structure):
    _fields_ = [("p", C.c_void_p), ("tok_stride", C.c_uint64), ("head_stride", C.c_uint64)]


_lib = None


def _kv():
    global _lib
    if _lib is None:
        L = lib()
        vp, u32, f32, size = C.c_void_p, C.c_uint32, C.c_float, C.c_size_t
        pool, seqs, rows = C.POINTER(PoolArgs), C.POINTER(SeqsArgs), C.POINTER(RowsArgs)
        sig = {
            "unison_kv_append": [vp, pool, seqs, rows, rows, vp],
            "unison_kv_attend_size": [pool, seqs, u32, C.c_int, u32, C.POINTER(size)],
            "unison_kv_attend": [vp, vp, size, pool, seqs, u32, rows, f32, C.c_int, f32, vp, vp],
            "unison_kv_attend_blocks": [vp, vp, size, pool, seqs, u32, rows, f32, u32, u32, u32, vp, vp, vp],
            "unison_kv_victims": [vp, pool, seqs, u32, u32, u32, u32, vp, vp, vp],
            "unison_kv_compact": [vp, pool, seqs, u32, vp, vp, vp],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = C.c_int
        _lib = L
    return _lib


_module = None


def _torch():
    global _module
    if _module is None:
        import torch as _module
    return _module


_raw = None


def _raw_stream(index):
    """The current stream's handle; the Stream object around it takes as long to make as a launch."""
    global _raw
    if _raw is None:
        torch = _torch()
        _raw = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _raw(index)


_count = 0


def _several():
    """Whether there is more than one device, of which another may be the current one."""
    global _count
    if not _count:
        _count = _torch().cuda.device_count()
    return _count > 1


def _refuse(why):
    raise UnisonError(E_INVALID, why)


def _need(t, name, dtype, shape, device):
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        _refuse("%s: contiguous %s %s on %s wanted, got %s %s on %s" % (
            name, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))


_dual = None


def _no_gradient(t, name):
    """The operators have no backward pass: what autograd follows is refused rather than dropped."""
    if t.requires_grad and _torch().is_grad_enabled():
        _refuse("%s requires a gradient, and there is no backward pass: detach it, or call under torch.no_grad()" % name)


def _no_tangent(t, name):
    global _dual
    if _dual is None:
        from torch.autograd.forward_ad import unpack_dual as _dual
    if _dual(t).tangent is not None:
        _refuse("%s has a tangent, and there is no forward-mode derivative" % name)


_bump = None


def _wrote(tensors):
    """Tells autograd that a kernel changed these tensors in place, so that a backward pass that saved their old
    values fails instead of using the new ones."""
    global _bump
    if _bump is None:
        from torch.autograd.graph import increment_version as _bump
    _bump(tensors)


class Pool:
    """Pages of a KV pool: k [n_pages, n_kv, page, head_dim], v [n_pages, n_kv, head_dim, page] in
    bfloat16 or float16; weight (float32) and pos (int32) [n_pages, n_kv, page]; box (int8)
    [n_pages, n_kv, 2, head_dim] with box_scale (float32) [n_pages, n_kv]."""

    def __init__(self, k, v, weight=None, pos=None, box=None, box_scale=None):
        torch = _torch()
        if k.dim() != 4 or k.dtype not in (torch.bfloat16, torch.float16):
            _refuse("k: bfloat16 or float16 [n_pages, n_kv, page, head_dim] wanted")
        n_pages, n_kv, page, dim = k.shape
        _need(k, "k", k.dtype, k.shape, k.device)
        _need(v, "v", k.dtype, (n_pages, n_kv, dim, page), k.device)
        words = (n_pages, n_kv, page)
        if weight is not None:
            _need(weight, "weight", torch.float32, words, k.device)
        if pos is not None:
            _need(pos, "pos", torch.int32, words, k.device)
        if (box is None) != (box_scale is None):
            _refuse("box and box_scale come together")
        if box is not None:
            _need(box, "box", torch.int8, (n_pages, n_kv, 2, dim), k.device)
            _need(box_scale, "box_scale", torch.float32, (n_pages, n_kv), k.device)
        self._floats = tuple(t for t in (k, v, weight) if t is not None)
        self._entries = tuple(t for t in (k, v, weight, pos, box, box_scale) if t is not None)
        for t in self._floats:
            _no_tangent(t, "the pool")
        self.k, self.v, self.weight, self.pos, self.box, self.box_scale = k, v, weight, pos, box, box_scale
        self.n_kv, self.page, self.head_dim, self.dtype, self.device = n_kv, page, dim, k.dtype, k.device
        ptr = lambda t: None if t is None else t.data_ptr()
        self._index = k.device.index if k.device.type == "cuda" else None
        self._args = PoolArgs(BF16 if k.dtype == torch.bfloat16 else FP16, dim, n_kv, page, n_pages, 0, ptr(k), ptr(v),
                              ptr(weight), ptr(pos), ptr(box), ptr(box_scale))
        self._ref = C.byref(self._args)

    @classmethod
    def empty(cls, n_pages, n_kv, page, head_dim, dtype=None, device="cuda", weight=True, pos=True, box=False):
        """A pool of zeroed pages."""
        torch = _torch()
        dtype = dtype or torch.bfloat16
        z = lambda *shape, dt: torch.zeros(shape, dtype=dt, device=device)
        return cls(z(n_pages, n_kv, page, head_dim, dt=dtype), z(n_pages, n_kv, head_dim, page, dt=dtype),
                   z(n_pages, n_kv, page, dt=torch.float32) if weight else None,
                   z(n_pages, n_kv, page, dt=torch.int32) if pos else None,
                   z(n_pages, n_kv, 2, head_dim, dt=torch.int8) if box else None,
                   z(n_pages, n_kv, dt=torch.float32) if box else None)


class Seqs:
    """A batch of sequences: pages int32 [n_seq, max_pages] (-1: no page), length int32 [n_seq] with
    the new tokens counted, tok int32 [n_seq + 1] the ranges of the new tokens' rows.  n_tok, max_new
    and max_len bound what the device arrays hold (max_len 0: the page table's capacity)."""

    def __init__(self, pages, length, tok=None, n_tok=0, max_new=0, max_len=0):
        torch = _torch()
        if pages.dim() != 2:
            _refuse("pages: int32 [n_seq, max_pages] wanted")
        n_seq, max_pages = pages.shape
        _need(pages, "pages", torch.int32, pages.shape, pages.device)
        _need(length, "length", torch.int32, (n_seq,), pages.device)
        if tok is not None:
            _need(tok, "tok", torch.int32, (n_seq + 1,), pages.device)
        elif n_tok:
            _refuse("tok is needed where there are new tokens")
        for name, x in (("n_tok", n_tok), ("max_new", max_new), ("max_len", max_len)):
            if not 0 <= int(x) < 1 << 31:
                _refuse("%s out of range" % name)
        self.pages, self.length, self.tok, self.n_tok, self.n_seq = pages, length, tok, int(n_tok), n_seq
        self.device = pages.device
        self._args = SeqsArgs(n_seq, max_pages, int(n_tok), int(max_new), int(max_len), 0, pages.data_ptr(),
                              length.data_ptr(), None if tok is None else tok.data_ptr())
        self._ref = C.byref(self._args)
        self._sizes = {}  # workspace bytes by the pool's sizes and the call's: no content is kept


class _On:
    """The device of a call made current, and its stream."""

    __slots__ = ("index", "before")

    def __init__(self, pool, seqs, whole=False):
        """whole: a call whose results are whole numbers, which have no gradient."""
        if seqs.device != pool.device:
            _refuse("the sequences are on %s, the pool on %s" % (seqs.device, pool.device))
        if not whole and (pool.k.requires_grad or pool.v.requires_grad or
                          (pool.weight is not None and pool.weight.requires_grad)):
            for t in pool._floats:
                _no_gradient(t, "the pool")
        self.index = pool._index

    def __enter__(self):
        index = self.index
        if index is None:
            _refuse("the operators run on the GPU, the pool is on another device")
        self.before = index
        if _several():
            cuda = _torch().cuda
            self.before = cuda.current_device()
            if self.before != index:
                cuda.set_device(index)
        return _raw_stream(index)

    def __exit__(self, *exc):
        if self.before != self.index:
            _torch().cuda.set_device(self.before)


def _rows(t, name, pool, n_tok, heads):
    shape = t.shape
    if len(shape) != 3 or t.dtype != pool.dtype or t.device != pool.device or shape[0] != n_tok or \
            shape[2] != pool.head_dim or (heads is not None and shape[1] != heads):
        _refuse("%s: %s [%d, heads, %d] on %s wanted, got %s %s on %s" % (
            name, pool.dtype, n_tok, pool.head_dim, pool.device, t.dtype, tuple(shape), t.device))
    _no_gradient(t, name)
    _no_tangent(t, name)
    tok, head, element = t.stride()
    if element != 1 or tok < 0 or head < 0:
        _refuse("%s: the head dimension has to be contiguous" % name)
    # the stride of a single row or head is never walked
    return RowsArgs(t.data_ptr(), tok if n_tok > 1 else 0, head if shape[1] > 1 else 0)


def _int32(t, name, shape, device):
    _need(t, name, _torch().int32, shape, device)
    return t.data_ptr()


def append(pool, seqs, k, v, positions=None):
    """Writes the new tokens' rows k, v [n_tok, n_kv, head_dim] (any strides with a contiguous last
    dimension that are multiples of 8) into their entries; positions int32 [n_tok] where the pool
    keeps them."""
    with _On(pool, seqs) as stream:
        rk, rv = _rows(k, "k", pool, seqs.n_tok, pool.n_kv), _rows(v, "v", pool, seqs.n_tok, pool.n_kv)
        pos = None if positions is None else _int32(positions, "positions", (seqs.n_tok,), pool.device)
        _check(_kv().unison_kv_append(stream, pool._ref, seqs._ref, C.byref(rk), C.byref(rv), pos))
        _wrote(pool._entries)


def _workspace(pool, seqs, n_q, weights, n_sel):
    key = (pool._args.dtype, pool.head_dim, pool.n_kv, pool.page, n_q, weights, n_sel)
    n = seqs._sizes.get(key)
    if n is None:
        out = C.c_size_t()
        _check(_kv().unison_kv_attend_size(pool._ref, seqs._ref, n_q, weights, n_sel, C.byref(out)))
        n = seqs._sizes[key] = out.value
    return n, _torch().empty(n, dtype=_torch().uint8, device=pool.device) if n else None


def _scale(scale, pool):
    return pool.head_dim ** -0.5 if scale is None else scale


def attend(pool, seqs, q, scale=None, decay=None, lse=False, out=None):
    """Attention of the new tokens q [n_tok, n_q, head_dim] over their sequences; scale: default
    1 / sqrt(head_dim).  decay: pool.weight becomes decay * weight + the tokens' attention weights
    (None: it stays).  out: a tensor for the result, whose memory may be q's own (out = q) only where
    decay is None.  Returns out, or (out, lse [n_tok, n_q]) with lse = True; rows that belong to no
    sequence are not written: in tensors made here they hold anything."""
    torch = _torch()
    with _On(pool, seqs) as stream:
        r = _rows(q, "q", pool, seqs.n_tok, None)
        n_q, given = q.shape[1], out is not None
        if out is None:
            out = torch.empty((seqs.n_tok, n_q, pool.head_dim), dtype=pool.dtype, device=pool.device)
        else:
            _need(out, "out", pool.dtype, (seqs.n_tok, n_q, pool.head_dim), pool.device)
            _no_gradient(out, "out")
            _no_tangent(out, "out")
        e = torch.empty((seqs.n_tok, n_q), dtype=torch.float32, device=pool.device) if lse else None
        n, ws = _workspace(pool, seqs, n_q, int(decay is not None), 0)
        _check(_kv().unison_kv_attend(stream, None if ws is None else ws.data_ptr(), n, pool._ref, seqs._ref, n_q,
                                      C.byref(r), _scale(scale, pool), int(decay is not None), decay or 0.0,
                                      out.data_ptr(), None if e is None else e.data_ptr()))
        if given:
            _wrote(out)
        if decay is not None:
            _wrote(pool.weight)
    return (out, e) if lse else out


def attend_blocks(pool, seqs, q, n_sel, first=0, last=1, scale=None, lse=False):
    """The same over at most n_sel pages a token and kv head: the first and the last of those it sees
    and the ones of highest box score.  Returns (out, sel int32 [n_tok, n_kv, n_sel]) and lse, whose
    rows that belong to no sequence hold anything."""
    torch = _torch()
    with _On(pool, seqs) as stream:
        r = _rows(q, "q", pool, seqs.n_tok, None)
        n_q = q.shape[1]
        for name, x in (("n_sel", n_sel), ("first", first), ("last", last)):
            if not 0 <= x < 1 << 31:
                _refuse("%s out of range" % name)
        if not 1 <= n_sel <= 4096:
            _refuse("n_sel out of range")
        out = torch.empty((seqs.n_tok, n_q, pool.head_dim), dtype=pool.dtype, device=pool.device)
        sel = torch.empty((seqs.n_tok, pool.n_kv, n_sel), dtype=torch.int32, device=pool.device)
        e = torch.empty((seqs.n_tok, n_q), dtype=torch.float32, device=pool.device) if lse else None
        n, ws = _workspace(pool, seqs, n_q, 0, n_sel)
        _check(_kv().unison_kv_attend_blocks(stream, None if ws is None else ws.data_ptr(), n, pool._ref, seqs._ref,
                                             n_q, C.byref(r), _scale(scale, pool), n_sel, first, last, out.data_ptr(),
                                             None if e is None else e.data_ptr(), sel.data_ptr()))
    return (out, sel, e) if lse else (out, sel)


def victims(pool, seqs, budget, first=0, recent=0, max_evict=1):
    """The entries that leave sequences of more than `budget`, by least weight: (victims, src, new_len),
    int32 [n_seq, n_kv, max_evict] twice and [n_seq]."""
    torch = _torch()
    with _On(pool, seqs, whole=True) as stream:
        for name, x in (("budget", budget), ("first", first), ("recent", recent), ("max_evict", max_evict)):
            if not 0 <= x < 1 << 31:
                _refuse("%s out of range" % name)
        if max_evict > 1 << 27:
            _refuse("max_evict out of range")
        shape = (seqs.n_seq, pool.n_kv, max_evict)
        gone = torch.empty(shape, dtype=torch.int32, device=pool.device)
        src = torch.empty(shape, dtype=torch.int32, device=pool.device)
        new_len = torch.empty(seqs.n_seq, dtype=torch.int32, device=pool.device)
        _check(_kv().unison_kv_victims(stream, pool._ref, seqs._ref, budget, first, recent, max_evict,
                                       gone.data_ptr(), src.data_ptr(), new_len.data_ptr()))
    return gone, src, new_len


def compact(pool, seqs, victims, src, new_len):
    """Carries victims()'s lists out; afterwards the caller sets the lengths to new_len."""
    with _On(pool, seqs) as stream:
        if victims.dim() != 3:
            _refuse("victims: int32 [n_seq, n_kv, max_evict] wanted")
        shape = (seqs.n_seq, pool.n_kv, victims.shape[2])
        v, s = _int32(victims, "victims", shape, pool.device), _int32(src, "src", shape, pool.device)
        n = _int32(new_len, "new_len", (seqs.n_seq,), pool.device)
        _check(_kv().unison_kv_compact(stream, pool._ref, seqs._ref, shape[2], v, s, n))
        _wrote(pool._entries)
