"""What the paged-KV operators write may not overlap what they read, or each other: the host side of the C calls,
built with stand-ins for the launches, so that a call that passes its checks ends without a GPU."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_09643_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
OK, INVALID = 0, -1

LAUNCHES = r"""
#include "kv_api.cpp"
namespace unison {
hipError_t launch_kv_append(const KvArgs&, const KvRows&, const KvRows&, const int32_t*, hipStream_t) { return hipSuccess; }
hipError_t launch_kv_victims(const KvArgs&, uint32_t, uint32_t, uint32_t, uint32_t, int32_t*, int32_t*, int32_t*,
                             hipStream_t) { return hipSuccess; }
hipError_t launch_kv_compact(const KvArgs&, uint32_t, const int32_t*, const int32_t*, const int32_t*, hipStream_t) {
  return hipSuccess;
}
size_t kv_attend_bytes(const KvArgs&, bool, uint32_t) { return 4096; }
bool kv_attend_fits(const KvArgs&, uint32_t) { return true; }
hipError_t launch_kv_attend(const KvArgs&, const KvRows&, float, bool, float, uint32_t, uint32_t, uint32_t, void*, float*,
                            int32_t*, void*, hipStream_t) { return hipSuccess; }
}
"""

# a place of its own for every array
AT = {name: (i + 1) << 32 for i, name in enumerate(
    ("k", "v", "weight", "pos", "box", "box_scale", "pages", "len", "tok", "q", "out", "lse", "sel", "ws", "victims",
     "src", "new_len", "rows_k", "rows_v", "tok_pos"))}
N_TOK, N_Q, N_KV, DIM, PAGE, N_PAGES, N_SEQ, MAX_PAGES, N_SEL, EVICT = 5, 4, 2, 128, 64, 10, 3, 4, 2, 7
BYTES = {"k": N_PAGES * N_KV * PAGE * DIM * 2, "v": N_PAGES * N_KV * PAGE * DIM * 2, "weight": N_PAGES * N_KV * PAGE * 4,
         "pos": N_PAGES * N_KV * PAGE * 4, "box": N_PAGES * N_KV * 2 * DIM, "box_scale": N_PAGES * N_KV * 4,
         "pages": N_SEQ * MAX_PAGES * 4, "len": N_SEQ * 4, "tok": (N_SEQ + 1) * 4, "q": N_TOK * N_Q * DIM * 2,
         "out": N_TOK * N_Q * DIM * 2, "lse": N_TOK * N_Q * 4, "sel": N_TOK * N_KV * N_SEL * 4, "ws": 4096,
         "victims": N_SEQ * N_KV * EVICT * 4, "src": N_SEQ * N_KV * EVICT * 4, "new_len": N_SEQ * 4}


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not os.path.exists(HIPCC) or shutil.which("g++") is None:
        pytest.skip("no hipcc")
    from paper_2609_09643_amd import kv
    d = tmp_path_factory.mktemp("kv_host")
    (d / "host.cpp").write_text(LAUNCHES)
    subprocess.check_call([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-fPIC",
                           "-I", CSRC, "-c", str(d / "host.cpp"), "-o", str(d / "host.o")], stderr=subprocess.DEVNULL)
    subprocess.check_call(["g++", "-shared", str(d / "host.o"), "-o", str(d / "host.so")])
    lib = C.CDLL(str(d / "host.so"))
    vp, u32, f32, size = C.c_void_p, C.c_uint32, C.c_float, C.c_size_t
    pool, seqs, rows = C.POINTER(kv.PoolArgs), C.POINTER(kv.SeqsArgs), C.POINTER(kv.RowsArgs)
    lib.unison_kv_attend.argtypes = [vp, vp, size, pool, seqs, u32, rows, f32, C.c_int, f32, vp, vp]
    lib.unison_kv_attend_blocks.argtypes = [vp, vp, size, pool, seqs, u32, rows, f32, u32, u32, u32, vp, vp, vp]
    lib.unison_kv_victims.argtypes = [vp, pool, seqs, u32, u32, u32, u32, vp, vp, vp]
    return kv, lib


def structs(kv, at, tok=N_Q * DIM, head=DIM):
    return (kv.PoolArgs(0, DIM, N_KV, PAGE, N_PAGES, 0, *(at[x] for x in ("k", "v", "weight", "pos", "box", "box_scale"))),
            kv.SeqsArgs(N_SEQ, MAX_PAGES, N_TOK, 2, 0, 0, at["pages"], at["len"], at["tok"]),
            kv.RowsArgs(at["q"], tok, head))


def attend(host, weights, blocks=False, tok=N_Q * DIM, head=DIM, **move):
    kv, lib = host
    at = dict(AT, **move)
    p, s, r = (C.byref(x) for x in structs(kv, at, tok, head))
    if blocks:
        return lib.unison_kv_attend_blocks(None, at["ws"], 1 << 20, p, s, N_Q, r, 0.1, N_SEL, 0, 1, at["out"], at["lse"],
                                           at["sel"])
    return lib.unison_kv_attend(None, at["ws"], 1 << 20, p, s, N_Q, r, 0.1, weights, 1.0, at["out"], at["lse"])


FORMS = [(0, False), (1, False), (0, True)]


@pytest.mark.parametrize("weights,blocks", FORMS)
def test_what_attention_writes_stands_apart(host, weights, blocks):
    assert attend(host, weights, blocks) == OK
    written = ["out", "lse", "ws"] + (["sel"] if blocks else [])
    read = ["k", "v", "weight", "pos", "box", "box_scale", "pages", "len", "tok", "q"]
    for w in written:
        align = {"out": 16, "ws": 256}.get(w, 4)
        for other in written + read:
            if other == w:
                continue
            end = AT[other] + BYTES[other]
            inside = (end - 1) // align * align                    # the last place that still overlaps
            assert attend(host, weights, blocks, **{w: inside}) == INVALID, (w, other)
            assert attend(host, weights, blocks, **{w: -(-end // align) * align}) == OK, (w, other, "behind")
            before = (AT[other] - BYTES[w]) // align * align
            assert attend(host, weights, blocks, **{w: before}) == OK, (w, other, "before")
            assert attend(host, weights, blocks, **{w: before + align}) == INVALID, (w, other)
    assert attend(host, weights, blocks, lse=None) == OK


def test_queries_written_over_in_place(host):
    """out = q: every row over itself, where nothing reads the queries again."""
    assert attend(host, 0, out=AT["q"]) == OK
    assert attend(host, 0, True, out=AT["q"]) == OK
    assert attend(host, 1, out=AT["q"]) == INVALID
    for more in (dict(tok=N_Q * DIM + 8), dict(head=DIM + 8), dict(tok=DIM, head=N_TOK * DIM), dict(tok=0), dict(head=0)):
        assert attend(host, 0, out=AT["q"], **more) == INVALID, more


def test_results_between_the_rows(host):
    """A result in the gap between two query rows touches none of them."""
    gap = AT["q"] + 2 * N_Q * DIM
    assert attend(host, 1, tok=1 << 20, out=gap) == OK
    assert attend(host, 1, tok=1 << 20, out=gap - 16) == INVALID
    assert attend(host, 1, tok=1 << 20, out=AT["q"] + (2 << 20) - BYTES["out"]) == OK
    assert attend(host, 1, tok=1 << 20, out=AT["q"] + (2 << 20) - BYTES["out"] + 16) == INVALID
    assert attend(host, 1, tok=DIM, head=1 << 20, out=AT["q"] + 2 * N_TOK * DIM) == OK
    assert attend(host, 1, tok=DIM, head=1 << 20, out=AT["q"] + 2 * N_TOK * DIM - 16) == INVALID
    assert attend(host, 0, tok=1 << 39, head=1 << 39) == OK


@pytest.mark.parametrize("change", [
    dict(k=AT["k"] + 8), dict(pages=AT["pages"] + 2), dict(q=AT["q"] + 8), dict(q=None), dict(tok=513), dict(head=4),
    dict(out=AT["out"] + 8), dict(out=None), dict(lse=AT["lse"] + 2), dict(ws=AT["ws"] + 128), dict(ws=None)])
@pytest.mark.parametrize("weights,blocks", FORMS)
def test_each_refusal_by_itself(host, weights, blocks, change):
    """The checks of the arguments, each with nothing else wrong."""
    assert attend(host, weights, blocks, **change) == INVALID


def test_eviction_lists_stand_apart(host):
    """The lengths among them: one head's block would write them while another's reads them."""
    kv, lib = host

    def victims(**move):
        at = dict(AT, **move)
        p, s, _ = (C.byref(x) for x in structs(kv, at))
        return lib.unison_kv_victims(None, p, s, 8, 0, 0, EVICT, at["victims"], at["src"], at["new_len"])

    assert victims() == OK
    assert victims(new_len=AT["len"]) == INVALID
    assert victims(new_len=AT["tok"]) == OK                        # token ranges are not read here
    written = ["victims", "src", "new_len"]
    for w in written:
        for other in written + ["weight", "pos", "pages", "len"]:
            if other == w:
                continue
            end = AT[other] + BYTES[other]
            assert victims(**{w: end - 4}) == INVALID, (w, other)
            assert victims(**{w: end}) == OK, (w, other, "behind")
            assert victims(**{w: AT[other] - BYTES[w]}) == OK, (w, other, "before")
            assert victims(**{w: AT[other] - BYTES[w] + 4}) == INVALID, (w, other)
