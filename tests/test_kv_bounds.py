"""What the paged-KV kernels make of the device arrays, on the CPU: kv_device.h compiled for the host and
driven with lengths, token ranges and page ids of any value.  Whatever they hold, the sequence a kernel
sees stays within the caller's bounds, and the elements of a page it may touch within the pool."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_09643_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

DRIVER = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "kv_device.h"
using namespace unison;

#define CHECK(x) do { if (!(x)) { std::fprintf(stderr, "failed: %s (line %d)\n", #x, __LINE__); return 1; } } while (0)

int main() {
  std::mt19937_64 rng(1);
  const auto any = [&](int32_t near) -> int32_t {
    switch (rng() % 6) {
      case 0: return (int32_t)rng();
      case 1: return -1;
      case 2: return INT32_MIN;
      case 3: return INT32_MAX;
      default: return near + (int32_t)(rng() % 7) - 3;
    }
  };
  for (int turn = 0; turn < 200000; ++turn) {
    KvArgs a = {};
    a.page_bits = 4 + rng() % 5;
    a.page = 1u << a.page_bits;
    a.dim = 64u << (rng() % 3);
    a.n_kv = 1 + rng() % 9;
    a.n_pages = 1 + rng() % 50;
    a.n_seq = 1 + rng() % 4;
    a.max_pages = 1 + rng() % 6;
    a.max_len = 1 + rng() % (a.max_pages * a.page);
    a.n_tok = 1 + rng() % 40;
    a.max_new = 1 + rng() % a.n_tok;
    std::vector<int32_t> len(a.n_seq), tok(a.n_seq + 1), pages(a.n_seq * a.max_pages);
    for (auto& x : len) x = any((int32_t)a.max_len);
    for (auto& x : tok) x = any((int32_t)(rng() % (a.n_tok + 1)));
    for (auto& x : pages) x = any((int32_t)a.n_pages);
    a.len = len.data();
    a.tok = rng() % 8 ? tok.data() : nullptr;
    a.pages = pages.data();
    const size_t elements = (size_t)a.n_pages * a.n_kv * a.page * a.dim, words = (size_t)a.n_pages * a.n_kv * a.page;
    for (uint32_t s = 0; s < a.n_seq; ++s) {
      const KvSeq q = kv_seq(a, s);
      CHECK(q.len >= 0 && (uint32_t)q.len <= a.max_len);
      CHECK(q.t0 >= 0 && q.n >= 0 && (uint32_t)q.n <= a.max_new && (uint32_t)(q.t0 + q.n) <= a.n_tok);
      CHECK(a.tok || q.n == 0);
      CHECK(q.pages == pages.data() + s * a.max_pages);
      CHECK((q.len + (int32_t)a.page - 1) >> a.page_bits <= (int32_t)a.max_pages);
      if (len[s] >= 0 && (uint32_t)len[s] <= a.max_len) CHECK(q.len == len[s]);
      for (uint32_t o = 0; o < a.max_pages; ++o) {
        const int32_t p = kv_page(a, q, (int32_t)o);
        CHECK(p == -1 || (p == q.pages[o] && p >= 0 && (uint32_t)p < a.n_pages));
        if (p < 0) continue;
        for (uint32_t h = 0; h < a.n_kv; ++h) {
          CHECK(kv_base(a, p, h) + (size_t)a.page * a.dim <= elements);
          CHECK(kv_word(a, p, h) + a.page <= words);
        }
      }
    }
  }
  // offsets past 32 bits
  KvArgs a = {};
  a.page = 256; a.dim = 256; a.n_kv = 1024;
  CHECK(kv_base(a, 0x7FFFFFFE, 1023) == (((size_t)0x7FFFFFFE * 1024 + 1023) << 16));
  CHECK(kv_word(a, 0x7FFFFFFE, 1023) == (((size_t)0x7FFFFFFE * 1024 + 1023) << 8));
  std::printf("ok\n");
  return 0;
}
"""


def test_whatever_the_device_arrays_hold(tmp_path):
    if not os.path.exists(HIPCC) or shutil.which("g++") is None:
        pytest.skip("no hipcc")
    src, obj, exe = tmp_path / "drv.cpp", tmp_path / "drv.o", tmp_path / "drv"
    src.write_text(DRIVER)
    subprocess.check_call([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-fPIC",
                           "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=all",
                           "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(obj)],
                          stderr=subprocess.DEVNULL)
    subprocess.check_call(["g++", str(obj), "-fsanitize=address,undefined", "-o", str(exe), "-L/opt/rocm/lib",
                           "-Wl,-rpath,/opt/rocm/lib", "-lamdhip64"])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout + r.stderr)[-2000:]
