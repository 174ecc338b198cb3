// kv_device.h -- arguments and small device functions of the paged-KV operators.
//
// A sequence's entries lie in pages of `page` entries, entry e in slot e % page of page
// pages[e / page].  Keys are rows [page][dim]; values are stored transposed, [dim][page], so that
// both products of attention read their matrix operands as 16-byte runs: a lane of the first takes
// 8 dimensions of one key, a lane of the second 8 entries of one dimension.
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

#include "../../include/unison.h"

#pragma clang fp contract(off)

namespace unison {

struct KvRows {  // rows of the new tokens, strides in elements
  const void* p;
  uint64_t tok, head;
};

struct KvArgs {
  uint32_t dtype, dim, n_kv, page, page_bits, n_pages;
  void *k, *v;
  float* weight;
  int32_t* pos;
  int8_t* box;
  float* box_scale;
  uint32_t n_seq, max_pages, n_tok, max_new, max_len;
  const int32_t *pages, *len, *tok;
  uint32_t n_q, group;
};

// A sequence as the kernels see it: whatever the device arrays hold, every index made from it stays
// inside the caller's arrays.
struct KvSeq {
  int32_t len;      // live entries
  int32_t t0, n;    // its new tokens are rows t0 .. t0 + n - 1, its last n entries
  const int32_t* pages;
};

__host__ __device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, uint32_t s) {
  KvSeq q;
  const int32_t l = a.len[s];
  q.len = l < 0 ? 0 : (uint32_t)l > a.max_len ? (int32_t)a.max_len : l;
  q.t0 = 0;
  q.n = 0;
  if (a.tok) {
    const int32_t b = a.tok[s], e = a.tok[s + 1], most = (int32_t)a.n_tok;
    q.t0 = b < 0 ? 0 : b > most ? most : b;
    const int32_t end = e < q.t0 ? q.t0 : e > most ? most : e;
    q.n = end - q.t0;
    if ((uint32_t)q.n > a.max_new) q.n = (int32_t)a.max_new;
  }
  q.pages = a.pages + (size_t)s * a.max_pages;
  return q;
}

// Blocks go to the eight XCDs in turn.  Where the fastest index walks a sequence in a multiple of 8 (or
// 4, or 2) pieces, the last pieces, which short sequences do not have, would all be the same XCD's: the
// walk starts one piece further for each kv head and sequence (a decode step of 64 ragged sequences: 594 us
// without this, 457 with it, 441 for equal lengths of the same sum).
__device__ __forceinline__ uint32_t spread_piece(uint32_t x, uint32_t n) { return (x + blockIdx.y + blockIdx.z) % n; }

// The page of ordinal `o` (below max_pages), or -1 where there is none.
__host__ __device__ __forceinline__ int32_t kv_page(const KvArgs& a, const KvSeq& q, int32_t o) {
  const int32_t p = q.pages[o];
  return (uint32_t)p < a.n_pages ? p : -1;
}
// First element of a page's keys (values) of kv head h.
__host__ __device__ __forceinline__ size_t kv_base(const KvArgs& a, int32_t page, uint32_t h) {
  return ((size_t)page * a.n_kv + h) * a.page * a.dim;
}
// First entry of a page's per-entry words (weights, positions) of kv head h.
__host__ __device__ __forceinline__ size_t kv_word(const KvArgs& a, int32_t page, uint32_t h) {
  return ((size_t)page * a.n_kv + h) * a.page;
}

// A power of two that brings a largest magnitude `top` into [64, 128), and its inverse; both 0 for
// magnitudes below 2^-120.  Multiplying by either is exact, so the int8 images and the scores made
// from them are the same whoever computes them.
struct KvStep {
  float inv, step;
};
__device__ __forceinline__ KvStep kv_step(float top) {
  const int32_t e = (__float_as_int(top) >> 23) & 255;
  return e < 7 ? KvStep{0.0f, 0.0f}
               : KvStep{__int_as_float((260 - e) << 23), __int_as_float((e - 6) << 23)};
}
__device__ __forceinline__ int32_t kv_clip(float x) {
  return (int32_t)fminf(fmaxf(x, -127.0f), 127.0f);
}

// An order of floats as unsigned words, -0 and 0 alike and NaN as 0.
__device__ __forceinline__ uint32_t kv_order(float x) {
  x = x != x ? 0.0f : x + 0.0f;
  const uint32_t b = __float_as_uint(x);
  return (b >> 31) ? ~b : b | 0x80000000u;
}

}  // namespace unison
