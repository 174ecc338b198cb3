// kv_api.cpp -- host side of the paged-KV operators (see include/unison.h): checks every size,
// pointer and stride that the kernels rely on, then launches them on the caller's stream.
#include <cmath>

#include "kv_device.h"

namespace unison {
hipError_t launch_kv_append(const KvArgs& a, const KvRows& k, const KvRows& v, const int32_t* pos,
                            hipStream_t st);
hipError_t launch_kv_victims(const KvArgs& a, uint32_t budget, uint32_t first, uint32_t recent,
                             uint32_t max_evict, int32_t* victims, int32_t* src, int32_t* new_len,
                             hipStream_t st);
hipError_t launch_kv_compact(const KvArgs& a, uint32_t max_evict, const int32_t* victims, const int32_t* src,
                             const int32_t* new_len, hipStream_t st);
size_t kv_attend_bytes(const KvArgs& a, bool weights, uint32_t n_sel);
bool kv_attend_fits(const KvArgs& a, uint32_t n_sel);
hipError_t launch_kv_attend(const KvArgs& a, const KvRows& q, float scale, bool weights, float decay,
                            uint32_t n_sel, uint32_t first, uint32_t last, void* out, float* lse, int32_t* sel,
                            void* ws, hipStream_t st);
}  // namespace unison

using namespace unison;

namespace {

constexpr uint32_t kMaxSeqs = 65535, kMaxKvHeads = 1024, kMaxGroup = 128, kMaxSelPages = 32768, kMaxSel = 4096;
constexpr uint64_t kMaxEntries = 1ull << 27;  // of a sequence: blocks of 16 stay below 2^32 threads a launch

bool on(const void* p, size_t bytes) { return p && reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// The sizes of a pool and a batch; no pointer is looked at.
int sizes(const unison_kv_pool* p, const unison_kv_seqs* s, KvArgs& a) {
  if (!p || !s) return UNISON_E_INVALID;
  if (p->dtype > UNISON_KV_FP16) return UNISON_E_INVALID;
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256) return UNISON_E_INVALID;
  if (p->n_kv < 1 || p->n_kv > kMaxKvHeads) return UNISON_E_INVALID;
  if (p->page < 16 || p->page > 256 || (p->page & (p->page - 1u))) return UNISON_E_INVALID;
  if (p->n_pages < 1 || p->n_pages > 0x7FFFFFFFu) return UNISON_E_INVALID;
  if (s->n_seq > kMaxSeqs) return UNISON_E_CAPACITY;
  if (s->max_pages < 1 || s->n_tok > 0x7FFFFFFFu) return UNISON_E_INVALID;
  const uint64_t entries = (uint64_t)s->max_pages * p->page;
  if (entries > kMaxEntries) return UNISON_E_CAPACITY;
  if (s->max_len > entries) return UNISON_E_INVALID;
  if (s->n_tok && s->max_new < 1) return UNISON_E_INVALID;
  a = KvArgs{};
  a.dtype = p->dtype;
  a.dim = p->head_dim;
  a.n_kv = p->n_kv;
  a.page = p->page;
  a.page_bits = (uint32_t)__builtin_ctz(p->page);
  a.n_pages = p->n_pages;
  a.k = p->k;
  a.v = p->v;
  a.weight = p->weight;
  a.pos = p->pos;
  a.box = p->box;
  a.box_scale = p->box_scale;
  a.n_seq = s->n_seq;
  a.max_pages = s->max_pages;
  a.n_tok = s->n_tok;
  a.max_new = s->max_new < s->n_tok ? s->max_new : s->n_tok;
  a.max_len = s->max_len ? s->max_len : (uint32_t)entries;
  a.pages = s->pages;
  a.len = s->len;
  a.tok = s->tok;
  return UNISON_OK;
}

int pointers(const KvArgs& a, bool tokens) {
  if (!on(a.k, 16) || !on(a.v, 16) || !on(a.pages, 4) || !on(a.len, 4)) return UNISON_E_INVALID;
  if ((a.weight && !on(a.weight, 16)) || (a.pos && !on(a.pos, 16))) return UNISON_E_INVALID;
  if (!a.box != !a.box_scale || (a.box && (!on(a.box, 16) || !on(a.box_scale, 16)))) return UNISON_E_INVALID;
  return tokens && !on(a.tok, 4) ? UNISON_E_INVALID : UNISON_OK;
}

bool rows(const unison_kv_rows* r, KvRows& out) {
  if (!r || !on(r->p, 16) || r->tok_stride % 8 || r->head_stride % 8) return false;
  if (r->tok_stride >> 40 || r->head_stride >> 40) return false;
  out = KvRows{r->p, r->tok_stride, r->head_stride};
  return true;
}

struct Span {
  uintptr_t at;
  uint64_t bytes;
};

Span span(const void* p, uint64_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), p ? bytes : 0}; }

bool meet(const Span& x, const Span& y) {
  return x.bytes && y.bytes && x.at < y.at + y.bytes && y.at < x.at + x.bytes;
}

// Whether one of the `n` written spans shares memory with another, with the pool or with the batch's arrays.
bool overlaps(const KvArgs& a, const Span* written, int n) {
  const uint64_t words = (uint64_t)a.n_pages * a.n_kv * a.page, boxes = (uint64_t)a.n_pages * a.n_kv;
  const Span read[] = {span(a.k, words * a.dim * 2), span(a.v, words * a.dim * 2), span(a.weight, words * 4),
                       span(a.pos, words * 4), span(a.box, boxes * 2 * a.dim), span(a.box_scale, boxes * 4),
                       span(a.pages, (uint64_t)a.n_seq * a.max_pages * 4), span(a.len, (uint64_t)a.n_seq * 4),
                       span(a.tok, ((uint64_t)a.n_seq + 1) * 4)};
  for (int i = 0; i < n; ++i) {
    for (const Span& r : read)
      if (meet(written[i], r)) return true;
    for (int j = 0; j < i; ++j)
      if (meet(written[i], written[j])) return true;
  }
  return false;
}

// The same for a written span and the query rows.  Strides may leave room between these, so where the span lies
// inside their extent the rows are looked at one by one.
bool meets_rows(const KvArgs& a, const KvRows& q, const Span& w) {
  typedef unsigned __int128 u128;
  const u128 head = (u128)(a.n_q - 1) * q.head + a.dim, all = (u128)(a.n_tok - 1) * q.tok + head;
  if (all >> 56) return true;  // no memory holds such rows
  const auto rows = [&](uint64_t at, uint64_t elements) { return span((const char*)q.p + 2 * at, 2 * elements); };
  if (!meet(w, rows(0, (uint64_t)all))) return false;
  for (uint64_t t = 0; t < a.n_tok; ++t) {
    if (!meet(w, rows(t * q.tok, (uint64_t)head))) continue;
    for (uint64_t h = 0; h < a.n_q; ++h)
      if (meet(w, rows(t * q.tok + h * q.head, a.dim))) return true;
  }
  return false;
}

// Whether the results are the query rows themselves, each over its own.
bool in_place(const KvArgs& a, const KvRows& q, const void* out) {
  return out == q.p && (a.n_tok == 1 || q.tok == (uint64_t)a.n_q * a.dim) && (a.n_q == 1 || q.head == a.dim);
}

int heads(KvArgs& a, uint32_t n_q) {
  if (n_q < 1 || n_q % a.n_kv || n_q / a.n_kv > kMaxGroup) return UNISON_E_INVALID;
  a.n_q = n_q;
  a.group = n_q / a.n_kv;
  // rows of a sequence, and a tile's behind them, are counted in 31 bits
  return (uint64_t)a.n_tok * n_q > 1ull << 30 ? UNISON_E_CAPACITY : UNISON_OK;
}

int done(hipError_t rc) { return rc == hipSuccess ? UNISON_OK : UNISON_E_HIP; }

int attend(void* hip_stream, void* ws, size_t ws_bytes, const unison_kv_pool* pool, const unison_kv_seqs* seqs,
           uint32_t n_q, const unison_kv_rows* q, float scale, int weights, float decay, uint32_t n_sel,
           uint32_t first, uint32_t last, void* out, float* lse, int32_t* sel) {
  KvArgs a;
  KvRows r;
  int rc = sizes(pool, seqs, a);
  if (rc == UNISON_OK) rc = heads(a, n_q);
  if (rc != UNISON_OK) return rc;
  if (!std::isfinite(scale)) return UNISON_E_INVALID;
  if (weights && (!a.weight || !(decay >= 0.0f && decay <= 1.0f))) return UNISON_E_INVALID;
  if (a.n_seq == 0 || a.n_tok == 0) return UNISON_OK;
  rc = pointers(a, true);
  if (rc != UNISON_OK) return rc;
  if (!rows(q, r) || !on(out, 16) || (lse && !on(lse, 4))) return UNISON_E_INVALID;
  if (!kv_attend_fits(a, n_sel)) return UNISON_E_CAPACITY;
  const size_t need = kv_attend_bytes(a, weights != 0, n_sel);
  if (need && (ws_bytes < need || !on(ws, 256))) return UNISON_E_INVALID;
  const uint64_t tok_rows = (uint64_t)a.n_tok * n_q;
  const Span written[] = {span(out, tok_rows * a.dim * 2), span(lse, tok_rows * 4), span(ws, need),
                          span(sel, (uint64_t)a.n_tok * a.n_kv * n_sel * 4)};
  if (overlaps(a, written, 4)) return UNISON_E_INVALID;
  // a block without weights has its query rows in registers before it writes their results; the weights' second
  // product reads them again
  for (const Span& w : written)
    if (meets_rows(a, r, w) && !(&w == written && !weights && in_place(a, r, out))) return UNISON_E_INVALID;
  return done(launch_kv_attend(a, r, scale, weights != 0, decay, n_sel, first, last, out, lse, sel, ws,
                               reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // namespace

extern "C" {

int unison_kv_append(void* hip_stream, const unison_kv_pool* pool, const unison_kv_seqs* seqs,
                     const unison_kv_rows* k, const unison_kv_rows* v, const int32_t* tok_pos) {
  KvArgs a;
  KvRows rk, rv;
  int rc = sizes(pool, seqs, a);
  if (rc != UNISON_OK) return rc;
  if (a.n_seq == 0 || a.n_tok == 0) return UNISON_OK;
  rc = pointers(a, true);
  if (rc != UNISON_OK) return rc;
  if (!rows(k, rk) || !rows(v, rv) || !a.pos != !tok_pos || (tok_pos && !on(tok_pos, 4))) return UNISON_E_INVALID;
  return done(launch_kv_append(a, rk, rv, tok_pos, reinterpret_cast<hipStream_t>(hip_stream)));
}

int unison_kv_attend_size(const unison_kv_pool* pool, const unison_kv_seqs* seqs, uint32_t n_q, int weights,
                          uint32_t n_sel, size_t* bytes) {
  KvArgs a;
  int rc = sizes(pool, seqs, a);
  if (rc == UNISON_OK) rc = heads(a, n_q);
  if (rc != UNISON_OK) return rc;
  if (!bytes) return UNISON_E_INVALID;
  if (n_sel && a.max_pages > kMaxSelPages) return UNISON_E_CAPACITY;
  *bytes = a.n_seq && a.n_tok ? kv_attend_bytes(a, weights != 0, n_sel) : 0;
  return UNISON_OK;
}

int unison_kv_attend(void* hip_stream, void* workspace, size_t workspace_bytes, const unison_kv_pool* pool,
                     const unison_kv_seqs* seqs, uint32_t n_q, const unison_kv_rows* q, float scale, int weights,
                     float decay, void* out, float* lse) {
  return attend(hip_stream, workspace, workspace_bytes, pool, seqs, n_q, q, scale, weights, decay, 0, 0, 0, out, lse,
                nullptr);
}

int unison_kv_attend_blocks(void* hip_stream, void* workspace, size_t workspace_bytes, const unison_kv_pool* pool,
                            const unison_kv_seqs* seqs, uint32_t n_q, const unison_kv_rows* q, float scale,
                            uint32_t n_sel, uint32_t first, uint32_t last, void* out, float* lse, int32_t* sel) {
  if (!pool || !seqs || n_sel < 1 || n_sel > kMaxSel || last < 1 || (uint64_t)first + last > n_sel)
    return UNISON_E_INVALID;
  if (seqs->max_pages > kMaxSelPages) return UNISON_E_CAPACITY;
  if (seqs->n_seq && seqs->n_tok && (!pool->box || !on(sel, 4))) return UNISON_E_INVALID;
  return attend(hip_stream, workspace, workspace_bytes, pool, seqs, n_q, q, scale, 0, 0.0f, n_sel, first, last, out,
                lse, sel);
}

int unison_kv_victims(void* hip_stream, const unison_kv_pool* pool, const unison_kv_seqs* seqs, uint32_t budget,
                      uint32_t first, uint32_t recent, uint32_t max_evict, int32_t* victims, int32_t* src,
                      int32_t* new_len) {
  KvArgs a;
  int rc = sizes(pool, seqs, a);
  if (rc != UNISON_OK) return rc;
  if (budget < 1 || (uint64_t)first + recent > budget || max_evict < 1 || max_evict > kMaxEntries)
    return UNISON_E_INVALID;
  if (a.n_seq == 0) return UNISON_OK;
  rc = pointers(a, false);
  if (rc != UNISON_OK) return rc;
  if (!a.weight || !a.pos || !on(victims, 4) || !on(src, 4) || !on(new_len, 4)) return UNISON_E_INVALID;
  // the lengths among what is read: a block of one head writes new_len while the other heads' read len
  const uint64_t list = (uint64_t)a.n_seq * a.n_kv * max_evict * 4;
  const Span written[] = {span(victims, list), span(src, list), span(new_len, (uint64_t)a.n_seq * 4)};
  a.tok = nullptr;  // not looked at
  if (overlaps(a, written, 3)) return UNISON_E_INVALID;
  return done(launch_kv_victims(a, budget, first, recent, max_evict, victims, src, new_len,
                                reinterpret_cast<hipStream_t>(hip_stream)));
}

int unison_kv_compact(void* hip_stream, const unison_kv_pool* pool, const unison_kv_seqs* seqs, uint32_t max_evict,
                      const int32_t* victims, const int32_t* src, const int32_t* new_len) {
  KvArgs a;
  int rc = sizes(pool, seqs, a);
  if (rc != UNISON_OK) return rc;
  if (max_evict < 1 || max_evict > kMaxEntries) return UNISON_E_INVALID;
  if (a.n_seq == 0) return UNISON_OK;
  rc = pointers(a, false);
  if (rc != UNISON_OK) return rc;
  if (!on(victims, 4) || !on(src, 4) || !on(new_len, 4)) return UNISON_E_INVALID;
  return done(launch_kv_compact(a, max_evict, victims, src, new_len, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
