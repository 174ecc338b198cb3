// kv_cache.hip -- the operators that write pages or choose among entries: append, victims, compact,
// and the page choice of sparse attention.
#include "kv_device.h"

#pragma clang fp contract(off)

namespace unison {

namespace {

constexpr uint32_t kBlock = 256;
constexpr uint32_t kSelBlock = 1024;

// Renews the box of one page of kv head h over its first `live` slots: a thread per dimension (the
// block has at least `dim`).  All threads of the block call it.
template <typename T>
__device__ void renew_box(const KvArgs& a, int32_t page, uint32_t h, int32_t live, float* lds) {
  const uint32_t tid = threadIdx.x;
  float lo = 0.0f, hi = 0.0f;
  if (tid < a.dim) {
    const T* k = (const T*)a.k + kv_base(a, page, h) + tid;
    lo = __int_as_float(0x7F800000);
    hi = -lo;
    for (int32_t i = 0; i < live; ++i) {
      const float x = to_f32(k[(size_t)i * a.dim]);
      lo = fminf(lo, x);
      hi = fmaxf(hi, x);
    }
  }
  float top = tid < a.dim ? fmaxf(fabsf(lo), fabsf(hi)) : 0.0f;
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((tid & 63u) == 0u) lds[tid >> 6] = top;
  __syncthreads();
  top = 0.0f;
  for (uint32_t w = 0; w < blockDim.x / 64u; ++w) top = fmaxf(top, lds[w]);
  __syncthreads();
  const KvStep st = kv_step(top);
  if (tid < a.dim) {
    int8_t* b = a.box + ((size_t)page * a.n_kv + h) * 2 * a.dim + tid;
    b[0] = (int8_t)kv_clip(floorf(lo * st.inv));
    b[a.dim] = (int8_t)kv_clip(ceilf(hi * st.inv));
  }
  if (tid == 0) a.box_scale[(size_t)page * a.n_kv + h] = st.step;
}

// One block per (page that may get entries, kv head, sequence).
template <typename T>
__global__ __launch_bounds__(kBlock) void kv_append_kernel(KvArgs a, KvRows nk, KvRows nv,
                                                           const int32_t* tok_pos) {
  __shared__ float lds[kBlock / 64];
  const uint32_t h = blockIdx.y, tid = threadIdx.x;
  const KvSeq q = kv_seq(a, blockIdx.z);
  const int32_t first = q.len - q.n;  // below 0: tokens without an entry
  const int32_t o = ((first < 0 ? 0 : first) >> a.page_bits) + (int32_t)blockIdx.x;
  const int32_t lo = o << a.page_bits, hi = lo + (int32_t)a.page;
  const int32_t b = first > lo ? first : lo, e = q.len < hi ? q.len : hi;
  if (b >= e) return;
  const int32_t page = kv_page(a, q, o);
  if (page < 0) return;
  T* k = (T*)a.k + kv_base(a, page, h);
  T* v = (T*)a.v + kv_base(a, page, h);
  for (uint32_t i = tid; i < (uint32_t)(e - b) * a.dim; i += kBlock) {
    const uint32_t r = i / a.dim, d = i % a.dim, slot = (uint32_t)(b - lo) + r;
    const size_t tok = (size_t)(q.t0 + (b - first)) + r;
    k[(size_t)slot * a.dim + d] = ((const T*)nk.p)[tok * nk.tok + h * nk.head + d];
    v[(size_t)d * a.page + slot] = ((const T*)nv.p)[tok * nv.tok + h * nv.head + d];
  }
  for (int32_t i = b + (int32_t)tid; i < e; i += (int32_t)kBlock) {
    const size_t w = kv_word(a, page, h) + (size_t)(i - lo);
    if (a.weight) a.weight[w] = 0.0f;
    if (a.pos) a.pos[w] = tok_pos[q.t0 + (i - first)];
  }
  if (a.box) {
    __threadfence_block();
    __syncthreads();
    renew_box<T>(a, page, h, e - lo, lds);
  }
}

// ------------------------------------------------------------------ the n smallest keys

// Inclusive sum over the block of a word per thread; `total` is the block's.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* lds, uint32_t& total) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o);
    if (lane >= (uint32_t)o) x += y;
  }
  if (lane == 63u) lds[wave] = x;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
  for (uint32_t w = 0; w < blockDim.x / 64u; ++w) {
    const uint32_t t = lds[w];
    before += w < wave ? t : 0u;
    total += t;
  }
  __syncthreads();
  return x + before;
}

struct Cut {
  uint32_t key;   // the largest chosen key
  uint32_t ties;  // how many entries with that key are chosen: the lowest slots
};

// The cut below which lie the `need` smallest of key(0) .. key(count - 1), 1 <= need <= count: four
// passes of 8 bits, each a histogram (of whole numbers: any order gives the same) and its prefix.
template <typename Key>
__device__ Cut smallest(uint32_t count, uint32_t need, Key key, uint32_t* hist /* 258 */) {
  const uint32_t tid = threadIdx.x;
  uint32_t prefix = 0, left = need;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (uint32_t i = tid; i < 256u; i += blockDim.x) hist[i] = 0;
    __syncthreads();
    for (uint32_t i = tid; i < count; i += blockDim.x) {
      const uint32_t x = key(i);
      if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8)))
        atomicAdd(&hist[(x >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid < 64u) {
      const uint32_t c0 = hist[4 * tid], c1 = hist[4 * tid + 1], c2 = hist[4 * tid + 2],
                     c3 = hist[4 * tid + 3];
      uint32_t upto = c0 + c1 + c2 + c3;
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(upto, o);
        if (tid >= (uint32_t)o) upto += y;
      }
      uint32_t at = upto - (c0 + c1 + c2 + c3);
      const uint32_t c[4] = {c0, c1, c2, c3};
      for (uint32_t j = 0; j < 4; ++j) {
        if (at < left && left <= at + c[j]) {
          hist[256] = 4 * tid + j;
          hist[257] = left - at;
        }
        at += c[j];
      }
    }
    __syncthreads();
    prefix |= hist[256] << shift;
    left = hist[257];
    __syncthreads();
  }
  return Cut{prefix, left};
}

// Entries' keys of one (sequence, kv head): the order of their weights, 0xFFFFFFFF where protected
// or not there.
struct WeightKey {
  KvArgs a;
  KvSeq q;
  uint32_t h;
  int64_t first, newest;  // protected: pos < first or pos > newest
  __device__ uint32_t operator()(uint32_t e) const {
    const int32_t p = kv_page(a, q, (int32_t)(e >> a.page_bits));
    if (p < 0) return 0xFFFFFFFFu;
    const size_t w = kv_word(a, p, h) + (e & (a.page - 1u));
    const int32_t pos = a.pos[w];
    return pos < first || pos > newest ? 0xFFFFFFFFu : kv_order(a.weight[w]);
  }
};

__global__ __launch_bounds__(kSelBlock) void kv_victims_kernel(KvArgs a, uint32_t budget, uint32_t first,
                                                               uint32_t recent, uint32_t max_evict,
                                                               int32_t* victims, int32_t* src,
                                                               int32_t* new_len) {
  __shared__ uint32_t hist[258];
  __shared__ uint32_t scan[kSelBlock / 64];
  const uint32_t h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x;
  KvArgs b = a;
  b.tok = nullptr;
  const KvSeq q = kv_seq(b, s);
  const uint32_t len = (uint32_t)q.len;
  uint32_t n = len > budget ? len - budget : 0u;
  n = n < max_evict ? n : max_evict;
  const uint32_t stay = len - n;
  if (h == 0 && tid == 0) new_len[s] = (int32_t)stay;
  const size_t row = ((size_t)s * a.n_kv + h) * max_evict;
  uint32_t got = 0, moved = 0;
  if (n) {
    // the newest position
    int32_t top = INT32_MIN;
    for (uint32_t e = tid; e < len; e += kSelBlock) {
      const int32_t p = kv_page(a, q, (int32_t)(e >> a.page_bits));
      if (p >= 0) {
        const int32_t x = a.pos[kv_word(a, p, h) + (e & (a.page - 1u))];
        top = x > top ? x : top;
      }
    }
    for (int o = 32; o; o >>= 1) {
      const int32_t y = __shfl_xor(top, o);
      top = y > top ? y : top;
    }
    if ((tid & 63u) == 0u) scan[tid >> 6] = (uint32_t)top;
    __syncthreads();
    for (uint32_t w = 0; w < kSelBlock / 64; ++w) top = (int32_t)scan[w] > top ? (int32_t)scan[w] : top;
    __syncthreads();
    const WeightKey key{a, q, h, (int64_t)first, (int64_t)top - (int64_t)recent};
    const Cut cut = smallest(len, n, key, hist);
    // in slot order: the victims, and the kept entries behind the new end
    uint32_t ties = 0;
    for (uint32_t base = 0; base < len; base += kSelBlock) {
      const uint32_t e = base + tid;
      const uint32_t x = e < len ? key(e) : 0u;
      uint32_t total;
      const uint32_t tie = e < len && x == cut.key ? 1u : 0u;
      const uint32_t rank = ties + block_scan(tie, scan, total) - tie;
      ties += total;
      const uint32_t out = e < len && (x < cut.key || (tie && rank < cut.ties)) ? 1u : 0u;
      const uint32_t fill = e < len && !out && e >= stay ? 1u : 0u;
      const uint32_t both = block_scan(out | (fill << 16), scan, total);
      if (out) victims[row + got + (both & 0xFFFFu) - 1u] = (int32_t)e;
      if (fill) src[row + moved + (both >> 16) - 1u] = (int32_t)e;
      got += total & 0xFFFFu;
      moved += total >> 16;
    }
  }
  for (uint32_t i = got + tid; i < max_evict; i += kSelBlock) victims[row + i] = -1;
  for (uint32_t i = moved + tid; i < max_evict; i += kSelBlock) src[row + i] = -1;
}

// A block per (16 moves, kv head, sequence), a move per 16 threads.
template <typename T>
__global__ __launch_bounds__(kBlock) void kv_compact_kernel(KvArgs a, uint32_t max_evict,
                                                            const int32_t* victims, const int32_t* src,
                                                            const int32_t* new_len) {
  const uint32_t h = blockIdx.y, s = blockIdx.z;
  const uint32_t i = blockIdx.x * (kBlock / 16) + (threadIdx.x >> 4), sub = threadIdx.x & 15u;
  if (i >= max_evict) return;
  KvArgs b = a;
  b.tok = nullptr;
  const KvSeq q = kv_seq(b, s);
  const int32_t stay = new_len[s];
  const size_t row = ((size_t)s * a.n_kv + h) * max_evict;
  const int32_t from = src[row + i], to = victims[row + i];
  if (to < 0 || to >= stay || from < stay || from >= q.len) return;
  const int32_t pf = kv_page(a, q, from >> a.page_bits), pt = kv_page(a, q, to >> a.page_bits);
  if (pf < 0 || pt < 0) return;
  const uint32_t sf = (uint32_t)from & (a.page - 1u), st = (uint32_t)to & (a.page - 1u);
  const T *kf = (const T*)a.k + kv_base(a, pf, h), *vf = (const T*)a.v + kv_base(a, pf, h);
  T *kt = (T*)a.k + kv_base(a, pt, h), *vt = (T*)a.v + kv_base(a, pt, h);
  for (uint32_t d = sub; d < a.dim; d += 16u) {
    kt[(size_t)st * a.dim + d] = kf[(size_t)sf * a.dim + d];
    vt[(size_t)d * a.page + st] = vf[(size_t)d * a.page + sf];
  }
  if (sub == 0) {
    if (a.weight) a.weight[kv_word(a, pt, h) + st] = a.weight[kv_word(a, pf, h) + sf];
    if (a.pos) a.pos[kv_word(a, pt, h) + st] = a.pos[kv_word(a, pf, h) + sf];
  }
}

// The boxes after the moves: a block per (page ordinal, kv head, sequence); renewed are the pages
// below new_len that hold a victim's place or a new end.
template <typename T>
__global__ __launch_bounds__(kBlock) void kv_rebox_kernel(KvArgs a, uint32_t max_evict,
                                                          const int32_t* victims, const int32_t* new_len) {
  __shared__ float lds[kBlock / 64];
  const uint32_t h = blockIdx.y, s = blockIdx.z;
  KvArgs b = a;
  b.tok = nullptr;
  const KvSeq q = kv_seq(b, s);
  const int32_t stay = new_len[s] < q.len ? new_len[s] : q.len;
  const int32_t lo = (int32_t)(blockIdx.x << a.page_bits), hi = lo + (int32_t)a.page;
  if (lo >= stay) return;
  const int32_t page = kv_page(a, q, (int32_t)blockIdx.x);
  if (page < 0) return;
  const int32_t* v = victims + ((size_t)s * a.n_kv + h) * max_evict;
  // the first victim at or past lo; -1 stands behind the last
  uint32_t l = 0, r = max_evict;
  while (l < r) {
    const uint32_t m = (l + r) >> 1;
    if ((uint32_t)v[m] < (uint32_t)lo) l = m + 1; else r = m;
  }
  const bool got = l < max_evict && v[l] >= lo && v[l] < hi, cut = stay < q.len && stay < hi;
  if (!got && !cut) return;
  renew_box<T>(a, page, h, stay < hi ? stay - lo : (int32_t)a.page, lds);
}

// ------------------------------------------------------------------ the pages of sparse attention

// Keys of the pages for one token and kv head: a block each.  keys [n_tok][n_kv][max_pages], a
// larger score a smaller key; 0: taken in any case, 0xFFFFFFFF: not there.
template <typename T>
__global__ __launch_bounds__(kBlock) void kv_score_kernel(KvArgs a, KvRows nq, uint32_t first, uint32_t last,
                                                          uint32_t* keys) {
  __shared__ int32_t neg[256], plus[256];
  __shared__ float lds[kBlock / 64];
  const uint32_t h = blockIdx.y, j = blockIdx.x, tid = threadIdx.x;
  const KvSeq q = kv_seq(a, blockIdx.z);
  if ((int32_t)j >= q.n) return;
  const size_t t = (size_t)q.t0 + j;
  const int32_t limit = q.len - q.n + (int32_t)j + 1;
  const int32_t count = limit > 0 ? (limit + (int32_t)a.page - 1) >> a.page_bits : 0;
  const T* row = (const T*)nq.p + t * nq.tok + (size_t)h * a.group * nq.head;
  float top = 0.0f;
  for (uint32_t i = tid; i < a.group * a.dim; i += kBlock)
    top = fmaxf(top, fabsf(to_f32(row[(size_t)(i / a.dim) * nq.head + i % a.dim])));
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((tid & 63u) == 0u) lds[tid >> 6] = top;
  __syncthreads();
  for (uint32_t w = 0; w < kBlock / 64; ++w) top = fmaxf(top, lds[w]);
  const float inv = kv_step(top).inv;
  if (tid < a.dim) {
    int32_t n = 0, p = 0;
    for (uint32_t g = 0; g < a.group; ++g) {
      const int32_t x = kv_clip(rintf(to_f32(row[(size_t)g * nq.head + tid]) * inv));
      n += x < 0 ? x : 0;
      p += x > 0 ? x : 0;
    }
    neg[tid] = n;
    plus[tid] = p;
  }
  __syncthreads();
  uint32_t* out = keys + (t * a.n_kv + h) * a.max_pages;
  for (int32_t o = (int32_t)tid; o < count; o += (int32_t)kBlock) {
    const int32_t page = kv_page(a, q, o);
    uint32_t key = 0xFFFFFFFFu;
    if (page >= 0) {
      if (o < (int32_t)first || o >= count - (int32_t)last) {
        key = 0;
      } else {
        const size_t at = (size_t)page * a.n_kv + h;
        const int8_t* b = a.box + at * 2 * a.dim;
        int32_t sum = 0;
        for (uint32_t d = 0; d < a.dim; ++d) sum += neg[d] * b[d] + plus[d] * b[a.dim + d];
        key = ~kv_order((float)sum * a.box_scale[at]);
      }
    }
    out[o] = key;
  }
}

__global__ __launch_bounds__(kBlock) void kv_choose_kernel(KvArgs a, uint32_t n_sel, const uint32_t* keys,
                                                           int32_t* sel) {
  __shared__ uint32_t hist[258];
  __shared__ uint32_t scan[kBlock / 64];
  const uint32_t h = blockIdx.y, j = blockIdx.x, tid = threadIdx.x;
  const KvSeq q = kv_seq(a, blockIdx.z);
  if ((int32_t)j >= q.n) return;
  const size_t t = (size_t)q.t0 + j;
  const int32_t limit = q.len - q.n + (int32_t)j + 1;
  const uint32_t count = limit > 0 ? (uint32_t)(limit + (int32_t)a.page - 1) >> a.page_bits : 0u;
  const uint32_t* in = keys + (t * a.n_kv + h) * a.max_pages;
  int32_t* out = sel + (t * a.n_kv + h) * n_sel;
  const uint32_t need = n_sel < count ? n_sel : count;
  uint32_t got = 0;
  if (need) {
    const Cut cut = smallest(count, need, [&](uint32_t i) { return in[i]; }, hist);
    uint32_t ties = 0;
    for (uint32_t base = 0; base < count; base += kBlock) {
      const uint32_t o = base + tid, x = o < count ? in[o] : 0xFFFFFFFFu;
      uint32_t total;
      const uint32_t tie = o < count && x == cut.key ? 1u : 0u;
      const uint32_t rank = ties + block_scan(tie, scan, total) - tie;
      ties += total;
      const uint32_t take = x != 0xFFFFFFFFu && (x < cut.key || (tie && rank < cut.ties)) ? 1u : 0u;
      const uint32_t at = block_scan(take, scan, total);
      if (take) out[got + at - 1u] = (int32_t)o;
      got += total;
    }
  }
  for (uint32_t i = got + tid; i < n_sel; i += kBlock) out[i] = -1;
}

}  // namespace

hipError_t launch_kv_append(const KvArgs& a, const KvRows& k, const KvRows& v, const int32_t* pos,
                            hipStream_t st) {
  const uint32_t most = a.max_new < a.max_len ? a.max_new : a.max_len;
  const dim3 grid((most + 2 * a.page - 2) / a.page, a.n_kv, a.n_seq);
  if (a.dtype == UNISON_KV_BF16)
    hipLaunchKernelGGL(kv_append_kernel<__hip_bfloat16>, grid, dim3(kBlock), 0, st, a, k, v, pos);
  else
    hipLaunchKernelGGL(kv_append_kernel<__half>, grid, dim3(kBlock), 0, st, a, k, v, pos);
  return hipGetLastError();
}

hipError_t launch_kv_victims(const KvArgs& a, uint32_t budget, uint32_t first, uint32_t recent,
                             uint32_t max_evict, int32_t* victims, int32_t* src, int32_t* new_len,
                             hipStream_t st) {
  hipLaunchKernelGGL(kv_victims_kernel, dim3(a.n_kv, a.n_seq), dim3(kSelBlock), 0, st, a, budget, first, recent,
                     max_evict, victims, src, new_len);
  return hipGetLastError();
}

hipError_t launch_kv_compact(const KvArgs& a, uint32_t max_evict, const int32_t* victims, const int32_t* src,
                             const int32_t* new_len, hipStream_t st) {
  const dim3 grid((max_evict + kBlock / 16 - 1) / (kBlock / 16), a.n_kv, a.n_seq);
  const dim3 pages((a.max_len + a.page - 1) / a.page, a.n_kv, a.n_seq);
  if (a.dtype == UNISON_KV_BF16) {
    hipLaunchKernelGGL(kv_compact_kernel<__hip_bfloat16>, grid, dim3(kBlock), 0, st, a, max_evict, victims, src,
                       new_len);
    if (a.box)
      hipLaunchKernelGGL(kv_rebox_kernel<__hip_bfloat16>, pages, dim3(kBlock), 0, st, a, max_evict, victims,
                         new_len);
  } else {
    hipLaunchKernelGGL(kv_compact_kernel<__half>, grid, dim3(kBlock), 0, st, a, max_evict, victims, src, new_len);
    if (a.box)
      hipLaunchKernelGGL(kv_rebox_kernel<__half>, pages, dim3(kBlock), 0, st, a, max_evict, victims, new_len);
  }
  return hipGetLastError();
}

hipError_t launch_kv_choose(const KvArgs& a, const KvRows& q, uint32_t n_sel, uint32_t first, uint32_t last,
                            uint32_t* keys, int32_t* sel, hipStream_t st) {
  const dim3 grid(a.max_new, a.n_kv, a.n_seq);
  if (a.dtype == UNISON_KV_BF16)
    hipLaunchKernelGGL(kv_score_kernel<__hip_bfloat16>, grid, dim3(kBlock), 0, st, a, q, first, last, keys);
  else
    hipLaunchKernelGGL(kv_score_kernel<__half>, grid, dim3(kBlock), 0, st, a, q, first, last, keys);
  hipLaunchKernelGGL(kv_choose_kernel, grid, dim3(kBlock), 0, st, a, n_sel, (const uint32_t*)keys, sel);
  return hipGetLastError();
}

}  // namespace unison
