// kv_attend.hip -- attention of the new tokens over their sequences' pages, and the accumulated
// attention weights of the entries.
#include "kv_device.h"

#pragma clang fp contract(off)

namespace unison {

namespace {

constexpr uint32_t kBlock = 256;
constexpr float kMinusInf = -__builtin_inff();

// One block per (new token, query head, sequence): 256 entries at a time, a score per thread, then a
// dimension per thread.  sel: the pages that the token reads, or null for all of them.
template <typename T>
__global__ __launch_bounds__(kBlock) void kv_attend_kernel(KvArgs a, KvRows nq, float scale, const int32_t* sel,
                                                           uint32_t n_sel, T* out, float* lse) {
  __shared__ float qs[256], ps[kBlock], red[kBlock / 64];
  __shared__ int32_t at[kBlock];
  const uint32_t j = blockIdx.x / a.n_q, hq = blockIdx.x % a.n_q, h = hq / a.group, tid = threadIdx.x;
  const KvSeq q = kv_seq(a, blockIdx.z);
  if ((int32_t)j >= q.n) return;
  const size_t t = (size_t)q.t0 + j;
  const int32_t limit = q.len - q.n + (int32_t)j + 1;
  if (tid < a.dim) qs[tid] = to_f32(((const T*)nq.p)[t * nq.tok + hq * nq.head + tid]);
  __syncthreads();
  const int32_t* mine = sel ? sel + (t * a.n_kv + h) * n_sel : nullptr;
  const int32_t total = sel ? (int32_t)(n_sel << a.page_bits) : limit > 0 ? limit : 0;
  float m = kMinusInf, l = 0.0f, o = 0.0f;
  for (int32_t base = 0; base < total; base += (int32_t)kBlock) {
    const int32_t i = base + (int32_t)tid;
    float s = kMinusInf;
    int32_t page = -1;
    if (i < total) {
      const int32_t ord = mine ? mine[i >> a.page_bits] : i >> a.page_bits;
      const int32_t e = (ord << a.page_bits) + (i & (int32_t)(a.page - 1u));
      if (ord >= 0 && e < limit) page = kv_page(a, q, ord);
      if (page >= 0) {
        const T* k = (const T*)a.k + kv_base(a, page, h) + (size_t)(e & (int32_t)(a.page - 1u)) * a.dim;
        s = 0.0f;
        for (uint32_t d = 0; d < a.dim; ++d) s = fmaf(qs[d], to_f32(k[d]), s);
        s *= scale;
      }
    }
    at[tid] = page;
    float top = s;
    for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    if ((tid & 63u) == 0u) red[tid >> 6] = top;
    __syncthreads();
    for (uint32_t w = 0; w < kBlock / 64; ++w) top = fmaxf(top, red[w]);
    const float next = fmaxf(m, top);
    if (next > kMinusInf) {
      const float shrink = m > kMinusInf ? expf(m - next) : 0.0f;
      ps[tid] = s > kMinusInf ? expf(s - next) : 0.0f;
      __syncthreads();
      l *= shrink;
      o *= shrink;
      for (uint32_t x = 0; x < kBlock; ++x) {
        if (at[x] < 0) continue;
        l += ps[x];
        if (tid < a.dim)
          o = fmaf(ps[x], to_f32(((const T*)a.v)[kv_base(a, at[x], h) + (size_t)tid * a.page +
                                                 ((uint32_t)(base + (int32_t)x) & (a.page - 1u))]), o);
      }
      m = next;
    }
    __syncthreads();
  }
  if (tid < a.dim) out[(t * a.n_q + hq) * a.dim + tid] = from_f32<T>(l > 0.0f ? o / l : 0.0f);
  if (lse && tid == 0) lse[t * a.n_q + hq] = l > 0.0f ? m + logf(l) : kMinusInf;
}

// weight = decay * weight + the sum of p over the sequence's new tokens: a thread per entry.
template <typename T>
__global__ __launch_bounds__(kBlock) void kv_weight_kernel(KvArgs a, KvRows nq, float scale, float decay,
                                                           const float* lse) {
  const uint32_t h = blockIdx.y;
  const KvSeq q = kv_seq(a, blockIdx.z);
  const int32_t e = (int32_t)(blockIdx.x * kBlock + threadIdx.x);
  if (q.n == 0 || e >= q.len) return;
  const int32_t page = kv_page(a, q, e >> a.page_bits);
  if (page < 0) return;
  const uint32_t slot = (uint32_t)e & (a.page - 1u);
  const T* k = (const T*)a.k + kv_base(a, page, h) + (size_t)slot * a.dim;
  float sum = 0.0f;
  for (int32_t j = 0; j < q.n; ++j) {
    if (e >= q.len - q.n + j + 1) continue;
    for (uint32_t g = 0; g < a.group; ++g) {
      const size_t t = (size_t)(q.t0 + j);
      const uint32_t hq = h * a.group + g;
      const T* row = (const T*)nq.p + t * nq.tok + hq * nq.head;
      float s = 0.0f;
      for (uint32_t d = 0; d < a.dim; ++d) s = fmaf(to_f32(row[d]), to_f32(k[d]), s);
      sum += expf(s * scale - lse[t * a.n_q + hq]);
    }
  }
  float* w = a.weight + kv_word(a, page, h) + slot;
  *w = fmaf(decay, *w, sum);
}

}  // namespace

size_t kv_attend_bytes(const KvArgs& a, bool weights, uint32_t n_sel) {
  (void)weights;
  const size_t lse = (size_t)a.n_tok * a.n_q * sizeof(float);
  const size_t keys = n_sel ? (size_t)a.n_tok * a.n_kv * a.max_pages * sizeof(uint32_t) : 0;
  return (lse + 255) / 256 * 256 + keys;
}

hipError_t launch_kv_choose(const KvArgs& a, const KvRows& q, uint32_t n_sel, uint32_t first, uint32_t last,
                            uint32_t* keys, int32_t* sel, hipStream_t st);

template <typename T>
static hipError_t attend(const KvArgs& a, const KvRows& q, float scale, bool weights, float decay, uint32_t n_sel,
                         const int32_t* sel, void* out, float* lse, void* ws, hipStream_t st) {
  float* l = lse ? lse : (float*)ws;
  hipLaunchKernelGGL(kv_attend_kernel<T>, dim3(a.max_new * a.n_q, 1, a.n_seq), dim3(kBlock), 0, st, a, q, scale, sel,
                     n_sel, (T*)out, l);
  if (weights)
    hipLaunchKernelGGL(kv_weight_kernel<T>, dim3((a.max_len + kBlock - 1) / kBlock, a.n_kv, a.n_seq), dim3(kBlock), 0,
                       st, a, q, scale, decay, (const float*)l);
  return hipGetLastError();
}

hipError_t launch_kv_attend(const KvArgs& a, const KvRows& q, float scale, bool weights, float decay,
                            uint32_t n_sel, uint32_t first, uint32_t last, void* out, float* lse, int32_t* sel,
                            void* ws, hipStream_t st) {
  if (n_sel) {
    const size_t at = ((size_t)a.n_tok * a.n_q * sizeof(float) + 255) / 256 * 256;
    const hipError_t rc = launch_kv_choose(a, q, n_sel, first, last, (uint32_t*)((char*)ws + at), sel, st);
    if (rc != hipSuccess) return rc;
  }
  return a.dtype == UNISON_KV_BF16
             ? attend<__hip_bfloat16>(a, q, scale, weights, decay, n_sel, sel, out, lse, ws, st)
             : attend<__half>(a, q, scale, weights, decay, n_sel, sel, out, lse, ws, st);
}

}  // namespace unison
