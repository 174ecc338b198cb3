// kv_attend.hip -- attention of the new tokens over their sequences' pages, and the accumulated
// attention weights of the entries.
//
// Both products run on the matrix cores transposed: S^T = K Q^T leaves a query row in every lane's
// column and the entries in its registers, which is the layout the second product
// O^T = V^T P^T takes its right operand in.  The scores therefore never leave the registers and
// are never exchanged between lanes: the rows of the left operand K are permuted (any order of
// entries gives the same sums) so that a lane's registers hold 8 consecutive entries, and V,
// stored transposed, is read in the same runs of 8.
//
// The softmax keeps a running maximum and sum in 32 bits.  The maximum is only moved when a score
// passes it by kSlack (in powers of two), which a ballot tells: p then stays below 2^kSlack, and the
// cross-lane maximum and the rescaling of the sums run a few times per row instead of once per tile.
#include "kv_device.h"

#include <type_traits>

#pragma clang fp contract(off)

namespace unison {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));

struct Bf16 {
  typedef __bf16 t;
  typedef b16x8 v8;
  static __device__ __forceinline__ f32x4 mma16(v8 a, v8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mma32(v8 a, v8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
struct Fp16 {
  typedef _Float16 t;
  typedef h16x8 v8;
  static __device__ __forceinline__ f32x4 mma16(v8 a, v8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mma32(v8 a, v8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

constexpr uint32_t kBlock = 256;
constexpr uint32_t kWaves = kBlock / 64;
constexpr uint32_t kRowsFew = 32;         // rows of a (sequence, kv head) up to which the few-rows kernel serves it
constexpr uint32_t kPagesLds = 1024;      // page ids of one block's entries
constexpr uint32_t kManyRows = 128, kManyKeys = 64;
constexpr float kInf = __builtin_inff();
constexpr float kSlack = 8.0f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Everything a launch of the attention kernels takes.
struct Attn {
  KvArgs a;
  KvRows q;
  float scale2;         // scale * log2(e): scores are powers of two
  void* out;
  float* lse;
  const int32_t* sel;   // [n_tok][n_kv][n_sel], or null: every page
  uint32_t n_sel;
  // Partial results of a split of the entries, for row r of (sequence s, kv head h):
  // index ((split * n_seq + s) * n_kv + h) * row_cap + r
  float* part_o;        // [..][dim], times the exponential of the maximum
  float2* part_ml;      // maximum (power of two) and sum
  float* scores;        // [n_seq][n_kv][row_cap][score_len], or null
  uint32_t n_split, chunk, row_cap, score_len;
  uint32_t rows_from, rows_to;  // rows of a sequence that this launch serves: rows_from < n * group <= rows_to
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float or_zero(float m) { return m == -kInf ? 0.0f : m; }

__device__ __forceinline__ size_t part_row(const Attn& p, uint32_t split, uint32_t s, uint32_t h) {
  return (((size_t)split * p.a.n_seq + s) * p.a.n_kv + h) * p.row_cap;
}

template <typename M, int N>
__device__ __forceinline__ void store4(typename M::t* out, const float (&x)[N]) {
  typedef typename M::t v4 __attribute__((ext_vector_type(4)));
  v4 y;
  for (int i = 0; i < 4; ++i) y[i] = (typename M::t)x[i];
  *(v4*)out = y;
}

// ------------------------------------------------------------------ few rows

// Attention of up to 16 * NT rows (new tokens x the kv head's query heads) over a chunk of entries:
// what a decode step is.  It reads every key and value once and computes little on each, so it is
// bound by HBM; the wavefronts of a block take tiles of 32 entries in turn, straight from memory
// into the matrix operands, and join their maxima, sums and products in LDS at the end.  With
// SPARSE a block serves one token and reads the pages of its choice instead of all.
template <typename M, int D, int NT, bool SPARSE, bool SCORES>
__global__ __launch_bounds__(kBlock, NT * D <= 128 ? 3 : NT * D <= 256 ? 2 : 1) void kv_few_kernel(Attn p) {
  typedef typename M::t T;
  typedef typename M::v8 v8;
  constexpr int KS = D / 32, DT = D / 16;
  __shared__ int32_t pg[kPagesLds + 1];
  __shared__ int32_t eb[SPARSE ? kPagesLds + 1 : 1];
  __shared__ f32x4 join[(kWaves / 2) * NT * DT * 64];
  __shared__ float2 join_ml[(kWaves / 2) * NT * 64];
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x, lane = tid & 63u;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const uint32_t split = blockIdx.x % p.n_split;
  const KvSeq q = kv_seq(a, s);
  uint32_t r0 = 0, rows;
  const int32_t* sel = nullptr;
  if (SPARSE) {
    const uint32_t tiles = (a.group + 16 * NT - 1) / (16 * NT), x = blockIdx.x / p.n_split;
    const uint32_t j = x / tiles, first = (x % tiles) * 16 * NT;
    if ((int32_t)j >= q.n) return;
    r0 = j * a.group + first;
    rows = a.group - first < 16u * NT ? a.group - first : 16u * NT;
    sel = p.sel + ((size_t)(q.t0 + (int32_t)j) * a.n_kv + h) * p.n_sel;
  } else {
    rows = (uint32_t)q.n * a.group;
    if (rows <= p.rows_from || rows > p.rows_to) return;
  }
  const uint32_t all = SPARSE ? p.n_sel << a.page_bits : (uint32_t)q.len;
  const uint32_t start = split * p.chunk, end = start + p.chunk < all ? start + p.chunk : all;
  if (start >= all && split) return;

  for (uint32_t i = tid; i < (p.chunk >> a.page_bits) + 1u; i += kBlock) {
    int32_t page = -1, o = -1;
    if (start + (i << a.page_bits) < end) {
      o = (int32_t)((start >> a.page_bits) + i);
      if (SPARSE) o = sel[o];
      if (o >= 0 && (o << a.page_bits) < q.len) page = kv_page(a, q, o);
    }
    pg[i] = page;
    if (SPARSE) eb[i] = o << a.page_bits;
  }
  __syncthreads();

  const uint32_t r16 = lane & 15u, g4 = lane >> 4;
  // the lane's query rows: the right operand of S^T, and how many entries each sees
  v8 qf[NT][KS];
  int32_t limit[NT];
  const int32_t old = q.len - q.n;  // entries before the new tokens
  for (int n = 0; n < NT; ++n) {
    const uint32_t r = r16 + 16u * n;
    const bool is = r < rows;
    const uint32_t j = (r0 + (is ? r : 0u)) / a.group, g = (r0 + (is ? r : 0u)) % a.group;
    const T* row = (const T*)p.q.p + (size_t)(q.t0 + (int32_t)j) * p.q.tok + (h * a.group + g) * p.q.head;
    limit[n] = is ? old + (int32_t)j + 1 : 0;
    for (int k = 0; k < KS; ++k) {
      v8 x = *(const v8*)(row + 32 * k + 8 * g4);
      if (!is) x = (v8)(T)0.0f;
      qf[n][k] = x;
    }
  }
  const int32_t seen_by_all = old + (int32_t)(r0 / a.group) + 1;

  f32x4 o[NT][DT];
  float m[NT], l[NT];
  for (int n = 0; n < NT; ++n) {
    m[n] = -kInf;
    l[n] = 0.0f;
    for (int t = 0; t < DT; ++t) o[n][t] = (f32x4)0.0f;
  }
  const size_t head = (size_t)h * a.page * D, per_page = (size_t)a.n_kv * a.page * D;
  const uint32_t in_page = a.page - 1u;
  // keys: lane r of the left operand has entry 8 (r / 4) + r % 4 of the tile, and 4 behind it
  const uint32_t k_of = 8u * (r16 >> 2);
  const auto load_k = [&](uint32_t i, v8 (&k)[2][KS]) {
    const uint32_t e = i + k_of;
    int32_t page = pg[(e - start) >> a.page_bits];
    page = page < 0 ? 0 : page;
    const T* at = (const T*)a.k + (size_t)page * per_page + head + ((e & in_page) + (r16 & 3u)) * D + 8 * g4;
    for (int x = 0; x < 2; ++x)
      for (int c = 0; c < KS; ++c) k[x][c] = *(const v8*)(at + x * 4 * D + 32 * c);
  };
  v8 k[2][KS];
  uint32_t i = start + 32u * wave;
  if (i < end) load_k(i, k);
  for (; i < end; i += 32u * kWaves) {
    // values: lane r has dimension r of each 16, entries 8 (lane / 16) to + 7
    v8 v[DT];
    const uint32_t ev = i + 8u * g4;
    const int32_t vpage = pg[(ev - start) >> a.page_bits];
    {
      const T* at = (const T*)a.v + (size_t)(vpage < 0 ? 0 : vpage) * per_page + head + (size_t)r16 * a.page +
                    (ev & in_page);
      for (int t = 0; t < DT; ++t) v[t] = *(const v8*)(at + (size_t)t * 16 * a.page);
    }
    f32x4 sc[NT][2];
    for (int n = 0; n < NT; ++n)
      for (int x = 0; x < 2; ++x) {
        sc[n][x] = (f32x4)0.0f;
        for (int c = 0; c < KS; ++c) sc[n][x] = M::mma16(k[x][c], qf[n][c], sc[n][x]);
      }
    if (i + 32u * kWaves < end) load_k(i + 32u * kWaves, k);
    // the entry of the lane's first value, and whether every row sees the whole tile
    const int32_t mine = SPARSE ? eb[(ev - start) >> a.page_bits] + (int32_t)(ev & in_page) : (int32_t)ev;
    const bool inside = vpage >= 0 && mine + 8 <= seen_by_all;
    const bool whole = __builtin_amdgcn_ballot_w64(!inside) == 0ull;
    if (!whole)
      for (int t = 0; t < DT; ++t)
        for (int x = 0; x < 8; ++x)  // what is not an entry may hold anything
          if (vpage < 0 || mine + x >= q.len) v[t][x] = (T)0.0f;
    for (int n = 0; n < NT; ++n) {
      float z[8];
      for (int x = 0; x < 8; ++x) z[x] = sc[n][x >> 2][x & 3] * p.scale2;
      if (!whole)
        for (int x = 0; x < 8; ++x)
          if (vpage < 0 || mine + x >= limit[n]) z[x] = -kInf;
      if (SCORES && r16 + 16u * n < rows) {
        float* to = p.scores + (((size_t)s * a.n_kv + h) * p.row_cap + r16 + 16u * n) * p.score_len + ev;
        *(f32x4*)to = f32x4{z[0], z[1], z[2], z[3]};
        *(f32x4*)(to + 4) = f32x4{z[4], z[5], z[6], z[7]};
      }
      float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
      if (__builtin_amdgcn_ballot_w64(top > m[n] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float next = fmaxf(m[n], top);
        const float f = exp2_fast(m[n] - or_zero(next));
        m[n] = next;
        l[n] *= f;
        for (int t = 0; t < DT; ++t) o[n][t] *= f;
      }
      const float base = or_zero(m[n]);
      v8 pf;
      for (int x = 0; x < 8; ++x) {
        const float e = exp2_fast(z[x] - base);
        l[n] += e;
        // p is rounded to the inputs' type for the second product (half a step of each term); the sum
        // it is divided by is not
        pf[x] = (T)e;
      }
      for (int t = 0; t < DT; ++t) o[n][t] = M::mma16(v[t], pf, o[n][t]);
    }
  }
  for (int n = 0; n < NT; ++n) {
    l[n] += __shfl_xor(l[n], 16);
    l[n] += __shfl_xor(l[n], 32);
  }
  // join the wavefronts, half of them at a time
  for (uint32_t half = kWaves / 2; half; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
      const uint32_t at = wave - half;
      for (int n = 0; n < NT; ++n) {
        join_ml[(at * NT + n) * 64 + lane] = make_float2(m[n], l[n]);
        for (int t = 0; t < DT; ++t) join[((at * NT + n) * DT + t) * 64 + lane] = o[n][t];
      }
    }
    __syncthreads();
    if (wave < half) {
      for (int n = 0; n < NT; ++n) {
        const float2 y = join_ml[(wave * NT + n) * 64 + lane];
        const float next = or_zero(fmaxf(m[n], y.x));
        const float f = exp2_fast(m[n] - next), g = exp2_fast(y.x - next);
        m[n] = fmaxf(m[n], y.x);
        l[n] = l[n] * f + y.y * g;
        for (int t = 0; t < DT; ++t) o[n][t] = o[n][t] * f + join[((wave * NT + n) * DT + t) * 64 + lane] * g;
      }
    }
    __syncthreads();
  }
  if (wave) return;
  for (int n = 0; n < NT; ++n) {
    const uint32_t r = r16 + 16u * n;
    if (r >= rows) continue;
    const size_t part = part_row(p, split, s, h) + r0 + r;
    if (g4 == 0 && (p.n_split > 1 || SCORES)) p.part_ml[part] = make_float2(m[n], l[n]);
    if (p.n_split > 1) {
      for (int t = 0; t < DT; ++t) *(f32x4*)(p.part_o + part * D + 16 * t + 4 * g4) = o[n][t];
    } else {
      const size_t row = (size_t)(q.t0 + (int32_t)((r0 + r) / a.group)) * a.n_q + h * a.group + (r0 + r) % a.group;
      const float inv = l[n] > 0.0f ? 1.0f / l[n] : l[n] == 0.0f ? 0.0f : l[n];
      for (int t = 0; t < DT; ++t) {
        const float x[4] = {o[n][t][0] * inv, o[n][t][1] * inv, o[n][t][2] * inv, o[n][t][3] * inv};
        store4<M>((T*)p.out + row * D + 16 * t + 4 * g4, x);
      }
      if (p.lse && g4 == 0) p.lse[row] = l[n] == 0.0f ? -kInf : (m[n] + log2f(l[n])) * kLn2;
    }
  }
}

// Joins the splits of a few- or many-rows launch: 1024 / dim rows a block, 4 dimensions a thread.
template <typename M, int D>
__global__ __launch_bounds__(kBlock) void kv_join_kernel(Attn p) {
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z;
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group, r = blockIdx.x * (4 * kBlock / D) + threadIdx.x / (D / 4);
  if (r >= rows || (!p.sel && (rows <= p.rows_from || rows > p.rows_to))) return;
  const uint32_t d = 4 * (threadIdx.x % (D / 4));
  const uint32_t all = p.sel ? p.n_sel << a.page_bits : (uint32_t)q.len;
  const uint32_t used = all ? (all + p.chunk - 1) / p.chunk : 1u;
  float m = -kInf;
  for (uint32_t i = 0; i < used; ++i) m = fmaxf(m, p.part_ml[part_row(p, i, s, h) + r].x);
  const float base = or_zero(m);
  float l = 0.0f;
  f32x4 o = (f32x4)0.0f;
  for (uint32_t i = 0; i < used; ++i) {
    const size_t part = part_row(p, i, s, h) + r;
    const float2 y = p.part_ml[part];
    const float f = exp2_fast(y.x - base);
    l += y.y * f;
    o += *(const f32x4*)(p.part_o + part * D + d) * f;
  }
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  const size_t row = (size_t)(q.t0 + (int32_t)(r / a.group)) * a.n_q + h * a.group + r % a.group;
  const float x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  store4<M>((typename M::t*)p.out + row * D + d, x);
  if (p.lse && d == 0) p.lse[row] = l == 0.0f ? -kInf : (m + log2f(l)) * kLn2;
}

// weight = decay * weight + sum of p, from the scores that the few-rows kernel left: a thread per
// four entries.
__global__ __launch_bounds__(kBlock) void kv_weight_few_kernel(Attn p, float decay) {
  __shared__ float base[kRowsFew];
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group;
  if (rows == 0 || blockIdx.x * 4 * kBlock >= (uint32_t)q.len) return;
  if (tid < rows) {
    const uint32_t used = ((uint32_t)q.len + p.chunk - 1) / p.chunk;
    float m = -kInf, l = 0.0f;
    for (uint32_t i = 0; i < used; ++i) m = fmaxf(m, p.part_ml[part_row(p, i, s, h) + tid].x);
    for (uint32_t i = 0; i < used; ++i) {
      const float2 y = p.part_ml[part_row(p, i, s, h) + tid];
      l += y.y * exp2_fast(y.x - or_zero(m));
    }
    base[tid] = l == 0.0f ? kInf : m + log2f(l);
  }
  __syncthreads();
  const uint32_t e = 4 * (blockIdx.x * kBlock + tid);
  if (e >= (uint32_t)q.len) return;
  const int32_t page = kv_page(a, q, (int32_t)(e >> a.page_bits));
  if (page < 0) return;
  const float* z = p.scores + ((size_t)s * a.n_kv + h) * p.row_cap * p.score_len + e;
  f32x4 sum = (f32x4)0.0f;
  for (uint32_t r = 0; r < rows; ++r) {
    const f32x4 x = *(const f32x4*)(z + (size_t)r * p.score_len);
    for (int i = 0; i < 4; ++i) sum[i] += exp2_fast(x[i] - base[r]);
  }
  float* w = a.weight + kv_word(a, page, h) + (e & (a.page - 1u));
  const f32x4 was = *(const f32x4*)w;
  for (int i = 0; i < 4; ++i)
    if (e + i < (uint32_t)q.len) w[i] = fmaf(decay, was[i], sum[i]);
}

// ------------------------------------------------------------------ many rows

// 16 bytes from memory into LDS without a register: lane i's go to lds + 16 i.
__device__ __forceinline__ void to_lds(const void* from, void* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// The order in which rows of a left operand hold entries: bits 2 and 3 change places.
__device__ __forceinline__ uint32_t swap23(uint32_t x) {
  return (x & ~12u) | ((x & 4u) << 1) | ((x & 8u) >> 1);
}

// Attention of 128 rows over a chunk of entries, 32 rows a wavefront, 64 entries at a time from
// double-buffered LDS: a turn's new tokens over their session.  The 16-byte pieces of a row are
// stored at places xored with the row, so that the 8 or 16 rows that a read takes at once lie in
// different banks.  Bound by the matrix cores and the exponentials beside them.
template <typename M, int D>
__global__ __launch_bounds__(kBlock, D <= 128 ? 2 : 1) void kv_many_kernel(Attn p) {
  typedef typename M::t T;
  typedef typename M::v8 v8;
  constexpr uint32_t CH = D / 8, MASK = CH - 1 < 15 ? CH - 1 : 15;
  constexpr int KS = D / 16, DT = D / 32, NK = CH / 4, NV = D / 32;
  __shared__ v8 kt[2][kManyKeys * CH];
  __shared__ v8 vt[2][D * 8];
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.x % a.n_kv, split = blockIdx.x / a.n_kv, s = blockIdx.z, tid = threadIdx.x;
  const uint32_t lane = tid & 63u, half = lane >> 5, r32 = lane & 31u;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group;
  const uint32_t tile = gridDim.y - 1u - blockIdx.y;  // the longest first
  if (rows <= p.rows_from || tile * kManyRows >= rows) return;
  const int32_t old = q.len - q.n;
  const uint32_t r = tile * kManyRows + 32u * wave + r32;
  const bool is = r < rows;
  const uint32_t j = (is ? r : 0u) / a.group, g = (is ? r : 0u) % a.group;
  const int32_t limit = is ? old + (int32_t)j + 1 : 0;
  // entries that some row of the block (of the wavefront) sees, and that all rows of the wavefront see
  const auto token = [&](uint32_t x) { return (int32_t)((x < rows ? x : rows - 1u) / a.group); };
  const int32_t block_end = old + token((tile + 1u) * kManyRows - 1u) + 1;
  const uint32_t w0 = tile * kManyRows + 32u * wave;
  const int32_t wave_end = w0 < rows ? old + token(w0 + 31u) + 1 : 0;
  const int32_t seen_by_all = old + token(w0) + 1;
  const int32_t start = (int32_t)(split * p.chunk);
  int32_t end = block_end < q.len ? block_end : q.len;
  if ((uint32_t)end > (uint32_t)start + p.chunk && end > 0) end = start + (int32_t)p.chunk;
  if (start >= q.len && split) return;

  v8 qf[KS];
  {
    const T* row = (const T*)p.q.p + (size_t)(q.t0 + (int32_t)j) * p.q.tok + (h * a.group + g) * p.q.head;
    for (int k = 0; k < KS; ++k) {
      v8 x = *(const v8*)(row + 16 * k + 8 * half);
      if (!is) x = (v8)(T)0.0f;
      qf[k] = x;
    }
  }
  f32x16 o[DT];
  for (int t = 0; t < DT; ++t) o[t] = (f32x16)0.0f;
  float m = -kInf, l = 0.0f;

  const size_t head = (size_t)h * a.page * D, per_page = (size_t)a.n_kv * a.page * D;
  const uint32_t in_page = a.page - 1u;
  // the pages of a tile's four runs of 16 entries; bit 4 i of the result: run i is there
  int32_t pg[4];
  const auto pages_of = [&](int32_t base, int32_t (&to)[4]) {
    for (int i = 0; i < 4; ++i) {
      const int32_t e = base + 16 * i;
      to[i] = e < q.len ? kv_page(a, q, e >> a.page_bits) : -1;
    }
  };
  const auto pick = [&](const int32_t (&from)[4], uint32_t i) {
    const int32_t x = i & 1u ? from[1] : from[0], y = i & 1u ? from[3] : from[2];
    const int32_t z = i & 2u ? y : x;
    return z < 0 ? 0 : z;
  };
  const auto load = [&](int32_t base, const int32_t (&from)[4], uint32_t buf) {
    for (int i = 0; i < NK; ++i) {
      const uint32_t at = (wave * NK + i) * 64u, c = at + lane, row = c / CH;
      const uint32_t key = swap23(row), part = (c % CH) ^ (row & MASK);
      const T* src = (const T*)a.k + (size_t)pick(from, key >> 4) * per_page + head +
                     (((uint32_t)base + key) & in_page) * D + 8 * part;
      to_lds(src, &kt[buf][at]);
    }
    for (int i = 0; i < NV; ++i) {
      const uint32_t at = (wave * NV + i) * 64u, c = at + lane, d = c >> 3;
      const uint32_t part = (c & 7u) ^ (d & 7u);
      const T* src = (const T*)a.v + (size_t)pick(from, part >> 1) * per_page + head + (size_t)d * a.page +
                     (((uint32_t)base + 8 * part) & in_page);
      to_lds(src, &vt[buf][at]);
    }
  };
  int32_t next_pg[4] = {-1, -1, -1, -1};
  if (start < end) {
    pages_of(start, pg);
    load(start, pg, 0);
    pages_of(start + (int32_t)kManyKeys, next_pg);
  }
  uint32_t buf = 0;
  for (int32_t base = start; base < end; base += (int32_t)kManyKeys, buf ^= 1u) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int32_t after[4];
    if (base + (int32_t)kManyKeys < end) {
      load(base + (int32_t)kManyKeys, next_pg, buf ^ 1u);
      pages_of(base + 2 * (int32_t)kManyKeys, after);
    } else {
      for (int i = 0; i < 4; ++i) after[i] = -1;
    }
    const bool there = (pg[0] | pg[1] | pg[2] | pg[3]) >= 0;
    if (!there || base + (int32_t)kManyKeys > q.len) {  // what is not an entry may hold anything
      for (uint32_t c = tid; c < D * 8u; c += kBlock) {
        const uint32_t part = (c & 7u) ^ ((c >> 3) & 7u);
        const int32_t run = part & 4u ? (part & 2u ? pg[3] : pg[2]) : (part & 2u ? pg[1] : pg[0]);
        v8 x = vt[buf][c];
        for (int i = 0; i < 8; ++i)
          if (run < 0 || base + (int32_t)(8 * part) + i >= q.len) x[i] = (T)0.0f;
        vt[buf][c] = x;
      }
      __syncthreads();
    }
    if (base < wave_end) {
      float z[32];
      for (int b = 0; b < 2; ++b) {
        f32x16 sc = (f32x16)0.0f;
        const uint32_t row = 32u * b + r32;
        for (int k = 0; k < KS; ++k) sc = M::mma32(kt[buf][row * CH + ((2 * k + half) ^ (row & MASK))], qf[k], sc);
        for (int i = 0; i < 16; ++i) z[16 * b + i] = sc[i] * p.scale2;
      }
      // register i of the lane is entry 16 (i / 8) + 8 half + i % 8 of the tile
      if (!there || base + (int32_t)kManyKeys > seen_by_all)
        for (int i = 0; i < 32; ++i) {
          const int32_t e = base + 16 * (i >> 3) + 8 * (int32_t)half + (i & 7);
          if (pg[i >> 3] < 0 || e >= limit) z[i] = -kInf;
        }
      float top = z[0];
      for (int i = 1; i < 32; ++i) top = fmaxf(top, z[i]);
      if (__builtin_amdgcn_ballot_w64(top > m + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float next = fmaxf(m, top);
        const float f = exp2_fast(m - or_zero(next));
        m = next;
        l *= f;
        for (int t = 0; t < DT; ++t) o[t] *= f;
      }
      const float sub = or_zero(m);
      v8 pf[4];
      for (int i = 0; i < 32; ++i) {
        const float e = exp2_fast(z[i] - sub);
        l += e;
        pf[i >> 3][i & 7] = (T)e;  // rounded for the second product only, as above
      }
      for (int t = 0; t < DT; ++t) {
        const uint32_t d = 32u * t + r32;
        for (int k = 0; k < 4; ++k) o[t] = M::mma32(vt[buf][d * 8 + ((2 * k + half) ^ (d & 7u))], pf[k], o[t]);
      }
    }
    for (int i = 0; i < 4; ++i) {
      pg[i] = next_pg[i];
      next_pg[i] = after[i];
    }
  }
  l += __shfl_xor(l, 32);
  if (!is) return;
  const size_t part = part_row(p, split, s, h) + r;
  if (p.n_split > 1) {
    if (half == 0) p.part_ml[part] = make_float2(m, l);
    for (int t = 0; t < DT; ++t)
      for (int c = 0; c < 4; ++c)
        *(f32x4*)(p.part_o + part * D + 32 * t + 8 * c + 4 * half) =
            f32x4{o[t][4 * c], o[t][4 * c + 1], o[t][4 * c + 2], o[t][4 * c + 3]};
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  const size_t row = (size_t)(q.t0 + (int32_t)j) * a.n_q + h * a.group + g;
  for (int t = 0; t < DT; ++t)
    for (int c = 0; c < 4; ++c) {
      const float x[4] = {o[t][4 * c] * inv, o[t][4 * c + 1] * inv, o[t][4 * c + 2] * inv, o[t][4 * c + 3] * inv};
      store4<M>((T*)p.out + row * D + 32 * t + 8 * c + 4 * half, x);
    }
  if (p.lse && half == 0) p.lse[row] = l == 0.0f ? -kInf : (m + log2f(l)) * kLn2;
}

// weight = decay * weight + the sum of p over a sequence's rows, which another product of the keys
// with the queries gives, the entries in the lanes now and the rows in their registers: 32 entries a
// wavefront with their keys in registers, 32 rows at a time from LDS.
template <typename M, int D>
__global__ __launch_bounds__(kBlock) void kv_weight_many_kernel(Attn p, float decay) {
  typedef typename M::t T;
  typedef typename M::v8 v8;
  constexpr uint32_t CH = D / 8, MASK = CH - 1 < 15 ? CH - 1 : 15;
  constexpr int KS = D / 16;
  __shared__ v8 qt[32 * CH];
  __shared__ float base[32];
  __shared__ int32_t lim[32];
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x, lane = tid & 63u, half = lane >> 5, c32 = lane & 31u;
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group;
  const int32_t first = (int32_t)(blockIdx.x * (kBlock / 2));
  if (rows == 0 || first >= q.len) return;
  const int32_t e = first + (int32_t)(32u * (tid >> 6) + c32), old = q.len - q.n;
  const int32_t page = e < q.len ? kv_page(a, q, e >> a.page_bits) : -1;
  const uint32_t slot = (uint32_t)e & (a.page - 1u);
  const T* key = (const T*)a.k + kv_base(a, page < 0 ? 0 : page, h) + (size_t)slot * D;
  v8 kf[KS];
  for (int k = 0; k < KS; ++k) kf[k] = *(const v8*)(key + 16 * k + 8 * half);
  float sum = 0.0f;
  // rows of tokens before entry `first` see nothing here
  const uint32_t from = first > old ? ((uint32_t)(first - old) * a.group) & ~31u : 0u;
  for (uint32_t r0 = from; r0 < rows; r0 += 32u) {
    for (uint32_t c = tid; c < 32u * CH; c += kBlock) {
      const uint32_t row = c / CH, part = c % CH, r = r0 + row;
      v8 x = (v8)(T)0.0f;
      if (r < rows)
        x = *(const v8*)((const T*)p.q.p + (size_t)(q.t0 + (int32_t)(r / a.group)) * p.q.tok +
                         (h * a.group + r % a.group) * p.q.head + 8 * part);
      qt[row * CH + (part ^ (row & MASK))] = x;
    }
    if (tid < 32u) {
      const uint32_t r = r0 + tid;
      float b = kInf;
      int32_t to = 0;
      if (r < rows) {
        const int32_t j = (int32_t)(r / a.group);
        b = p.lse[(size_t)(q.t0 + j) * a.n_q + h * a.group + r % a.group] * kLog2e;
        if (b == -kInf) b = kInf;
        to = old + j + 1;
      }
      base[tid] = b;
      lim[tid] = to;
    }
    __syncthreads();
    f32x16 sc = (f32x16)0.0f;
    for (int k = 0; k < KS; ++k) sc = M::mma32(qt[c32 * CH + ((2 * k + half) ^ (c32 & MASK))], kf[k], sc);
    float part = 0.0f;  // a tile's sum first: thousands of rows added one by one would lose bits
    for (int i = 0; i < 16; ++i) {
      const uint32_t row = 8u * (i >> 2) + 4u * half + (i & 3);
      const float x = exp2_fast(sc[i] * p.scale2 - base[row]);
      part += e < lim[row] ? x : 0.0f;
    }
    sum += part;
    __syncthreads();
  }
  sum += __shfl_xor(sum, 32);
  if (page < 0 || half) return;
  float* w = a.weight + kv_word(a, page, h) + slot;
  *w = fmaf(decay, *w, sum);
}

// ------------------------------------------------------------------ plans

size_t up(size_t x, size_t to) { return (x + to - 1) / to * to; }

// How a call is split and where its workspace lies.
struct Plan {
  uint32_t few_rows;       // rows of a tile of the few-rows kernel: 16 or 32
  bool few, many;          // which kernels run
  uint32_t few_chunk, few_split, few_cap, many_chunk, many_split, score_len;
  size_t o, ml, many_o, many_ml, scores, lse, keys, bytes;
};

constexpr uint64_t kBlocksWanted = 2048;  // eight blocks a compute unit: enough loads in flight

// The entries of a split: at least 256, few enough that `units` of them give the blocks wanted, at
// most what LDS has page ids for, whole pages and whole rounds of the block's tiles.
uint32_t chunk_of(const KvArgs& a, uint64_t entries, uint64_t units, uint64_t wanted, uint32_t least) {
  const uint64_t splits = units >= wanted ? 1 : (wanted + units - 1) / units;
  uint64_t c = (entries + splits - 1) / splits;
  c = c < least ? least : c;
  const uint64_t most = (uint64_t)kPagesLds * a.page;
  c = c > most ? most : c;
  return (uint32_t)up(c, a.page > 128 ? a.page : 128);
}

Plan plan_of(const KvArgs& a, bool weights, uint32_t n_sel) {
  Plan p = {};
  const uint64_t row_most = (uint64_t)a.max_new * a.group;
  const uint64_t pairs = (uint64_t)a.n_seq * a.n_kv;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t was = at;
    at = up(at + bytes, 256);
    return was;
  };
  if (n_sel) {
    p.few = true;
    p.few_rows = a.group > 16 ? 32 : 16;
    const uint64_t all = (uint64_t)n_sel << a.page_bits;
    // a token of each sequence at least; ragged batches have fewer tokens than n_seq * max_new
    const uint64_t tokens = a.n_tok > a.n_seq ? a.n_tok : a.n_seq;
    p.few_chunk = chunk_of(a, all, tokens * a.n_kv, kBlocksWanted, 256);
    p.few_split = (uint32_t)((all + p.few_chunk - 1) / p.few_chunk);
    p.few_cap = (uint32_t)row_most;
    p.keys = take((size_t)a.n_tok * a.n_kv * a.max_pages * sizeof(uint32_t));
  } else {
    p.few = true;
    p.few_rows = row_most > 16 ? 32 : 16;
    p.many = row_most > kRowsFew;
    p.few_chunk = chunk_of(a, a.max_len, pairs, kBlocksWanted, 256);
    p.few_split = (a.max_len + p.few_chunk - 1) / p.few_chunk;
    p.few_cap = (uint32_t)(row_most < kRowsFew ? row_most : kRowsFew);
    if (p.many) {
      const uint64_t row_tiles = (row_most + kManyRows - 1) / kManyRows;
      p.many_chunk = chunk_of(a, a.max_len, pairs * row_tiles, 512, 512);
      p.many_split = (a.max_len + p.many_chunk - 1) / p.many_chunk;
    }
  }
  if (p.few_split > 1) p.o = take((size_t)p.few_split * pairs * p.few_cap * a.dim * sizeof(float));
  if (p.few_split > 1 || weights) p.ml = take((size_t)p.few_split * pairs * p.few_cap * sizeof(float2));
  if (p.many && p.many_split > 1) {
    p.many_o = take((size_t)p.many_split * pairs * row_most * a.dim * sizeof(float));
    p.many_ml = take((size_t)p.many_split * pairs * row_most * sizeof(float2));
  }
  if (weights && !p.many) {
    p.score_len = (uint32_t)up(a.max_len, 32);
    p.scores = take(pairs * p.few_cap * p.score_len * sizeof(float));
  }
  if (weights && p.many) p.lse = take((size_t)a.n_tok * a.n_q * sizeof(float));
  p.bytes = at;
  return p;
}

template <typename M, int D>
hipError_t attend(const KvArgs& a, const KvRows& q, const Plan& plan, float scale, bool weights, float decay,
                  uint32_t n_sel, const int32_t* sel, void* out, float* lse, char* ws, hipStream_t st) {
  Attn p = {};
  p.a = a;
  p.q = q;
  p.scale2 = scale * kLog2e;
  p.out = out;
  p.lse = weights && plan.many && !lse ? (float*)(ws + plan.lse) : lse;
  p.sel = sel;
  p.n_sel = n_sel;
  const uint32_t row_most = a.max_new * a.group;
  const auto launch = [&](auto kernel, dim3 grid, auto... more) {
    hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, st, p, more...);
  };
  const auto join = [&](uint32_t rows) {
    const uint32_t per = 4 * kBlock / D;
    launch(kv_join_kernel<M, D>, dim3((rows + per - 1) / per, a.n_kv, a.n_seq));
  };
  p.part_o = (float*)(ws + plan.o);
  p.part_ml = (float2*)(ws + plan.ml);
  p.n_split = plan.few_split;
  p.chunk = plan.few_chunk;
  p.row_cap = plan.few_cap;
  p.rows_from = 0;
  p.rows_to = plan.few_rows;
  if (n_sel) {
    const dim3 grid(plan.few_split * a.max_new * ((a.group + plan.few_rows - 1) / plan.few_rows), a.n_kv, a.n_seq);
    if (plan.few_rows == 16) launch(kv_few_kernel<M, D, 1, true, false>, grid);
    else launch(kv_few_kernel<M, D, 2, true, false>, grid);
    if (plan.few_split > 1) join(row_most);
    return hipGetLastError();
  }
  const dim3 grid(plan.few_split, a.n_kv, a.n_seq);
  const bool scores = weights && !plan.many;
  if (scores) {
    p.scores = (float*)(ws + plan.scores);
    p.score_len = plan.score_len;
    if (plan.few_rows == 16) launch(kv_few_kernel<M, D, 1, false, true>, grid);
    else launch(kv_few_kernel<M, D, 2, false, true>, grid);
  } else {
    if (plan.few_rows == 16) launch(kv_few_kernel<M, D, 1, false, false>, grid);
    else launch(kv_few_kernel<M, D, 2, false, false>, grid);
  }
  if (plan.few_split > 1) join(plan.few_cap);
  if (scores) launch(kv_weight_few_kernel, dim3((a.max_len + 4 * kBlock - 1) / (4 * kBlock), a.n_kv, a.n_seq), decay);
  if (plan.many) {
    p.part_o = (float*)(ws + plan.many_o);
    p.part_ml = (float2*)(ws + plan.many_ml);
    p.n_split = plan.many_split;
    p.chunk = plan.many_chunk;
    p.row_cap = row_most;
    p.rows_from = kRowsFew;
    p.rows_to = row_most;
    launch(kv_many_kernel<M, D>, dim3(a.n_kv * plan.many_split, (row_most + kManyRows - 1) / kManyRows, a.n_seq));
    if (plan.many_split > 1) join(row_most);
    if (weights) launch(kv_weight_many_kernel<M, D>, dim3((a.max_len + kBlock / 2 - 1) / (kBlock / 2), a.n_kv, a.n_seq),
                        decay);
  }
  return hipGetLastError();
}

}  // namespace

size_t kv_attend_bytes(const KvArgs& a, bool weights, uint32_t n_sel) { return plan_of(a, weights, n_sel).bytes; }

// Whether the launches of a call fit the device's counts of blocks (2^32 threads, 65,535 in y and z).
bool kv_attend_fits(const KvArgs& a, uint32_t n_sel) {
  const Plan p = plan_of(a, false, n_sel);
  const uint64_t rows = (uint64_t)a.max_new * a.group, most = (1ull << 24) - 1;
  if (rows / (4 * kBlock / a.dim) >= most) return false;
  if (n_sel) {
    const uint64_t tiles = (a.group + p.few_rows - 1) / p.few_rows, scored = (a.max_len >> a.page_bits) / 64 + 1;
    return p.few_split * tiles * a.max_new <= most && scored * a.max_new <= most;
  }
  return (uint64_t)a.n_kv * p.many_split <= most && (rows + kManyRows - 1) / kManyRows <= 65535;
}

hipError_t launch_kv_choose(const KvArgs& a, const KvRows& q, uint32_t n_sel, uint32_t first, uint32_t last,
                            uint32_t* keys, int32_t* sel, hipStream_t st);

hipError_t launch_kv_attend(const KvArgs& a, const KvRows& q, float scale, bool weights, float decay,
                            uint32_t n_sel, uint32_t first, uint32_t last, void* out, float* lse, int32_t* sel,
                            void* ws, hipStream_t st) {
  const Plan plan = plan_of(a, weights, n_sel);
  if (n_sel) {
    const hipError_t rc = launch_kv_choose(a, q, n_sel, first, last, (uint32_t*)((char*)ws + plan.keys), sel, st);
    if (rc != hipSuccess) return rc;
  }
  const auto run = [&](auto m, auto d) {
    return attend<decltype(m), decltype(d)::value>(a, q, plan, scale, weights, decay, n_sel, sel, out, lse, (char*)ws,
                                                   st);
  };
  const auto typed = [&](auto d) { return a.dtype == UNISON_KV_BF16 ? run(Bf16{}, d) : run(Fp16{}, d); };
  return a.dim == 64 ? typed(std::integral_constant<int, 64>{})
         : a.dim == 128 ? typed(std::integral_constant<int, 128>{})
                        : typed(std::integral_constant<int, 256>{});
}

}  // namespace unison
