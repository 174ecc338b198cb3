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
// In fp16 a p below 2^-25 would be rounded to 0, and thousands of weak entries with it that the sum counts.
// Scores are therefore taken against the maximum less kLift there: a row's largest p lies in 2^7 .. 2^15
// (the type ends at 2^16), and what is rounded away lies under 2^-32 of it.
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
  static constexpr float kLift = 0.0f;  // the exponents of 32 bits
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
  static constexpr float kLift = 7.0f;
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
constexpr uint32_t kManyKeys = 64;
// The many-rows kernel: wavefronts of a block, 32 rows each, and tiles of 64 entries in LDS.
constexpr uint32_t many_waves(uint32_t dim) { return dim <= 128 ? 8 : 4; }
constexpr uint32_t many_rows(uint32_t dim) { return 32 * many_waves(dim); }

// Bytes of scores that a few-rows block keeps in LDS and writes at its end, in one run (64 sequences of 3,300
// to 16,384 entries, 32 query heads: 573 us, written as they come 584).
constexpr size_t kScoresLds = 40960;
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
  // Partial results of a split of the entries (part_row)
  float* part_o;        // [..][dim], times the exponential of the maximum
  float2* part_ml;      // maximum (power of two, less kLift) and sum
  float* scores;        // of the dense few-rows kernel (score_at), or null
  uint32_t n_split, chunk, row_cap, score_len, score_lds;
  float* part_w;        // weights' sums of a split of the rows, [w_split][n_seq][n_kv][w_len]
  uint32_t w_split, w_rows, w_len;
  uint32_t rows_from, rows_to;  // rows of a sequence that this launch serves: rows_from < n * group <= rows_to
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float or_zero(float m) { return m == -kInf ? 0.0f : m; }

// Where the partial results of row r of (sequence, kv head) lie: row_cap rows of every pair, or, where
// sequences may have many, the tokens' own rows (row_cap 0).
__device__ __forceinline__ size_t part_row(const Attn& p, uint32_t split, uint32_t s, uint32_t h, int32_t t0, uint32_t r) {
  if (p.row_cap) return (((size_t)split * p.a.n_seq + s) * p.a.n_kv + h) * p.row_cap + r;
  return ((size_t)split * p.a.n_tok + (uint32_t)t0 + r / p.a.group) * p.a.n_q + h * p.a.group + r % p.a.group;
}

// Scores of row r and 32 entries, those 8 g + 4 x to + 3 of them in word g: rows side by side, so that the
// lanes of a store write runs of 64 bytes a row.
__device__ __forceinline__ f32x4* score_at(const Attn& p, uint32_t s, uint32_t h, uint32_t group32, uint32_t x,
                                           uint32_t r) {
  const size_t unit = (size_t)s * p.a.n_kv + h;
  return (f32x4*)p.scores + (((unit * (p.score_len / 32) + group32) * 2 + x) * p.row_cap + r) * 4;
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
// bound by HBM; the wavefronts of a block take runs of 64 entries in turn, straight from memory into
// the matrix operands, and join their maxima, sums and products in LDS at the end.  64 entries of a
// dimension are a line of V (of 128 bytes): with 32 a wavefront, two of them fetched every line.  With
// SPARSE a block serves one token and reads the pages of its choice instead of all.
// 64 sequences of 9,856 entries, 8 kv heads of 128, one token each: 450 us, 5.7 TB/s (a plain read of as many
// scattered pages of 16 KiB reaches 6.1); ragged ones of the same sum 460 to 500.  The scores for the weights
// cost 80 us more.
template <typename M, int D, int NT, bool SPARSE, bool SCORES>
__global__ __launch_bounds__(kBlock, NT * D <= 256 ? 2 : 1) void kv_few_kernel(Attn p) {
  typedef typename M::t T;
  typedef typename M::v8 v8;
  // H groups of 32 entries an iteration; wide heads or two row tiles leave registers for one, two in a row
  constexpr int KS = D / 32, DT = D / 16, H = NT * D > 128 ? 1 : 2;
  __shared__ int32_t pg[kPagesLds + 4];
  __shared__ int32_t eb[SPARSE ? kPagesLds + 4 : 1];
  __shared__ f32x4 join[(kWaves / 2) * NT * DT * 64];
  __shared__ float2 join_ml[(kWaves / 2) * NT * 64];
  extern __shared__ f32x4 kept[];  // the chunk's scores until the end, where they fit
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x, lane = tid & 63u;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const uint32_t split = spread_piece(blockIdx.x % p.n_split, p.n_split);
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

  // a run of 64 may end past the chunk: up to three pages more, which are not there
  for (uint32_t i = tid; i < (p.chunk >> a.page_bits) + 4u; i += kBlock) {
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
  // keys: lane r of the left operand has entry 8 (r / 4) + r % 4 of a group, and 4 behind it
  const uint32_t k_of = 8u * (r16 >> 2);
  const auto load_k = [&](uint32_t i, v8 (&k)[H][2][KS]) {
    for (int y = 0; y < H; ++y) {
      const uint32_t e = i + 32u * y + k_of;
      int32_t page = pg[(e - start) >> a.page_bits];
      page = page < 0 ? 0 : page;
      const T* at = (const T*)a.k + (size_t)page * per_page + head + ((e & in_page) + (r16 & 3u)) * D + 8 * g4;
      for (int x = 0; x < 2; ++x)
        for (int c = 0; c < KS; ++c) k[y][x][c] = *(const v8*)(at + x * 4 * D + 32 * c);
    }
  };
  // the wavefront's groups: runs of 64 entries, every kWaves-th
  const auto after = [&](uint32_t i) {
    return H == 2 ? i + 64u * kWaves : ((i - start) & 32u) ? i + 64u * kWaves - 32u : i + 32u;
  };
  v8 k[H][2][KS];
  uint32_t i = start + 64u * wave;
  if (i < end) load_k(i, k);
  while (i < end) {
    // values: lane r has dimension r of each 16, entries 8 (lane / 16) to + 7 of a group
    v8 v[H][DT];
    int32_t vpage[H], mine[H];
    bool inside = true;
    for (int y = 0; y < H; ++y) {
      const uint32_t ev = i + 32u * y + 8u * g4, at_page = (ev - start) >> a.page_bits;
      vpage[y] = pg[at_page];
      // the entry of the lane's first value, and whether every row sees all of them
      mine[y] = SPARSE ? eb[at_page] + (int32_t)(ev & in_page) : (int32_t)ev;
      inside = inside && vpage[y] >= 0 && mine[y] + 8 <= seen_by_all;
      const T* at = (const T*)a.v + (size_t)(vpage[y] < 0 ? 0 : vpage[y]) * per_page + head + (size_t)r16 * a.page +
                    (ev & in_page);
      for (int t = 0; t < DT; ++t) v[y][t] = *(const v8*)(at + (size_t)t * 16 * a.page);
    }
    f32x4 sc[NT][H][2];
    for (int n = 0; n < NT; ++n)
      for (int y = 0; y < H; ++y)
        for (int x = 0; x < 2; ++x) {
          sc[n][y][x] = (f32x4)0.0f;
          for (int c = 0; c < KS; ++c) sc[n][y][x] = M::mma16(k[y][x][c], qf[n][c], sc[n][y][x]);
        }
    const uint32_t next_i = after(i);
    if (next_i < end) load_k(next_i, k);
    const bool whole = __builtin_amdgcn_ballot_w64(!inside) == 0ull;
    if (!whole)
      for (int y = 0; y < H; ++y)
        for (int x = 0; x < 8; ++x)  // what is not an entry may hold anything
          if (vpage[y] < 0 || mine[y] + x >= q.len)
            for (int t = 0; t < DT; ++t) v[y][t][x] = (T)0.0f;
    for (int n = 0; n < NT; ++n) {
      float z[H][8];
      float top = -kInf;
      for (int y = 0; y < H; ++y) {
        for (int x = 0; x < 8; ++x) z[y][x] = sc[n][y][x >> 2][x & 3] * p.scale2;
        if (!whole)
          for (int x = 0; x < 8; ++x)
            if (vpage[y] < 0 || mine[y] + x >= limit[n]) z[y][x] = -kInf;
        if (SCORES && r16 + 16u * n < rows) {
          const uint32_t at = (((i - start) >> 5) + y) * 2 * p.row_cap + r16 + 16u * n;
          f32x4* to = (p.score_lds ? kept : score_at(p, s, h, start >> 5, 0, 0)) + 4u * at + g4;
          to[0] = f32x4{z[y][0], z[y][1], z[y][2], z[y][3]};
          to[4u * p.row_cap] = f32x4{z[y][4], z[y][5], z[y][6], z[y][7]};
        }
        for (int x = 0; x < 8; ++x) top = fmaxf(top, z[y][x]);
      }
      if (__builtin_amdgcn_ballot_w64(top > m[n] + (kSlack + M::kLift))) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float next = fmaxf(m[n], top - M::kLift);
        const float f = exp2_fast(m[n] - or_zero(next));
        m[n] = next;
        l[n] *= f;
        for (int t = 0; t < DT; ++t) o[n][t] *= f;
      }
      const float base = or_zero(m[n]);
      for (int y = 0; y < H; ++y) {
        // p in two parts for the second product, what the inputs' type holds of it and of the rest, which leaves
        // 2^-16 of each term in bf16: the matrix cores have time for both here (the 64 sequences of kScoresLds:
        // 567 us either way; 30 rows of 256 dimensions 23.8 in place of 23.2)
        v8 pf, rest;
        for (int x = 0; x < 8; ++x) {
          const float e = exp2_fast(z[y][x] - base);
          l[n] += e;
          pf[x] = (T)e;
          rest[x] = (T)(e - (float)pf[x]);
        }
        for (int t = 0; t < DT; ++t) {
          o[n][t] = M::mma16(v[y][t], rest, o[n][t]);
          o[n][t] = M::mma16(v[y][t], pf, o[n][t]);
        }
      }
    }
    i = next_i;
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
  if (SCORES && p.score_lds && start < end) {  // everybody's scores are there: one run of memory
    f32x4* to = score_at(p, s, h, start >> 5, 0, 0);
    const uint32_t words = ((end - start + 63u) >> 6) * 16u * p.row_cap;
    // past the caches, which keys and values pass through (the 64 sequences of kScoresLds: 566 us, through them 573)
    for (uint32_t x = tid; x < words; x += kBlock) __builtin_nontemporal_store(kept[x], to + x);
  }
  if (wave) return;
  for (int n = 0; n < NT; ++n) {
    const uint32_t r = r16 + 16u * n;
    if (r >= rows) continue;
    const size_t part = part_row(p, split, s, h, q.t0, r0 + r);
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

// Joins the splits of a few- or many-rows launch: 1024 / dim rows a block, 4 dimensions a thread.  Bound by
// latency: 16 splits are asked for at once (4 us for 16 splits of 32 rows; one after the other 11 us).
template <typename M, int D>
__global__ __launch_bounds__(kBlock) void kv_join_kernel(Attn p) {
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z;
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group, r = blockIdx.x * (4 * kBlock / D) + threadIdx.x / (D / 4);
  if (r >= rows || (!p.sel && (rows <= p.rows_from || rows > p.rows_to))) return;
  const uint32_t d = 4 * (threadIdx.x % (D / 4));
  const int32_t limit = q.len - q.n + (int32_t)(r / a.group) + 1;  // splits behind it may not be written
  const uint32_t all = p.sel ? p.n_sel << a.page_bits : limit > 0 ? (uint32_t)limit : 0u;
  const uint32_t used = (all + p.chunk - 1) / p.chunk;
  float m = -kInf, l = 0.0f;
  f32x4 o = (f32x4)0.0f;
  constexpr uint32_t B = 16;  // splits' loads in flight
  for (uint32_t i0 = 0; i0 < used; i0 += B) {
    float2 y[B];
    f32x4 x[B];
    for (uint32_t i = 0; i < B; ++i) {
      y[i] = make_float2(-kInf, 0.0f);
      x[i] = (f32x4)0.0f;
      if (i0 + i >= used) continue;
      const size_t part = part_row(p, i0 + i, s, h, q.t0, r);
      y[i] = p.part_ml[part];
      x[i] = *(const f32x4*)(p.part_o + part * D + d);
    }
    float next = m;
    for (uint32_t i = 0; i < B; ++i) next = fmaxf(next, y[i].x);
    const float base = or_zero(next), f = exp2_fast(m - base);
    m = next;
    l *= f;
    o *= f;
    for (uint32_t i = 0; i < B; ++i) {
      const float g = exp2_fast(y[i].x - base);
      l += y[i].y * g;
      o += x[i] * g;
    }
  }
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  const size_t row = (size_t)(q.t0 + (int32_t)(r / a.group)) * a.n_q + h * a.group + r % a.group;
  const float x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  store4<M>((typename M::t*)p.out + row * D + d, x);
  if (p.lse && d == 0) p.lse[row] = l == 0.0f ? -kInf : (m + log2f(l)) * kLn2;
}

// weight = decay * weight + sum of p, from the scores that the few-rows kernel left: a thread per
// four entries.  Bound by memory: 26 us for 5 million entries of 4 rows each (120 MB, 4.6 TB/s).
__global__ __launch_bounds__(kBlock) void kv_weight_few_kernel(Attn p, float decay) {
  __shared__ float base[kRowsFew];
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group;
  const uint32_t piece = spread_piece(blockIdx.x, gridDim.x);
  if (rows == 0 || piece * 4 * kBlock >= (uint32_t)q.len) return;
  if (tid < rows) {
    const uint32_t used = ((uint32_t)q.len + p.chunk - 1) / p.chunk;
    float m = -kInf, l = 0.0f;
    for (uint32_t i0 = 0; i0 < used; i0 += 8) {
      float2 y[8];
      float next = m;
      for (uint32_t i = 0; i < 8; ++i) {
        y[i] = p.part_ml[part_row(p, i0 + i < used ? i0 + i : i0, s, h, q.t0, tid)];
        if (i0 + i >= used) y[i] = make_float2(-kInf, 0.0f);
        next = fmaxf(next, y[i].x);
      }
      l *= exp2_fast(m - or_zero(next));
      m = next;
      for (uint32_t i = 0; i < 8; ++i) l += y[i].y * exp2_fast(y[i].x - or_zero(m));
    }
    base[tid] = l == 0.0f ? kInf : m + log2f(l);
  }
  __syncthreads();
  const uint32_t e = 4 * (piece * kBlock + tid);
  if (e >= (uint32_t)q.len) return;
  const int32_t page = kv_page(a, q, (int32_t)(e >> a.page_bits));
  if (page < 0) return;
  const f32x4* z = score_at(p, s, h, e >> 5, (e >> 2) & 1u, 0) + ((e >> 3) & 3u);
  f32x4 sum = (f32x4)0.0f;
  for (uint32_t r = 0; r < rows; ++r) {
    const f32x4 x = z[4u * r];
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

// Waits for the wavefront's loads, those into LDS among them (vmcnt(0)).
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// The order in which rows of a left operand hold entries: bits 2 and 3 change places.
__device__ __forceinline__ uint32_t swap23(uint32_t x) {
  return (x & ~12u) | ((x & 4u) << 1) | ((x & 8u) >> 1);
}

// Where rows of CH 16-byte pieces lie in LDS, so that 16 rows' pieces c, which a read takes at once, lie in
// different banks (64 of them: 256 bytes): a kibibyte (64 pieces, what a wavefront loads at once) takes kRun
// bytes, the 64 more turning the next one's banks by a quarter, and inside it a row's pieces are xored with two
// bits of the row.  The address of piece c is then the lane's for c mod 4 and a constant.
constexpr uint32_t kRun = 1024 + 64;
template <uint32_t CH>
__device__ __forceinline__ uint32_t turn(uint32_t row) {
  return CH == 8 ? (row >> 1) & 3u : CH == 16 ? row & 3u : (row & 1u) | ((row >> 2) & 2u);
}
template <uint32_t CH>
__device__ __forceinline__ uint32_t piece_at(uint32_t row, uint32_t c) {
  const uint32_t at = row * CH;  // in pieces
  return at / 64u * kRun + at % 64u * 16u + (c ^ turn<CH>(row)) * 16u;
}

// A row of the queries, negated where the scale is negative: the kernels below scale by its magnitude.
template <typename v8>
__device__ __forceinline__ v8 signed_row(v8 x, bool negate) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  const u4 y = __builtin_bit_cast(u4, x) ^ (negate ? 0x80008000u : 0u);
  return __builtin_bit_cast(v8, y);
}
// A scale of 0 would make NaN of the scores that a mask sets to -inf.
__device__ __forceinline__ float magnitude(float scale2) { return fmaxf(fabsf(scale2), 1e-35f); }

// Attention of 128 or 256 rows over a chunk of entries, 32 rows a wavefront, 64 entries at a time from
// double-buffered LDS: a turn's new tokens over their session.  Bound by the matrix cores and, nearly as
// much, by the exponentials (at half the rate of an addition) and the additions and roundings beside them, so the
// two are put side by side: while the exponentials of a group of 32 entries run, the matrix cores do
// the second product of the group before and the first product of the group behind.
// 4 sequences of up to 2,000 tokens over up to 12,001 entries, 32 query and 8 kv heads of 128 (928 GFLOP seen):
// 900 us, 1.03 PFLOP/s; a large library product reaches 1.38.  Its matrix cores are busy 54 % of the time, its
// vector units 41 %.  Four tiles in LDS in place of two, their loads awaited by number, took 2 to 5 % longer.
template <typename M, int D>
__global__ __launch_bounds__(64 * many_waves(D), D <= 128 ? 2 : 1) void kv_many_kernel(Attn p) {
  typedef typename M::t T;
  typedef typename M::v8 v8;
  constexpr uint32_t CH = D / 8;
  constexpr uint32_t WAVES = many_waves(D), ROWS = many_rows(D);
  constexpr int KS = D / 16, DT = D / 32, NK = CH / WAVES, NV = D / 8 / WAVES;
  // an array for each buffer: the compiler waits for every load into an array before it reads the array
  constexpr uint32_t KB = kManyKeys * D * 2 / 1024 * kRun, VB = D * 128 / 1024 * kRun;
  __shared__ alignas(16) char kt0[KB], kt1[KB], vt0[VB], vt1[VB];
  __shared__ int32_t pg[kPagesLds];
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.x % a.n_kv, split = blockIdx.x / a.n_kv, s = blockIdx.z, tid = threadIdx.x;
  const uint32_t lane = tid & 63u, half = lane >> 5, r32 = lane & 31u;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group;
  const uint32_t tile = gridDim.y - 1u - blockIdx.y;  // the longest first
  if (rows <= p.rows_from || tile * ROWS >= rows) return;
  const int32_t old = q.len - q.n;
  const uint32_t r = tile * ROWS + 32u * wave + r32;
  const bool is = r < rows;
  const uint32_t j = (is ? r : 0u) / a.group, g = (is ? r : 0u) % a.group;
  const int32_t limit = is ? old + (int32_t)j + 1 : 0;
  // entries that some row of the block (of the wavefront) sees, and that all rows of the wavefront see
  const auto token = [&](uint32_t x) { return (int32_t)((x < rows ? x : rows - 1u) / a.group); };
  const int32_t block_end = old + token((tile + 1u) * ROWS - 1u) + 1;
  const uint32_t w0 = tile * ROWS + 32u * wave;
  const int32_t start = (int32_t)(split * p.chunk);
  if (split && start >= block_end) return;  // the join knows
  int32_t end = block_end < q.len ? block_end : q.len;
  if (end > 0 && (uint32_t)end > (uint32_t)start + p.chunk) end = start + (int32_t)p.chunk;
  const int32_t tiles = end > start ? (end - start + 63) >> 6 : 0;
  const int32_t wave_end = w0 < rows ? old + token(w0 + 31u) + 1 : 0;
  int32_t wave_tiles = (wave_end < end ? wave_end : end) - start;
  wave_tiles = wave_tiles > 0 ? (wave_tiles + 63) >> 6 : 0;
  const int32_t seen_by_all = old + token(w0) + 1;
  const float scale = magnitude(p.scale2);

  v8 qf[KS];
  {
    const T* row = (const T*)p.q.p + (size_t)(q.t0 + (int32_t)j) * p.q.tok + (h * a.group + g) * p.q.head;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      v8 x = signed_row(*(const v8*)(row + 16 * k + 8 * half), p.scale2 < 0.0f);
      if (!is) x = (v8)(T)0.0f;
      qf[k] = x;
    }
  }
  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = (f32x16)0.0f;
  float m = -kInf, l = 0.0f;

  const size_t head = (size_t)h * a.page * D, per_page = (size_t)a.n_kv * a.page * D;
  const uint32_t in_page = a.page - 1u;
  const bool wide = a.page >= kManyKeys;
  // The page ids of the next kPagesLds pages, from tile `ids_from` on (whole pages); a tile's are read a
  // tile ahead of their use.
  const uint32_t n_ids = end > start ? (uint32_t)(end - start + (int32_t)in_page) >> a.page_bits : 0u;
  const int32_t window = (int32_t)((kPagesLds << a.page_bits) / kManyKeys);
  int32_t ids_from = 0;
  const auto fill_ids = [&] {
    const uint32_t first_id = (uint32_t)ids_from * kManyKeys >> a.page_bits;
    for (uint32_t i = tid; i < kPagesLds; i += 64u * WAVES) {
      const uint32_t id = first_id + i;
      pg[i] = id < n_ids ? kv_page(a, q, (int32_t)(((uint32_t)start >> a.page_bits) + id)) : -1;
    }
    __syncthreads();
  };
  fill_ids();
  struct Pages {  // of a tile's four runs of 16 entries, x[0] of all where a page holds the tile
    int32_t x[4];
  };
  const auto ids_of = [&](int32_t t) __attribute__((always_inline)) {
    Pages to;
    const uint32_t e = (uint32_t)(t - ids_from) * kManyKeys;
    to.x[0] = pg[e >> a.page_bits];
    to.x[1] = to.x[2] = to.x[3] = to.x[0];
    if (!wide)
#pragma unroll
      for (int i = 1; i < 4; ++i) to.x[i] = pg[(e + 16u * i) >> a.page_bits];
    return to;
  };
  const auto uniform = [&](const Pages& from) __attribute__((always_inline)) {
    Pages to;
    to.x[0] = __builtin_amdgcn_readfirstlane(from.x[0]);
    to.x[1] = to.x[2] = to.x[3] = to.x[0];
    if (!wide)
#pragma unroll
      for (int i = 1; i < 4; ++i) to.x[i] = __builtin_amdgcn_readfirstlane(from.x[i]);
    return to;
  };
  const auto pick = [&](const Pages& from, uint32_t i) {
    const int32_t x = i & 1u ? from.x[1] : from.x[0], y = i & 1u ? from.x[3] : from.x[2];
    const int32_t z = i & 2u ? y : x;
    return z < 0 ? 0 : z;
  };
  // Where a lane's pieces of a tile lie in a page of 64 entries or more, which holds the whole tile: the rest
  // of their address is the same for all lanes.
  uint32_t k_off[NK], v_off[NV];
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const uint32_t c = (wave * NK + i) * 64u + lane, row = c / CH;
    k_off[i] = (swap23(row) * D + 8 * ((c % CH) ^ turn<CH>(row))) * 2u;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const uint32_t c = (wave * NV + i) * 64u + lane, d = c >> 3;
    v_off[i] = (d * a.page + 8 * ((c & 7u) ^ turn<8>(d))) * 2u;
  }
  const auto load_k = [&](int32_t t, const Pages& from, char* kt) __attribute__((always_inline)) {
    const uint32_t e = (uint32_t)(start + 64 * t);
    if (wide) {
      const char* at = (const char*)((const T*)a.k + (size_t)pick(from, 0) * per_page + head + (e & in_page) * D);
#pragma unroll
      for (int i = 0; i < NK; ++i) to_lds(at + k_off[i], kt + (wave * NK + i) * kRun);
      return;
    }
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const uint32_t at = (wave * NK + i) * 64u, c = at + lane, row = c / CH;
      const uint32_t key = swap23(row), part = (c % CH) ^ turn<CH>(row);
      to_lds((const T*)a.k + (size_t)pick(from, key >> 4) * per_page + head + ((e + key) & in_page) * D + 8 * part,
             kt + at / 64u * kRun);
    }
  };
  const auto load_v = [&](int32_t t, const Pages& from, char* vt) __attribute__((always_inline)) {
    const uint32_t e = (uint32_t)(start + 64 * t);
    if (wide) {
      const char* at = (const char*)((const T*)a.v + (size_t)pick(from, 0) * per_page + head + (e & in_page));
#pragma unroll
      for (int i = 0; i < NV; ++i) to_lds(at + v_off[i], vt + (wave * NV + i) * kRun);
      return;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t at = (wave * NV + i) * 64u, c = at + lane, d = c >> 3;
      const uint32_t part = (c & 7u) ^ turn<8>(d);
      to_lds((const T*)a.v + (size_t)pick(from, part >> 1) * per_page + head + (size_t)d * a.page +
                 ((e + 8 * part) & in_page), vt + at / 64u * kRun);
    }
  };
  const auto landed = [&] {
    wait_loads();
    __syncthreads();
  };
  // the lane's pieces of rows r32, by their number's second bit: the rest of the number is a constant offset
  uint32_t k_at[2], v_at[2];
#pragma unroll
  for (uint32_t k = 0; k < 2; ++k) {
    k_at[k] = piece_at<CH>(r32, 2 * k + half);
    v_at[k] = piece_at<8>(r32, 2 * k + half);
  }
  const auto k_piece = [&](const char* kb, int k, uint32_t group) __attribute__((always_inline)) {
    return *(const v8*)(kb + k_at[k & 1] + (k >> 1) * 64 + group * (32 * CH / 64) * kRun);
  };
  const auto v_piece = [&](const char* vb, int k, int dims) __attribute__((always_inline)) {
    return *(const v8*)(vb + v_at[k & 1] + (k >> 1) * 64 + dims * 4 * kRun);
  };

  v8 pend[2];  // the rounded p of the group before, whose second product is still to come
  pend[0] = pend[1] = (v8)(T)0.0f;
  f32x16 sc = (f32x16)0.0f;

  // One group of 32 entries, c = 0 or 1 of tile t, its scores in sc.  `vb` and `kb`: the buffers of the group
  // before's values (its pieces from 2 (1 - c) on) and of the group behind's keys (its rows from 32 (1 - c) on).
  const auto group = [&](auto c_, int32_t t, const Pages& pages, const char* vb,
                         const char* kb) __attribute__((always_inline)) {
    constexpr int c = decltype(c_)::value;
    const int32_t base = start + 64 * t + 32 * c;
    const bool there = (c ? pages.x[2] | pages.x[3] : pages.x[0] | pages.x[1]) >= 0;
    if (!there || base + 32 > seen_by_all)
      // register i of the lane is entry 16 (i / 8) + 8 half + i % 8 of the group
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (pages.x[2 * c + (i >> 3)] < 0 || base + 16 * (i >> 3) + 8 * (int32_t)half + (i & 7) >= limit)
          sc[i] = -kInf;
    float top = sc[0];
    for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
    top *= scale;
    float f = 1.0f;
    const bool moved = __builtin_amdgcn_ballot_w64(top > m + (kSlack + M::kLift)) != 0ull;
    if (moved) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = fmaxf(m, top - M::kLift);
      f = exp2_fast(m - or_zero(next));
      m = next;
      l *= f;
    }
    const float sub = -or_zero(m);
    // A product, a later product's read and an element in turn.  The order is held as written: left alone, the
    // exponentials sink behind the next branch and each read goes next to its product.
    static_assert(KS == 2 * DT, "as many products of each kind");
    constexpr int N = 2 * KS, AHEAD = 6;
    v8 pf[2], f_[N];
    f32x16 behind = (f32x16)0.0f;
    float e_[16], l0 = 0.0f, l1 = 0.0f;
    const auto read = [&](int u) __attribute__((always_inline)) {
      const int i = u >> 1;
      f_[u] = u & 1 ? k_piece(kb, i, 1 - c) : v_piece(vb, 2 * (1 - c) + i / DT, i % DT);
    };
    const auto rest = [&](int x) __attribute__((always_inline)) {
      if (x & 1) l1 += e_[x]; else l0 += e_[x];
      // rounded for the second product only, half a step of each term; in two parts, as the few rows' p is, it would
      // take half as many products again
      pf[x >> 3][x & 7] = (T)e_[x];
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) read(u);
    // Ahead of the SIMD's other wavefront while there are products, which then does what has none beside it
    // (two prompts of 8,000 tokens: 1,040 us without, 1,007 with).
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      __builtin_amdgcn_sched_barrier(0);
      const int i = u >> 1;
      if (u & 1) behind = M::mma32(f_[u], qf[i], behind);
      else o[i % DT] = M::mma32(f_[u], pend[i / DT], o[i % DT]);
      if (u + AHEAD < N) read(u + AHEAD);
#pragma unroll
      for (int x = u * 16 / N; x < (u + 1) * 16 / N; ++x) {
        e_[x] = exp2_fast(fmaf(sc[x], scale, sub));
        if (x) rest(x - 1);  // the result of an exponential is not there at once
      }
    }
    __builtin_amdgcn_s_setprio(0);
    rest(15);
    l0 += l1;
    asm volatile("" : "+v"(pf[0]), "+v"(pf[1]), "+v"(l0));
    __builtin_amdgcn_sched_barrier(0);
    l += l0;
    if (moved)
#pragma unroll
      for (int t2 = 0; t2 < DT; ++t2) o[t2] *= f;
    pend[0] = pf[0];
    pend[1] = pf[1];
    sc = behind;
  };
  const std::integral_constant<int, 0> c0;
  const std::integral_constant<int, 1> c1;

  Pages now = uniform(ids_of(0)), next = uniform(ids_of(1)), then = ids_of(2);
  if (tiles) {
    load_k(0, now, kt0);
    load_v(0, now, vt0);
    if (tiles > 1) load_k(1, next, kt1);
    // in the place of the values before the first tile's, which the first group takes: zeros times zero
    for (uint32_t i = tid; i < VB / 16u; i += 64u * WAVES) ((v8*)vt1)[i] = (v8)(T)0.0f;
    landed();
#pragma unroll
    for (int k = 0; k < KS; ++k) sc = M::mma32(k_piece(kt0, k, 0), qf[k], sc);
  }
  // Tile t: its first group while V of tile t - 1 and K of tile t are there; then everybody is done with
  // both, and V of tile t + 1 and K of tile t + 2 take their places.
  const auto body = [&](auto odd_, int32_t t) __attribute__((always_inline)) {
    constexpr bool odd = decltype(odd_)::value;
    char *const k_now = odd ? kt1 : kt0, *const k_next = odd ? kt0 : kt1;
    char *const v_now = odd ? vt1 : vt0, *const v_before = odd ? vt0 : vt1;
    if (t < wave_tiles) group(c0, t, now, v_before, k_now);
    landed();
    if (t + 1 < tiles) load_v(t + 1, next, v_before);
    const Pages behind = uniform(then);
    if (t + 2 < tiles) load_k(t + 2, behind, k_now);
    if (t + 3 - ids_from >= window) {  // nobody reads the old ids any more: the last are in registers
      ids_from = (t + 3) & ~3;         // pages of 256 hold four tiles
      fill_ids();
    }
    then = ids_of(t + 3);
    const int32_t base = start + 64 * t;
    if ((now.x[0] | now.x[1] | now.x[2] | now.x[3]) < 0 || base + 64 > q.len) {
      for (uint32_t i = tid; i < D * 8u; i += 64u * WAVES) {  // what is not an entry may hold anything
        const uint32_t part = (i & 7u) ^ turn<8>(i >> 3);
        const int32_t run = part & 4u ? (part & 2u ? now.x[3] : now.x[2]) : (part & 2u ? now.x[1] : now.x[0]);
        v8 x = *(const v8*)(v_now + i / 64u * kRun + i % 64u * 16u);
        for (int y = 0; y < 8; ++y)
          if (run < 0 || base + (int32_t)(8 * part) + y >= q.len) x[y] = (T)0.0f;
        *(v8*)(v_now + i / 64u * kRun + i % 64u * 16u) = x;
      }
      __syncthreads();
    }
    if (t < wave_tiles) {
      group(c1, t, now, v_now, k_next);
      if (t + 1 == wave_tiles)
#pragma unroll
        for (int u = 0; u < 2 * DT; ++u)
          o[u % DT] = M::mma32(v_piece(v_now, 2 + u / DT, u % DT), pend[u / DT], o[u % DT]);
    }
    now = next;
    next = behind;
  };
  for (int32_t t = 0; t < tiles; t += 2) {
    body(std::false_type{}, t);
    if (t + 1 < tiles) body(std::true_type{}, t + 1);
  }
  l += __shfl_xor(l, 32);
  if (!is) return;
  const size_t part = part_row(p, split, s, h, q.t0, r);
  if (p.n_split > 1) {
    if (half == 0) p.part_ml[part] = make_float2(m, l);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *(f32x4*)(p.part_o + part * D + 32 * t + 8 * c + 4 * half) =
            f32x4{o[t][4 * c], o[t][4 * c + 1], o[t][4 * c + 2], o[t][4 * c + 3]};
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  const size_t row = (size_t)(q.t0 + (int32_t)j) * a.n_q + h * a.group + g;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float x[4] = {o[t][4 * c] * inv, o[t][4 * c + 1] * inv, o[t][4 * c + 2] * inv, o[t][4 * c + 3] * inv};
      store4<M>((T*)p.out + row * D + 32 * t + 8 * c + 4 * half, x);
    }
  if (p.lse && half == 0) p.lse[row] = l == 0.0f ? -kInf : (m + log2f(l)) * kLn2;
}

// weight = decay * weight + the sum of p over a sequence's rows, which another product of the keys with
// the queries gives, the entries in the lanes now and the rows in their registers: 64 entries a wavefront
// with their keys in registers, 64 rows at a time from double-buffered LDS.  As above, the exponentials of
// 32 rows run beside the products of the next 32; the two take about the same time.  565 us for the sequences
// named there (464 GFLOP; matrix cores 44 % busy, vector units 62 %).
constexpr uint32_t kWeightKeys = 256, kWeightRows = 64;

template <typename M, int D>
__global__ __launch_bounds__(kBlock, D <= 128 ? 2 : 1) void kv_weight_many_kernel(Attn p, float decay) {
  typedef typename M::t T;
  typedef typename M::v8 v8;
  constexpr uint32_t CH = D / 8, QB = kWeightRows * D * 2 / 1024 * kRun;
  constexpr int KS = D / 16, NQ = CH / 4;
  __shared__ alignas(16) char qt0[QB], qt1[QB];
  __shared__ f32x4 base[4][kWeightRows / 4];  // minus the rows' log sums, in powers of two, of tile t in t % 4
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x, lane = tid & 63u, half = lane >> 5, c32 = lane & 31u;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const KvSeq q = kv_seq(a, s);
  const uint32_t rows = (uint32_t)q.n * a.group;
  const uint32_t split = blockIdx.x % p.w_split, piece_of = spread_piece(blockIdx.x / p.w_split, gridDim.x / p.w_split);
  const int32_t first = (int32_t)(piece_of * kWeightKeys), mine = first + (int32_t)(64u * wave);
  if (rows == 0 || first >= q.len) return;
  const int32_t old = q.len - q.n;
  const float scale = magnitude(p.scale2);
  const bool negate = p.scale2 < 0.0f;
  v8 kf[2][KS];
  int32_t page[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int32_t e = mine + 32 * y + (int32_t)c32;
    page[y] = e < q.len ? kv_page(a, q, e >> a.page_bits) : -1;
    const T* key = (const T*)a.k + kv_base(a, page[y] < 0 ? 0 : page[y], h) + (size_t)((uint32_t)e & (a.page - 1u)) * D;
#pragma unroll
    for (int k = 0; k < KS; ++k) kf[y][k] = signed_row(*(const v8*)(key + 16 * k + 8 * half), negate);
  }
  // the split's rows; those of tokens before entry `first` see nothing here
  uint32_t from = first > old ? ((uint32_t)(first - old) * a.group) & ~(kWeightRows - 1u) : 0u;
  from = from > split * p.w_rows ? from : split * p.w_rows;
  const uint32_t to = rows < (split + 1u) * p.w_rows ? rows : (split + 1u) * p.w_rows;
  const int32_t tiles = from < to ? (int32_t)((to - from + kWeightRows - 1u) / kWeightRows) : 0;
  // the first tile with a row that sees an entry of the wavefront
  const uint32_t seen_from = mine > old ? (uint32_t)(mine - old) * a.group : 0u;
  const int32_t begin = seen_from > from ? (int32_t)((seen_from - from) / kWeightRows) : 0;
  // token and head of the lane's rows of the next tile, moved on without dividing
  const uint32_t dj = kWeightRows / a.group, dg = kWeightRows % a.group;
  uint32_t rj[NQ], rg[NQ], part[NQ], bj = 0, bg = 0;
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const uint32_t c = (wave * NQ + i) * 64u + lane, row = c / CH;
    rj[i] = (from + row) / a.group;
    rg[i] = (from + row) % a.group;
    part[i] = 8 * ((c % CH) ^ turn<CH>(row));
  }
  if (tid < kWeightRows) {
    bj = (from + tid) / a.group;
    bg = (from + tid) % a.group;
  }
  const auto on = [&](uint32_t& j, uint32_t& g) __attribute__((always_inline)) {
    j += dj;
    g += dg;
    if (g >= a.group) {
      g -= a.group;
      ++j;
    }
  };
  const auto load = [&](char* qt) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const uint32_t j = rj[i] < (uint32_t)q.n ? rj[i] : (uint32_t)q.n - 1u;  // a row behind the last counts nothing
      to_lds((const T*)p.q.p + (size_t)(q.t0 + (int32_t)j) * p.q.tok + (h * a.group + rg[i]) * p.q.head + part[i],
             qt + (wave * NQ + i) * kRun);
      on(rj[i], rg[i]);
    }
  };
  float b = 0.0f;
  const auto load_base = [&]() __attribute__((always_inline)) {
    if (tid < kWeightRows) {
      b = bj < (uint32_t)q.n ? p.lse[(size_t)(q.t0 + (int32_t)bj) * a.n_q + h * a.group + bg] : kInf;
      on(bj, bg);
    }
  };
  const auto put_base = [&](int32_t t) __attribute__((always_inline)) {  // a row that sees nothing has -inf
    if (tid < kWeightRows) ((float*)base[t & 3])[tid] = b == -kInf ? -kInf : b * -kLog2e;
  };
  uint32_t q_at[2];
  q_at[0] = piece_at<CH>(c32, half);
  q_at[1] = piece_at<CH>(c32, 2 + half);
  const auto piece = [&](const char* qt, int k, uint32_t x) __attribute__((always_inline)) {
    return *(const v8*)(qt + q_at[k & 1] + (k >> 1) * 64 + x * (32 * CH / 64) * kRun);
  };
  float sum[2] = {0.0f, 0.0f};
  f32x16 sc[2];
  sc[0] = sc[1] = (f32x16)0.0f;
  // Rows 32 x to 32 x + 31 of tile t, their scores in sc; the next rows' from `qt`, rows 32 (1 - x) on.
  const auto rows32 = [&](auto x_, auto whole_, int32_t t, const char* qt) __attribute__((always_inline)) {
    constexpr int x = decltype(x_)::value;
    constexpr bool whole = decltype(whole_)::value;
    constexpr int N = 2 * KS, AHEAD = 3, PER = 32 / N;
    f32x4 n[4];  // register i is row 8 (i / 4) + 4 half + i % 4 of the 32
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) n[i] = base[t & 3][8 * x + 2 * i + half];
    // entry e is seen from row (e - old) * group on
    int32_t behind[2];
#pragma unroll
    for (int y = 0; y < 2; ++y)
      behind[y] = (int32_t)(from + (uint32_t)t * kWeightRows + 32u * x + 4u * half) -
                  (mine + 32 * y + (int32_t)c32 > old ? (mine + 32 * y + (int32_t)c32 - old) * (int32_t)a.group : 0);
    f32x16 nx[2];
    nx[0] = nx[1] = (f32x16)0.0f;
    v8 f_[KS];
    float e_[32], part[2] = {0.0f, 0.0f};  // a tile's sums first: thousands of rows added one by one would lose bits
    const auto add = [&](int z) __attribute__((always_inline)) {
      const int y = z >> 4, i = z & 15;
      part[y] += whole || behind[y] + 8 * (i >> 2) + (i & 3) >= 0 ? e_[z] : 0.0f;
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) f_[k] = piece(qt, k, 1 - x);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      __builtin_amdgcn_sched_barrier(0);
      nx[u & 1] = M::mma32(f_[u >> 1], kf[u & 1][u >> 1], nx[u & 1]);
      if (!(u & 1) && (u >> 1) + AHEAD < KS) f_[(u >> 1) + AHEAD] = piece(qt, (u >> 1) + AHEAD, 1 - x);
#pragma unroll
      for (int z = u * PER; z < (u + 1) * PER; ++z) {
        e_[z] = exp2_fast(fmaf(sc[z >> 4][z & 15], scale, n[(z & 15) >> 2][z & 3]));
        asm volatile("" : "+v"(e_[z]));  // here, not in pairs behind the products
        if (z) add(z - 1);
      }
    }
    add(31);
    asm volatile("" : "+v"(part[0]), "+v"(part[1]));
    __builtin_amdgcn_sched_barrier(0);
    sum[0] += part[0];
    sum[1] += part[1];
    sc[0] = nx[0];
    sc[1] = nx[1];
  };
  const auto step = [&](auto x_, int32_t t, const char* qt) __attribute__((always_inline)) {
    const uint32_t r = from + (uint32_t)t * kWeightRows + 32u * decltype(x_)::value;
    if (old + (int32_t)(r / a.group) + 1 >= mine + 64) rows32(x_, std::true_type{}, t, qt);
    else rows32(x_, std::false_type{}, t, qt);
  };
  const std::integral_constant<int, 0> x0;
  const std::integral_constant<int, 1> x1;
  if (tiles) {
    load(qt0);
    load_base();
    put_base(0);
    if (tiles > 1) {
      load(qt1);
      load_base();
      put_base(1);
    }
    wait_loads();
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2 * KS; ++u) sc[u & 1] = M::mma32(piece(qt0, u >> 1, 0), kf[u & 1][u >> 1], sc[u & 1]);
  }
  // Tile t: its first 32 rows while its second 32 are there; then everybody is done with its queries, and tile
  // t + 2 takes their place.  Scores are made one step ahead, so a wavefront begins a tile early.
  const auto body = [&](auto odd_, int32_t t) __attribute__((always_inline)) {
    constexpr bool odd = decltype(odd_)::value;
    char *const qt = odd ? qt1 : qt0, *const qt_next = odd ? qt0 : qt1;
    if (t + 1 >= begin) step(x0, t, qt);
    wait_loads();
    __syncthreads();
    if (t + 2 < tiles) {
      load(qt);
      load_base();
    }
    if (t + 1 >= begin) step(x1, t, qt_next);
    if (t + 2 < tiles) put_base(t + 2);
  };
  for (int32_t t = 0; t < tiles; t += 2) {
    body(std::false_type{}, t);
    if (t + 1 < tiles) body(std::true_type{}, t + 1);
  }
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    sum[y] += __shfl_xor(sum[y], 32);
    if (page[y] < 0 || half) continue;
    const uint32_t e = (uint32_t)mine + 32u * y + c32;
    if (p.w_split > 1) {
      p.part_w[(((size_t)split * a.n_seq + s) * a.n_kv + h) * p.w_len + e] = sum[y];
      continue;
    }
    float* w = a.weight + kv_word(a, page[y], h) + (e & (a.page - 1u));
    *w = fmaf(decay, *w, sum[y]);
  }
}

// weight = decay * weight + the sums of the splits of the rows, in their order.
__global__ __launch_bounds__(kBlock) void kv_weight_join_kernel(Attn p, float decay) {
  const KvArgs& a = p.a;
  const uint32_t h = blockIdx.y, s = blockIdx.z, e = blockIdx.x * kBlock + threadIdx.x;
  const KvSeq q = kv_seq(a, s);
  if (q.n <= 0 || e >= (uint32_t)q.len) return;
  const int32_t page = kv_page(a, q, (int32_t)(e >> a.page_bits));
  if (page < 0) return;
  float sum = 0.0f;
#pragma unroll 8
  for (uint32_t i = 0; i < p.w_split; ++i) sum += p.part_w[(((size_t)i * a.n_seq + s) * a.n_kv + h) * p.w_len + e];
  float* w = a.weight + kv_word(a, page, h) + (e & (a.page - 1u));
  *w = fmaf(decay, *w, sum);
}

// ------------------------------------------------------------------ plans

size_t up(size_t x, size_t to) { return (x + to - 1) / to * to; }

// How a call is split and where its workspace lies.
struct Plan {
  uint32_t few_rows;       // rows of a tile of the few-rows kernel: 16 or 32
  uint32_t few_most;       // rows of a pair up to which that kernel serves it; 0: none
  bool many;               // whether the many-rows kernel runs, for sequences of more rows
  uint32_t few_chunk, few_split, few_cap, many_chunk, many_split, many_cap, score_len;
  uint32_t w_split, w_rows, w_len;
  size_t o, ml, many_o, many_ml, scores, lse, part_w, keys, bytes;
};

// Blocks of a few-rows launch, 16 a compute unit: enough loads under way and even ends (64 ragged sequences as
// above: 613 us with 2,048, 583 with 4,096, 600 with 8,192).
constexpr uint64_t kBlocksWanted = 4096;

// Blocks of the many-rows weights: two a compute unit, the rows split, at least 128 of them each, where the entries
// alone give fewer (2,000 tokens over themselves, 32 query and 8 kv heads: 50 us, with unsplit rows 183).
constexpr uint64_t kWeightBlocks = 512, kWeightLeast = 128;

// The entries (or rows) of a split: at least `least`, few enough that `units` of them give the blocks wanted, at
// most `most`, a multiple of `whole` (whole pages and whole rounds of a block's wavefronts).
uint32_t chunk_of(uint64_t entries, uint64_t units, uint64_t wanted, uint64_t least, uint64_t most,
                  uint32_t whole = 256) {
  const uint64_t splits = units >= wanted ? 1 : (wanted + units - 1) / units;
  uint64_t c = (entries + splits - 1) / splits;
  c = c < least ? least : c;
  c = c > most ? most : c;
  return (uint32_t)up(c, whole);
}

// The entries of a split of the many-rows kernel, a block of which fills a compute unit.  A block takes the time of
// its split's tiles, of 3 more to begin and, where rows are split, of 7 to write and read what is joined, and the
// join's launch that of 2.  One sequence's blocks are alike and run in rounds of 256; of more sequences, whose
// lengths differ, the blocks' sum counts, three quarters of what the longest would give, and half of the longest
// block for the end, and the longest at least.  (46 sequences' up to 137 tokens over 6,000 to 29,296 entries, 2
// heads of 3: 374 us, by rounds 573; 2,000 tokens over themselves, 32
// query and 8 kv heads: 65 us unsplit, 105 in two; 512 tokens over 20,000: 178 in 4, 192 in 8, 225 in 16; 64 over
// 60,000: 93 in 32, 107 in 64; 200 of 4 sequences over 20,000: 320 in 2, 331 in 4.)
uint32_t many_chunk_of(const KvArgs& a) {
  constexpr uint64_t UNITS = 256;
  const uint64_t rows = many_rows(a.dim), one = ((uint64_t)a.max_new * a.group + rows - 1) / rows;
  // ragged batches have fewer tokens than n_seq * max_new
  const uint64_t by_seq = one * a.n_seq, by_tok = (uint64_t)a.n_tok * a.group / rows + a.n_seq;
  const uint64_t blocks = (by_seq < by_tok ? by_seq : by_tok) * a.n_kv;
  const uint64_t whole = a.page > kManyKeys ? a.page : kManyKeys, least = 2 * kManyKeys;
  uint64_t chunk = up(a.max_len, whole);
  const auto cost_of = [&](uint64_t n, uint64_t tiles) {  // of n blocks, times 4
    const uint64_t rounds = 4 * ((n + UNITS - 1) / UNITS) * tiles, sum = 3 * n * tiles / UNITS + 2 * tiles;
    return a.n_seq == 1 ? rounds : sum > 4 * tiles ? sum : 4 * tiles;
  };
  uint64_t best = cost_of(blocks, chunk / kManyKeys + 3);
  // two rounds even out by themselves: lengths differ, and the longest blocks come first
  for (uint64_t rounds = 1; rounds <= 8 && blocks < 2 * UNITS; ++rounds) {
    uint64_t splits = UNITS * rounds / blocks;
    splits = splits * least > a.max_len ? a.max_len / least : splits;
    if (splits < 2) continue;
    const uint64_t c = up((a.max_len + splits - 1) / splits, whole);
    splits = (a.max_len + c - 1) / c;
    if (splits < 2) continue;
    const uint64_t cost = cost_of(blocks * splits, c / kManyKeys + 10) + 8;
    if (cost < best) {
      best = cost;
      chunk = c;
    }
  }
  return (uint32_t)chunk;
}

Plan plan_of(const KvArgs& a, bool weights, uint32_t n_sel) {
  Plan p = {};
  const uint64_t row_most = (uint64_t)a.max_new * a.group;
  const uint64_t pairs = (uint64_t)a.n_seq * a.n_kv;
  const uint64_t lds_most = (uint64_t)kPagesLds * a.page;  // entries that the few-rows kernel has page ids for
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t was = at;
    at = up(at + bytes, 256);
    return was;
  };
  if (n_sel) {
    p.few_rows = p.few_most = a.group > 16 ? 32 : 16;
    const uint64_t all = (uint64_t)n_sel << a.page_bits;
    // a token of each sequence at least; ragged batches have fewer tokens than n_seq * max_new
    const uint64_t tokens = a.n_tok > a.n_seq ? a.n_tok : a.n_seq;
    p.few_chunk = chunk_of(all, tokens * a.n_kv, kBlocksWanted, 256, lds_most);
    p.few_split = (uint32_t)((all + p.few_chunk - 1) / p.few_chunk);
    p.few_cap = 0;
    p.keys = take((size_t)a.n_tok * a.n_kv * a.max_pages * sizeof(uint32_t));
  } else {
    // 17 to 32 rows: two row tiles leave the few-rows kernel fewer loads under way, but it needs no second pass
    // for the weights and ends sooner where there is little to read.  (8 heads, 8 tokens of 4 query heads: 16
    // sequences of 8,192 entries 142 us against 113 on the many-rows kernel, 4 of them 48 against 43 and with
    // weights 66 against 59, one of them 20 on both; one head of 256, up to 5,003 entries: 13 sequences 24 against
    // 30, 20 of them 38 against 35.)
    const bool wide = a.dim >= 128 && pairs * a.max_len * a.dim * 4 >= 100000000ull;
    // Up to 16 rows: of 256 dimensions the few-rows kernel has two wavefronts' registers only (the same 16
    // sequences, one token each: 130 us against 113).
    p.few_most = !wide ? kRowsFew : a.dim == 256 && !weights ? 0 : 16;
    p.few_rows = row_most > 16 && !wide ? 32 : 16;
    p.many = row_most > p.few_most;
    if (p.many && a.n_seq == 1) p.few_most = 0;  // nobody else may have few: no launches for them
    // One block: no second launch.  It pays where a block is done within a few tiles (777 entries of 64
    // dimensions: 9 us in one, 13 split; but 1,000 of 128: 18 in one, 13 split) and where the pairs alone fill the
    // card (2,048 pairs of up to 1,000 entries: 128 us in one, 161 split).
    const bool one = (uint64_t)a.max_len * a.dim <= 65536 || (a.max_len <= 1024 && pairs >= 512);
    p.few_chunk = one ? (uint32_t)up(a.max_len, 256) : chunk_of(a.max_len, pairs, kBlocksWanted, 256, lds_most);
    p.few_split = (a.max_len + p.few_chunk - 1) / p.few_chunk;
    p.few_cap = (uint32_t)(row_most < p.few_most ? row_most : p.few_most);
    if (p.many) {
      p.many_chunk = many_chunk_of(a);
      p.many_split = (a.max_len + p.many_chunk - 1) / p.many_chunk;
    }
  }
  const size_t all_rows = (size_t)a.n_tok * a.n_q, few_part = p.few_cap ? pairs * p.few_cap : all_rows;
  if (p.few_most == 0) p.few_split = 0;
  if (p.few_split > 1) p.o = take(p.few_split * few_part * a.dim * sizeof(float));
  if (p.few_split > 1 || (weights && !p.many)) p.ml = take(p.few_split * few_part * sizeof(float2));
  if (p.many && p.many_split > 1) {
    // token arrays may hold more rows than these sequences can have
    p.many_cap = (uint64_t)a.n_seq * a.max_new < a.n_tok ? (uint32_t)row_most : 0;
    const size_t many_part = p.many_cap ? pairs * p.many_cap : all_rows;
    p.many_o = take(p.many_split * many_part * a.dim * sizeof(float));
    p.many_ml = take(p.many_split * many_part * sizeof(float2));
  }
  if (weights && !p.many) {
    p.score_len = (uint32_t)up(a.max_len, 64);
    p.scores = take(pairs * p.few_cap * p.score_len * sizeof(float));
  }
  if (weights && p.many) {
    p.lse = take((size_t)a.n_tok * a.n_q * sizeof(float));
    p.w_len = (uint32_t)up(a.max_len, kWeightKeys);
    p.w_rows = chunk_of(row_most, pairs * (p.w_len / kWeightKeys), kWeightBlocks, kWeightLeast, row_most, kWeightRows);
    p.w_split = (uint32_t)((row_most + p.w_rows - 1) / p.w_rows);
    if (p.w_split > 1) p.part_w = take(p.w_split * pairs * p.w_len * sizeof(float));
  }
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
  p.rows_to = plan.few_most;
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
    const size_t bytes = (size_t)plan.few_chunk * plan.few_cap * sizeof(float);
    p.score_lds = bytes <= kScoresLds;
    const auto scored = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), p.score_lds ? bytes : 0, st, p);
    };
    if (plan.few_rows == 16) scored(kv_few_kernel<M, D, 1, false, true>);
    else scored(kv_few_kernel<M, D, 2, false, true>);
  } else if (plan.few_most) {
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
    p.row_cap = plan.many_cap;
    p.rows_from = plan.few_most;
    p.rows_to = row_most;
    hipLaunchKernelGGL((kv_many_kernel<M, D>),
                       dim3(a.n_kv * plan.many_split, (row_most + many_rows(D) - 1) / many_rows(D), a.n_seq),
                       dim3(64 * many_waves(D)), 0, st, p);
    if (plan.many_split > 1) join(row_most);
    if (weights) {
      p.part_w = (float*)(ws + plan.part_w);
      p.w_split = plan.w_split;
      p.w_rows = plan.w_rows;
      p.w_len = plan.w_len;
      launch(kv_weight_many_kernel<M, D>, dim3(plan.w_len / kWeightKeys * plan.w_split, a.n_kv, a.n_seq), decay);
      if (plan.w_split > 1) launch(kv_weight_join_kernel, dim3((a.max_len + kBlock - 1) / kBlock, a.n_kv, a.n_seq), decay);
    }
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
  return (uint64_t)a.n_kv * p.many_split <= most && rows / many_rows(a.dim) < 65535;
}

hipError_t launch_kv_choose(const KvArgs& a, const KvRows& q, bool negate, uint32_t n_sel, uint32_t first,
                            uint32_t last, uint32_t* keys, int32_t* sel, hipStream_t st);

hipError_t launch_kv_attend(const KvArgs& a, const KvRows& q, float scale, bool weights, float decay,
                            uint32_t n_sel, uint32_t first, uint32_t last, void* out, float* lse, int32_t* sel,
                            void* ws, hipStream_t st) {
  const Plan plan = plan_of(a, weights, n_sel);
  if (n_sel) {
    const hipError_t rc =
        launch_kv_choose(a, q, scale < 0.0f, n_sel, first, last, (uint32_t*)((char*)ws + plan.keys), sel, st);
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
