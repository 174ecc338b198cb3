// kv_cache.hip -- the operators that write pages or choose among entries: append, victims, compact,
// and the page choice of sparse attention.
#include <type_traits>

#include "kv_device.h"

#pragma clang fp contract(off)

namespace unison {

namespace {

constexpr uint32_t kBlock = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

template <typename T>
__device__ __forceinline__ float bits_f32(uint16_t b);
template <>
__device__ __forceinline__ float bits_f32<__hip_bfloat16>(uint16_t b) {
  return __uint_as_float((uint32_t)b << 16);
}
template <>
__device__ __forceinline__ float bits_f32<__half>(uint16_t b) {
  return (float)__builtin_bit_cast(_Float16, b);
}

// ------------------------------------------------------------------ boxes

// The lower and upper sides of a page's keys, gathered 8 dimensions at a time: thread t of the block
// has the dimensions 8 (t % (D / 8)) of rows t / (D / 8), t / (D / 8) + kBlock / (D / 8), ...
struct Sides {
  float lo[8], hi[8];
  __device__ __forceinline__ void clear() {
    for (int i = 0; i < 8; ++i) {
      lo[i] = __builtin_inff();
      hi[i] = -__builtin_inff();
    }
  }
  template <typename T>
  __device__ __forceinline__ void add(u16x8 x) {
    for (int i = 0; i < 8; ++i) {
      const float f = bits_f32<T>(x[i]);
      lo[i] = fminf(lo[i], f);
      hi[i] = fmaxf(hi[i], f);
    }
  }
};

// Writes a page's box from the threads' sides; `lds` has 16 words a thread.  All threads call it.
template <int D>
__device__ void write_box(const KvArgs& a, int32_t page, uint32_t h, const Sides& x, float* lds) {
  constexpr uint32_t CH = D / 8, RG = kBlock / CH;
  const uint32_t tid = threadIdx.x, c = tid % CH, g = tid / CH;
  for (int i = 0; i < 8; ++i) {
    lds[g * D + 8 * c + i] = x.lo[i];
    lds[(RG + g) * D + 8 * c + i] = x.hi[i];
  }
  __syncthreads();
  float lo = 0.0f, hi = 0.0f, top = 0.0f;
  if (tid < D) {
    lo = lds[tid];
    hi = lds[RG * D + tid];
    for (uint32_t i = 1; i < RG; ++i) {
      lo = fminf(lo, lds[i * D + tid]);
      hi = fmaxf(hi, lds[(RG + i) * D + tid]);
    }
    top = fmaxf(fabsf(lo), fabsf(hi));
  }
  __syncthreads();
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((tid & 63u) == 0u) lds[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  const KvStep st = kv_step(top);
  if (tid < D) {
    int8_t* b = a.box + ((size_t)page * a.n_kv + h) * 2 * D + tid;
    b[0] = (int8_t)kv_clip(floorf(lo * st.inv));
    b[D] = (int8_t)kv_clip(ceilf(hi * st.inv));
  }
  if (tid == 0) a.box_scale[(size_t)page * a.n_kv + h] = st.step;
}

// ------------------------------------------------------------------ append

// One block per (page that may get entries, kv head, sequence).  Keys go over in 16-byte pieces and,
// where the pool has boxes, through the box's sides on the way, together with the page's older rows.
// Values change their order: 64 slots of the page are put together in LDS, two slots to a word, and
// leave in 16-byte runs of slots; up to kDirect new rows (a decode step) go straight to their places.
// Bound by memory: 16 sequences' turns of up to 2,000 tokens, 8 heads of 128 (158 MB): 42 us, 3.8 TB/s; a step of
// 64 tokens 5.8 us, most of it latency.  A step of 4 tokens each takes 10.3 us direct, 10.9 through LDS; of
// 8 12.5 and 10.5.
constexpr int32_t kDirect = 4;

template <typename T, int D>
__global__ __launch_bounds__(kBlock) void kv_append_kernel(KvArgs a, KvRows nk, KvRows nv,
                                                           const int32_t* tok_pos) {
  constexpr uint32_t CH = D / 8, RG = kBlock / CH, S = 33;  // an odd stride spreads the words over the banks
  __shared__ uint32_t lds[D * S > 16 * kBlock ? D * S : 16 * kBlock];
  const uint32_t h = blockIdx.y, tid = threadIdx.x, c = tid % CH, g = tid / CH;
  const KvSeq q = kv_seq(a, blockIdx.z);
  const int32_t first = q.len - q.n;  // below 0: tokens without an entry
  const int32_t o = ((first < 0 ? 0 : first) >> a.page_bits) + (int32_t)blockIdx.x;
  const int32_t lo = o << a.page_bits, hi = lo + (int32_t)a.page;
  const int32_t b = first > lo ? first : lo, e = q.len < hi ? q.len : hi;
  if (b >= e) return;
  const int32_t page = kv_page(a, q, o);
  if (page < 0) return;
  uint16_t* k = (uint16_t*)a.k + kv_base(a, page, h);
  uint16_t* v = (uint16_t*)a.v + kv_base(a, page, h);
  const int32_t t0 = q.t0 - first;  // row of entry x: t0 + x
  const uint16_t* sk = (const uint16_t*)nk.p + h * nk.head + 8 * c;
  const uint16_t* sv = (const uint16_t*)nv.p + h * nv.head;
  for (int32_t i = b + (int32_t)tid; i < e; i += (int32_t)kBlock) {
    const size_t w = kv_word(a, page, h) + (size_t)(i - lo);
    if (a.weight) a.weight[w] = 0.0f;
    if (a.pos) a.pos[w] = tok_pos[t0 + i];
  }
  if (e - b <= kDirect) {
    for (uint32_t i = tid; i < (uint32_t)(e - b) * D; i += kBlock) {
      const int32_t x = b + (int32_t)(i / D);
      v[(size_t)(i % D) * a.page + (uint32_t)(x - lo)] = sv[(size_t)(t0 + x) * nv.tok + i % D];
    }
  } else {
    for (int32_t s0 = b & ~63; s0 < e; s0 += 64) {
      const int32_t base = s0 > lo ? s0 : lo;  // pages of 16 and 32 are narrower than 64 slots
      const int32_t stop = base + 64 < hi ? base + 64 : hi;
      for (uint32_t x = g; x < (uint32_t)(stop - base) / 2; x += RG) {
        const int32_t r = base + 2 * (int32_t)x;
        u16x8 u = (u16x8)(uint16_t)0, w = (u16x8)(uint16_t)0;
        if (r >= b && r < e) u = *(const u16x8*)(sv + (size_t)(t0 + r) * nv.tok + 8 * c);
        if (r + 1 >= b && r + 1 < e) w = *(const u16x8*)(sv + (size_t)(t0 + r + 1) * nv.tok + 8 * c);
        for (uint32_t i = 0; i < 8; ++i) lds[(8 * c + i) * S + x] = u[i] | ((uint32_t)w[i] << 16);
      }
      __syncthreads();
      const uint32_t runs = (uint32_t)(stop - base) / 8;  // 2, 4 or 8
      for (uint32_t i = tid; i < D * runs; i += kBlock) {
        const uint32_t d = i / runs, run = i % runs;
        const int32_t r = base + 8 * (int32_t)run;
        const uint32_t* from = lds + d * S + 4 * run;
        const u32x4 x = {from[0], from[1], from[2], from[3]};
        uint16_t* to = v + (size_t)d * a.page + (uint32_t)(r - lo);
        if (r >= b && r + 8 <= e) {
          *(u32x4*)to = x;
        } else {
          for (int32_t y = 0; y < 8; ++y)
            if (r + y >= b && r + y < e) to[y] = (uint16_t)(x[y >> 1] >> (16 * (y & 1)));
        }
      }
      __syncthreads();
    }
  }
  Sides side;
  side.clear();
  for (int32_t x = (a.box ? lo : b) + (int32_t)g; x < e; x += (int32_t)RG) {
    uint16_t* at = k + (size_t)(uint32_t)(x - lo) * D + 8 * c;
    u16x8 row;
    if (x >= b) {
      row = *(const u16x8*)(sk + (size_t)(t0 + x) * nk.tok);
      *(u16x8*)at = row;
    } else {
      row = *(const u16x8*)at;
    }
    if (a.box) side.add<T>(row);
  }
  if (a.box) write_box<D>(a, page, h, side, (float*)lds);
}

// ------------------------------------------------------------------ the n smallest keys

// Finds the `need` smallest of up to BLOCK * PER keys that the block holds in registers: element i of
// a thread is number wave * 64 PER + (i / 4) * 256 + 4 lane + i % 4, so that its memory is read in
// 16-byte pieces side by side and still follows in the order of numbers.
template <int BLOCK, int PER>
struct Pick {
  uint32_t hist[2048];
  uint32_t sums[2][BLOCK / 64];
  uint32_t found[3];
  unsigned long long best;
};

struct Numbers {
  uint32_t base;
  template <int PER>
  static __device__ __forceinline__ Numbers of() {
    return Numbers{(threadIdx.x >> 6) * 64u * PER + 4u * (threadIdx.x & 63u)};
  }
  __device__ __forceinline__ uint32_t operator()(int i) const { return base + (uint32_t)(i / 4) * 256u + (uint32_t)(i % 4); }
  // Made anew where a new pass begins: kept from the first one, the numbers and what was compared with them
  // take more registers than the keys.
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(base)); }
};

struct Cut {
  uint32_t key;   // the largest chosen key
  uint32_t ties;  // how many entries with that key are chosen: the lowest numbers
};

// The cut of the `need` smallest keys, 1 <= need <= the keys' count; a key of 0xFFFFFFFF is chosen only when
// the others do not suffice, and elements at and past the keys' count hold it.  Digits of 11, 11 and 10 bits from
// the top: a histogram (whole numbers: any order of additions gives the same), its prefix, and the
// digit the cut is in.  It ends early once a digit is taken whole.
template <int BLOCK, int PER>
__device__ __forceinline__ Cut pick_cut(const uint32_t (&key)[PER], uint32_t need, Pick<BLOCK, PER>& s) {
  constexpr uint32_t BINS = 2048 / BLOCK;
  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
  for (uint32_t i = 0; i < BINS; ++i) s.hist[tid * BINS + i] = 0;
  uint32_t prefix = 0, left = need, top = 0;  // bits of the key at and above `top` are known
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const uint32_t shift = pass == 0 ? 21u : pass == 1 ? 10u : 0u, mask = pass == 2 ? 1023u : 2047u;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool in = key[i] != 0xFFFFFFFFu && (pass == 0 || (key[i] >> top) == (prefix >> top));
      const uint32_t bin = (key[i] >> shift) & mask;
      const uint64_t who = __builtin_amdgcn_ballot_w64(in);
      if (who == 0ull) continue;
      // equal digits in a whole wavefront (weights that were never added to) count once
      const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)bin, (int)__builtin_ctzll(who));
      if (__builtin_amdgcn_ballot_w64(in && bin == one) == who) {
        if (lane == 0) atomicAdd(&s.hist[one], (uint32_t)__builtin_popcountll(who));
      } else if (in) {
        atomicAdd(&s.hist[bin], 1u);
      }
    }
    __syncthreads();
    uint32_t n[BINS], sum = 0;
    for (uint32_t i = 0; i < BINS; ++i) {
      n[i] = s.hist[tid * BINS + i];
      s.hist[tid * BINS + i] = 0;
      sum += n[i];
    }
    uint32_t upto = sum;
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(upto, o);
      if (lane >= (uint32_t)o) upto += y;
    }
    if (lane == 63u) s.sums[0][wave] = upto;
    if (tid == 0) s.found[2] = 0;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (uint32_t w = 0; w < BLOCK / 64; ++w) {
      before += w < wave ? s.sums[0][w] : 0u;
      all += s.sums[0][w];
    }
    uint32_t at = before + upto - sum;
    for (uint32_t i = 0; i < BINS; ++i) {
      if (at < left && left <= at + n[i]) {
        s.found[0] = tid * BINS + i;
        s.found[1] = left - at;
        s.found[2] = left == at + n[i] ? 2u : 1u;
      }
      at += n[i];
    }
    __syncthreads();
    const uint32_t how = s.found[2];
    // all keys below 0xFFFFFFFF are taken, and some of those
    if (how == 0u) return Cut{0xFFFFFFFFu, left - all};
    prefix |= s.found[0] << shift;
    left = s.found[1];
    top = shift;
    if (how == 2u) return Cut{prefix | ((1u << shift) - 1u), 0xFFFFFFFFu};
  }
  return Cut{prefix, left};
}

// Calls emit(i, place) for the flagged elements, their places in the order of their numbers; the block's
// total.  Of up to 32 elements the wavefront's flags stay in scalar registers; more are taken twice.
template <int BLOCK, int PER, typename Flag, typename Emit>
__device__ __forceinline__ uint32_t pick_places(Flag flag, Emit emit, uint32_t* sums) {
  constexpr bool KEEP = PER <= 32;
  const uint32_t wave = threadIdx.x >> 6;
  uint64_t kept[KEEP ? PER : 1];
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t w = __builtin_amdgcn_ballot_w64(flag(i));
    if (KEEP) kept[KEEP ? i : 0] = w;
    n += (uint32_t)__builtin_popcountll(w);
  }
  if ((threadIdx.x & 63u) == 0u) sums[wave] = n;
  __syncthreads();
  uint32_t at = 0, all = 0;
  for (uint32_t w = 0; w < BLOCK / 64; ++w) {
    at += w < wave ? sums[w] : 0u;
    all += sums[w];
  }
  const uint64_t below = (1ull << (threadIdx.x & 63u));
#pragma unroll
  for (int c = 0; c < PER / 4; ++c) {
    uint32_t x = at;
    bool is[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t w = KEEP ? kept[KEEP ? 4 * c + i : 0] : __builtin_amdgcn_ballot_w64(flag(4 * c + i));
      x += __builtin_amdgcn_mbcnt_hi((uint32_t)(w >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)w, 0u));
      at += (uint32_t)__builtin_popcountll(w);
      is[i] = (w & below) != 0ull;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (is[i]) emit(4 * c + i, x++);
  }
  __syncthreads();
  return all;
}

// A bit for each of a thread's elements.
template <int PER>
struct Bits {
  uint32_t w[(PER + 31) / 32];
  __device__ __forceinline__ bool operator()(int i) const { return (w[i / 32] >> (i % 32)) & 1u; }
  __device__ __forceinline__ void set(int i, bool x) { w[i / 32] |= (x ? 1u : 0u) << (i % 32); }
  __device__ __forceinline__ void drop(int i) { w[i / 32] &= ~(1u << (i % 32)); }
};

// Which elements the cut chooses: at least as many keys as it takes, so never an element past the last key.
template <int BLOCK, int PER>
__device__ __forceinline__ Bits<PER> pick_chosen(const uint32_t (&key)[PER], Cut cut, Pick<BLOCK, PER>& s) {
  Bits<PER> out = {};
#pragma unroll
  for (int i = 0; i < PER; ++i) out.set(i, key[i] <= cut.key);
  if (cut.ties != 0xFFFFFFFFu) {
    const Bits<PER> before = out;
    pick_places<BLOCK, PER>([&](int i) { return before(i) && key[i] == cut.key; },
                            [&](int i, uint32_t at) { if (at >= cut.ties) out.drop(i); }, s.sums[0]);
  }
  return out;
}

// ------------------------------------------------------------------ victims

// Up to so many victims, rounds of a minimum beat the digits' histograms (one of 20,000 entries: 16 us, 38 with
// histograms; one of 4,097 in 512 pairs: 14 and 20).
constexpr uint32_t kFewVictims = 4;

// One block per (kv head, sequence) of up to BLOCK * PER entries: weights and positions are read once into
// registers (twice of more than 32 a thread).  Bound by vector instructions (busy 65 to 71 % of the time) and the
// barriers between them: 8 sequences of up to 32,768 entries and 8 heads (64 blocks) down to 8,192: 39 us for 25 MB.
template <int BLOCK, int PER>
__global__ __launch_bounds__(BLOCK, PER <= 8 ? 8 : 4) void kv_victims_kernel(KvArgs a, uint32_t budget, uint32_t first,
                                                           uint32_t recent, uint32_t max_evict,
                                                           int32_t* victims, int32_t* src, int32_t* new_len) {
  __shared__ Pick<BLOCK, PER> s;
  const uint32_t h = blockIdx.x, seq = blockIdx.y, tid = threadIdx.x;
  a.tok = nullptr;
  const KvSeq q = kv_seq(a, seq);
  const uint32_t len = (uint32_t)q.len;
  uint32_t n = len > budget ? len - budget : 0u;
  n = n < max_evict ? n : max_evict;
  const uint32_t stay = len - n;
  if (h == 0 && tid == 0) new_len[seq] = (int32_t)stay;
  const size_t row = ((size_t)seq * a.n_kv + h) * max_evict;
  uint32_t got = 0, moved = 0;
  if (n) {
    // the highest position first; more than 32 a thread are read again rather than kept
    constexpr bool KEEP = PER <= 32;
    uint32_t key[PER];
    i32x4 pos[KEEP ? PER / 4 : 1];
    int32_t top = INT32_MIN;
    Numbers num = Numbers::of<PER>();
    // the word of entry e, any word for one that is not there
    const auto word = [&](uint32_t e, bool& in) __attribute__((always_inline)) {
      const int32_t p = kv_page(a, q, (int32_t)((e < len ? e : len - 1u) >> a.page_bits));
      in = e < len && p >= 0;
      return kv_word(a, p < 0 ? 0 : p, h) + (e & (a.page - 1u));
    };
#pragma unroll
    for (int c = 0; c < PER / 4; ++c) {
      const uint32_t e = num(4 * c);
      bool in = false;
      i32x4 x = (i32x4)0;
      f32x4 w = (f32x4)0.0f;
      if (__builtin_amdgcn_ballot_w64(e < len)) {  // a wavefront behind the end reads nothing
        const size_t at = word(e, in);
        x = *(const i32x4*)(a.pos + at);
        w = *(const f32x4*)(a.weight + at);
      }
      if (KEEP) pos[KEEP ? c : 0] = x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool is = in && e + i < len;
        key[4 * c + i] = is ? kv_order(w[i]) : 0xFFFFFFFFu;
        top = is && x[i] > top ? x[i] : top;
      }
      if (!KEEP && c % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // no more loads under way than registers
    }
    for (int o = 32; o; o >>= 1) {
      const int32_t y = __shfl_xor(top, o);
      top = y > top ? y : top;
    }
    if ((tid & 63u) == 0u) s.sums[1][tid >> 6] = (uint32_t)top;
    __syncthreads();
    for (uint32_t w = 0; w < BLOCK / 64; ++w) top = (int32_t)s.sums[1][w] > top ? (int32_t)s.sums[1][w] : top;
    const int64_t newest = (int64_t)top - (int64_t)recent;
    num.renew();
#pragma unroll
    for (int c = 0; c < PER / 4; ++c) {
      bool in;
      const i32x4 x = KEEP ? pos[KEEP ? c : 0] : *(const i32x4*)(a.pos + word(num(4 * c), in));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (x[i] < (int64_t)first || x[i] > newest) key[4 * c + i] = 0xFFFFFFFFu;
      if (!KEEP && c % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    if (KEEP && n <= kFewVictims) {  // a step's victim or two: the smallest of key and slot, one after the other
      int32_t gone[kFewVictims];
      uint64_t last = 0;
      for (uint32_t v = 0; v < kFewVictims; ++v) gone[v] = INT32_MAX;
      for (uint32_t v = 0; v < n; ++v) {
        uint64_t best = ~0ull;
        num.renew();
#pragma unroll
        for (int i = 0; i < PER; ++i) {  // what is no entry has the largest key and a larger number than any entry
          const uint64_t x = ((uint64_t)key[i] << 32) | num(i);
          if ((v == 0 || x > last) && x < best) best = x;
        }
        if (tid == 0) s.best = ~0ull;
        __syncthreads();
        atomicMin(&s.best, (unsigned long long)best);
        __syncthreads();
        last = s.best;
        __syncthreads();
        // in the order of slots
        int32_t e = (int32_t)(uint32_t)last;
        for (uint32_t w = 0; w < kFewVictims; ++w) {
          const int32_t x = gone[w];
          gone[w] = e < x ? e : x;
          e = e < x ? x : e;
        }
      }
      if (tid < max_evict) {
        int32_t mine = -1, from = -1;
        if (tid < n) {
          uint32_t filled = 0;
          for (uint32_t e = stay; e < len; ++e) {
            bool is = false;
            for (uint32_t w = 0; w < kFewVictims; ++w) is = is || gone[w] == (int32_t)e;
            if (!is) {
              if (filled == tid) from = (int32_t)e;
              ++filled;
            }
          }
          for (uint32_t w = 0; w < kFewVictims; ++w) mine = w == tid ? gone[w] : mine;
        }
        victims[row + tid] = mine;
        src[row + tid] = from;
      }
      for (uint32_t i = BLOCK + tid; i < max_evict; i += BLOCK) victims[row + i] = src[row + i] = -1;
      return;
    }
    const Cut cut = pick_cut<BLOCK, PER>(key, n, s);
    const Bits<PER> out = pick_chosen<BLOCK, PER>(key, cut, s);
    num.renew();
    got = pick_places<BLOCK, PER>(out, [&](int i, uint32_t at) { victims[row + at] = (int32_t)num(i); }, s.sums[0]);
    num.renew();
    moved = pick_places<BLOCK, PER>([&](int i) { return num(i) >= stay && num(i) < len && !out(i); },
                                    [&](int i, uint32_t at) { src[row + at] = (int32_t)num(i); }, s.sums[0]);
  }
  for (uint32_t i = got + tid; i < max_evict; i += BLOCK) victims[row + i] = -1;
  for (uint32_t i = moved + tid; i < max_evict; i += BLOCK) src[row + i] = -1;
}

// Longer sequences than a block's registers hold are read again in every pass (8 of up to 66,000 entries:
// 420 us; of 65,536 in registers 89).
constexpr uint32_t kSelBlock = 1024;

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

__global__ __launch_bounds__(kSelBlock) void kv_victims_long_kernel(KvArgs a, uint32_t budget, uint32_t first,
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

// ------------------------------------------------------------------ compact

// Where the moves of a block read and write; -1: no move.
struct Move {
  int64_t from, to;   // first elements of the two pages' keys and values
  uint32_t sf, st;    // their slots
};

__device__ __forceinline__ Move move_of(const KvArgs& a, uint32_t h, uint32_t s, uint32_t i, uint32_t max_evict,
                                        const int32_t* victims, const int32_t* src, const int32_t* new_len) {
  Move m = {-1, -1, 0, 0};
  if (i >= max_evict) return m;
  KvArgs b = a;
  b.tok = nullptr;
  const KvSeq q = kv_seq(b, s);
  const int32_t stay = new_len[s];
  const size_t row = ((size_t)s * a.n_kv + h) * max_evict;
  const int32_t from = src[row + i], to = victims[row + i];
  if (to < 0 || to >= stay || from < stay || from >= q.len) return m;
  const int32_t pf = kv_page(a, q, from >> a.page_bits), pt = kv_page(a, q, to >> a.page_bits);
  if (pf < 0 || pt < 0) return m;
  m.from = (int64_t)kv_base(a, pf, h);
  m.to = (int64_t)kv_base(a, pt, h);
  m.sf = (uint32_t)from & (a.page - 1u);
  m.st = (uint32_t)to & (a.page - 1u);
  return m;
}

// Few moves (a step that evicts an entry or two): 64 lanes each, a lane per dimension of the values.
template <int D>
__global__ __launch_bounds__(kBlock) void kv_compact_few_kernel(KvArgs a, uint32_t max_evict,
                                                                const int32_t* victims, const int32_t* src,
                                                                const int32_t* new_len) {
  const uint32_t h = blockIdx.y, lane = threadIdx.x & 63u;
  const Move m = move_of(a, h, blockIdx.z, blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6), max_evict, victims, src,
                         new_len);
  if (m.from < 0) return;
  uint16_t *k = (uint16_t*)a.k, *v = (uint16_t*)a.v;
  if (lane < D / 8) *(u32x4*)(k + m.to + m.st * D + 8 * lane) = *(const u32x4*)(k + m.from + m.sf * D + 8 * lane);
  uint16_t x[D / 64];
  for (uint32_t i = 0; i < D / 64; ++i) x[i] = v[m.from + (size_t)(64 * i + lane) * a.page + m.sf];
  for (uint32_t i = 0; i < D / 64; ++i) v[m.to + (size_t)(64 * i + lane) * a.page + m.st] = x[i];
  if (lane == 0) {
    if (a.weight) a.weight[m.to / D + m.st] = a.weight[m.from / D + m.sf];
    if (a.pos) a.pos[m.to / D + m.st] = a.pos[m.from / D + m.sf];
  }
}

// Many moves: 64 of a block, whose places lie close together, with a lane per move for the values, so
// that a load takes its 64 slots of a dimension from a few lines (a lane per dimension took 64 lines for 64
// values: 312 us for 8 sequences of up to 32,768 entries down to 8,192, 8 heads of 128; now 190).  Bound by the
// lines that the values touch: a dimension's 64 slots are one, and most lines behind the new end and
// most of those before it are touched, 0.7 GB in all where the moved entries are 0.37.
template <int D>
__global__ __launch_bounds__(kBlock) void kv_compact_kernel(KvArgs a, uint32_t max_evict,
                                                            const int32_t* victims, const int32_t* src,
                                                            const int32_t* new_len) {
  constexpr uint32_t CH = D / 8;
  __shared__ Move moves[64];
  const uint32_t h = blockIdx.y, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
  if (tid < 64u) moves[tid] = move_of(a, h, blockIdx.z, blockIdx.x * 64u + tid, max_evict, victims, src, new_len);
  __syncthreads();
  uint16_t *k = (uint16_t*)a.k, *v = (uint16_t*)a.v;
  u32x4 x[CH / 4];
  for (uint32_t i = 0; i < CH / 4; ++i) {
    const Move m = moves[(i * kBlock + tid) / CH];
    if (m.from >= 0) x[i] = *(const u32x4*)(k + m.from + m.sf * D + 8 * (tid % CH));
  }
  for (uint32_t i = 0; i < CH / 4; ++i) {
    const Move m = moves[(i * kBlock + tid) / CH];
    if (m.from >= 0) *(u32x4*)(k + m.to + m.st * D + 8 * (tid % CH)) = x[i];
  }
  const Move m = moves[lane];
  if (m.from < 0) return;
  const uint16_t* vf = v + m.from + m.sf + (size_t)(wave * (D / 4)) * a.page;
  uint16_t* vt = v + m.to + m.st + (size_t)(wave * (D / 4)) * a.page;
  for (uint32_t d = 0; d < D / 4; d += 16) {
    uint16_t y[16];
    for (uint32_t i = 0; i < 16; ++i) y[i] = vf[(size_t)(d + i) * a.page];
    for (uint32_t i = 0; i < 16; ++i) vt[(size_t)(d + i) * a.page] = y[i];
  }
  if (wave == 0 && a.weight) a.weight[m.to / D + m.st] = a.weight[m.from / D + m.sf];
  if (wave == 1 && a.pos) a.pos[m.to / D + m.st] = a.pos[m.from / D + m.sf];
}

// The boxes after the moves: a block per (page ordinal, kv head, sequence); renewed are the pages
// below new_len that hold a victim's place or a new end.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void kv_rebox_kernel(KvArgs a, uint32_t max_evict,
                                                          const int32_t* victims, const int32_t* new_len) {
  constexpr uint32_t CH = D / 8, RG = kBlock / CH;
  __shared__ float lds[16 * kBlock];
  const uint32_t h = blockIdx.y, s = blockIdx.z, c = threadIdx.x % CH, g = threadIdx.x / CH;
  a.tok = nullptr;
  const KvSeq q = kv_seq(a, s);
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
  const int32_t live = stay < hi ? stay - lo : (int32_t)a.page;
  const uint16_t* k = (const uint16_t*)a.k + kv_base(a, page, h) + 8 * c;
  Sides side;
  side.clear();
  for (int32_t x = (int32_t)g; x < live; x += (int32_t)RG) side.add<T>(*(const u16x8*)(k + (size_t)x * D));
  write_box<D>(a, page, h, side, lds);
}

// ------------------------------------------------------------------ the pages of sparse attention

constexpr uint32_t kScorePages = 64;  // of a block, 16 a wavefront

// Keys of 64 pages for one token and kv head.  keys [n_tok][n_kv][max_pages], a larger score a smaller
// key; 0: taken in any case, 0xFFFFFFFF: not there.
//   sum over heads and dimensions of max(qi lower, qi upper)
//     = sum over dimensions of (sum over heads of min(qi, 0)) lower + (sum over heads of max(qi, 0)) upper,
// one product with the box's bytes for all heads of the group.  The summed query has up to 15 bits: two
// 7-bit halves, so that the products are byte dot products.  Bound by latency and the boxes' bytes: 2,047 pages,
// 8 heads of 128: 5.4 us; 24 sequences of up to 512 pages and 2 tokens: 12.5 us (32 MB of boxes).
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void kv_score_kernel(KvArgs a, KvRows nq, bool negate, uint32_t first,
                                                          uint32_t last, uint32_t* keys) {
  constexpr uint32_t LP = 2 * D / 16, PP = 64 / LP;  // lanes of a page, pages of a wavefront's load
  __shared__ alignas(16) uint8_t half[2][2 * D];     // low and high 7 bits: D of the lower side, D of the upper
  __shared__ float lds[kBlock / 64];
  const uint32_t h = blockIdx.y, tid = threadIdx.x, lane = tid & 63u;
  const uint32_t chunks = (a.max_len + a.page * kScorePages - 1) / (a.page * kScorePages);
  const uint32_t j = blockIdx.x / chunks, base = spread_piece(blockIdx.x % chunks, chunks) * kScorePages;
  const KvSeq q = kv_seq(a, blockIdx.z);
  if ((int32_t)j >= q.n) return;
  const size_t t = (size_t)q.t0 + j;
  const int32_t limit = q.len - q.n + (int32_t)j + 1;
  const int32_t count = limit > 0 ? (limit + (int32_t)a.page - 1) >> a.page_bits : 0;
  if ((int32_t)base >= count) return;
  // the wavefront's 16 pages
  const int32_t mine = (int32_t)(base + (tid >> 6) * (kScorePages / 4) + (lane & 15u));
  const int32_t page = mine < count ? kv_page(a, q, mine) : -1;
  const uint16_t* row = (const uint16_t*)nq.p + t * nq.tok + (size_t)h * a.group * nq.head;
  float top = 0.0f;
  for (uint32_t i = tid; i < a.group * D; i += kBlock)
    top = fmaxf(top, fabsf(bits_f32<T>(row[(size_t)(i / D) * nq.head + i % D])));
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if ((tid & 63u) == 0u) lds[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  const float inv = negate ? -kv_step(top).inv : kv_step(top).inv;  // a negative scale prefers the smallest q.k
  if (tid < D) {
    int32_t n = 0, p = 0;
    for (uint32_t g = 0; g < a.group; ++g) {
      const int32_t x = kv_clip(rintf(bits_f32<T>(row[(size_t)g * nq.head + tid]) * inv));
      n -= x < 0 ? x : 0;
      p += x > 0 ? x : 0;
    }
    half[0][tid] = (uint8_t)(n & 127);
    half[1][tid] = (uint8_t)(n >> 7);
    half[0][D + tid] = (uint8_t)(p & 127);
    half[1][D + tid] = (uint8_t)(p >> 7);
  }
  __syncthreads();
  const uint32_t sub = lane % LP;
  const i32x4 ql = *(const i32x4*)&half[0][16 * sub], qh = *(const i32x4*)&half[1][16 * sub];
  i32x4 b[16 / PP];
  for (uint32_t i = 0; i < 16 / PP; ++i) {
    const int32_t p = __shfl(page, (int)(i * PP + lane / LP));
    b[i] = (i32x4)0;
    if (p >= 0) b[i] = *(const i32x4*)(a.box + ((size_t)p * a.n_kv + h) * 2 * D + 16 * sub);
  }
  int32_t score = 0;  // of page `mine`, in lanes 0 to 15
  for (uint32_t i = 0; i < 16 / PP; ++i) {
    int32_t x = 0, y = 0;
    for (int w = 0; w < 4; ++w) {
      x = __builtin_amdgcn_sdot4(ql[w], b[i][w], x, false);
      y = __builtin_amdgcn_sdot4(qh[w], b[i][w], y, false);
    }
    x += y * 128;
    x = sub < LP / 2 ? -x : x;
    for (uint32_t o = LP / 2; o; o >>= 1) x += __shfl_xor(x, (int)o);
    // lane l of 0 to 15 takes page l, which lanes (l % PP) LP have in step l / PP
    const int32_t got = __shfl(x, (int)((lane % PP) * LP));
    score = (lane & 15u) / PP == i ? got : score;
  }
  if (lane >= 16u || mine >= count) return;
  uint32_t key = 0xFFFFFFFFu;
  if (page >= 0)
    key = mine < (int32_t)first || mine >= count - (int32_t)last
              ? 0u : ~kv_order((float)score * a.box_scale[(size_t)page * a.n_kv + h]);
  keys[(t * a.n_kv + h) * a.max_pages + (uint32_t)mine] = key;
}

// The n_sel pages of smallest key, one block per (token, kv head).  Bound by latency: 8.5 us for 64 of 2,047.
template <int BLOCK, int PER>
__global__ __launch_bounds__(BLOCK, PER <= 8 ? 8 : 4) void kv_choose_kernel(KvArgs a, uint32_t n_sel, const uint32_t* keys,
                                                          int32_t* sel) {
  __shared__ Pick<BLOCK, PER> s;
  const uint32_t h = blockIdx.y, j = blockIdx.x, tid = threadIdx.x;
  const KvSeq q = kv_seq(a, blockIdx.z);
  if ((int32_t)j >= q.n) return;
  const size_t t = (size_t)q.t0 + j;
  const int32_t limit = q.len - q.n + (int32_t)j + 1;
  const uint32_t count = limit > 0 ? (uint32_t)(limit + (int32_t)a.page - 1) >> a.page_bits : 0u;
  const uint32_t* in = keys + (t * a.n_kv + h) * a.max_pages;
  int32_t* out = sel + (t * a.n_kv + h) * n_sel;
  uint32_t got = 0;
  if (count) {
    uint32_t key[PER];
    Numbers num = Numbers::of<PER>();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      key[i] = in[num(i) < count ? num(i) : count - 1u];
      key[i] = num(i) < count ? key[i] : 0xFFFFFFFFu;
    }
    Cut cut = {0xFFFFFFFEu, 0xFFFFFFFFu};  // every page that is there
    if (count > n_sel) cut = pick_cut<BLOCK, PER>(key, n_sel, s);
    const Bits<PER> take = pick_chosen<BLOCK, PER>(key, cut, s);
    num.renew();
    got = pick_places<BLOCK, PER>([&](int i) { return take(i) && key[i] != 0xFFFFFFFFu; },
                                  [&](int i, uint32_t at) { out[at] = (int32_t)num(i); }, s.sums[0]);
  }
  for (uint32_t i = got + tid; i < n_sel; i += BLOCK) out[i] = -1;
}

}  // namespace

namespace {

template <typename F>
hipError_t with_dim(uint32_t dim, F f) {
  if (dim == 64) f(std::integral_constant<int, 64>{});
  else if (dim == 128) f(std::integral_constant<int, 128>{});
  else f(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

template <typename F>
hipError_t with_type(const KvArgs& a, F f) {
  return with_dim(a.dim, [&](auto d) {
    if (a.dtype == UNISON_KV_BF16) f(__hip_bfloat16{}, d);
    else f(__half{}, d);
  });
}

// The smallest block whose registers hold `n` keys, of 1,024 threads rather than more keys a thread (2,047
// keys: 8.5 us with 1,024 x 4, 12.2 with 256 x 16).
template <typename F>
bool with_pick(uint32_t n, F f) {
  if (n <= 1024) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
  else if (n <= 4096) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
  else if (n <= 8192) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 8>{});
  else if (n <= 16384) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 16>{});
  else if (n <= 32768) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 32>{});
  else return false;
  return true;
}

}  // namespace

hipError_t launch_kv_append(const KvArgs& a, const KvRows& k, const KvRows& v, const int32_t* pos,
                            hipStream_t st) {
  const uint32_t most = a.max_new < a.max_len ? a.max_new : a.max_len;
  const dim3 grid((most + 2 * a.page - 2) / a.page, a.n_kv, a.n_seq);
  return with_type(a, [&](auto t, auto d) {
    hipLaunchKernelGGL((kv_append_kernel<decltype(t), decltype(d)::value>), grid, dim3(kBlock), 0, st, a, k, v, pos);
  });
}

hipError_t launch_kv_victims(const KvArgs& a, uint32_t budget, uint32_t first, uint32_t recent,
                             uint32_t max_evict, int32_t* victims, int32_t* src, int32_t* new_len,
                             hipStream_t st) {
  const dim3 grid(a.n_kv, a.n_seq);
  const auto picked = [&](auto block, auto per) {
    hipLaunchKernelGGL((kv_victims_kernel<decltype(block)::value, decltype(per)::value>), grid,
                       dim3(decltype(block)::value), 0, st, a, budget, first, recent, max_evict, victims, src, new_len);
  };
  if (with_pick(a.max_len, picked)) return hipGetLastError();
  if (a.max_len <= 65536)
    picked(std::integral_constant<int, 1024>{}, std::integral_constant<int, 64>{});
  else
    hipLaunchKernelGGL(kv_victims_long_kernel, grid, dim3(kSelBlock), 0, st, a, budget, first, recent, max_evict,
                       victims, src, new_len);
  return hipGetLastError();
}

hipError_t launch_kv_compact(const KvArgs& a, uint32_t max_evict, const int32_t* victims, const int32_t* src,
                             const int32_t* new_len, hipStream_t st) {
  // a wavefront per move up to a few: one entry of 512 pairs 7.3 us against 8.2, 8 of them 13.4 against 12.4, 16
  // 24.7 against 20.4
  const bool few = max_evict < 8;
  const uint32_t per = few ? kBlock / 64 : 64;
  const dim3 grid((max_evict + per - 1) / per, a.n_kv, a.n_seq);
  const dim3 pages((a.max_len + a.page - 1) / a.page, a.n_kv, a.n_seq);
  return with_type(a, [&](auto t, auto d) {
    constexpr int D = decltype(d)::value;
    if (few)
      hipLaunchKernelGGL(kv_compact_few_kernel<D>, grid, dim3(kBlock), 0, st, a, max_evict, victims, src, new_len);
    else
      hipLaunchKernelGGL(kv_compact_kernel<D>, grid, dim3(kBlock), 0, st, a, max_evict, victims, src, new_len);
    if (a.box)
      hipLaunchKernelGGL((kv_rebox_kernel<decltype(t), D>), pages, dim3(kBlock), 0, st, a, max_evict, victims,
                         new_len);
  });
}

hipError_t launch_kv_choose(const KvArgs& a, const KvRows& q, bool negate, uint32_t n_sel, uint32_t first,
                            uint32_t last, uint32_t* keys, int32_t* sel, hipStream_t st) {
  const uint32_t pages = (a.max_len + a.page - 1) / a.page;
  const dim3 grid(a.max_new * ((pages + kScorePages - 1) / kScorePages), a.n_kv, a.n_seq);
  const hipError_t rc = with_type(a, [&](auto t, auto d) {
    hipLaunchKernelGGL((kv_score_kernel<decltype(t), decltype(d)::value>), grid, dim3(kBlock), 0, st, a, q, negate,
                       first, last, keys);
  });
  if (rc != hipSuccess) return rc;
  const bool fits = with_pick(pages, [&](auto block, auto per) {
    hipLaunchKernelGGL((kv_choose_kernel<decltype(block)::value, decltype(per)::value>),
                       dim3(a.max_new, a.n_kv, a.n_seq), dim3(decltype(block)::value), 0, st, a, n_sel,
                       (const uint32_t*)keys, sel);
  });
  return fits ? hipGetLastError() : hipErrorInvalidValue;
}

}  // namespace unison
