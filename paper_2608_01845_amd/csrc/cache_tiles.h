// Device helpers of the attention kernels over a paged key/value cache: which rows
// and keys a block works on, where its pages lie, and the pieces of a tile's
// softmax and products that the caches of both element types share.
#pragma once

#include "common.h"

#include <algorithm>
#include <cfloat>

namespace wdc {
namespace {

constexpr int RSRC_WORD3 = 0x00020000;   // raw buffer descriptor word 3
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Buffer of `bytes` bytes from base + off: what lies outside reads as zero
__device__ __forceinline__ u32x4_t buffer_at(const void *base, int64_t off, int bytes) {
  const uint64_t p = (uint64_t)base + (uint64_t)off;
  return u32x4_t{(uint32_t)uni((int)(uint32_t)p), (uint32_t)uni((int)(uint32_t)(p >> 32) & 0xffff), (uint32_t)uni(bytes),
                 (uint32_t)RSRC_WORD3};
}
// LDS address of a pointer into it, the same in every lane
__device__ __forceinline__ uint32_t lds_addr(const void *p) {
  return (uint32_t)uni((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p);
}
// waits until at most N loads are under way
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Four rows of 16 columns of 2 bytes, each read as 4 x 8 bytes by the lanes of a
// group of 16 in row order, come back transposed: lane c of the group gets column c.
__device__ __forceinline__ s16x4 lds_read_tr(const char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
}

__device__ __forceinline__ float quad_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// First slots in the pool of one sequence's pages and a kv head, asked for in rising order by a whole
// wave: 64 table entries in a register, the next 64 on their way in another. EARLY: slots are found for all 64
// at once (long chunks over small pages: 59 -> 56 us for 2,048 rows of 16 heads of 128; single
// tokens, which touch few entries of a page table, lose by it: 86 -> 93).
template <bool EARLY>
struct PageWalk {
  const int32_t *tab;
  int last, base, cur, next;
  __device__ __forceinline__ int fetch(int i) const { return tab[min(i + (int)(threadIdx.x & 63), last)]; }
  __device__ __forceinline__ static int slot(const CacheArgs &a, int h, int entry) {   // (pools hold fewer than 2^31)
    return (cache_page(a, entry) * a.kvh + h) << a.plog;
  }
  __device__ __forceinline__ void init(const CacheArgs &a, const int32_t *tab_, int last_, int h, int first) {
    tab = tab_;
    last = last_;
    base = first;
    cur = fetch(base);
    next = fetch(base + 64);
    if (EARLY) cur = slot(a, h, cur);
  }
  // before get(i); the entries that share i's group of 64 from the first on need no further call
  __device__ __forceinline__ void advance(const CacheArgs &a, int h, int i) {
    while (i - base >= 64) {
      cur = EARLY ? slot(a, h, next) : next;
      base += 64;
      next = fetch(base + 64);
    }
  }
  __device__ __forceinline__ int get(const CacheArgs &a, int h, int i) const {
    const int x = __builtin_amdgcn_readlane(cur, i - base);
    return EARLY ? x : slot(a, h, x);
  }
};

// a sequence's lengths as wave-uniform values
__device__ __forceinline__ CacheSeq uniform_seq(const CacheArgs &a, int b) {
  CacheSeq s = cache_seq(a, b);
  s.q0 = uni(s.q0);
  s.nq = uni(s.nq);
  s.n = uni(s.n);
  s.start = uni(s.start);
  return s;
}

// Keys that the rows of group g share: whole pages of its first sequence (*lead)
__device__ __forceinline__ int shared_keys(const CacheArgs &c, const CacheShared &sh, int g, int *lead) {
  *lead = min(max(sh.group_start[g], 0), c.batch - 1);
  const int n = min(max(c.kv_len[*lead], 0), c.cap);
  return min(min(max(sh.prefix_len[g], 0), sh.max_prefix), n) >> c.plog << c.plog;
}
// Group of sequence b, -1: none (group_start rises)
__device__ __forceinline__ int shared_group(const CacheShared &sh, int b) {
  int lo = 0, hi = sh.groups;                    // groups that end at or before b are before lo
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sh.group_start[mid + 1] <= b)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo < sh.groups && sh.group_start[lo] <= b ? lo : -1;
}

// Entry of a launch's list: rows and keys, the row of the page table and the pages left out at its start. Where groups
// share a past, their rows over the shared keys come first, all of them seen, then each sequence's rows over its own
// keys, slots counted from the first of them.
struct AttnSeq {
  CacheSeq s;
  int row, skip;   // table row, pages
  int shared;      // 0: all of the rows' keys, 1: those that their group shares, 2: the others
};
__device__ __forceinline__ AttnSeq shared_entry(const CacheAttnArgs &a, int g) {
  const CacheArgs &c = a.c;
  AttnSeq x;
  x.s.n = shared_keys(c, a.sh, g, &x.row);
  const int b0 = min(max(a.sh.group_start[g], 0), c.batch), b1 = min(max(a.sh.group_start[g + 1], b0), c.batch);
  x.s.q0 = min(max(c.q_start[b0], 0), c.rows);
  x.s.nq = x.s.n > 0 ? min(max(c.q_start[b1], x.s.q0), c.rows) - x.s.q0 : 0;
  x.s.start = x.s.n;                             // (cache_limit: every row sees all)
  x.skip = 0;
  x.shared = 1;
  return x;
}
__device__ __forceinline__ AttnSeq own_entry(const CacheAttnArgs &a, int b) {
  AttnSeq x;
  x.s = cache_seq(a.c, b);
  x.row = b;
  x.skip = x.shared = 0;
  if (a.sh.groups > 0) {
    const int g = shared_group(a.sh, b);
    int lead;
    const int p = g < 0 ? 0 : shared_keys(a.c, a.sh, g, &lead), q = x.s.n - x.s.start;
    x.s.n = min(max(x.s.n - p, 0), a.sh.max_own);
    x.s.start = x.s.n - q;
    x.skip = p >> a.c.plog;
    x.shared = p > 0 ? 2 : 0;
  }
  return x;
}

// Ranges of keys that the rows of a block which see up to `keys` of them are cut
// into, one block each (the first is always there: it writes zeros where nothing is seen)
__device__ __forceinline__ int range_count(const CacheAttnArgs &a, int keys, bool past = false) {
  const int range = past ? a.past_range : a.range;
  return (past ? a.past_splits : a.splits) > 1 ? max(1, (keys + range - 1) / range) : 1;
}

// Part sp (ranges of shared keys come first) of packed row `row` and a head: HD unnormalised values at
// part + slot * HD, its reference and sum at part + slots * HD + 2 slot
__device__ __forceinline__ int64_t part_slot(const CacheAttnArgs &a, int sp, int row, int head) {
  return ((int64_t)sp * a.c.rows + row) * a.c.heads + head;
}
__device__ __forceinline__ float *part_ml(const CacheAttnArgs &a, int64_t slot) {
  return a.part + (int64_t)(a.past_splits + a.splits) * a.c.rows * a.c.heads * a.c.hd + 2 * slot;
}

// What a block of an attention launch works on: query rows [m0, m0 + rpb) of
// `count` of sequence b and kv head h, range sp of nr of the keys that they see.
// Blocks are numbered sequence by sequence with the lengths of the device, so those that the host's bounds
// allow for but no chunk needs come last. (2,048 single tokens over 100 keys each, 16 heads of 64: 1,432 us when every
// block counted the sequences before its own, 515 without.) Within a sequence kv heads go fastest: with 8 (or a divisor
// or multiple) of them the blocks of one run on one XCD (or its group) and share K and V in that L2; the last rows,
// which see the most, come first (8,192 rows causal over themselves, 16 heads of 128: 312 us from the first, 271 so).
struct AttnBlock {
  CacheSeq s;
  const int32_t *tab;   // its pages, and the last one's number
  int tab_last;
  int h, m0, count, group, sp, nr;
  int range;            // keys of a range
  int lim_lo, lim_hi;   // keys seen by the first and the last row
  int part;             // the range's number among the parts of its rows, -1: what the block computes is the result
  bool live;
  __device__ __forceinline__ explicit AttnBlock(const CacheAttnArgs &a) : live(false) {
    const CacheArgs &c = a.c;
    int row, skip = 0, shared = 0;
    const int lane = threadIdx.x & 63;
    group = c.heads / c.kvh;
    int li = blockIdx.x;
    // the entry whose blocks have this one among them; li counts within it, or past all of them
    auto among = [&](int entries, bool past) {
      for (int e0 = 0; e0 < entries; e0 += 64) {
        int cnt = 0;
        AttnSeq x{};
        if (e0 + lane < entries) {
          x = past ? shared_entry(a, e0 + lane) : own_entry(a, e0 + lane);
          cnt = (x.s.nq * group + a.rpb - 1) / a.rpb * range_count(a, x.s.n, past) * c.kvh;
        }
        const int sum = wave_scan(cnt);
        const uint64_t found = __ballot(sum > li);
        if (found) {
          const int k = __builtin_ctzll(found);
          li -= __builtin_amdgcn_readlane(sum - cnt, k);
          s.q0 = __builtin_amdgcn_readlane(x.s.q0, k);
          s.nq = __builtin_amdgcn_readlane(x.s.nq, k);
          s.n = __builtin_amdgcn_readlane(x.s.n, k);
          s.start = __builtin_amdgcn_readlane(x.s.start, k);
          row = __builtin_amdgcn_readlane(x.row, k);
          skip = __builtin_amdgcn_readlane(x.skip, k);
          shared = __builtin_amdgcn_readlane(x.shared, k);
          return true;
        }
        li -= __builtin_amdgcn_readlane(sum, 63);
      }
      return false;
    };
    if (a.sh.groups == 0 || a.only == 2 || !among(a.sh.groups, true)) {
      if (a.only == 1) return;
      if (c.batch == 1 || (a.splits == 1 && c.max_q * group <= a.rpb)) {   // one sequence, or a block for each and kv head
        int b = 0;
        if (c.batch > 1) {
          b = uni(li / c.kvh);
          if (b >= c.batch) return;
          li -= b * c.kvh;
        }
        const AttnSeq x = own_entry(a, b);
        s.q0 = uni(x.s.q0);
        s.nq = uni(x.s.nq);
        s.n = uni(x.s.n);
        s.start = uni(x.s.start);
        row = b;
        skip = uni(x.skip);
        shared = uni(x.shared);
      } else if (!among(c.batch, false)) {
        return;
      }
    }
    li = uni(li);
    skip = min(skip, c.table_ld - 1);            // (pages beyond the table hold no keys)
    tab = c.table + (int64_t)row * c.table_ld + skip;
    tab_last = c.table_ld - 1 - skip;
    range = shared == 1 ? a.past_range : a.range;
    count = s.nq * group;
    const int q = uni(li / c.kvh), nrg = range_count(a, s.n, shared == 1), back = uni(q / nrg);
    const int rb = (count + a.rpb - 1) / a.rpb - 1 - back;
    h = li - q * c.kvh;
    sp = q - back * nrg;
    m0 = rb * a.rpb;
    if (m0 < 0) return;
    lim_lo = uni(cache_limit(c, s, cache_row(c, m0)));
    lim_hi = uni(cache_limit(c, s, cache_row(c, min(m0 + a.rpb, count) - 1)));
    nr = uni(range_count(a, lim_hi, shared == 1));
    part = nr > 1 || shared ? (shared == 1 ? sp : a.past_splits + sp) : -1;
    live = sp < nr;
  }
};

// ---------------------------------------------------------------- parts of a split launch
// o = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s with M the largest m_s, ranges
// in order (of shared keys first); thread: one row, 4 columns. 4.4 us for 384 rows, 16 heads of 64, five ranges: a launch and its
// latency.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_cache_attn_combine(CacheAttnArgs a) {
  constexpr int TPR = HD / 4;
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh, b = blockIdx.y;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int e = 4 * (int)(gid % TPR), q = (int)(gid / TPR);   // q: chunk row x heads + head
  const AttnSeq as = own_entry(a, b);
  const CacheSeq s = as.s;
  if (q >= s.nq * c.heads) return;
  const int i = q / c.heads, head = q - i * c.heads, h = head / group, mr = i * group + head - h * group;
  const int last = min(mr / a.rpb * a.rpb + a.rpb, s.nq * group) - 1;   // of the row's block
  const int own = range_count(a, cache_limit(c, s, cache_row(c, last)));
  if (own == 1 && !as.shared) return;            // finished by its block
  const int past = as.shared ? range_count(a, as.skip << c.plog, true) : 0;
  const int nr = past + own, gap = a.past_splits - past;   // part of range u: u, or u + gap of the own ones
  const int64_t at0 = part_slot(a, 0, s.q0 + i, head), step = (int64_t)c.rows * c.heads;
  float mx = -INFINITY, den = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int u0 = 0; u0 < nr; u0 += 8) {           // eight ranges' loads at a time
    float2 ml[8];
    f32x4 y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (u0 + u < nr) {
        const int64_t at = at0 + (u0 + u + (u0 + u < past ? 0 : gap)) * step;
        ml[u] = *(const float2 *)part_ml(a, at);
        y[u] = *(const f32x4 *)(a.part + at * HD + e);
      }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (u0 + u < nr) {
        const float mn = fmaxf(mx, ml[u].x), ref = mn == -INFINITY ? 0.f : mn;
        const float wo = __builtin_amdgcn_exp2f(mx - ref), wn = __builtin_amdgcn_exp2f(ml[u].x - ref);
        mx = mn;
        den = wo * den + wn * ml[u].y;
#pragma unroll
        for (int d = 0; d < 4; ++d) x[d] = wo * x[d] + wn * y[u][d];
      }
  }
  T *O = (T *)a.o + (int64_t)(s.q0 + i) * a.ldo + (int64_t)head * HD + e;
  if constexpr (sizeof(T) == 2) {
    bf16x4 y;
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] = (__bf16)(den == 0.f ? 0.f : x[d] / den);
    *(bf16x4 *)O = y;
  } else {
#pragma unroll
    for (int d = 0; d < 4; ++d) O[d] = den == 0.f ? 0.f : x[d] / den;
  }
  if (a.lse && e == 0)
    a.lse[(int64_t)(s.q0 + i) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
}

// The same for few rows of many parts: a block for each row and head, whose groups of HD / 4 threads take every
// 1024 / HD-th part each and meet in LDS. (32 rows of 32 heads of 128, 33 parts: 9.7 us with a thread for all of them, 7.6 so.)
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_cache_attn_combine_few(CacheAttnArgs a) {
  constexpr int TPR = HD / 4, G = 256 / TPR;
  __shared__ f32x4 xs[G][TPR];
  __shared__ float2 mls[G];
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh, b = blockIdx.y, q = blockIdx.x;   // q: chunk row x heads + head
  const int e = 4 * (int)(threadIdx.x % TPR), g = threadIdx.x / TPR;
  const AttnSeq as = own_entry(a, b);
  const CacheSeq s = as.s;
  if (q >= s.nq * c.heads) return;
  const int i = q / c.heads, head = q - i * c.heads, h = head / group, mr = i * group + head - h * group;
  const int last = min(mr / a.rpb * a.rpb + a.rpb, s.nq * group) - 1;   // of the row's block
  const int own = range_count(a, cache_limit(c, s, cache_row(c, last)));
  if (own == 1 && !as.shared) return;            // finished by its block
  const int past = as.shared ? range_count(a, as.skip << c.plog, true) : 0;
  const int nr = past + own, gap = a.past_splits - past;
  const int64_t at0 = part_slot(a, 0, s.q0 + i, head), step = (int64_t)c.rows * c.heads;
  float mx = -INFINITY, den = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  auto join = [&](float2 ml, f32x4 y) __attribute__((always_inline)) {
    const float mn = fmaxf(mx, ml.x), ref = mn == -INFINITY ? 0.f : mn;
    const float wo = __builtin_amdgcn_exp2f(mx - ref), wn = __builtin_amdgcn_exp2f(ml.x - ref);
    mx = mn;
    den = wo * den + wn * ml.y;
#pragma unroll
    for (int d = 0; d < 4; ++d) x[d] = wo * x[d] + wn * y[d];
  };
  for (int u0 = g; u0 < nr; u0 += 4 * G) {       // four ranges' loads at a time
    float2 ml[4];
    f32x4 y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int p = u0 + u * G;
      if (p < nr) {
        const int64_t at = at0 + (p + (p < past ? 0 : gap)) * step;
        ml[u] = *(const float2 *)part_ml(a, at);
        y[u] = *(const f32x4 *)(a.part + at * HD + e);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (u0 + u * G < nr) join(ml[u], y[u]);
  }
  xs[g][e / 4] = x;
  if (e == 0) mls[g] = make_float2(mx, den);
  __syncthreads();
  if (g > 0) return;
#pragma unroll
  for (int u = 1; u < G; ++u) join(mls[u], xs[u][e / 4]);
  T *O = (T *)a.o + (int64_t)(s.q0 + i) * a.ldo + (int64_t)head * HD + e;
  if constexpr (sizeof(T) == 2) {
    bf16x4 y;
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] = (__bf16)(den == 0.f ? 0.f : x[d] / den);
    *(bf16x4 *)O = y;
  } else {
#pragma unroll
    for (int d = 0; d < 4; ++d) O[d] = den == 0.f ? 0.f : x[d] / den;
  }
  if (a.lse && e == 0)
    a.lse[(int64_t)(s.q0 + i) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
}

// ---------------------------------------------------------------- tiles
__device__ __forceinline__ float unround(float sum, float rounded) { return rounded == 0.f ? 1.f : sum / rounded; }

template <int HD>
struct Few {
  static constexpr int ROWB = HD * 2;            // bytes of a row
  static constexpr int RPL = 1024 / ROWB;        // rows per LDS load of a wave (4 or 8)
  static constexpr int KT = HD == 128 ? 16 : 32; // keys per tile
  static constexpr int NK = KT / 16;
  static constexpr int LPH = 16 / RPL;           // LDS loads per 16 rows (4 or 2)
  static constexpr int TILE = KT * ROWB;
  // 16-byte chunk c of row r lies at c ^ key(r): the 16 rows of a K fragment, and
  // the 4 rows that 16 lanes of a transposed V read take (a pair of chunks each), spread over the banks
  static __device__ __forceinline__ int kkey(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int vkey(int r) { return HD == 128 ? 2 * (r & 3) : 2 * ((r >> 1) & 1); }
  // transposed V reads of dims 16 i ..: lane offset i % VR, the rest a constant
  static constexpr int VR = HD == 128 ? 4 : 2;
};

// V^T fragment (16 dims, 32 keys): keys 4 lg .. of the first and the second 16 rows
template <int HD>
__device__ __forceinline__ bf16x8 v_frag(const char *p) {
  const s16x4 v0 = lds_read_tr(p), v1 = lds_read_tr(p + 16 * Few<HD>::ROWB);
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Element offset of row `slot` of a sequence (entries tab) and kv head h in k and v
__device__ __forceinline__ int64_t slot_row(const CacheArgs &c, const int32_t *tab, int h, int slot) {
  return ((((int64_t)cache_page(c, tab[slot >> c.plog]) * c.kvh + h) << c.plog) + (slot & ((1 << c.plog) - 1))) * c.hd;
}

// ---------------------------------------------------------------- weights of 32 rows over KK tiles of 16 keys
template <int HD, int KK>
__device__ __forceinline__ float rowmax(const f32x4 (&S)[KK][2], int t) {
  float mx = S[0][t][0];
#pragma unroll
  for (int k = 0; k < KK; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) mx = fmaxf(mx, S[k][t][e]);
  return quad_max(mx);
}
// Whether a row of the wave has a reference so large that its rounding, half a step of m = sc max S, changes what
// fma(S, sc, -m) is for the largest S by more than 2^-4: the weights of such a row would pass float32's range or all vanish.
__device__ __forceinline__ bool far_out(float m) { return __any(fabsf(m) > 0x1p20f); }

// P of one row tile, its lane sums. Far out S sc is rounded like the reference before m is taken off (S is scaled in
// place), so that the largest score has weight 1.
template <int KK>
__device__ __forceinline__ float weights(f32x4 (&S)[KK][2], bf16x8 (&pf)[KK / 2], int t, float sc, float m) {
  float ls = 0.f;
  if (far_out(m)) {
#pragma unroll
    for (int k = 0; k < KK; ++k) S[k][t] *= sc;
    sc = 1.f;
  }
#pragma unroll
  for (int k = 0; k < KK; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(S[k][t][e], sc, -m));
      ls += p;
      pf[k >> 1][4 * (k & 1) + e] = (__bf16)p;
    }
  return ls;
}

// ---------------------------------------------------------------- launches
// most blocks of one range of keys each
inline int64_t attn_blocks(int rpb, const CacheArgs &c) {
  const int64_t group = c.heads / c.kvh, per = (c.max_q * group + rpb - 1) / rpb;
  return c.kvh * std::min<int64_t>(c.batch * per, c.rows * group / rpb + c.batch);
}
inline size_t attn_part_bytes(const CacheArgs &c, int splits) {
  return (size_t)splits * c.rows * c.heads * (c.hd + 2) * sizeof(float);
}

template <typename T, int HD>
hipError_t launch_combine_t(const CacheAttnArgs &a, bool few, hipStream_t s) {
  const int64_t items = (int64_t)a.c.max_q * a.c.heads;
  if (few)
    hipLaunchKernelGGL((k_cache_attn_combine_few<T, HD>), dim3((unsigned)items, a.c.batch), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_cache_attn_combine<T, HD>), dim3((unsigned)((items * (HD / 4) + 255) / 256), a.c.batch), dim3(256), 0, s, a);
  return hipGetLastError();
}
// few: where parts are many and their rows do not fill the device
inline hipError_t launch_combine(int dtype, const CacheAttnArgs &a, bool few, hipStream_t s) {
  if (dtype == 1) return a.c.hd == 128 ? launch_combine_t<bf16_t, 128>(a, few, s) : launch_combine_t<bf16_t, 64>(a, few, s);
  return a.c.hd == 128 ? launch_combine_t<float, 128>(a, few, s) : launch_combine_t<float, 64>(a, few, s);
}
inline bool few_rows_of_many_parts(const CacheAttnArgs &a) {
  return a.past_splits + a.splits > 8 && (int64_t)a.c.max_q * a.c.batch * a.c.heads <= 4096;
}

// Rows per block and ranges over the keys that groups share [0] and over their sequences' own keys [1].
// Both kinds of blocks go out in one launch, so that the compute units that one leaves idle do the other, or
// in two, each with blocks of its own height: many sequences with few own keys want low ones (1,024 tokens of 32 heads on 8
// of 128 off 8,128 shared keys, 65 own ones each: 542 us in one launch, 230 in two; 64 of 16 heads of 64 off 16,000, up to 442 own
// ones: 65 and 45; 32 of 32 heads on 8 off 24,448, up to 900 own ones: 48 and 53,
// both before waves without rows were spared the work).
//
// By estimate: all blocks' times over the places for them (two a compute unit for blocks of 16 rows), of several
// groups or sequences two thirds of the blocks that the bounds allow for, and a third of the longest one's; 5 us for a start and
// end and tile[] us per 64 keys in blocks of 16, 32, 128 and 256 rows; the parts written and read; 8 us for a further launch.
//
// All rows are divided into parts, for few rows the price of reading shared keys once (32 tokens of 32 heads on 8 off 24,448
// keys: 45.2 us, 273 with the unshared call over the same pages). Whole frames, which the products bound, pay it for nothing: four
// of 384 rows, 16 heads of 64, off 3,456 keys 54.8 us, 47.5 unshared; of 2,040 rows, 16 heads of 128, off 24,448 keys 1,537 and 1,446.
inline SharedPlan plan_shared(int dtype, const CacheArgs &c, const CacheShared &sh, const double (&tile)[4]) {
  CacheArgs of[2] = {c, c};
  of[0].batch = sh.groups;
  of[0].max_q = c.rows;
  of[0].cap = std::min(c.cap, sh.max_prefix);
  of[1].cap = std::min(c.cap, sh.max_own);
  const double cus = std::max(1, device_cus()), part = (double)attn_part_bytes(c, 1) * 2 / 4e6;
  constexpr int ROWS[4] = {16, 32, 128, 256};
  // one kind of blocks at ROWS[r] and n ranges: their number, the ranges, and for the estimate the sum of the
  // times and the longest
  struct Kind {
    int64_t blocks, range, splits;
    double sum, there, top;
  };
  auto kind = [&](int k, int r, int64_t n) {
    const int64_t step = ROWS[r] == 128 && c.hd == 64 ? 128 : 64, cap = std::max(of[k].cap, 1);
    Kind x;
    x.range = ((cap + n - 1) / n + step - 1) / step * step;
    x.splits = std::max<int64_t>(1, (cap + x.range - 1) / x.range);
    x.blocks = std::max<int64_t>(1, attn_blocks(ROWS[r], of[k])) * x.splits;
    x.there = (double)x.blocks * (of[k].batch > 1 ? 2.0 / 3 : 1.0);
    x.top = (double)x.range / 64 * tile[r] + 5.0;
    x.sum = x.top * x.there;
    return x;
  };
  auto time = [&](double sum, double there, double top, int r) {
    const double places = r == 0 ? 2 * cus : cus;
    return there <= places ? top : sum / places + 0.35 * top;
  };
  // heights for so many rows of a (group or sequence, kv head)
  auto first = [&](int64_t m) { return dtype == 0 || (m > 16 && m <= 32) ? 1 : 0; };
  auto last = [&](int64_t m) { return dtype == 0 || (m > 16 && m <= 32) ? 1 : m <= 16 ? 0 : 3; };
  // 1, 2, 3, 4, 6, 8, 12, .. 64 ranges, or as many as fill the compute units
  auto ranges = [&](int k, int r, int i) -> int64_t {
    const int64_t n = i == 12           ? (int64_t)cus / std::max<int64_t>(1, attn_blocks(ROWS[r], of[k]))
                      : i % 2 || i == 0 ? int64_t(1) << (i + 1) / 2
                                        : int64_t(3) << (i / 2 - 1);
    return n == 1 || (n > 1 && of[k].cap >= 256 * n) ? n : 0;
  };
  const int64_t group = c.heads / c.kvh, m[2] = {c.rows * group, c.max_q * group};
  SharedPlan best{}, apart{};
  double t_best = 0, t_apart = 8.0;
  for (int r = first(m[0]); r <= last(m[0]); ++r)
    for (int i = 0; i < 13; ++i) {
      const int64_t n0 = ranges(0, r, i);
      if (n0 == 0) continue;
      const Kind x = kind(0, r, n0);
      for (int64_t n1 = 1; n1 <= 4; n1 *= 2) {
        if (n1 > 1 && of[1].cap < 256 * n1) continue;
        const Kind y = kind(1, r, n1);
        const double t = time(x.sum + y.sum, x.there + y.there, std::max(x.top, y.top), r) + part * (double)(x.splits + y.splits);
        if (t_best == 0 || t < t_best) {
          t_best = t;
          best = SharedPlan{true, {x.blocks, y.blocks}, {ROWS[r], ROWS[r]}, {(int)x.range, (int)y.range},
                            {(int)x.splits, (int)y.splits}, 0};
        }
      }
    }
  for (int k = 0; k < 2; ++k) {
    double t_kind = 0;
    for (int r = first(m[k]); r <= last(m[k]); ++r)
      for (int i = 0; i < 13; ++i) {
        const int64_t n = ranges(k, r, i);
        if (n == 0) continue;
        const Kind x = kind(k, r, n);
        const double t = time(x.sum, x.there, x.top, r) + part * (double)x.splits;
        if (t_kind == 0 || t < t_kind) {
          t_kind = t;
          apart.blocks[k] = x.blocks;
          apart.rpb[k] = ROWS[r];
          apart.range[k] = (int)x.range;
          apart.splits[k] = (int)x.splits;
        }
      }
    t_apart += t_kind;
  }
  SharedPlan &p = t_apart < t_best ? apart : best;
  p.scratch = attn_part_bytes(c, p.splits[0] + p.splits[1]);
  return p;
}
template <class Launch>
hipError_t launch_shared(int dtype, const CacheAttnArgs &in, const SharedPlan &p, Launch &&launch, hipStream_t s) {
  if (in.c.rows <= 0 || in.c.max_q <= 0) return hipSuccess;
  CacheAttnArgs a = in;
  a.past_range = p.range[0];
  a.past_splits = p.splits[0];
  a.range = p.range[1];
  a.splits = p.splits[1];
  hipError_t e = hipSuccess;
  if (!p.together) {
    a.only = 1;
    a.blocks = (unsigned)p.blocks[0];
    a.rpb = p.rpb[0];
    e = launch(dtype, a, s);
    if (e != hipSuccess) return e;
    a.only = 2;
  }
  a.blocks = (unsigned)(p.blocks[1] + (p.together ? p.blocks[0] : 0));
  a.rpb = p.rpb[1];
  e = launch(dtype, a, s);
  return e != hipSuccess ? e : launch_combine(dtype, a, few_rows_of_many_parts(a), s);
}
// a launch over all keys of every sequence
inline unsigned attn_grid(const CacheAttnArgs &a) { return (unsigned)(attn_blocks(a.rpb, a.c) * a.splits); }

}  // namespace
}  // namespace wdc
