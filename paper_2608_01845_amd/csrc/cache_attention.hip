// Attention of chunks of new rows over a paged key/value cache, and the weight
// that each cached key received from it.
//
// A chunk's rows and the query heads that share a kv head are one axis of query
// rows, m = i * group + g, so a key tile is read once for all of them. Row i sees
// the slots below cache_limit(i): limits grow with i, so of the key tiles of a
// block of rows a first part is seen by all rows whole, a second part in part, and
// the rest by none and is left out.
#include "common.h"

#include <algorithm>
#include <type_traits>

namespace wdc {
namespace {

constexpr int RSRC_WORD3 = 0x00020000;   // raw buffer descriptor word 3
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ void lds_load16(__amdgpu_buffer_rsrc_t r, char *lds, int voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)lds, 16, voff, soff, 0, 0);
}
// Four rows of 16 columns of 2 bytes, each read as 4 x 8 bytes by the lanes of a
// group of 16 in row order, come back transposed: lane c of the group gets column c.
__device__ __forceinline__ s16x4 lds_read_tr(const char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
}
// s_waitcnt vmcnt(N), the other counters untouched
template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
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

// Entries of one sequence's page table, asked for in rising order by a whole
// wave: 64 entries in a register, the next 64 on their way.
struct PageWalk {
  const int32_t *tab;
  int last, base, pages, cur, next;
  __device__ __forceinline__ int fetch(int i) const { return tab[min(i + (int)(threadIdx.x & 63), last)]; }
  __device__ __forceinline__ void init(const CacheArgs &a, int b, int first) {
    tab = a.table + (int64_t)b * a.table_ld;
    last = a.table_ld - 1;
    pages = a.pages;
    base = first;
    cur = fetch(base);
    next = fetch(base + 64);
  }
  __device__ __forceinline__ int get(int i) {
    while (i - base >= 64) {
      cur = next;
      base += 64;
      next = fetch(base + 64);
    }
    return min(max(__builtin_amdgcn_readlane(cur, i - base), 0), pages - 1);
  }
};

// a sequence's lengths as wave-uniform values
__device__ __forceinline__ CacheSeq uniform_seq(const CacheArgs &a, int b) {
  CacheSeq s = cache_seq(a, b);
  s.q0 = __builtin_amdgcn_readfirstlane(s.q0);
  s.nq = __builtin_amdgcn_readfirstlane(s.nq);
  s.n = __builtin_amdgcn_readfirstlane(s.n);
  s.start = __builtin_amdgcn_readfirstlane(s.start);
  return s;
}

// Block of a launch over (sequence, kv head) x per blocks each. With the XCD order
// the blocks of one (sequence, kv head) share an XCD, and so its K and V in that L2.
__device__ __forceinline__ void cache_block(const CacheArgs &c, int per, int &bh, int &li) {
  if (c.xcd_order) {
    li = blockIdx.x >> 3;
    bh = (blockIdx.x & 7) + 8 * (li / per);
  } else {
    li = blockIdx.x;
    bh = li / per;
  }
  li %= per;
}

// ---------------------------------------------------------------- bf16, few rows
// RT tiles of 16 query rows per block of four waves; wave w takes key tiles w, w +
// 4, .. of 32 keys of the block's range and the four partial softmaxes meet at the
// end. What bounds it is the stream of K and V: a wave keeps one tile of 32 keys
// under way (direct buffer loads into its own part of LDS, no block barrier) while it
// works on the other: hd 128: 16 KB a tile, 64 to 128 KB under way per CU.
//
// S^T = K Q^T (A: 16 keys, B: 16 rows) leaves lane (lr, lg) the keys 4 lg + e of
// row lr; these values of two key tiles are the B operand of O^T = V^T P^T, whose A
// operand is V^T: rows 4 lg .. 4 lg + 3 of V read transposed from LDS.
//
// Softmax in base 2 with a reference m per row that moves when a score passes it
// by more than 8: scores are scaled by log2(e)/sqrt(hd) in float32, weights are summed in
// float32 and rounded to bf16 once for the product with V (as its operand type).
template <int HD>
struct Few {
  static constexpr int ROWB = HD * 2;            // bytes of a row
  static constexpr int RPL = 1024 / ROWB;        // rows per load of a wave (4 or 8)
  static constexpr int LPT = 32 / RPL;           // loads per tile of 32 rows
  static constexpr int TILE = 32 * ROWB;
  static constexpr int WAVE = 4 * TILE;          // two K and two V tiles
  // 16-byte chunk c of row r lies at c ^ key(r): the 16 rows of a K fragment, and
  // the rows of a transposed V read in pairs of chunks, spread over the banks
  static __device__ __forceinline__ int kkey(int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int vkey(int r) { return HD == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
};

template <int HD, int RT>
__global__ __launch_bounds__(256, 1) void k_cache_attn_few(CacheAttnArgs a) {
  using F = Few<HD>;
  constexpr int NC = HD / 32, NI = HD / 16;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float ml[4][2][16 * RT];
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh;
  const int nrb = (c.max_q * group + 16 * RT - 1) / (16 * RT);
  int bh, li;                                    // (sequence, kv head); row block and key range
  cache_block(c, nrb * a.splits, bh, li);
  const int sp = li % a.splits, rb = li / a.splits;
  const int b = bh / c.kvh, h = bh % c.kvh;
  const CacheSeq s = uniform_seq(c, b);
  const int m0 = rb * 16 * RT, count = s.nq * group;
  if (m0 >= count) return;

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mlast = min(m0 + 16 * RT, count) - 1;
  const int lim_lo = cache_limit(c, s, m0 / group), lim_hi = cache_limit(c, s, mlast / group);
  const int tiles = (lim_hi + 31) / 32;
  const int t0 = (int)((int64_t)sp * tiles / a.splits), t1 = (int)((int64_t)(sp + 1) * tiles / a.splits);

  const float sc = LOG2E / sqrtf((float)HD);
  bf16x8 qf[RT][NC];
  int lim[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int m = m0 + 16 * t + lr, mm = min(m, mlast), i = mm / group;
    lim[t] = m < count ? cache_limit(c, s, i) : 0;
    const bf16_t *Q = (const bf16_t *)a.q + (int64_t)(s.q0 + i) * a.ldq + (int64_t)(h * group + mm % group) * HD + 8 * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) qf[t][j] = *(const bf16x8 *)(Q + 32 * j);
  }

  char *mine = smem + w * F::WAVE;
  int kvo[F::LPT / 2], vvo[F::LPT / 2];          // byte offsets in 16 rows of K and V
#pragma unroll
  for (int i = 0; i < F::LPT / 2; ++i) {
    const int r = i * F::RPL + lane / (HD / 8), ch = lane % (HD / 8);
    kvo[i] = r * F::ROWB + (ch ^ F::kkey(r)) * 16;
    vvo[i] = r * F::ROWB + (ch ^ F::vkey(r)) * 16;
  }
  int kro[NC];                                   // K fragment of rows lr, dims 32 c + 8 lg
#pragma unroll
  for (int j = 0; j < NC; ++j) kro[j] = lr * F::ROWB + ((4 * j + lg) ^ F::kkey(lr)) * 16;
  int vro[NI];                                   // transposed V read of rows 4 lg .. + 3, dims 16 i ..
  {
    const int r = 4 * lg + ((lane & 15) >> 2), j = lane & 3;
#pragma unroll
    for (int i = 0; i < NI; ++i) vro[i] = r * F::ROWB + ((2 * i + (j >> 1)) ^ F::vkey(r)) * 16 + 8 * (j & 1);
  }
  PageWalk pw;
  pw.init(c, b, (32 * t0) >> c.plog);
  const int pmask = (1 << c.plog) - 1;
  // tile t into slot j: halves of 16 rows, each on one page. Rows past the cache's
  // end lie outside the buffer range and arrive as zeros, whatever they hold.
  auto load = [&](int t, int j) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int key = 32 * t + 16 * hf;
      const int pg = pw.get(key >> c.plog);
      const int64_t off = (((((int64_t)pg * c.kvh + h) << c.plog) + (key & pmask)) * HD) * 2;
      const int bytes = min(max(s.n - key, 0), 16) * F::ROWB;
      const __amdgpu_buffer_rsrc_t kd = __builtin_amdgcn_make_buffer_rsrc((char *)c.k + off, (short)0, bytes, RSRC_WORD3);
      const __amdgpu_buffer_rsrc_t vd = __builtin_amdgcn_make_buffer_rsrc((char *)c.v + off, (short)0, bytes, RSRC_WORD3);
#pragma unroll
      for (int i = 0; i < F::LPT / 2; ++i)
        lds_load16(kd, mine + j * F::TILE + hf * 16 * F::ROWB + i * 1024, kvo[i], 0);
#pragma unroll
      for (int i = 0; i < F::LPT / 2; ++i)
        lds_load16(vd, mine + (2 + j) * F::TILE + hf * 16 * F::ROWB + i * 1024, vvo[i], 0);
    }
  };

  f32x4 o[RT][NI];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  int slot = 0;
  if (t0 + w < t1) load(t0 + w, 0);
  for (int t = t0 + w; t < t1; t += 4, slot ^= 1) {
    if (t + 4 < t1) {
      load(t + 4, slot ^ 1);
      wait_vm<2 * F::LPT>();
    } else {
      wait_vm<0>();
    }
    asm volatile("" ::: "memory");
    const char *kt = mine + slot * F::TILE, *vt = mine + (2 + slot) * F::TILE;
    f32x4 S[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int k = 0; k < 2; ++k) S[r][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bf16x8 kf = *(const bf16x8 *)(kt + k * 16 * F::ROWB + kro[j]);
#pragma unroll
        for (int r = 0; r < RT; ++r) S[r][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][j], S[r][k], 0, 0, 0);
      }
    const bool part = 32 * t + 32 > lim_lo;      // some row does not see the whole tile
    bf16x8 pf[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = S[r][k][e] * sc;
          if (part && 32 * t + 16 * k + 4 * lg + e >= lim[r]) x = -INFINITY;
          S[r][k][e] = x;
          mx = fmaxf(mx, x);
        }
      mx = quad_max(mx);
      if (__any(mx > m[r] + 8.f)) {
        const float mn = fmaxf(m[r], mx), al = mn == m[r] ? 1.f : __builtin_amdgcn_exp2f(m[r] - mn);
        m[r] = mn;
        l[r] *= al;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[r][i][e] *= al;
      }
      const float ref = m[r] == -INFINITY ? 0.f : m[r];   // a row that has seen nothing yet
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(S[r][k][e] - ref);
          l[r] += p;
          pf[r][4 * k + e] = (__bf16)p;
        }
    }
    // A key that a row does not see has weight 0, but 0 times an infinity or NaN
    // of its V is NaN in a matrix product. Tiles seen in part are looked over, and
    // one that holds such a value is multiplied key by key.
    bool odd = false;
    if (part) {
#pragma unroll
      for (int i = 0; i < F::LPT; ++i) {
        const uint4 u = *(const uint4 *)(vt + i * 1024 + lane * 16);
        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) odd |= (x[q] & 0x7f80u) == 0x7f80u || (x[q] & 0x7f800000u) == 0x7f800000u;
      }
      odd = __any(odd);
    }
    if (odd) {
      for (int k = 0; k < 2; ++k)
        for (int e = 0; e < 4; ++e)
          for (int g = 0; g < 4; ++g) {
            const int key = 16 * k + 4 * g + e;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
              float p = 0.f;                     // of key and row lr, held by lane group g
#pragma unroll
              for (int q = 0; q < 8; ++q)
                if (q == 4 * k + e) p = (float)pf[r][q];
              p = __shfl(p, 16 * g + lr, 64);
              if (32 * t + key < lim[r])
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                  for (int d = 0; d < 4; ++d) {
                    const int col = 16 * i + 4 * lg + d;
                    o[r][i][d] += p * bf2f(*(const bf16_t *)(vt + key * F::ROWB + ((col >> 3) ^ F::vkey(key)) * 16 + (col & 7) * 2));
                  }
            }
          }
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const s16x4 v0 = lds_read_tr(vt + vro[i]), v1 = lds_read_tr(vt + 16 * F::ROWB + vro[i]);
        bf16x8 vf;
        s16x4 *vp = (s16x4 *)&vf;
        vp[0] = v0;
        vp[1] = v1;
#pragma unroll
        for (int r = 0; r < RT; ++r) o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r], o[r][i], 0, 0, 0);
      }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0): the slot has been read before it is loaded again
  }

  // the four waves' parts: each leaves its rows in its own part of LDS
  float *po = (float *)mine;                     // [16 RT rows][HD]
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] = quad_sum(l[t]);
#pragma unroll
    for (int i = 0; i < NI; ++i) *(f32x4 *)(po + (16 * t + lr) * HD + 4 * ((4 * i + lg) ^ (lr & 7))) = o[t][i];
    if (lg == 0) {
      ml[w][0][16 * t + lr] = m[t];
      ml[w][1][16 * t + lr] = l[t];
    }
  }
  __syncthreads();
  constexpr int TPR = HD / 4, RPI = 256 / TPR;   // threads per row, rows per turn
  for (int r = tid / TPR; r < 16 * RT; r += RPI) {
    const int mr = m0 + r, e = tid % TPR;
    if (mr >= count) continue;
    float mx = ml[0][0][r];
#pragma unroll
    for (int u = 1; u < 4; ++u) mx = fmaxf(mx, ml[u][0][r]);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float den = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float wt = __builtin_amdgcn_exp2f(ml[u][0][r] - ref);
      den += wt * ml[u][1][r];
      const f32x4 y = *(const f32x4 *)(smem + u * F::WAVE + (r * HD + 4 * (e ^ (r & 7))) * 4);
#pragma unroll
      for (int d = 0; d < 4; ++d) x[d] += wt * y[d];
    }
    if (a.splits > 1) {
      const int64_t at = ((int64_t)bh * a.splits + sp) * (c.max_q * group) + mr;
      *(f32x4 *)(a.part + at * HD + 4 * e) = x;
      if (e == 0) {
        float *pm = a.part + (int64_t)c.batch * c.kvh * a.splits * (c.max_q * group) * HD + 2 * at;
        pm[0] = mx;
        pm[1] = den;
      }
      continue;
    }
    const float inv = den > 0.f ? 1.f / den : den != den ? den : 0.f;
    const int i = mr / group, head = h * group + mr % group;
    bf16x4 y;
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] = (__bf16)(den == 0.f ? 0.f : x[d] * inv);
    *(bf16x4 *)((bf16_t *)a.o + (int64_t)(s.q0 + i) * a.ldo + (int64_t)head * HD + 4 * e) = y;
    if (a.lse && e == 0)
      a.lse[(int64_t)(s.q0 + i) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
  }
}

// ---------------------------------------------------------------- parts of a split launch
// o = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s with M the largest m_s, ranges
// in order; thread: one row, 8 columns.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_cache_attn_combine(CacheAttnArgs a) {
  constexpr int TPR = HD / 8;
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh, rows = c.max_q * group;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int e = 8 * (int)(gid % TPR);
  const int64_t q = gid / TPR;
  const int bh = (int)(q / rows), mr = (int)(q % rows);
  if (bh >= c.batch * c.kvh) return;
  const int b = bh / c.kvh, h = bh % c.kvh;
  const CacheSeq s = cache_seq(c, b);
  if (mr >= s.nq * group) return;
  const int64_t at0 = (int64_t)bh * a.splits * rows + mr;
  const float *pm = a.part + (int64_t)c.batch * c.kvh * a.splits * rows * HD;
  float mx = -INFINITY;
  for (int u = 0; u < a.splits; ++u) mx = fmaxf(mx, pm[2 * (at0 + (int64_t)u * rows)]);
  const float ref = mx == -INFINITY ? 0.f : mx;
  float den = 0.f, x[8] = {};
  for (int u = 0; u < a.splits; ++u) {
    const int64_t at = at0 + (int64_t)u * rows;
    const float wt = __builtin_amdgcn_exp2f(pm[2 * at] - ref);
    den += wt * pm[2 * at + 1];
    const f32x4 y0 = *(const f32x4 *)(a.part + at * HD + e), y1 = *(const f32x4 *)(a.part + at * HD + e + 4);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      x[d] += wt * y0[d];
      x[4 + d] += wt * y1[d];
    }
  }
  const int i = mr / group, head = h * group + mr % group;
  T *O = (T *)a.o + (int64_t)(s.q0 + i) * a.ldo + (int64_t)head * HD + e;
  if constexpr (sizeof(T) == 2) {
    bf16x8 y;
#pragma unroll
    for (int d = 0; d < 8; ++d) y[d] = (__bf16)(den == 0.f ? 0.f : x[d] / den);
    *(bf16x8 *)O = y;
  } else {
#pragma unroll
    for (int d = 0; d < 8; ++d) O[d] = den == 0.f ? 0.f : x[d] / den;
  }
  if (a.lse && e == 0)
    a.lse[(int64_t)(s.q0 + i) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
}

// ---------------------------------------------------------------- float32
// Element offset of row `slot` of a sequence (entries tab) and kv head h in k and v
__device__ __forceinline__ int64_t slot_row(const CacheArgs &c, const int32_t *tab, int h, int slot) {
  return ((((int64_t)cache_page(c, tab[slot >> c.plog]) * c.kvh + h) << c.plog) + (slot & ((1 << c.plog) - 1))) * c.hd;
}

// float32 attention on v_mfma_f32_32x32x2_f32 (64 cycles each): a block's four
// waves share 32 rows and take every fourth key tile of 32 of the block's range. S^T = K Q^T
// leaves a lane one row and 16 keys, which O^T = V^T P^T takes one by one as its B
// operand. Bound by the matrix instructions, so K and V come straight from the
// caches: K of the next tile is asked for under this tile's softmax and P V. Keys past
// the cache's end are read as its last key and get weight 0.
template <int HD>
__global__ __launch_bounds__(256, 1) void k_cache_attn_f32(CacheAttnArgs a) {
  constexpr int NI = HD / 32, NC = HD / 8;
  typedef __attribute__((ext_vector_type(NI))) float vecn;
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh, nrb = (c.max_q * group + 31) / 32;
  int bh, li;
  cache_block(c, nrb * a.splits, bh, li);
  const int sp = li % a.splits, rb = li / a.splits, b = bh / c.kvh, h = bh % c.kvh;
  const CacheSeq s = uniform_seq(c, b);
  const int m0 = rb * 32, count = s.nq * group;
  if (m0 >= count) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int mlast = min(m0 + 32, count) - 1, mm = min(m0 + lr, mlast), row = mm / group;
  const int lim_lo = cache_limit(c, s, m0 / group), lim_hi = cache_limit(c, s, mlast / group);
  const int lim = m0 + lr < count ? cache_limit(c, s, row) : 0;
  const int tiles = (lim_hi + 31) / 32;
  const int t0 = (int)((int64_t)sp * tiles / a.splits), t1 = (int)((int64_t)(sp + 1) * tiles / a.splits);
  const int32_t *tab = c.table + (int64_t)b * c.table_ld;
  const float *Q = (const float *)a.q + (int64_t)(s.q0 + row) * a.ldq + (int64_t)(h * group + mm % group) * HD + 4 * lg;
  const float *K = (const float *)c.k + 4 * lg, *V = (const float *)c.v + NI * lr;
  const float sc = LOG2E / sqrtf((float)HD);
  f32x4 qf[NC], kf[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) qf[j] = *(const f32x4 *)(Q + 8 * j) * sc;
  f32x16 o[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  auto load_k = [&](int t) {
    const float *p = K + slot_row(c, tab, h, min(32 * t + lr, s.n - 1));
#pragma unroll
    for (int j = 0; j < NC; ++j) kf[j] = *(const f32x4 *)(p + 8 * j);
  };
  if (t0 + w < t1) load_k(t0 + w);
  for (int t = t0 + w; t < t1; t += 4) {
    vecn v[16];
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {             // four keys of one page
      const int key = 32 * t + 8 * e4 + 4 * lg, k0 = min(key, s.n - 1);
      const float *p = V + slot_row(c, tab, h, k0);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * e4 + e] = *(const vecn *)(p + (min(key + e, s.n - 1) - k0) * HD);
    }
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int d = 0; d < 4; ++d) x = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j][d], qf[j][d], x, 0, 0, 0);
    if (t + 4 < t1) load_k(t + 4);
    const bool part = 32 * t + 32 > lim_lo;
    bool odd = false;
    if (part) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (32 * t + 8 * (e / 4) + 4 * lg + e % 4 >= lim) x[e] = -INFINITY;
#pragma unroll
        for (int i = 0; i < NI; ++i) odd |= (__float_as_uint(v[e][i]) & 0x7f800000u) == 0x7f800000u;
      }
      odd = __any(odd);
    }
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, x[e]);
    const float mn = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32, 64)));
    const float ref = mn == -INFINITY ? 0.f : mn;   // a row that has seen nothing yet
    if (__any(mn > m)) {
      const float al = exp2f(m - ref);
      m = mn;
      l *= al;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= al;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      x[e] = exp2f(x[e] - ref);
      l += x[e];
    }
    if (odd) {
      // infinities or NaN among the V of keys that some row does not see: key by key
#pragma unroll
      for (int e = 0; e < 16; ++e)
        for (int g = 0; g < 2; ++g) {
          const int key = 32 * t + 8 * (e / 4) + 4 * g + e % 4;
          const float p = __shfl(x[e], 32 * g + lr, 64);
          if (key >= lim) continue;
          const float *vp = (const float *)c.v + slot_row(c, tab, h, key);
#pragma unroll
          for (int d = 0; d < 16; ++d)
#pragma unroll
            for (int i = 0; i < NI; ++i) o[i][d] += p * vp[NI * (8 * (d / 4) + 4 * lg + d % 4) + i];
        }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int i = 0; i < NI; ++i) o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e][i], x[e], o[i], 0, 0, 0);
    }
  }
  l += __shfl_xor(l, 32, 64);
  // lane: row lr, dimensions NI r + i of rows r = 8 (e / 4) + 4 lg + e % 4
  __shared__ float po[4][NI * 16][64], ml[4][2][32];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) po[w][i * 16 + e][lane] = o[i][e];
  if (lg == 0) {
    ml[w][0][lr] = m;
    ml[w][1][lr] = l;
  }
  __syncthreads();
  if (m0 + lr >= count) return;
  float mx = ml[0][0][lr], den = 0.f, wt[4];
#pragma unroll
  for (int u = 1; u < 4; ++u) mx = fmaxf(mx, ml[u][0][lr]);
  const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    wt[u] = exp2f(ml[u][0][lr] - ref);
    den += wt[u] * ml[u][1][lr];
  }
  // wave w finishes entries e = 4 w .. 4 w + 3: NI x 4 consecutive dimensions per lane
  const int head = h * group + mm % group, dim0 = NI * (8 * w + 4 * lg);
  const int64_t at = ((int64_t)bh * a.splits + sp) * (c.max_q * group) + mm;
  float *O = a.splits > 1 ? a.part + at * HD + dim0
                          : (float *)a.o + (int64_t)(s.q0 + row) * a.ldo + (int64_t)head * HD + dim0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float y = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) y += wt[u] * po[u][i * 16 + 4 * w + e][lane];
      O[NI * e + i] = a.splits > 1 ? y : den == 0.f ? 0.f : y / den;
    }
  if (w != 0 || lg != 0) return;
  if (a.splits > 1) {
    float *pm = a.part + (int64_t)c.batch * c.kvh * a.splits * (c.max_q * group) * HD + 2 * at;
    pm[0] = mx;
    pm[1] = den;
  } else if (a.lse) {
    a.lse[(int64_t)(s.q0 + row) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
  }
}

// ---------------------------------------------------------------- accumulated weights
// out[j] = decay * mass[j] (0 for the chunk's own keys) + sum over the rows that
// see key j of exp(score - lse): the row's softmax weights again from its scores and
// its log-sum-exp. Sums over rows in a fixed order, in float32.

// First chunk row that sees slot `key`
__device__ __forceinline__ int first_row(const CacheArgs &c, const CacheSeq &s, int key) {
  if (c.frame <= 0 || key < s.start) return 0;
  return (int)min((int64_t)((key - s.start) / c.frame) * c.frame, (int64_t)s.nq);
}

// The sum of key `key` (a slot of sequence b and kv head h)
__device__ __forceinline__ void mass_store(const CacheMassArgs &a, const CacheSeq &s, int b, int h, int key, float sum) {
  const CacheArgs &c = a.c;
  const int e = c.table[(int64_t)b * c.table_ld + (key >> c.plog)];
  if ((unsigned)e >= (unsigned)c.pages) return;   // a slot on no page of the cache
  const int64_t at = (((int64_t)e * c.kvh + h) << c.plog) + (key & ((1 << c.plog) - 1));
  a.out[at] = (key < s.start && a.decay != 0.f ? a.decay * a.mass[at] : 0.f) + sum;
}

// Four waves share KT keys and take every fourth tile of rows (16 of bf16, 32 of
// float32). K stays in registers (A operand), rows stream past it as the B operand; a lane
// holds one row and KT / 4 (float32: 16) keys, whose sums stay in its registers until the end.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_cache_mass(CacheMassArgs a) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int KT = BF ? 64 : 32, RQ = BF ? 16 : 32, NK = BF ? 4 : 1, NE = BF ? 4 : 16;
  constexpr int NC = BF ? HD / 32 : HD / 8;
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh, nkt = (c.cap + KT - 1) / KT;
  int bh, li;
  cache_block(c, nkt * a.splits, bh, li);
  const int sp = li % a.splits, kt = li / a.splits, b = bh / c.kvh, h = bh % c.kvh;
  const CacheSeq s = uniform_seq(c, b);
  const int key0 = kt * KT;
  if (key0 >= s.n) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane % RQ, lg = lane / RQ;
  const int32_t *tab = c.table + (int64_t)b * c.table_ld;
  const int count = s.nq * group;
  const int r_lo = first_row(c, s, key0) * group / RQ, r_hi = (count + RQ - 1) / RQ;
  const int span = max(r_hi - r_lo, 0);
  const int r0 = r_lo + (int)((int64_t)sp * span / a.splits), r1 = r_lo + (int)((int64_t)(sp + 1) * span / a.splits);
  typedef typename std::conditional<BF, bf16x8, f32x4>::type frag;
  typedef typename std::conditional<BF, f32x4, f32x16>::type acc;
  constexpr int STEP = BF ? 32 : 8, PER = BF ? 8 : 4;   // elements of a row per fragment: of the wave, of a lane
  frag kf[NK][NC];
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const T *p = (const T *)c.k + slot_row(c, tab, h, min(key0 + RQ * k + lr, s.n - 1)) + PER * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) kf[k][j] = *(const frag *)(p + STEP * j);
  }
  const float sc = LOG2E / sqrtf((float)HD);
  float sum[NK][NE] = {};
  for (int r = r0 + w; r < r1; r += 4) {
    const int m = r * RQ + lr, mm = min(m, count - 1), i = mm / group, head = h * group + mm % group;
    const T *Q = (const T *)a.q + (int64_t)(s.q0 + i) * a.ldq + (int64_t)head * HD + PER * lg;
    const float lse = a.lse[(int64_t)(s.q0 + i) * c.heads + head] * LOG2E;
    const int lim = m < count ? cache_limit(c, s, i) : 0;
    frag qf[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) qf[j] = *(const frag *)(Q + STEP * j);
    const bool part = __any(key0 + KT > lim);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      acc x;
#pragma unroll
      for (int e = 0; e < NE; ++e) x[e] = 0.f;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        if constexpr (BF) {
          x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k][j], qf[j], x, 0, 0, 0);
        } else {
#pragma unroll
          for (int d = 0; d < 4; ++d) x = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[k][j][d], qf[j][d], x, 0, 0, 0);
        }
      }
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const int key = key0 + (BF ? 16 * k + 4 * lg + e : 8 * (e / 4) + 4 * lg + e % 4);
        float p = BF ? __builtin_amdgcn_exp2f(x[e] * sc - lse) : exp2f(x[e] * sc - lse);
        if (part && key >= lim) p = 0.f;
        sum[k][e] += p;
      }
    }
  }
  __shared__ float ws[4][KT];
#pragma unroll
  for (int k = 0; k < NK; ++k)
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      float v = group_sum<16>(sum[k][e]);
      if (!BF) v += __shfl_xor(v, 16, 64);
      if (lr == 0) ws[w][BF ? 16 * k + 4 * lg + e : 8 * (e / 4) + 4 * lg + e % 4] = v;
    }
  __syncthreads();
  if (tid >= KT || key0 + tid >= s.n) return;
  const float total = ws[0][tid] + ws[1][tid] + ws[2][tid] + ws[3][tid];
  if (a.splits > 1)
    a.part[((int64_t)bh * a.splits + sp) * c.cap + key0 + tid] = total;
  else
    mass_store(a, s, b, h, key0 + tid, total);
}

__global__ __launch_bounds__(256) void k_cache_mass_combine(CacheMassArgs a) {
  const CacheArgs &c = a.c;
  const int key = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
  const CacheSeq s = cache_seq(c, b);
  if (key >= s.n) return;
  const float *p = a.part + ((int64_t)b * c.kvh + h) * a.splits * c.cap + key;
  float sum = 0.f;
  for (int u = 0; u < a.splits; ++u) sum += p[(int64_t)u * c.cap];
  mass_store(a, s, b, h, key, sum);
}

// ---------------------------------------------------------------- launches
int rows_per_block(int dtype, const CacheArgs &c) {
  if (dtype == 0) return 32;
  const int64_t m = (int64_t)c.max_q * (c.heads / c.kvh);
  return m <= 16 ? 16 : m <= 32 ? 32 : 64;
}
int64_t attn_blocks(int dtype, const CacheArgs &c) {
  const int rpb = rows_per_block(dtype, c);
  return (int64_t)c.batch * c.kvh * (((int64_t)c.max_q * (c.heads / c.kvh) + rpb - 1) / rpb);
}
size_t attn_part_bytes(const CacheArgs &c, int splits) {
  return (size_t)c.batch * c.kvh * splits * c.max_q * (c.heads / c.kvh) * (c.hd + 2) * sizeof(float);
}

template <int HD, int RT>
hipError_t launch_few(const CacheAttnArgs &a, hipStream_t s) {
  constexpr int LDS = 4 * Few<HD>::WAVE;
  static DeviceOnce once;
  const hipError_t lim = once_on_device(once, [] {
    return hipFuncSetAttribute((const void *)k_cache_attn_few<HD, RT>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  });
  if (lim != hipSuccess) return lim;
  hipLaunchKernelGGL((k_cache_attn_few<HD, RT>), dim3((unsigned)(attn_blocks(1, a.c) * a.splits)), dim3(256), LDS, s, a);
  return hipGetLastError();
}
template <int HD>
hipError_t launch_bf16(const CacheAttnArgs &a, hipStream_t s) {
  const int rpb = rows_per_block(1, a.c);
  return rpb == 16 ? launch_few<HD, 1>(a, s) : rpb == 32 ? launch_few<HD, 2>(a, s) : launch_few<HD, 4>(a, s);
}

}  // namespace

// Ranges of at least 256 keys, as many as fill the compute units once
static int wanted_splits(int dtype, const CacheArgs &c) {
  const int cus = device_cus();
  const int64_t blocks = std::max<int64_t>(1, attn_blocks(dtype, c));
  const int64_t fill = cus / blocks, most = ((int64_t)c.cap + 255) / 256;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(fill, most), 64));
}
int cache_attn_splits(int dtype, const CacheArgs &c, size_t scratch) {
  int s = wanted_splits(dtype, c);
  while (s > 1 && attn_part_bytes(c, s) > scratch) --s;
  return s;
}
size_t cache_attn_scratch(int dtype, const CacheArgs &c) {
  const int s = wanted_splits(dtype, c);
  return s > 1 ? attn_part_bytes(c, s) : 0;
}

hipError_t launch_cache_attention(int dtype, const CacheAttnArgs &in, hipStream_t s) {
  CacheAttnArgs a = in;
  a.c.xcd_order = a.c.batch * a.c.kvh % 8 == 0 ? 1 : 0;
  if (attn_blocks(dtype, a.c) <= 0) return hipSuccess;
  hipError_t e;
  if (dtype == 1) {
    e = a.c.hd == 128 ? launch_bf16<128>(a, s) : launch_bf16<64>(a, s);
  } else {
    const dim3 grid((unsigned)(attn_blocks(0, a.c) * a.splits));
    if (a.c.hd == 128)
      hipLaunchKernelGGL((k_cache_attn_f32<128>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_cache_attn_f32<64>), grid, dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.splits <= 1) return e;
  const int64_t items = (int64_t)a.c.batch * a.c.max_q * a.c.heads * (a.c.hd / 8);
  const dim3 grid((unsigned)((items + 255) / 256));
  if (dtype == 1) {
    if (a.c.hd == 128)
      hipLaunchKernelGGL((k_cache_attn_combine<bf16_t, 128>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_cache_attn_combine<bf16_t, 64>), grid, dim3(256), 0, s, a);
  } else {
    if (a.c.hd == 128)
      hipLaunchKernelGGL((k_cache_attn_combine<float, 128>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_cache_attn_combine<float, 64>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

static int64_t mass_blocks(int dtype, const CacheArgs &c) {
  const int kt = dtype == 1 ? 64 : 32;
  return (int64_t)c.batch * c.kvh * (((int64_t)c.cap + kt - 1) / kt);
}
static size_t mass_part_bytes(const CacheArgs &c, int splits) {
  return (size_t)c.batch * c.kvh * splits * c.cap * sizeof(float);
}
// Row ranges of at least 256 rows, as many as give every compute unit two blocks
static int mass_wanted(int dtype, const CacheArgs &c) {
  const int64_t fill = 2 * device_cus() / std::max<int64_t>(1, mass_blocks(dtype, c));
  const int64_t most = ((int64_t)c.max_q * (c.heads / c.kvh) + 255) / 256;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(fill, most), 64));
}
int cache_mass_splits(int dtype, const CacheArgs &c, size_t scratch) {
  int s = mass_wanted(dtype, c);
  while (s > 1 && mass_part_bytes(c, s) > scratch) --s;
  return s;
}
size_t cache_mass_scratch(int dtype, const CacheArgs &c) {
  const int s = mass_wanted(dtype, c);
  return s > 1 ? mass_part_bytes(c, s) : 0;
}

hipError_t launch_cache_mass(int dtype, const CacheMassArgs &in, hipStream_t s) {
  CacheMassArgs a = in;
  a.c.xcd_order = a.c.batch * a.c.kvh % 8 == 0 ? 1 : 0;
  const int64_t blocks = mass_blocks(dtype, a.c);
  if (blocks <= 0) return hipSuccess;
  const dim3 grid((unsigned)(blocks * a.splits));
  if (dtype == 1) {
    if (a.c.hd == 128)
      hipLaunchKernelGGL((k_cache_mass<bf16_t, 128>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_cache_mass<bf16_t, 64>), grid, dim3(256), 0, s, a);
  } else {
    if (a.c.hd == 128)
      hipLaunchKernelGGL((k_cache_mass<float, 128>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_cache_mass<float, 64>), grid, dim3(256), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits <= 1) return e;
  hipLaunchKernelGGL(k_cache_mass_combine, dim3((a.c.cap + 255) / 256, a.c.kvh, a.c.batch), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace wdc
