// Attention of chunks of new rows over a paged cache of e4m3 codes with a power of two
// per slot and kv head. A code times its power is exact in bf16 and in float32, so
// these kernels compute what those of cache_attention.hip compute over the values.
#include "cache_tiles.h"

#include <type_traits>

namespace wdc {
namespace {

// Eight codes of two words as float32, times a power of two
__device__ __forceinline__ void values8(uint32_t u, uint32_t v, float up, float (&x)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(u, up, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(u, up, true);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, up, false), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, up, true);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    x[e] = a[e];
    x[2 + e] = b[e];
    x[4 + e] = c[e];
    x[6 + e] = d[e];
  }
}
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
// Buffer of `bytes` bytes from base + off (both the same in every lane): what lies outside reads as zero
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_at(const void *base, int64_t off, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((char *)base + off, 0, bytes, RSRC_WORD3);
}
// power of two of an exponent byte
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float((byte & 255u) << 23); }

// ---------------------------------------------------------------- float32
// As over a cache in float32: v_mfma_f32_32x32x2_f32, four waves share 32 rows and take every fourth key
// tile of 32 of the block's range. S^T = K Q^T leaves a lane one row and 16 keys, which O^T = V^T P^T takes one by
// one as its B operand. Codes come straight from the cache, those of K 16 at a time (which dimension a lane
// takes in which step is free as long as K and Q agree: lane group g has [g hd / 2, + hd / 2)). Keys past the
// cache's end are read as its last key and get weight 0. Bound by the matrix instructions: chunks of 256 and 100 rows over
// 1,500 and 777 keys, 4 heads of 64, 14.7 us and 4 of the parts' launch, as over float32 (14.2), most of it latency.
template <int HD>
__global__ __launch_bounds__(256, 1) void k_cache8_attn_f32(CacheAttnArgs a) {
  constexpr int NI = HD / 32, NC = HD / 2;
  typedef __attribute__((ext_vector_type(NI))) float vecn;
  typedef typename std::conditional<NI == 4, uint32_t, uint16_t>::type codes_t;
  const CacheArgs &c = a.c;
  const AttnBlock k_(a);
  if (!k_.live) return;
  const CacheSeq s = k_.s;
  const int32_t *tab = k_.tab;
  const int h = k_.h, m0 = k_.m0, count = k_.count, group = k_.group, sp = k_.sp, nr = k_.nr, part_ = k_.part;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 31, lg = lane >> 5;
  const int mlast = min(m0 + 32, count) - 1, mm = min(m0 + lr, mlast), row = cache_row(c, mm);
  const int lim_lo = k_.lim_lo, lim = m0 + lr < count ? cache_limit(c, s, row) : 0;
  const int tiles = (k_.lim_hi + 31) / 32;
  const int t0 = nr > 1 ? sp * (k_.range / 32) : 0, t1 = nr > 1 ? min(t0 + k_.range / 32, tiles) : tiles;
  const float *Q = (const float *)a.q + (int64_t)(s.q0 + row) * a.ldq + (int64_t)(h * group + mm - row * group) * HD + NC * lg;
  const uint8_t *K = (const uint8_t *)c.k + NC * lg, *V = (const uint8_t *)c.v + NI * lr;
  const float sc = LOG2E / sqrtf((float)HD);
  float qf[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) qf[j] = Q[j] * sc;
  uint4 kq[NC / 16];
  float kup;
  f32x16 o[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  auto load_k = [&](int t) {
    const int64_t at = slot_row(c, tab, h, min(32 * t + lr, s.n - 1));
#pragma unroll
    for (int j = 0; j < NC / 16; ++j) kq[j] = *(const uint4 *)(K + at + 16 * j);
    kup = power(c.scale[at / HD * 2]);
  };
  if (t0 + w < t1) load_k(t0 + w);
  for (int t = t0 + w; t < t1; t += 4) {
    vecn v[16];
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {             // four keys of one page
      const int key = 32 * t + 8 * e4 + 4 * lg, k0 = min(key, s.n - 1);
      const int64_t at = slot_row(c, tab, h, k0);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t x = at / HD + min(key + e, s.n - 1) - k0;   // past the end: the last key
        const codes_t u = *(const codes_t *)(V + x * HD);
        const float up = power(c.scale[2 * x + 1]);
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((uint32_t)u, up, false);
        v[4 * e4 + e][0] = lo[0];
        v[4 * e4 + e][1] = lo[1];
        if constexpr (NI == 4) {
          const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((uint32_t)u, up, true);
          v[4 * e4 + e][2] = hi[0];
          v[4 * e4 + e][3] = hi[1];
        }
      }
    }
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
    for (int j = 0; j < NC / 8; ++j) {
      float kf[8];
      const uint4 u = kq[j / 2];
      values8(j & 1 ? u.z : u.x, j & 1 ? u.w : u.y, kup, kf);
#pragma unroll
      for (int d = 0; d < 8; ++d) x = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[d], qf[8 * j + d], x, 0, 0, 0);
    }
    if (t + 4 < t1) load_k(t + 4);
    const bool part = 32 * t + 32 > lim_lo;
    bool odd = false;
    if (part) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (32 * t + 8 * (e / 4) + 4 * lg + e % 4 >= lim) x[e] = -INFINITY;
#pragma unroll
        for (int i = 0; i < NI; ++i) odd |= !(fabsf(v[e][i]) < INFINITY);
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
      // NaN among the V of keys that some row does not see: key by key
#pragma unroll
      for (int e = 0; e < 16; ++e)
        for (int g = 0; g < 2; ++g) {
          const int key = 32 * t + 8 * (e / 4) + 4 * g + e % 4;
          const float p = __shfl(x[e], 32 * g + lr, 64);
          if (key >= lim) continue;
          const int64_t at = slot_row(c, tab, h, key);
          const uint8_t *vp = (const uint8_t *)c.v + at;
          const float up = power(c.scale[at / HD * 2 + 1]);
#pragma unroll
          for (int d = 0; d < 16; ++d)
#pragma unroll
            for (int i = 0; i < NI; ++i)
              o[i][d] += p * __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((uint32_t)vp[NI * (8 * (d / 4) + 4 * lg + d % 4) + i], up, false)[0];
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
  const int head = h * group + mm - row * group, dim0 = NI * (8 * w + 4 * lg);
  const int64_t at = part_slot(a, max(part_, 0), s.q0 + row, head);
  float *O = (float *)a.o + (int64_t)(s.q0 + row) * a.ldo + (int64_t)head * HD + dim0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float y = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) y += wt[u] * po[u][i * 16 + 4 * w + e][lane];
      if (part_ >= 0)
        a.part[at * HD + dim0 + NI * e + i] = y;
      else
        O[NI * e + i] = den == 0.f ? 0.f : y / den;
    }
  if (w != 0 || lg != 0) return;
  if (part_ >= 0) {
    *(float2 *)part_ml(a, at) = make_float2(mx, den);
  } else if (a.lse) {
    a.lse[(int64_t)(s.q0 + row) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
  }
}

// ---------------------------------------------------------------- bf16, few rows
// RT tiles of 16 query rows per block of four waves; wave w takes key tiles w, w + 4, .. of 32 keys of the block's range and
// the four partial softmaxes meet at the end. What bounds it is the stream of codes: each wave has a tile under way in registers
// beside the one it works on.
//
// S^T = K Q^T (A: 16 keys, B: 16 rows): lane (lr, lg) loads hd / 4 consecutive codes of key lr, and Q in the same order of
// dimensions, so K needs no LDS; its powers ride on the conversion to bf16. The lane is left the
// scores of row lr and keys 4 lg + e of both halves of the tile, the B operand of O^T = V^T P^T. V goes through LDS, from which rows
// come back transposed, 8 keys of one dimension a lane. It goes there in bf16, converted while a lane's codes are of one key, its
// power with them: powers multiplied into the weights would take weights of 2^-9 and below out of bf16's normal numbers at the smallest
// power. The softmax is the one of the cache in bf16.
//
// Eight tokens over 1 to 32,768 keys, 32 heads on 8 of 128 (235 MB): 47.4 us and 4.8 of the parts' launch, 5.0 TB/s, where
// the cache in bf16 takes 80 for twice the bytes (5.4 TB/s; a large copy, which writes too, 4.9). 182 registers allow two blocks
// per compute unit (at hd 64 112 do four; with 32 rows 172 do two, and 364 at hd 128 one).
template <int HD>
struct Codes {
  static constexpr int KT = 32;                  // keys per tile
  static constexpr int NL = HD / 64;             // 16-byte loads of a lane per 16 keys
  static constexpr int CH = HD / 16;             // 16-byte chunks of a row
};

// Eight codes as bf16, times a power of two. (The conversion's result is taken as a word: its second half taken as an element
// comes out as the first.)
__device__ __forceinline__ bf16x8 bf16_values8(uint32_t u, uint32_t v, float up) {
  const u32x4_t w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, up, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, up, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, up, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, up, true))};
  return __builtin_bit_cast(bf16x8, w);
}
// Whether one of sixteen codes may be no finite number: one is NaN, or not all are zeros and the power makes the largest codes
// infinite (256 * 2^120 on)
__device__ __forceinline__ bool not_finite(u32x4_t u, float up) {
  uint32_t nan = 0, some = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    nan |= (u[q] & 0x7f7f7f7fu) + 0x01010101u;
    some |= u[q];
  }
  return (nan & 0x80808080u) != 0 || (up >= 0x1p120f && (some & 0x7f7f7f7fu) != 0);
}

template <int HD, int RT>
__global__ __launch_bounds__(256, HD * RT == 256 ? 1 : 2) void k_cache8_attn_few(CacheAttnArgs a) {
  using F = Codes<HD>;
  using L = Few<HD>;                             // layout of V in LDS
  constexpr int NC = HD / 32, NI = HD / 16, KT = F::KT, NL = F::NL, WAVE = 64 * RT * HD;
  static_assert(WAVE >= KT * L::ROWB, "a tile of V in bf16");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float ml[4][2][16 * RT];
  const CacheArgs &c = a.c;
  const AttnBlock k_(a);
  if (!k_.live) return;
  const CacheSeq s = k_.s;
  const int h = k_.h, m0 = k_.m0, count = k_.count, group = k_.group, sp = k_.sp, nr = k_.nr, part_ = k_.part;

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mlast = min(m0 + 16 * RT, count) - 1;
  const int lim_lo = k_.lim_lo, tiles = (k_.lim_hi + KT - 1) / KT;
  const int t0 = nr > 1 ? sp * (k_.range / KT) : 0, t1 = nr > 1 ? min(t0 + k_.range / KT, tiles) : tiles;

  const float sc = LOG2E / sqrtf((float)HD);
  bf16x8 qf[RT][NC];
  int lim[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int m = m0 + 16 * t + lr, mm = min(m, mlast), i = cache_row(c, mm);
    lim[t] = m < count ? cache_limit(c, s, i) : 0;
    const bf16_t *Q = (const bf16_t *)a.q + (int64_t)(s.q0 + i) * a.ldq + (int64_t)(h * group + mm - i * group) * HD + HD / 4 * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) qf[t][j] = *(const bf16x8 *)(Q + 8 * j);
  }

  char *mine = smem + w * WAVE;
  // LDS offsets in 16 rows of V in bf16: of the first half of the lane's 16 codes (the second: ^ 16), and of the transposed
  // read of rows 4 lg .. + 3, dims 16 i ..
  const int vrow = lane / F::CH;                 // row of the lane's codes, of load j: + 64 / CH j
  int vwo[NL], vro[L::VR];
#pragma unroll
  for (int j = 0; j < NL; ++j) {
    const int r = vrow + j * (64 / F::CH);
    vwo[j] = r * L::ROWB + ((2 * (lane % F::CH)) ^ L::vkey(r)) * 16;
  }
  {
    const int r = 4 * lg + (lr >> 2), j = lane & 3;
#pragma unroll
    for (int i = 0; i < L::VR; ++i) vro[i] = r * L::ROWB + ((2 * i + (j >> 1)) ^ L::vkey(r)) * 16 + 8 * (j & 1);
  }
  PageWalk<false> pw;
  pw.init(c, k_.tab, k_.tab_last, h, (KT * t0) >> c.plog);
  const int pmask = (1 << c.plog) - 1;
  struct Tile {
    u32x4_t k[2][NL], v[2][NL];
    uint32_t ks[2];                              // powers' bytes of (k, v) of key lr
  } tile[2];
  // Tile t: halves of 16 rows, each on one page. Rows past the cache's end lie outside the buffer range and arrive as
  // zeros, whatever they hold; so do tiles past the range.
  auto load = [&](int t, Tile &x) __attribute__((always_inline)) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int key = KT * t + 16 * hf;
      const bool live = t < t1;
      if (live) pw.advance(c, h, key >> c.plog);
      const int64_t slot = live ? pw.get(c, h, key >> c.plog) + (key & pmask) : 0;
      const int rows = live ? min(max(s.n - key, 0), 16) : 0;
      const auto kd = rsrc_at(c.k, slot * HD, rows * HD), vd = rsrc_at(c.v, slot * HD, rows * HD);
      const auto ed = rsrc_at(c.scale, slot * 2, rows * 2);
      x.ks[hf] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(ed, 2 * lr, 0, 0);
#pragma unroll
      for (int j = 0; j < NL; ++j)
        x.k[hf][j] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(kd, lr * HD + HD / 4 * lg + 16 * j, 0, 0));
#pragma unroll
      for (int j = 0; j < NL; ++j)
        x.v[hf][j] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(vd, lane * 16 + 1024 * j, 0, 0));
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  f32x4 o[RT][NI];
  float m[RT], l[RT], d[RT];                     // d: sum of the rounded weights
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = -INFINITY;
    l[t] = d[t] = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto step = [&](const Tile &x, int t) __attribute__((always_inline)) {
    f32x4 S[RT][2];
    float vup[2][NL];                            // powers of the lane's rows of V
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float up = power(x.ks[k]);
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const u32x4_t u = x.k[k][j / 2];
        const bf16x8 kf = bf16_values8(u[2 * (j & 1)], u[2 * (j & 1) + 1], up);
#pragma unroll
        for (int r = 0; r < RT; ++r)
          S[r][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][j], j == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : S[r][k], 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        // (255, which no append writes, would make codes of 0 NaN)
        vup[k][j] = power(min((uint32_t)__shfl((int)x.ks[k], vrow + j * (64 / F::CH), 64) >> 8, 254u));
        char *to = mine + k * 16 * L::ROWB;
#pragma unroll
        for (int q = 0; q < 2; ++q)
          *(bf16x8 *)(to + (vwo[j] ^ 16 * q)) = bf16_values8(x.v[k][j][2 * q], x.v[k][j][2 * q + 1], vup[k][j]);
      }
    }
    const bool part = KT * t + KT > lim_lo;      // some row does not see the whole tile
    bf16x8 pf[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y = S[r][k][e] * sc;
          if (KT * t + 16 * k + 4 * lg + e >= lim[r]) y = -INFINITY;
          S[r][k][e] = y;
          mx = fmaxf(mx, y);
        }
      mx = quad_max(mx);
      if (__any(mx > m[r] + 8.f)) {
        const float mn = fmaxf(m[r], mx), al = mn == m[r] ? 1.f : __builtin_amdgcn_exp2f(m[r] - mn);
        m[r] = mn;
        l[r] *= al;
        d[r] *= al;
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
          d[r] += (float)pf[r][4 * k + e];
        }
    }
    // A key that a row does not see has weight 0, but 0 times an infinity or NaN of its V is NaN in a matrix product.
    // Tiles seen in part are looked over, and one that may hold such a value is multiplied key by key.
    bool odd = false;
    if (part) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < NL; ++j) odd |= not_finite(x.v[k][j], vup[k][j]);
      odd = __any(odd);
    }
    asm volatile("" ::: "memory");
    if (odd) {
#pragma unroll 1
      for (int y = 0; y < KT; ++y) {             // key 16 (q / 4) + 4 g + q % 4
        const int q = y >> 2, g = y & 3, key = 16 * (q >> 2) + 4 * g + (q & 3);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          float p = 0.f;                         // of key and row lr, held by lane group g
#pragma unroll
          for (int z = 0; z < 8; ++z)
            if (z == q) p = (float)pf[r][z];
          p = __shfl(p, 16 * g + lr, 64);
          if (KT * t + key < lim[r])
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int col = 16 * i + 4 * lg + e;
                o[r][i][e] += p * bf2f(*(const bf16_t *)(mine + key * L::ROWB + ((col >> 3) ^ L::vkey(key)) * 16 + (col & 7) * 2));
              }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const bf16x8 vf = v_frag<HD>(mine + vro[i % L::VR] + i / L::VR * L::VR * 32);
#pragma unroll
        for (int r = 0; r < RT; ++r) o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r], o[r][i], 0, 0, 0);
      }
    }
    asm volatile("" ::: "memory");
  };
  if (t0 + w < t1) {
    load(t0 + w, tile[0]);
    for (int t = t0 + w; t < t1; t += 8) {
      load(t + 4, tile[1]);
      step(tile[0], t);
      if (t + 4 >= t1) break;
      load(t + 8, tile[0]);
      step(tile[1], t + 4);
    }
  }

  // the four waves' parts: each leaves its rows in its own part of LDS
  float *po = (float *)mine;                     // [16 RT rows][HD]
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] = quad_sum(l[t]);
    const float f = unround(l[t], quad_sum(d[t]));
#pragma unroll
    for (int i = 0; i < NI; ++i) *(f32x4 *)(po + (16 * t + lr) * HD + 4 * ((4 * i + lg) ^ (lr & 7))) = o[t][i] * f;
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
      const f32x4 y = *(const f32x4 *)(smem + u * WAVE + (r * HD + 4 * (e ^ (r & 7))) * 4);
#pragma unroll
      for (int d = 0; d < 4; ++d) x[d] += wt * y[d];
    }
    const int i = cache_row(c, mr), head = h * group + mr - i * group;
    if (part_ >= 0) {
      const int64_t at = part_slot(a, part_, s.q0 + i, head);
      *(f32x4 *)(a.part + at * HD + 4 * e) = x;
      if (e == 0) *(float2 *)part_ml(a, at) = make_float2(mx, den);
      continue;
    }
    const float inv = 1.f / den;
    bf16x4 y;
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] = (__bf16)(den == 0.f ? 0.f : x[d] * inv);
    *(bf16x4 *)((bf16_t *)a.o + (int64_t)(s.q0 + i) * a.ldo + (int64_t)head * HD + 4 * e) = y;
    if (a.lse && e == 0)
      a.lse[(int64_t)(s.q0 + i) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
  }
}

// ---------------------------------------------------------------- bf16, many rows
// The software pipeline of the cache in bf16 (32 query rows a wave, key tiles of 64, step t: P V of tile t, Q K of tile t + 2
// and the exponentials of tile t + 1 in one stream), with its tiles made from codes on the way: direct buffer loads of four waves bring
// a tile's codes and exponent bytes to LDS, and in every step all waves turn one tile of K and one of V into bf16 tiles
// of the same layout, each code once for all rows of the block. Step t asks for the codes of K_t+5 and V_t+4, converts K_t+3
// and V_t+2, and reads K_t+2, V_t and the first of V_t+1: two, four and three slots of K, V and codes.
//
// Tiles that some row sees in part, and the cache's last one, follow one at a time with their masks, tile u + 1 converted
// while u is worked on.
//
// Bound like the kernel over bf16 by the matrix cores, the exponentials and their power: 4,080 rows over 67,320 keys, 16 heads of
// 128, 1,906 to 2,005 us by device, 1,100 to 1,160 TFLOP/s, where that one takes 1,760 to 1,850; the conversion adds 8% to
// a step's vector instructions and half of its LDS traffic again. Blocks of 128 rows: at hd 64 KG = 2 groups of four waves take every
// second tile each; at hd 128 two such rings do not fit into LDS, and KH = 2 groups of four take half of every tile's keys
// (32 rows of 32 heads on 8 over 40,000 keys: 50 us with four waves over all of them, 45 so).
//
// A wave whose 32 rows are all past the last one only loads and converts, which leaves LDS and the matrix cores to the
// others: 60 rows of a kv head over 40,000 keys, 39.7 us with every wave at work and 35.6 so, at hd 64 43.1 and 37.8.
//
// References move when a lane's sum of weights over a tile passes 2^8 (2^16 over bf16), to the row's largest score: sums of weights
// times v are finite while |v| is below 2^120 over the number of keys.
constexpr int KV = 64, KS = 2, VS = 4, RS = 3, ES = 4;   // keys a tile; slots of K, V, codes and exponent bytes
constexpr int EB = 256;                          // bytes of a slot of exponent bytes
constexpr float SUM_LIMIT = 0x1p8f;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// Direct global -> LDS loads: lane l's 16 (4) bytes at `voff` of the buffer arrive at lds + 16 l (4 l). Instructions
// and wait states as in the kernels over bf16 (five between a vector instruction's scalar result and its use as
// part of a descriptor, one behind M0).
__device__ __forceinline__ void lds_load16(u32x4_t buf, uint32_t lds, int voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uni((int)lds)), "v"(voff), "s"(buf)
               : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(u32x4_t buf, uint32_t lds, int voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(uni((int)lds)), "v"(voff), "s"(buf)
               : "memory", "m0");
}

// The lane's number, at hd 128 found anew, by instructions that are not moved out of a loop: a register kept for it, or for
// what follows from it, would be spilled, and its reload in every step would wait for all loads under way (4,080 rows over
// 67,320 keys: 2.03 ms, 1.92 with what the pipeline needs kept in registers and the rest found anew). Blocks of 256 rows over pages
// of 16 or 32 slots still have one such reload a step, of four registers.
template <int HD>
__device__ __forceinline__ int lane_anew() {
  if (HD == 64) return threadIdx.x & 63;
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

// Loads of one wave (of four): stripe i of a tile is rows [(4 i + w) RPL, + RPL). SMALL:
// pages of 16 or 32 slots, where every stripe has its own page; otherwise a tile lies on one page.
template <int HD, bool SMALL>
struct CodeLoads {
  static constexpr int RPL = 1024 / HD;          // rows per load (8 or 16)
  static constexpr int NS = KV / (4 * RPL);      // stripes of a wave per tile (2 or 1)
  static constexpr int NP = SMALL ? NS : 1;
  static constexpr int NK = NS + 1;              // loads of K, exponent bytes included
  struct Where {
    int64_t off[NP];                             // bytes from the pool to the stripe (SMALL), or to the tile
    int bytes[NP];                               // what lies before the end of the cache
  };
  PageWalk<true> pw;                             // SMALL only
  int w, h, n;
  __device__ __forceinline__ void init(const CacheArgs &c, const CacheSeq &s, const int32_t *tab, int tab_last, int h_, int w_,
                                       int tile0) {
    w = w_;
    h = h_;
    n = s.n;
    if (SMALL) pw.init(c, tab, tab_last, h, (KV * tile0) >> c.plog);
  }
  // page of a whole tile, by a scalar load (the table does not change during a launch)
  __device__ __forceinline__ int page(const CacheArgs &c, const int32_t *tab, int tab_last, int tile) const {
    typedef const __attribute__((address_space(4))) int32_t *scalar_ptr;
    const int e = min((KV * tile) >> c.plog, tab_last);
    return cache_page(c, ((scalar_ptr)(uint64_t)tab)[e]);
  }
  // where a tile lies, its page given (unless SMALL), and the load of its exponent bytes, 2 keys a lane
  __device__ __forceinline__ void find(const CacheArgs &c, int tile, int page, Where &x, uint32_t lds) {
    const int pmask = (1 << c.plog) - 1, key0 = KV * tile, lane = lane_anew<HD>();
    if (SMALL) pw.advance(c, h, key0 >> c.plog);   // a tile's pages are of one group of 64
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = SMALL ? (4 * i + w) * RPL : 0, key = key0 + at, rows = SMALL ? RPL : KV;
      const int slot = SMALL ? pw.get(c, h, key >> c.plog) : ((page * c.kvh + h) << c.plog);   // (pools hold fewer than 2^31)
      x.off[i] = (int64_t)(slot + (key & pmask)) * HD;
      x.bytes[i] = min(max(n - key, 0), rows) * HD;
    }
    // lanes of keys past the end, and the upper half, ask for what is outside (pools have fewer than 2^32 of these bytes)
    const int key = key0 + 2 * (lane & 31);
    const int slot = SMALL ? __shfl(pw.cur, (key >> c.plog) - pw.base, 64) : (page * c.kvh + h) << c.plog;
    const uint32_t all = (uint32_t)(((int64_t)c.pages * c.kvh << c.plog) * 2);
    const uint32_t voff = lane < 32 && key < n ? (uint32_t)(slot + (key & pmask)) * 2 : all;
    lds_load4(buffer_at(c.scale, 0, (int)all), lds, (int)voff);
  }
  __device__ __forceinline__ void load(const void *pool, const Where &x, uint32_t lds) const {
    const int lane = lane_anew<HD>();
#pragma unroll
    for (int i = 0; i < NS; ++i)
      lds_load16(buffer_at(pool, x.off[SMALL ? i : 0], x.bytes[SMALL ? i : 0]), lds + (4 * i + w) * 1024,
                 16 * lane + (SMALL ? 0 : (4 * i + w) * 1024));
  }
};

template <int HD, bool SMALL, int W, int KG, int KH>
__global__ __launch_bounds__(64 * W, 8 / W) void k_cache8_attn_many(CacheAttnArgs a) {
  using F = Few<HD>;
  using TL = CodeLoads<HD, SMALL>;
  constexpr int NC = HD / 32, NI = HD / 16;
  constexpr int TB = KV * F::ROWB, RB = KV * HD; // bytes of a tile in bf16, in codes
  constexpr int V_BASE = KS * TB, RK_BASE = V_BASE + VS * TB, RV_BASE = RK_BASE + RS * RB, E_BASE = RV_BASE + RS * RB;
  constexpr int RING = E_BASE + ES * EB;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int odd_tile[KG][4];
  const CacheArgs &c = a.c;
  const AttnBlock k_(a);
  if (!k_.live) return;
  const CacheSeq s = k_.s;
  const int32_t *tab = k_.tab;
  const int tab_last = k_.tab_last;
  const int h = k_.h, m0 = k_.m0, count = k_.count, group = k_.group, sp = k_.sp, nr = k_.nr, part_ = k_.part;

  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  static_assert(KG == 1 || KH == 1, "keys are shared out in one way");
  constexpr int WG = W / KG, WR = WG / KH;       // waves over a ring; over the block's rows
  constexpr int KK = 4 / KH;                     // tiles of 16 keys of a wave
  // (rows of few waves lie on different SIMDs: waves w and w + 4 share one)
  const int kg = KG == 1 ? 0 : wid / WR, kh = KH == 1 ? 0 : wid / WR, wr = (wid + (kg + kh) * (WR / 2)) % WR, cw = wid % WG;
  const bool grp_a = KG == 2 || wid < 4;         // loads tiles
  const int mlast = min(m0 + 32 * WR, count) - 1;
  const int lim_lo = k_.lim_lo, tiles = (k_.lim_hi + KG * KV - 1) / (KG * KV);   // in steps of KG tiles
  const int range = k_.range / (KG * KV), t_first = nr > 1 ? sp * range : 0, t_end = nr > 1 ? min(t_first + range, tiles) : tiles;
  // steps of the range, relative to t_first: `nf` that every row sees whole, then masked ones
  const int tot = t_end - t_first, nf = min(max(lim_lo / (KG * KV) - t_first, 0), tot);
  const int ahead = min(tot, nf + RS);           // codes that the pipeline asks for
  const bool none = m0 + 32 * wr >= count;       // the wave has no rows: it loads and converts, and works on nothing

  const float sc = LOG2E / sqrtf((float)HD);
  bf16x8 qf[2][NC];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int mm = min(m0 + 32 * wr + 16 * t + lr, mlast), i = cache_row(c, mm);
    const bf16_t *Q = (const bf16_t *)a.q + (int64_t)(s.q0 + i) * a.ldq + (int64_t)(h * group + mm - i * group) * HD + 8 * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) qf[t][j] = *(const bf16x8 *)(Q + 32 * j);
  }
  // LDS offsets of the K fragment of rows lr, dims 8 lg .. (dims 32 j on: kro ^ 64 j), and of the transposed V read of rows
  // 4 lg .. + 3, dims 0 .. (dims 16 i on, i < VR: vro ^ 32 i). At hd 128 the others are made where they are needed.
  int kro = kh * 16 * KK * F::ROWB + lr * F::ROWB + (lg ^ F::kkey(lr)) * 16, vro;
  {
    const int r = 4 * lg + (lr >> 2), j = lane & 3;
    vro = V_BASE + kh * 16 * KK * F::ROWB + r * F::ROWB + ((j >> 1) ^ F::vkey(r)) * 16 + 8 * (j & 1);
  }
  char *ring = smem + kg * RING;
  const uint32_t lds0 = lds_addr(ring);
  TL tl;
  typename TL::Where wk, wv;                     // of the latest K tile asked for, and of the one before
  auto page_of = [&](int t) { return SMALL ? 0 : tl.page(c, tab, tab_last, KG * (t_first + t) + kg); };
  // codes of K and the exponent bytes of tile t; codes of V of the tile at x
  auto load_k = [&](int t, int slot, int page) __attribute__((always_inline)) {
    wv = wk;
    tl.find(c, KG * (t_first + t) + kg, page, wk, lds0 + E_BASE + (t % ES) * EB);
    tl.load(c.k, wk, lds0 + RK_BASE + slot * RB);
  };
  auto load_v = [&](int slot, const typename TL::Where &x) { tl.load(c.v, x, lds0 + RV_BASE + slot * RB); };

  // Conversion: 16 codes of a row a lane. NCV pieces of 1,024 codes for each wave of both K and V, or (BOTH false) one of K
  // for the first half of the waves and one of V for the others.
  constexpr int PIECES = RB / 1024;
  constexpr bool BOTH = WG <= PIECES;
  constexpr int NCV = BOTH ? PIECES / WG : 1;
  const bool conv_k = BOTH || cw < PIECES, conv_v = BOTH || cw >= PIECES;
  const int piece = BOTH ? cw : cw % PIECES;
  // A lane's two chunks go out one after the other, in the rows whose bit is set the upper one first: with V's swizzle
  // (even) half of the banks would be idle in each.
  auto upper_of = [](int row) { return HD == 128 ? row & 1 : (row >> 1) & 1; };
  const int prow = piece * TL::RPL + lane / (HD / 16), pch = 2 * (lane % (HD / 16));
  const int to_k = prow * F::ROWB + (pch ^ F::kkey(prow)) * 16, to_v = prow * F::ROWB + ((pch + upper_of(prow)) ^ F::vkey(prow)) * 16;
  int to2 = to_k | to_v << 16;                   // where the first chunk goes in a tile of K, and of V
  u32x4_t raw[NCV];
  float up[NCV];
  // (the rows of a wave's pieces differ by a multiple of 16 or of 32, which the swizzles do not see)
  static_assert(NCV == 1 || WG * (1024 / HD) % 16 == 0, "rows of a wave's pieces");
  auto take = [&](const char *codes, const char *bytes, int which) __attribute__((always_inline)) {
    const int ln = lane_anew<HD>(), row = ln / (HD / 16), up8 = which ? 8 * upper_of(row) : 0;   // (a piece starts at an even row pair)
#pragma unroll
    for (int i = 0; i < NCV; ++i) {
      const char *p = codes + (piece + i * WG) * 1024 + 16 * ln;
      const u32x2_t x = *(const u32x2_t *)(p + up8), y = *(const u32x2_t *)(p + (up8 ^ 8));
      raw[i] = u32x4_t{x[0], x[1], y[0], y[1]};
      // (past the end any byte may follow an odd key: 255 would make the zeros there NaN)
      up[i] = power(min((uint32_t)*(const uint8_t *)(bytes + 2 * (row + (piece + i * WG) * TL::RPL) + which), 254u));
    }
  };
  auto put = [&](char *to, int which, int half) __attribute__((always_inline)) {
    const int at = (HD == 64 ? (which ? to_v : to_k) : which ? (uint32_t)to2 >> 16 : to2 & 0xffff) ^ (16 * half);
#pragma unroll
    for (int i = 0; i < NCV; ++i)
      *(bf16x8 *)(to + at + i * WG * TL::RPL * F::ROWB) = bf16_values8(raw[i][2 * half], raw[i][2 * half + 1], up[i]);
  };
  auto raw_k = [&](int slot) { return ring + RK_BASE + slot * RB; };
  auto raw_v = [&](int slot) { return ring + RV_BASE + slot * RB; };
  auto bytes_of = [&](int t) { return ring + E_BASE + (t % ES) * EB; };
  // both tiles t at once; whether V may hold an infinity or NaN
  auto convert = [&](int t, bool k, bool v) __attribute__((always_inline)) {
    bool odd = false;
    if (k && conv_k) {
      take(raw_k(t % RS), bytes_of(t), 0);
      put(ring + (t % KS) * TB, 0, 0);
      put(ring + (t % KS) * TB, 0, 1);
    }
    if (v && conv_v) {
      take(raw_v(t % RS), bytes_of(t), 1);
      put(ring + V_BASE + (t % VS) * TB, 1, 0);
      put(ring + V_BASE + (t % VS) * TB, 1, 1);
#pragma unroll
      for (int i = 0; i < NCV; ++i) odd |= not_finite(raw[i], up[i]);
    }
    return odd;
  };

  int page[4];                                   // of the K tiles that the next four steps ask for
  if (grp_a) {                                   // tiles 0 to 2
    tl.init(c, s, tab, tab_last, h, wid & 3, KG * t_first + kg);
    wk = typename TL::Where{};
#pragma unroll
    for (int j = 0; j < RS; ++j)
      if (j < tot) {
        load_k(j, j, page_of(j));
        load_v(j, wk);
      }
    wait_vm<0>();
  }
  if (tid < 4 * KG) odd_tile[tid >> 2][tid & 3] = 0;
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

  f32x4 o[NI][2];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int t = 0; t < 2; ++t) o[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  auto qk = [&](f32x4 (&S)[KK][2], const char *kb) {
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        const bf16x8 kf = *(const bf16x8 *)(kb + (kro ^ 64 * j) + k * 16 * F::ROWB);
#pragma unroll
        for (int t = 0; t < 2; ++t)
          S[k][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][j], j == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : S[k][t], 0, 0, 0);
      }
  };
  auto vfrag = [&](const char *vb, int i, int p) {   // V^T fragment: dims 16 i .., keys of the 32-key group p
    return v_frag<HD>(vb + (vro ^ 32 * (i % F::VR)) + i / F::VR * F::VR * 32 + p * 32 * F::ROWB);
  };

  if (nf > 0) {
    f32x4 S[2][KK][2];                           // S of tiles t + 1 and t + 2 (index tile & 1)
    bf16x8 pf[2][2][KK / 2];                        // P of tiles t and t + 1 (index tile & 1), [row tile][32-key group]
    convert(0, true, true);
    convert(1, true, true);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (grp_a) {                                 // K_3, V_3, K_4
      if (3 < ahead) {
        load_k(3, 0, page_of(3));
        load_v(0, wk);
      }
      if (4 < ahead) load_k(4, 1, page_of(4));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) page[j] = page_of(5 + j);
    qk(S[0], ring);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      m[t] = fmaxf(rowmax<HD>(S[0], t) * sc, -FLT_MAX);   // (scores of -inf: weight 0)
      l[t] = weights(S[0], pf[0][t], t, sc, m[t]);
    }
    // a lane's sum of weights above which a tile's weights are taken again; far out all are
    float limit = far_out(fmaxf(fabsf(m[0]), fabsf(m[1]))) ? -1.f : SUM_LIMIT;
    if (nf > 1) qk(S[1], ring + TB);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    convert(2, true, false);                     // into the slot of K_0
    if (grp_a) wait_vm<0>();                     // K_3
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    constexpr int NPV = KK / 2 * NI, NMF = NPV + KK * NC;   // fragment reads of P V, and of a step; two MFMAs each
    constexpr int EPM = 8 * KK / NMF;            // exponentials per pair of MFMAs
    static_assert(NMF == 16 || NMF == 32, "hd 64 or 128");
    // Where V's codes are taken and put. Behind the last of them come the reads of four V fragments, two instructions
    // each, which are all that the step's last wait leaves under way: what was put is there when the barrier opens.
    constexpr int TAKE_V = NMF == 32 ? 16 : 7, PUT_V = NMF == 32 ? 22 : 9, LAST_PUT = NMF == 32 ? 26 : 11;
    static_assert(LAST_PUT <= NMF - 5 && NPV >= 4, "tiles put before the last eight reads");
    bf16x8 fr_[NMF];
    // One step, P = t % 4 at compile time, as in the kernel over bf16; the conversions lie in the stream: K's codes are
    // taken at its start and put a fourth later, V's likewise in its second half. Past the last tile they run on stale slots, unused.
    auto read = [&](int r, const char *vb, const char *kb) __attribute__((always_inline)) {
      const int g = r >= NPV ? r - NPV : 0;
      if (r < NPV)
        fr_[r] = vfrag(vb, r % NI, (r < NPV ? r : 0) / NI);
      else
        fr_[r] = *(const bf16x8 *)(kb + (kro ^ 64 * (g / KK)) + (g % KK) * 16 * F::ROWB);
    };
#pragma unroll
    for (int r = 0; r < 4; ++r) read(r, ring, ring);
    int rs = 0;                                  // t % RS
    auto step = [&](auto pc, int t, int page) __attribute__((always_inline)) {
      constexpr int P = decltype(pc)::value, cur = (P + 1) & 1, n = P & 1;
      const int r1 = rs == RS - 1 ? 0 : rs + 1, r2 = rs == 0 ? RS - 1 : rs - 1;   // (t + 1) % RS, (t + 2) % RS
      int issued = 0;
      if (grp_a) {
        if (t + 5 < ahead) {
          load_k(t + 5, r2, page);
          issued += TL::NK;
        } else {
          wv = wk;
        }
        if (t + 4 < ahead) {
          load_v(r1, wv);
          issued += TL::NS;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      const char *vb = ring + P * TB, *kb = ring + (P % KS) * TB, *vn = ring + ((P + 1) % VS) * TB;
      if (HD == 128) asm volatile("" : "+v"(kro), "+v"(vro), "+v"(to2));
      float ls[2] = {0.f, 0.f}, ex[2];
      auto mma = [&](int q, int t_) __attribute__((always_inline)) {
        if (q < NPV) {
          o[q % NI][t_] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr_[q], pf[n][t_][(q < NPV ? q : 0) / NI], o[q % NI][t_], 0, 0, 0);
        } else {
          const int g = q >= NPV ? q - NPV : 0;
          S[n][g % KK][t_] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr_[q], qf[t_][g / KK],
                                                                     g < KK ? f32x4{0.f, 0.f, 0.f, 0.f} : S[n][g % KK][t_], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      auto expo = [&](int x) __attribute__((always_inline)) {
        const int k = x / 8, t_ = (x / 4) % 2, e = x % 4;
        float y = __builtin_amdgcn_exp2f(__builtin_fmaf(S[cur][k][t_][e], sc, -m[t_]));
        asm volatile("" : "+v"(y));
        return y;
      };
#pragma unroll
      for (int q = 0; q < NMF; ++q) {
        if constexpr (EPM == 2) {
          ex[0] = expo(2 * q);
          ex[1] = expo(2 * q + 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        mma(q, 0);
        if constexpr (EPM == 1) {
          ex[q & 1] = expo(q);
          __builtin_amdgcn_sched_barrier(0);
        }
        mma(q, 1);
        if (q + 4 < NMF)
          read(q + 4, vb, kb);
        else                                     // the next step's first reads: V of tile t + 1
          read(q + 4 - NMF, vn, kb);
        __builtin_amdgcn_sched_barrier(0);
        if (EPM == 2 || (q & 1)) {
          const int x = EPM == 2 ? 2 * q : q - 1, k = x / 8, t_ = (x / 4) % 2, e = x % 4;
          const bf16x2_t pr = {(__bf16)ex[0], (__bf16)ex[1]};
          uint32_t u = __builtin_bit_cast(uint32_t, pr);
          ls[t_] += ex[0] + ex[1];
          asm volatile("" : "+v"(u), "+v"(ls[t_]));
          u32x4_t w_ = __builtin_bit_cast(u32x4_t, pf[cur][t_][k / 2]);
          w_[2 * (k & 1) + e / 2] = u;
          pf[cur][t_][k / 2] = __builtin_bit_cast(bf16x8, w_);
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (BOTH) {
          char *kt = ring + ((P + 3) % KS) * TB, *vt = ring + V_BASE + ((P + 2) % VS) * TB;
          if (q == 0) take(raw_k(rs), bytes_of(P + 3), 0);
          if (q == NMF / 4 - 2) put(kt, 0, 0);
          if (q == NMF / 4 + 2) put(kt, 0, 1);
          if (q == TAKE_V) take(raw_v(r2), bytes_of(P + 2), 1);
          if (q == PUT_V) put(vt, 1, 0);
          if (q == LAST_PUT) put(vt, 1, 1);
        } else {
          char *to = ring + (conv_k ? ((P + 3) % KS) * TB : V_BASE + ((P + 2) % VS) * TB);
          if (q == 0) take(conv_k ? raw_k(rs) : raw_v(r2), conv_k ? bytes_of(P + 3) : bytes_of(P + 2), conv_k ? 0 : 1);
          if (q == NMF / 2) put(to, conv_k ? 0 : 1, 0);
          if (q == LAST_PUT) put(to, conv_k ? 0 : 1, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (t + 1 < nf) {
        if (__any(!(fmaxf(ls[0], ls[1]) <= limit))) {
#pragma unroll
          for (int t_ = 0; t_ < 2; ++t_) {
            const float mx = rowmax<HD>(S[cur], t_) * sc, mn = fmaxf(mx, m[t_]);
            const float al = __builtin_amdgcn_exp2f(m[t_] - mn);
            m[t_] = mn;
            l[t_] *= al;
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i][t_][e] *= al;
            ls[t_] = weights(S[cur], pf[cur][t_], t_, sc, m[t_]);
          }
          limit = far_out(fmaxf(fabsf(m[0]), fabsf(m[1]))) ? -1.f : SUM_LIMIT;
        }
        l[0] += ls[0];
        l[1] += ls[1];
      }
      rs = r1;
      // the loads of earlier steps are done, this step's tiles are written, and all reads but the four just issued
      if (grp_a) {
        if (issued == TL::NK + TL::NS)
          wait_vm<TL::NK + TL::NS>();
        else if (issued == TL::NS)
          wait_vm<TL::NS>();
        else
          wait_vm<0>();
      }
      asm volatile("s_waitcnt lgkmcnt(%0)\n\ts_barrier" ::"n"(8) : "memory");
    };
    // A step of a wave without rows: its share of the loads and the conversion.
    auto serve = [&](int t) __attribute__((always_inline)) {
      const int r1 = rs == RS - 1 ? 0 : rs + 1, r2 = rs == 0 ? RS - 1 : rs - 1;
      int issued = 0;
      if (grp_a) {
        if (t + 5 < ahead) {
          load_k(t + 5, r2, page_of(t + 5));
          issued += TL::NK;
        } else {
          wv = wk;
        }
        if (t + 4 < ahead) {
          load_v(r1, wv);
          issued += TL::NS;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (conv_k) {
        take(raw_k(rs), bytes_of(t + 3), 0);
        put(ring + ((t + 3) % KS) * TB, 0, 0);
        put(ring + ((t + 3) % KS) * TB, 0, 1);
      }
      if (conv_v) {
        take(raw_v(r2), bytes_of(t + 2), 1);
        put(ring + V_BASE + ((t + 2) % VS) * TB, 1, 0);
        put(ring + V_BASE + ((t + 2) % VS) * TB, 1, 1);
      }
      rs = r1;
      if (grp_a) {
        if (issued == TL::NK + TL::NS)
          wait_vm<TL::NK + TL::NS>();
        else if (issued == TL::NS)
          wait_vm<TL::NS>();
        else
          wait_vm<0>();
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    if (none) {
#pragma unroll 1
      for (int t = 0; t < nf; ++t) serve(t);
    } else
    for (int t = 0; t < nf; t += 4) {
      int next[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) next[j] = page_of(t + 9 + j);
      step(std::integral_constant<int, 0>{}, t, page[0]);
      if (t + 1 >= nf) break;
      step(std::integral_constant<int, 1>{}, t + 1, page[1]);
      if (t + 2 >= nf) break;
      step(std::integral_constant<int, 2>{}, t + 2, page[2]);
      if (t + 3 >= nf) break;
      step(std::integral_constant<int, 3>{}, t + 3, page[3]);
#pragma unroll
      for (int j = 0; j < 4; ++j) page[j] = next[j];
    }
  }

  // Masked tiles, one at a time: the codes of tiles nf to nf + 2 have been asked for. A key that a row does not see has weight
  // 0, but 0 times an infinity or NaN is NaN in a matrix product: a tile whose V may hold one is multiplied key by key.
  int lim[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int mr = m0 + 32 * wr + 16 * t + lr;
    lim[t] = mr < count ? cache_limit(c, s, cache_row(c, mr)) : 0;
  }
  auto masked_convert = [&](int u) __attribute__((always_inline)) {
    if (__any(convert(u, true, true)) && lane == 0) odd_tile[kg][u & 3] = 1;
  };
  if (nf < tot) {
    if (nf > 0) {
      if (grp_a) wait_vm<0>();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    masked_convert(nf);
  }
  for (int u = nf; u < tot; ++u) {
    if (grp_a) wait_vm<0>();                     // codes of tile u + 1 (and u + 2)
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (grp_a && u + 3 < tot) {
      load_k(u + 3, u % RS, page_of(u + 3));
      load_v(u % RS, wk);
    }
    const bool odd = odd_tile[kg][u & 3];
    if (lane == 0 && cw == 0) odd_tile[kg][(u + 2) & 3] = 0;
    if (u + 1 < tot) masked_convert(u + 1);
    if (none) continue;
    const char *kb = ring + (u % KS) * TB, *vb = ring + (u % VS) * TB;   // vro holds V_BASE
    const int key0 = KV * (KG * (t_first + u) + kg) + 16 * KK * kh;
    f32x4 S[KK][2];
    bf16x8 pf[2][KK / 2];
    qk(S, kb);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int k = 0; k < KK; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key0 + 16 * k + 4 * lg + e >= lim[t]) S[k][t][e] = -INFINITY;
      const float mx = rowmax<HD>(S, t) * sc;
      if (__any(mx > m[t])) {                    // the largest itself: its weight is 1, without rounding
        const float mn = fmaxf(m[t], mx), al = mn == m[t] ? 1.f : __builtin_amdgcn_exp2f(m[t] - mn);
        m[t] = mn;
        l[t] *= al;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][t][e] *= al;
      }
      l[t] += weights(S, pf[t], t, sc, m[t] == -INFINITY ? 0.f : m[t]);
    }
    if (odd) {
      for (int k = 0; k < KK; ++k)
        for (int e = 0; e < 4; ++e)
          for (int g = 0; g < 4; ++g) {
            const int key = 16 * k + 4 * g + e;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              float p = 0.f;                     // of key and row lr, held by lane group g
#pragma unroll
              for (int q = 0; q < 4 * KK; ++q)
                if (q == 4 * k + e) p = (float)pf[t][q >> 3][q & 7];
              p = __shfl(p, 16 * g + lr, 64);
              if (key0 + key < lim[t])
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                  for (int d = 0; d < 4; ++d) {
                    const int col = 16 * i + 4 * lg + d;
                    o[i][t][d] += p * bf2f(*(const bf16_t *)(vb + V_BASE + (16 * KK * kh + key) * F::ROWB + ((col >> 3) ^ F::vkey(key)) * 16 + (col & 7) * 2));
                  }
            }
          }
    } else {
#pragma unroll
      for (int p = 0; p < KK / 2; ++p)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const bf16x8 vf = vfrag(vb, i, p);
#pragma unroll
          for (int t = 0; t < 2; ++t) o[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t][p], o[i][t], 0, 0, 0);
        }
    }
  }

  if constexpr (KG * KH == 2) {                       // the two softmaxes of every row meet
    f32x4 *xo = (f32x4 *)smem + (wr * 2 * NI) * 64 + lane;
    float2 *xm = (float2 *)((f32x4 *)smem + WR * 2 * NI * 64) + wr * 128 + lane;
    __syncthreads();
    if (kg + kh == 1) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < NI; ++i) xo[(t * NI + i) * 64] = o[i][t];
        xm[64 * t] = make_float2(m[t], l[t]);
      }
    }
    __syncthreads();
    if (kg + kh == 1) return;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float2 y = xm[64 * t];
      const float mn = fmaxf(m[t], y.x), ref = mn == -INFINITY ? 0.f : mn;
      const float a0 = __builtin_amdgcn_exp2f(m[t] - ref), a1 = __builtin_amdgcn_exp2f(y.x - ref);
      m[t] = mn;
      l[t] = a0 * l[t] + a1 * y.y;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const f32x4 z = xo[(t * NI + i) * 64];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][t][e] = a0 * o[i][t][e] + a1 * z[e];
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float den = quad_sum(l[t]);
    const int mr = m0 + 32 * wr + 16 * t + lr;
    if (mr >= count) continue;
    const int i0 = cache_row(c, mr), head = h * group + mr - i0 * group;
    if (part_ >= 0) {
      const int64_t at = part_slot(a, part_, s.q0 + i0, head);
#pragma unroll
      for (int i = 0; i < NI; ++i) *(f32x4 *)(a.part + at * HD + 16 * i + 4 * lg) = o[i][t];
      if (lg == 0) *(float2 *)part_ml(a, at) = make_float2(m[t], den);
      continue;
    }
    const float inv = 1.f / den;
    bf16_t *O = (bf16_t *)a.o + (int64_t)(s.q0 + i0) * a.ldo + (int64_t)head * HD + 4 * lg;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      bf16x4 y;
#pragma unroll
      for (int d = 0; d < 4; ++d) y[d] = (__bf16)(den == 0.f ? 0.f : o[i][t][d] * inv);
      *(bf16x4 *)(O + 16 * i) = y;
    }
    if (a.lse && lg == 0)
      a.lse[(int64_t)(s.q0 + i0) * c.heads + head] = den == 0.f ? -INFINITY : (m[t] + log2f(den)) * LN2;
  }
}

// ---------------------------------------------------------------- launches
// Rows per block and key ranges from the host's bounds, as over bf16.
//
// Up to 32 rows, and float32: blocks of 16 or 32 rows and enough ranges to fill the compute units, of several sequences
// (bf16) four times over, since they may be unlike (eight tokens over 1 to 32,768 keys, 32 heads on 8 of 128: 76 us with 1.5
// times, 54.5 with 4; of 64: 58 and 35), twice where their blocks alone do (sixteen over 4,000 each, 16 heads of 64: 41 us in
// one range, 34 in two or four, of 128: 56.5, 57.7 and 64). No range is shorter than
// 256 keys (one token over 4,000 keys, 32 heads on 8 of 64: 17.6 us in 4 ranges, 13.2 in 16), in float32 beyond 256 keys than 128.
//
// More rows: blocks of 32, 128 or 256 rows and the number of ranges by estimate: rounds of blocks on the compute units, 7 us for
// a block's start and end, a time per 64 keys (measured alone on a compute unit), then the second launch and the scratch written and
// read. It is within 10% of what was measured for 200 to 1,024 rows over 2,000 to 40,000 keys (32 rows of 32 heads on 8 of 128 over
// 40,000 keys: 44 us said and 46.5 measured; 1,024 rows over 8,192, 16 heads of 128: 83 and 82).
void plan8(int dtype, const CacheArgs &c, size_t scratch, int *rpb, int *range, int *splits) {
  const int64_t m = (int64_t)c.max_q * (c.heads / c.kvh);
  const int64_t cus = std::max(1, device_cus());
  auto set = [&](int r, int64_t keys) {
    *rpb = r;
    const int64_t step = r == 128 && c.hd == 64 ? 128 : 64;   // keys that a block works on at a time
    *range = (int)((std::max<int64_t>(keys, 64) + step - 1) / step * step);
    *splits = std::max(1, (c.cap + *range - 1) / *range);
  };
  if (dtype == 0 || m <= 32) {
    const int r = dtype == 1 && m <= 16 ? 16 : 32;
    const int64_t blocks = std::max<int64_t>(1, attn_blocks(r, c));
    const int64_t slots = c.batch == 1 ? cus : dtype == 0 ? cus * 3 / 2 : blocks < cus ? 4 * cus : 2 * cus;
    const int64_t want = std::max<int64_t>(1, slots / blocks);
    set(r, std::max<int64_t>(dtype == 1 || c.cap <= 256 ? 256 : 128, (c.cap + want - 1) / want));
  } else {
    // of several sequences not all ranges that the bounds allow for are there, the fewer the less the chunks fill their bound
    const int64_t most = std::max<int64_t>(1, (int64_t)c.batch * c.max_q);
    const int64_t slots = c.batch == 1 ? cus : cus + cus * 7 / 10 * (most - std::min<int64_t>(most, c.rows)) / most;
    const int64_t tiles = std::max(1, (c.cap + 63) / 64);
    const double part = (double)attn_part_bytes(c, 1) * 2 / 4e6;
    double best = 0;
    for (int r : {256, 128, 32}) {
      const double tile = c.hd == 128 ? (r == 256 ? 1.69 : r == 128 ? 1.15 : 0.95) : (r == 256 ? 1.09 : r == 128 ? 0.67 : 0.71);
      const int64_t blocks = std::max<int64_t>(1, attn_blocks(r, c));
      for (int64_t rounds = 0; rounds <= 4; ++rounds) {   // 0: not split; else the most ranges that fit so many rounds
        const int64_t most_n = std::max<int64_t>(1, std::min(rounds * slots / blocks, tiles / 4));
        const int64_t each = (tiles + most_n - 1) / most_n, n = (tiles + each - 1) / each;
        double t = (double)((blocks * n + slots - 1) / slots) * (each * tile + 7.0);
        if (n > 1) t += 5.0 + part * n;
        if (best == 0 || t < best) {
          best = t;
          set(r, each * 64);
        }
      }
    }
  }
  while (*splits > 1 && attn_part_bytes(c, *splits) > scratch) {
    *range = (int)std::min<int64_t>((int64_t)*range * 2, 1 << 30);
    *splits = (c.cap + *range - 1) / *range;
  }
}

template <int HD, int RT>
hipError_t launch_few8(const CacheAttnArgs &a, hipStream_t s) {
  constexpr int LDS = 4 * 64 * RT * HD;
  static DeviceOnce once;
  const hipError_t lim = once_on_device(once, [] {
    return hipFuncSetAttribute((const void *)k_cache8_attn_few<HD, RT>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  });
  if (lim != hipSuccess) return lim;
  hipLaunchKernelGGL((k_cache8_attn_few<HD, RT>), dim3(a.blocks), dim3(256), LDS, s, a);
  return hipGetLastError();
}
template <int HD, bool SMALL, int W, int KG, int KH>
hipError_t launch_many8(const CacheAttnArgs &a, hipStream_t s) {
  constexpr int LDS = KG * (KV * HD * (2 * (KS + VS) + 2 * RS) + ES * EB);
  static DeviceOnce once;
  const hipError_t lim = once_on_device(once, [] {
    return hipFuncSetAttribute((const void *)k_cache8_attn_many<HD, SMALL, W, KG, KH>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  });
  if (lim != hipSuccess) return lim;
  hipLaunchKernelGGL((k_cache8_attn_many<HD, SMALL, W, KG, KH>), dim3(a.blocks), dim3(64 * W), LDS, s, a);
  return hipGetLastError();
}
template <int HD>
hipError_t launch_hd(int dtype, const CacheAttnArgs &a, hipStream_t s) {
  constexpr int KG = HD == 64 ? 2 : 1, KH = HD == 64 ? 1 : 2;   // of blocks of 128 rows
  const bool small = a.c.plog < 6;
  if (dtype == 1 && a.rpb == 256) return small ? launch_many8<HD, true, 8, 1, 1>(a, s) : launch_many8<HD, false, 8, 1, 1>(a, s);
  if (dtype == 1 && a.rpb == 128) return small ? launch_many8<HD, true, 8, KG, KH>(a, s) : launch_many8<HD, false, 8, KG, KH>(a, s);
  if (dtype == 1) return a.rpb == 16 ? launch_few8<HD, 1>(a, s) : launch_few8<HD, 2>(a, s);
  hipLaunchKernelGGL((k_cache8_attn_f32<HD>), dim3(a.blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_pass8(int dtype, const CacheAttnArgs &a, hipStream_t s) {
  return a.c.hd == 128 ? launch_hd<128>(dtype, a, s) : launch_hd<64>(dtype, a, s);
}

}  // namespace

size_t cache8_attn_scratch(int dtype, const CacheArgs &c) {
  int rpb, range, splits;
  plan8(dtype, c, ~(size_t)0, &rpb, &range, &splits);
  return splits > 1 ? attn_part_bytes(c, splits) : 0;
}

hipError_t launch_cache8_attention(int dtype, const CacheAttnArgs &in, hipStream_t s) {
  CacheAttnArgs a = in;
  plan8(dtype, a.c, a.part ? a.part_bytes : 0, &a.rpb, &a.range, &a.splits);
  a.blocks = attn_grid(a);
  if (a.c.rows <= 0 || a.c.max_q <= 0) return hipSuccess;
  const hipError_t e = launch_pass8(dtype, a, s);
  return e != hipSuccess || a.splits <= 1 ? e : launch_combine(dtype, a, few_rows_of_many_parts(a), s);
}

// us per 64 keys in blocks of 16, 32, 128 and 256 rows (alone on a compute unit)
SharedPlan cache8_shared_plan(int dtype, const CacheArgs &c, const CacheShared &sh) {
  static const double tile[4][4] = {{0, 1.0, 0, 0}, {0, 2.0, 0, 0}, {0.55, 0.71, 0.67, 1.09}, {0.72, 0.95, 1.15, 1.69}};
  return plan_shared(dtype, c, sh, tile[2 * dtype + (c.hd == 128)]);
}

hipError_t launch_cache8_attention_shared(int dtype, const CacheAttnArgs &in, const SharedPlan &p, hipStream_t s) {
  return launch_shared(dtype, in, p, launch_pass8, s);
}

}  // namespace wdc
