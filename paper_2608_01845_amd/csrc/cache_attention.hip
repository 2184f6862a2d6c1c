// Attention of chunks of new rows over a paged key/value cache, and the weight
// that each cached key received from it.
//
// A chunk's rows and the query heads that share a kv head are one axis of query
// rows, m = i * group + g, so a key tile is read once for all of them. Row i sees
// the slots below cache_limit(i): limits grow with i, so of the key tiles of a
// block of rows a first part is seen by all rows whole, a second part in part, and
// the rest by none and is left out.
#include "cache_tiles.h"

#include <algorithm>
#include <type_traits>

namespace wdc {
namespace {

// Direct global -> LDS loads: lane l's 16 (4) bytes at `voff` of the buffer arrive
// at lds + 16 l (4 l). Written as instructions because the compiler lets no transposed LDS read pass while one
// of its own direct loads is under way (it waits for all of them); nothing is returned in
// registers, and the waits for the data are wait_vm's. The wait states are ours as well, since the compiler
// looks for hazards between its own instructions only: a scalar register written by a vector instruction
// (v_readfirstlane makes the descriptor's words) is there for a memory instruction five wait states later, one
// of s_mov_b32 and four of s_nop 3; M0 needs one of them.
__device__ __forceinline__ void lds_load16(u32x4_t buf, uint32_t lds, int voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(buf)
               : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(u32x4_t buf, uint32_t lds, int voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(buf)
               : "memory", "m0");
}
// Block of a launch over (sequence, kv head) x per blocks each. With the XCD order
// the blocks of one (sequence, kv head) share an XCD, and so its K and V in that L2.
__device__ __forceinline__ void cache_block(const CacheArgs &c, int per, int &bh, int &li) {
  li = c.xcd_order ? blockIdx.x >> 3 : blockIdx.x;
  const int q = uni(li / per);
  li -= q * per;
  bh = c.xcd_order ? (blockIdx.x & 7) + 8 * q : q;
}

// ---------------------------------------------------------------- bf16, few rows
// RT tiles of 16 query rows per block of four waves; wave w takes key tiles w, w +
// 4, .. of the block's range and the four partial softmaxes meet at the end. What
// bounds it is the stream of K and V, so each wave keeps a tile under way beside the
// one it works on, without a block barrier: direct loads into its own part of LDS, 8 KB a
// tile (32 keys of 64, 16 of 128). Eight tokens over 1 to 32,768 keys, 32 heads on 8 kv heads of 128: 85 to 87 us,
// 5.4 TB/s, also over four caches in turn, more than the last-level cache holds (a large copy, which writes too: 4.9).
//
// S^T = K Q^T (A: 16 keys, B: 16 rows) leaves lane (lr, lg) the keys 4 lg + e of
// row lr; these values of one (hd 128) or two key tiles are the B operand of O^T = V^T P^T, whose A
// operand is V^T: rows 4 lg .. 4 lg + 3 of V read transposed from LDS.
//
// Softmax in base 2 with a reference m per row that moves when a score passes it
// by more than 8: scores are scaled by log2(e)/sqrt(hd) in float32, weights are summed in
// float32 and rounded to bf16 once for the product with V (as its operand type). The rounded ones are summed as well
// and O is scaled by the ratio of the two sums: then it is a mean of V whatever their rounding, so that a key which
// has nearly all of the weight comes out as it is (else off by up to half a bf16 step, 1.6 times the error of a single
// rounding over keys of which a few dominate).
// Slots of a wave's K and V tiles: one in use, the other under way. Two blocks per compute unit with two slots each do
// more than one with four (16 heads of 64: 16 tokens over 4,000 keys 52.7 us, 57.1 with four; 2,048 over 100: 240, 479).
constexpr int FSL = 2;

template <int HD, int RT>
__global__ __launch_bounds__(256, 1) void k_cache_attn_few(CacheAttnArgs a) {
  using F = Few<HD>;
  constexpr int NC = HD / 32, NI = HD / 16, KT = F::KT, NB = FSL, WAVE = 2 * NB * F::TILE;   // K slots, V slots
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
    const bf16_t *Q = (const bf16_t *)a.q + (int64_t)(s.q0 + i) * a.ldq + (int64_t)(h * group + mm - i * group) * HD + 8 * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) qf[t][j] = *(const bf16x8 *)(Q + 32 * j);
  }

  char *mine = smem + w * WAVE;
  const uint32_t lds0 = lds_addr(mine);
  int kvo[F::LPH], vvo[F::LPH];                  // byte offsets in 16 rows of K and V
#pragma unroll
  for (int i = 0; i < F::LPH; ++i) {
    const int r = i * F::RPL + lane / (HD / 8), ch = lane % (HD / 8);
    kvo[i] = r * F::ROWB + (ch ^ F::kkey(r)) * 16;
    vvo[i] = r * F::ROWB + (ch ^ F::vkey(r)) * 16;
  }
  int kro[NC];                                   // K fragment of rows lr, dims 32 j + 8 lg
#pragma unroll
  for (int j = 0; j < NC; ++j) kro[j] = lr * F::ROWB + ((4 * j + lg) ^ F::kkey(lr)) * 16;
  int vro[F::VR];                                // transposed V read of rows 4 lg .. + 3, dims 16 i ..
  {
    const int r = 4 * lg + (lr >> 2), j = lane & 3;
#pragma unroll
    for (int i = 0; i < F::VR; ++i) vro[i] = r * F::ROWB + ((2 * i + (j >> 1)) ^ F::vkey(r)) * 16 + 8 * (j & 1);
  }
  PageWalk<false> pw;
  pw.init(c, k_.tab, k_.tab_last, h, (KT * t0) >> c.plog);
  const int pmask = (1 << c.plog) - 1;
  // Tile t into slot j: halves of 16 rows, each on one page. Rows past the cache's
  // end lie outside the buffer range and arrive as zeros, whatever they hold; so do tiles
  // past the range, which are asked for like the others so that the count of loads under way is fixed.
  auto load = [&](int t, int j) __attribute__((always_inline)) {
#pragma unroll
    for (int hf = 0; hf < F::NK; ++hf) {
      const int key = KT * t + 16 * hf;
      const bool live = t < t1;
      if (live) pw.advance(c, h, key >> c.plog);
      const int64_t off = (int64_t)(live ? pw.get(c, h, key >> c.plog) + (key & pmask) : 0) * F::ROWB;
      const int bytes = live ? min(max(s.n - key, 0), 16) * F::ROWB : 0;
      const u32x4_t kd = buffer_at(c.k, off, bytes), vd = buffer_at(c.v, off, bytes);
      const uint32_t to = lds0 + j * F::TILE + hf * 16 * F::ROWB;
#pragma unroll
      for (int i = 0; i < F::LPH; ++i) lds_load16(kd, to + i * 1024, kvo[i]);
#pragma unroll
      for (int i = 0; i < F::LPH; ++i) lds_load16(vd, to + NB * F::TILE + i * 1024, vvo[i]);
    }
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
  constexpr int LT = 2 * F::NK * F::LPH;         // loads per tile
  // tile t in slot J, with tile t + 4 (NB - 1) asked for
  auto step = [&](auto jc, int t) __attribute__((always_inline)) {
    constexpr int J = decltype(jc)::value;
    load(t + 4 * (NB - 1), (J + NB - 1) % NB);
    wait_vm<(NB - 1) * LT>();
    asm volatile("" ::: "memory");
    const char *kt = mine + J * F::TILE, *vt = kt + NB * F::TILE;
    f32x4 S[RT][F::NK];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int k = 0; k < F::NK; ++k) S[r][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int k = 0; k < F::NK; ++k) {
        const bf16x8 kf = *(const bf16x8 *)(kt + k * 16 * F::ROWB + kro[j]);
#pragma unroll
        for (int r = 0; r < RT; ++r) S[r][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][j], S[r][k], 0, 0, 0);
      }
    const bool part = KT * t + KT > lim_lo;      // some row does not see the whole tile
    bf16x4 pf[RT][F::NK];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < F::NK; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = S[r][k][e] * sc;
          if (KT * t + 16 * k + 4 * lg + e >= lim[r]) x = -INFINITY;
          S[r][k][e] = x;
          mx = fmaxf(mx, x);
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
      for (int k = 0; k < F::NK; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(S[r][k][e] - ref);
          l[r] += p;
          pf[r][k][e] = (__bf16)p;
          d[r] += (float)pf[r][k][e];
        }
    }
    // A key that a row does not see has weight 0, but 0 times an infinity or NaN
    // of its V is NaN in a matrix product. Tiles seen in part are looked over, and
    // one that holds such a value is multiplied key by key.
    bool odd = false;
    if (part) {
#pragma unroll
      for (int i = 0; i < F::TILE / 1024; ++i) {
        const u32x4_t u = *(const u32x4_t *)(vt + i * 1024 + lane * 16);
#pragma unroll
        for (int q = 0; q < 4; ++q) odd |= (u[q] & 0x7f80u) == 0x7f80u || (u[q] & 0x7f800000u) == 0x7f800000u;
      }
      odd = __any(odd);
    }
    if (odd) {
#pragma unroll 1
      for (int x = 0; x < KT; ++x) {             // key 16 (q / 4) + 4 g + q % 4
        const int q = x >> 2, g = x & 3, key = 16 * (q >> 2) + 4 * g + (q & 3);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          float p = 0.f;                         // of key and row lr, held by lane group g
#pragma unroll
          for (int y = 0; y < 4 * F::NK; ++y)
            if (y == q) p = (float)pf[r][y / 4][y % 4];
          p = __shfl(p, 16 * g + lr, 64);
          if (KT * t + key < lim[r])
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
        const char *vp = vt + vro[i % F::VR] + i / F::VR * F::VR * 32;
        if constexpr (F::NK == 2) {
          const bf16x8 vf = v_frag<HD>(vp);
#pragma unroll
          for (int r = 0; r < RT; ++r)
            o[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                vf, __builtin_shufflevector(pf[r][0], pf[r][F::NK - 1], 0, 1, 2, 3, 4, 5, 6, 7), o[r][i], 0, 0, 0);
        } else {
          const s16x4 vf = lds_read_tr(vp);
#pragma unroll
          for (int r = 0; r < RT; ++r)
            o[r][i] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf, __builtin_bit_cast(s16x4, pf[r][0]), o[r][i], 0, 0, 0);
        }
      }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0): the slot has been read before it is loaded again
  };
  if (t0 + w < t1) {
    static_assert(NB == 2, "slots of the unrolled steps");
    load(t0 + w, 0);
    for (int t = t0 + w; t < t1; t += 4 * NB) {
      step(std::integral_constant<int, 0>{}, t);
      if (t + 4 >= t1) break;
      step(std::integral_constant<int, 1>{}, t + 4);
    }
    wait_vm<0>();                                // what is still under way goes to this wave's part of LDS
    asm volatile("" ::: "memory");
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
// 32 query rows (two tiles of 16) a wave; key tiles of 64 reach four K and four V slots of LDS by direct buffer loads
// of four waves, up to four tiles ahead. Bound by the matrix cores, with the
// exponentials close behind, and by the power that both draw: 4,080 rows over 67,320 keys, 16 heads of 128, 1,750 to 1,860 us
// by device, 1,190 to 1,260 TFLOP/s (a large library product: 1,200 to 1,580), the matrix cores busy in 65% of the
// cycles of a clock that falls to 1.8 GHz.
//
// Blocks of 256 rows are 8 waves, two per SIMD: 1.0 us a tile at hd 64, 1.4 at hd 128. Few rows or keys leave
// compute units idle with them, so there are blocks of 128 rows too. At hd 128 they are 4 waves, 1.05 us a tile: one
// wave alone on a SIMD waits for its own results (1,720 cycles, of which 960 issue). At hd 64 two
// tiles fit into LDS at a time: KG = 2 groups of 4 waves take every second one each, 0.58 us a
// tile (0.77 with 4 waves), and their softmaxes meet at the end (2,048 rows causal over themselves, 16 heads: 26.7 us,
// 38.4 with 256 rows; 4,096 over 4,096 in full: 88.6, 77.4 with 256). Over a shared past the 128 rows at hd 128 have KH = 2
// groups of 4 waves, which take half of every tile's keys each and meet the same way (32 rollouts of a token, 32 heads on 8, off
// 24,448 shared keys: 56.7 us with 4 waves, 49 so).
//
// Tiles that all rows see whole run through a software pipeline: step t holds the P V
// products of tile t, the Q K products of tile t + 2 and, in the same instruction
// stream, the vector work of tile t + 1 (P = exp2(sc S - m), its row sum in float32, its
// rounding to bf16). m is a reference per row, not a running maximum: the first tile's
// maximum, moved only when a lane's sum of weights over a tile passes 2^16 (then O and the
// sum are rescaled and P is taken again): weights of up to that are as exact as those below 1, and sums of them times v
// stay within float32 while |v| is below 2^112 over the number of keys. Where a wave has references beyond 2^20, every
// tile's P is taken again (see far_out).
// Tiles that some row sees in part, and the cache's last, partial one, follow one at a
// time with their masks. There m is the row's largest score so far, so that a key with nearly all
// of the weight of a row that sees few has weight 1, without rounding. (Summing the rounded weights too, as with few
// rows, costs 5% on the call above and 20% on 2,048 rows causal over themselves.) At hd 128 a wave's 256 registers do not
// hold everything: 148 bytes a lane are in scratch, what only the masked tiles need: 21 to 23 reloads in each of them; none
// in the pipeline over pages of 64 slots and more, two a step over smaller ones.
constexpr int KV = 64, NB = 4;
constexpr float SUM_LIMIT = 0x1p16f;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// Loads of one wave (of four): stripe i of a tile is rows [(4 i + w) RPL, + RPL). SMALL:
// pages of 16 or 32 slots, where every stripe has its own page; otherwise a tile lies on one page.
template <int HD, bool SMALL>
struct TileLoads {
  using F = Few<HD>;
  static constexpr int NS = KV / (4 * F::RPL);   // stripes of a wave per tile (4 or 2)
  static constexpr int NP = SMALL ? NS : 1;
  struct Where {
    int64_t off[NP];                             // bytes from the pool to the tile (SMALL: the stripe's 16 rows)
    int bytes[NP];                               // what lies before the end of the cache
  };
  PageWalk<true> pw;                             // SMALL only
  int kvo_, w, h, n;                             // kvo_: the lane's byte offset in its stripe's rows of K
  __device__ __forceinline__ void init(const CacheArgs &c, const CacheSeq &s, const int32_t *tab, int tab_last, int h_, int w_,
                                       int lane, int tile0) {
    w = w_;
    h = h_;
    n = s.n;
    kvo_ = offset(lane);
    if (SMALL) pw.init(c, tab, tab_last, h, (KV * tile0) >> c.plog);
  }
  __device__ __forceinline__ int offset(int lane) const {
    const int r = w * F::RPL + lane / (HD / 8), ch = lane % (HD / 8);
    return (SMALL ? r & 15 : r) * F::ROWB + (ch ^ F::kkey(r)) * 16;
  }
  // With small pages it is found again each time: a register kept for it would be spilled as well, and its reload in every
  // step would wait for all loads under way. (The lane's number by an instruction that is not moved out of the loop.)
  __device__ __forceinline__ int kvo() const {
    if (!SMALL || HD == 64) return kvo_;
    int lane;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
    return offset(lane);
  }
  // the same of V, whose rows have another swizzle
  __device__ __forceinline__ int vvo() const {
    const int r = w * F::RPL + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)) / (HD / 8);
    return kvo() ^ ((F::kkey(r) ^ F::vkey(r)) * 16);
  }
  // page of a whole tile, by a scalar load (the table does not change during a launch)
  __device__ __forceinline__ int page(const CacheArgs &c, const int32_t *tab, int tab_last, int tile) const {
    typedef const __attribute__((address_space(4))) int32_t *scalar_ptr;
    const int e = min((KV * tile) >> c.plog, tab_last);
    return cache_page(c, ((scalar_ptr)(uint64_t)tab)[e]);
  }
  // where a tile lies; page: its page (unless SMALL)
  __device__ __forceinline__ void find(const CacheArgs &c, int tile, int page, Where &x) {
    const int pmask = (1 << c.plog) - 1, key0 = KV * tile, rest = n - key0;
    if (SMALL) pw.advance(c, h, key0 >> c.plog);   // a tile's pages are of one group of 64
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = SMALL ? (4 * i + w) * F::RPL / 16 * 16 : 0, key = key0 + at;
      const int slot = SMALL ? pw.get(c, h, key >> c.plog) : ((page * c.kvh + h) << c.plog);   // (pools hold fewer than 2^31)
      x.off[i] = (int64_t)(slot + (key & pmask)) * F::ROWB;
      x.bytes[i] = rest >= KV ? (SMALL ? 16 : KV) * F::ROWB : min(max(rest - at, 0), SMALL ? 16 : KV) * F::ROWB;
    }
  }
  __device__ __forceinline__ void load(const void *pool, const Where &x, uint32_t lds, int vo) const {
#pragma unroll
    for (int i = 0; i < NS; ++i)
      lds_load16(buffer_at(pool, x.off[SMALL ? i : 0], x.bytes[SMALL ? i : 0]), lds + i * 4096 + w * 1024,
                 SMALL ? vo : vo + i * 4096);
  }
};

template <int HD, bool SMALL, int W, int KG, int KH>
__global__ __launch_bounds__(64 * W, 8 / W) void k_cache_attn_many(CacheAttnArgs a) {
  using F = Few<HD>;
  using TL = TileLoads<HD, SMALL>;
  constexpr int NC = HD / 32, NI = HD / 16;
  constexpr int TB = KV * F::ROWB;               // bytes of a K or V tile
  constexpr int V_BASE = NB * TB;
  extern __shared__ __attribute__((aligned(16))) char smem[];
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
  constexpr int WR = W / (KG * KH);              // waves over the block's rows
  constexpr int KK = 4 / KH;                     // tiles of 16 keys of a wave
  // (rows of few waves lie on different SIMDs: waves w and w + 4 share one)
  const int kg = KG == 1 ? 0 : wid / WR, kh = KH == 1 ? 0 : wid / WR, wr = (wid + (kg + kh) * (WR / 2)) % WR;
  const bool grp_a = KG == 2 || wid < 4;         // loads tiles
  const int mlast = min(m0 + 32 * WR, count) - 1;
  const int lim_lo = k_.lim_lo, tiles = (k_.lim_hi + KG * KV - 1) / (KG * KV);   // in steps of KG tiles
  const int range = k_.range / (KG * KV), t_first = nr > 1 ? sp * range : 0, t_end = nr > 1 ? min(t_first + range, tiles) : tiles;
  // steps of the range, relative to t_first: `nf` that every row sees whole, then masked ones
  const int tot = t_end - t_first, nf = min(max(lim_lo / (KG * KV) - t_first, 0), tot);
  // The wave has no rows: it loads, and works on nothing (60 rows of a kv head over 40,000 keys, hd 64: 47.4 us with every wave
  // at work and 42.2 so; 32 of 32 heads on 8 off 24,448 shared keys: 49 and 45.7). In the other forms the
  // second loop costs registers: 4,080 rows over 67,320 keys 1,760 us without it, 1,860 with. Short ranges lose by the code
  // that they fetch (six causal chunks, hd 64, pages of 16: 28.3 us, 29.3 where the rule was for all lengths).
  const bool none = KG * KH == 2 && nf >= 8 && m0 + 32 * wr >= count;

  const float sc = LOG2E / sqrtf((float)HD);
  bf16x8 qf[2][NC];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int mm = min(m0 + 32 * wr + 16 * t + lr, mlast), i = cache_row(c, mm);
    const bf16_t *Q = (const bf16_t *)a.q + (int64_t)(s.q0 + i) * a.ldq + (int64_t)(h * group + mm - i * group) * HD + 8 * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) qf[t][j] = *(const bf16x8 *)(Q + 32 * j);
  }
  int kro[NC];                                   // K fragment of rows lr, dims 32 c + 8 lg
#pragma unroll
  for (int j = 0; j < NC; ++j) kro[j] = (16 * KK * kh + lr) * F::ROWB + ((4 * j + lg) ^ F::kkey(lr)) * 16;
  int vro[F::VR];                                // transposed V read of rows 4 lg .. + 3, dims 16 i ..
  {
    const int r = 4 * lg + (lr >> 2), j = lane & 3;
#pragma unroll
    for (int i = 0; i < F::VR; ++i) vro[i] = V_BASE + (16 * KK * kh + r) * F::ROWB + ((2 * i + (j >> 1)) ^ F::vkey(r)) * 16 + 8 * (j & 1);
  }
  char *ring = smem + kg * 2 * NB * TB;
  const uint32_t lds0 = lds_addr(ring);
  TL tl;
  typename TL::Where wk, wv;                     // of the latest K tile asked for, and of the one before
  auto page_of = [&](int t) { return SMALL ? 0 : tl.page(c, tab, tab_last, KG * (t_first + t) + kg); };
  auto load_k = [&](int t, int page) __attribute__((always_inline)) {
    wv = wk;
    tl.find(c, KG * (t_first + t) + kg, page, wk);
    tl.load(c.k, wk, lds0 + (t % NB) * TB, tl.kvo());
  };
  auto load_v = [&](int t, const typename TL::Where &x) { tl.load(c.v, x, lds0 + V_BASE + (t % NB) * TB, tl.vvo()); };

  int page[NB];                                  // of the K tiles that the next NB steps ask for
  if (grp_a) {                                   // K_0 .. K_3, V_0 .. V_2; the first products wait for K_0 and K_1 alone
    tl.init(c, s, tab, tab_last, h, wid & 3, lane, KG * t_first + kg);
    wk = typename TL::Where{};
    int first[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) first[j] = page_of(j);
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (j < tot) {
        load_k(j, first[j]);
        if (j > 0) load_v(j - 1, wv);
      }
    if (tot < NB && tot > 0) load_v(tot - 1, wk);
    if (nf >= 2 && tot >= NB)
      wait_vm<(NB + 1) * TL::NS>();              // K_0, V_0's neighbour K_1
    else
      wait_vm<0>();
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) page[j] = page_of(NB + j);
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
        const bf16x8 kf = *(const bf16x8 *)(kb + kro[j] + k * 16 * F::ROWB);
#pragma unroll
        for (int t = 0; t < 2; ++t)
          S[k][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][j], j == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : S[k][t], 0, 0, 0);
      }
  };
  auto vfrag = [&](const char *vb, int i, int p) {   // V^T fragment: dims 16 i .., keys of the 32-key group p
    return v_frag<HD>(vb + vro[i % F::VR] + i / F::VR * F::VR * 32 + p * 32 * F::ROWB);
  };

  if (nf > 0) {
    f32x4 S[2][KK][2];                           // S of tiles t + 1 and t + 2 (index tile & 1)
    bf16x8 pf[2][2][KK / 2];                          // P of tiles t and t + 1 (index tile & 1), [row tile][32-key group]
    qk(S[0], ring);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      m[t] = fmaxf(rowmax<HD>(S[0], t) * sc, -FLT_MAX);   // (scores of -inf: weight 0)
      l[t] = weights(S[0], pf[0][t], t, sc, m[t]);
    }
    // a lane's sum of weights above which a tile's weights are taken again; far out all are
    float limit = far_out(fmaxf(fabsf(m[0]), fabsf(m[1]))) ? -1.f : SUM_LIMIT;
    if (nf > 1) qk(S[1], ring + TB);
    if (grp_a) {                                 // K_2 and V_1: at most K_3 and V_2 are still under way
      if (tot >= NB)
        wait_vm<2 * TL::NS>();
      else
        wait_vm<0>();
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // step 0 refills the slot of K_0
    constexpr int NPV = KK / 2 * NI, NMF = NPV + KK * NC;   // fragment reads of P V, and of a step; two MFMAs each
    constexpr int EPM = 8 * KK / NMF;            // exponentials per pair of MFMAs
    static_assert(NMF == 16 || NMF == 32, "hd 64 or 128");
    bf16x8 fr_[NMF];
    // One step, P = t % NB at compile time. c indexes S of tile t + 1 and the P it becomes, n S of tile t
    // + 2 and the P of tile t. Pairs of MFMAs (one per row tile) in a fixed order: P V (32-key group q / NI, O tile
    // q % NI), then Q K (dims 32 (g / 4).., key tile g % 4, g = q - NPV); fragment q is read four pairs ahead of its
    // use (0 to 3 in the step before). Past the last tile the stream runs on stale slots and S, unused.
    // Exponential x is key tile x / 8, row tile (x / 4) % 2, entry x % 4; the empty asm pins it under these MFMAs.
    auto read = [&](int r, const char *vb, const char *kb) __attribute__((always_inline)) {
      const int g = r >= NPV ? r - NPV : 0;
      if (r < NPV)
        fr_[r] = vfrag(vb, r % NI, (r < NPV ? r : 0) / NI);
      else
        fr_[r] = *(const bf16x8 *)(kb + kro[g / KK] + (g % KK) * 16 * F::ROWB);
    };
#pragma unroll
    for (int r = 0; r < 4; ++r) read(r, ring, ring);
    auto step = [&](auto pc, int t, int page) __attribute__((always_inline)) {
      constexpr int P = decltype(pc)::value, cur = (P + 1) & 1, n = P & 1;
      int issued = 0;
      if (grp_a) {
        if (t + 4 < tot) {
          load_k(t + 4, page);
          issued += TL::NS;
        } else {
          wv = wk;
        }
        if (t + 3 < tot) {
          load_v(t + 3, wv);
          issued += TL::NS;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      const char *vb = ring + P * TB, *kb = ring + ((P + 2) % NB) * TB, *vn = ring + ((P + 1) % NB) * TB;
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
      }
      if (t + 1 < nf) {
        if (__any(!(fmaxf(ls[0], ls[1]) <= limit))) {
#pragma unroll
          for (int t_ = 0; t_ < 2; ++t_) {
            const float mx = rowmax<HD>(S[cur], t_) * sc, mn = mx > m[t_] + 8.f ? mx : m[t_];
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
      // the loads of earlier steps are done, and all reads but the four just issued
      if (grp_a) {
        if (issued == 2 * TL::NS)
          wait_vm<2 * TL::NS>();
        else if (issued == TL::NS)
          wait_vm<TL::NS>();
        else
          wait_vm<0>();
      }
      asm volatile("s_waitcnt lgkmcnt(%0)\n\ts_barrier" ::"n"(8) : "memory");
    };
    if (none) {
#pragma unroll 1
      for (int t = 0; t < nf; ++t) {
        int issued = 0;
        if (grp_a) {
          if (t + 4 < tot) {
            load_k(t + 4, page_of(t + 4));
            issued += TL::NS;
          } else {
            wv = wk;
          }
          if (t + 3 < tot) {
            load_v(t + 3, wv);
            issued += TL::NS;
          }
          if (issued == 2 * TL::NS)
            wait_vm<2 * TL::NS>();
          else if (issued == TL::NS)
            wait_vm<TL::NS>();
          else
            wait_vm<0>();
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      }
    } else
    for (int t = 0; t < nf; t += NB) {
      int next[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) next[j] = page_of(t + 2 * NB + j);
      step(std::integral_constant<int, 0>{}, t, page[0]);
      if (t + 1 >= nf) break;
      step(std::integral_constant<int, 1>{}, t + 1, page[1]);
      if (t + 2 >= nf) break;
      step(std::integral_constant<int, 2>{}, t + 2, page[2]);
      if (t + 3 >= nf) break;
      step(std::integral_constant<int, 3>{}, t + 3, page[3]);
#pragma unroll
      for (int j = 0; j < NB; ++j) page[j] = next[j];
    }
  }

  // masked tiles, one at a time: tile u with K and V of u + 1 and u + 2 under way
  int lim[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int mr = m0 + 32 * wr + 16 * t + lr;
    lim[t] = mr < count ? cache_limit(c, s, cache_row(c, mr)) : 0;
  }
  for (int u = nf; u < tot; ++u) {
    if (grp_a) wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (grp_a && u + 3 < tot) {
      if (u > nf) load_k(u + 3, page_of(u + 3));                 // at u = nf the pipeline has asked for it already
      load_v(u + 3, wk);
    }
    const char *kb = ring + (u % NB) * TB, *vb = ring + (u % NB) * TB;   // vro holds V_BASE
    // A key that a row does not see has weight 0, but 0 times an infinity or NaN of
    // its V is NaN in a matrix product: a tile that holds one is multiplied key by key.
    bool odd = false;
#pragma unroll
    for (int i = 0; i < TB / (1024 * WR); ++i) {   // (with KH of 2 both waves of a row part look over all of it)
      const u32x4_t y = *(const u32x4_t *)(vb + V_BASE + (i * 64 * WR + 64 * wr + lane) * 16);
#pragma unroll
      for (int q = 0; q < 4; ++q) odd |= (y[q] & 0x7f80u) == 0x7f80u || (y[q] & 0x7f800000u) == 0x7f800000u;
    }
    odd = __syncthreads_or(odd);
    if (none) continue;
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

// ---------------------------------------------------------------- float32
// float32 attention on v_mfma_f32_32x32x2_f32 (64 cycles each): a block's four
// waves share 32 rows and take every fourth key tile of 32 of the block's range. S^T = K Q^T
// leaves a lane one row and 16 keys, which O^T = V^T P^T takes one by one as its B
// operand. Bound by the matrix instructions, so K and V come straight from the
// caches: K of the next tile is asked for under this tile's softmax and P V. Keys past
// the cache's end are read as its last key and get weight 0. Chunks of 256 and 100 rows over 1,500 and 777 keys, 4 heads of 64:
// 14 us and 4 of the parts' launch; a wave has two tiles there, most of it latency. 2,040 rows over 10,200 keys, 8 heads of
// 128: 786 us, 108 TFLOP/s of a library product's 153.
template <int HD>
__global__ __launch_bounds__(256, 1) void k_cache_attn_f32(CacheAttnArgs a) {
  constexpr int NI = HD / 32, NC = HD / 8;
  typedef __attribute__((ext_vector_type(NI))) float vecn;
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
  const float *Q = (const float *)a.q + (int64_t)(s.q0 + row) * a.ldq + (int64_t)(h * group + mm - row * group) * HD + 4 * lg;
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
  const int head = h * group + mm - row * group, dim0 = NI * (8 * w + 4 * lg);
  const int64_t at = part_slot(a, max(part_, 0), s.q0 + row, head);
  float *O = part_ >= 0 ? a.part + at * HD + dim0
                          : (float *)a.o + (int64_t)(s.q0 + row) * a.ldo + (int64_t)head * HD + dim0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float y = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) y += wt[u] * po[u][i * 16 + 4 * w + e][lane];
      O[NI * e + i] = part_ >= 0 ? y : den == 0.f ? 0.f : y / den;
    }
  if (w != 0 || lg != 0) return;
  if (part_ >= 0) {
    *(float2 *)part_ml(a, at) = make_float2(mx, den);
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

// Rows of a key tile's launch part: tiles of `step` query rows from the first that sees key0
struct MassRows {
  int r0, r1;
  __device__ __forceinline__ MassRows(const CacheMassArgs &a, const CacheSeq &s, int group, int key0, int step, int sp) {
    const int lo = first_row(a.c, s, key0) * group / step, hi = (s.nq * group + step - 1) / step;
    const int span = max(hi - lo, 0);
    r0 = lo + (int)((int64_t)sp * span / a.splits);
    r1 = lo + (int)((int64_t)(sp + 1) * span / a.splits);
  }
};

// bf16: a block of four waves holds 256 keys, 64 a wave, in registers (A operand)
// and streams the rows past them, 128 a stage through two LDS slots of direct loads; every wave
// reads all rows (B operand). A lane holds one row and 16 keys of a tile of 16 x 64 and adds
// exp2(sc x - lse) to its 16 sums. Multiply-add, exponential and sum are 16 cycles for 64 weights, as many as hd 128's
// matrix work; the vector units are busy in 69% of the cycles and the matrix cores in 48%. What is lost: the blocks' last
// round, and in each stage one turn of nine without exponentials and one without products. 2,040 rows over 34,680 keys, 16
// heads of 128, 287 to 310 us by device and load (1,010 to 930 TFLOP/s; two waves per SIMD that share the rows' tiles: 339).
constexpr int MKT = 256, MST = 128, MNB = 2;
template <int HD>
__global__ __launch_bounds__(256, 2) void k_cache_mass_bf16(CacheMassArgs a) {
  using F = Few<HD>;
  constexpr int NC = HD / 32, NL = MST / (4 * F::RPL);   // loads of a wave per stage (8 or 4)
  constexpr int NZ = MST / 64, NQ = MST / 16;
  constexpr int QB = MST * F::ROWB;
  __shared__ __attribute__((aligned(16))) char qs[MNB * QB];
  __shared__ __attribute__((aligned(16))) float zs[MNB][4][MST];
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh, nkt = (c.cap + MKT - 1) / MKT;
  int bh, li;
  cache_block(c, nkt * a.splits, bh, li);
  const int kt = uni(li / a.splits), sp = li - kt * a.splits, b = uni(bh / c.kvh), h = bh - b * c.kvh;
  const CacheSeq s = uniform_seq(c, b);
  const int key0 = kt * MKT;
  if (key0 >= s.n) return;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int count = s.nq * group, kw = key0 + 64 * w;
  const MassRows rows(a, s, group, key0, MST, sp);
  const int32_t *tab = c.table + (int64_t)b * c.table_ld;
  bf16x8 kf[4][NC];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const bf16_t *p = (const bf16_t *)c.k + slot_row(c, tab, h, min(kw + 16 * k + lr, s.n - 1)) + 8 * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) kf[k][j] = *(const bf16x8 *)(p + 32 * j);
  }
  // Stage r into slot j: its rows lie at fixed offsets from its first chunk row i0
  // if the group divides 128; for other groups, and for rows past the last (read as the last), they are found per stage.
  int qo[NL], zo[NZ];
  const uint32_t qa = lds_addr(qs), za = lds_addr(zs);
  auto place = [&](int r, int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int x = (4 * i + w) * F::RPL + lane / (HD / 8), m = min(r * MST + x, count - 1), row = cache_row(c, m);
      qo[i] = (int)((row - i0) * a.ldq + (m - row * group) * HD) * 2 + ((lane % (HD / 8)) ^ F::kkey(x)) * 16;
    }
#pragma unroll
    for (int i = 0; i < NZ; ++i) {
      const int m = min(r * MST + 64 * i + lane, count - 1), row = cache_row(c, m);
      zo[i] = ((row - i0) * c.heads + m - row * group) * 4;
    }
  };
  const bool fixed = (group & (group - 1)) == 0;   // group <= 64
  auto load = [&](int r, int j) {
    const int i0 = cache_row(c, r * MST);
    if (!fixed || r * MST + MST > count) place(r, i0);
    const u32x4_t qd = buffer_at(a.q, ((int64_t)(s.q0 + i0) * a.ldq + (int64_t)h * group * HD) * 2, 0x7fffffff);
    const u32x4_t zd = buffer_at(a.lse, ((int64_t)(s.q0 + i0) * c.heads + h * group) * 4, 0x7fffffff);
#pragma unroll
    for (int i = 0; i < NL; ++i) lds_load16(qd, qa + j * QB + (4 * i + w) * 1024, qo[i]);
#pragma unroll
    for (int i = 0; i < NZ; ++i) lds_load4(zd, za + ((j * 4 + w) * MST + 64 * i) * 4, zo[i]);
  };
  int qro[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) qro[j] = lr * F::ROWB + ((4 * j + lg) ^ F::kkey(lr)) * 16;
  const float sc = LOG2E / sqrtf((float)HD);
  float sum[4][4] = {};
  const int n = rows.r1 - rows.r0;
  // from this chunk row on, every row sees all of the wave's keys
  const int whole = first_row(c, s, min(kw + 63, s.n - 1));
  if (n > 0) {
    place(rows.r0, cache_row(c, rows.r0 * MST));
    load(rows.r0, 0);
  }
  for (int t = 0; t < n; ++t) {
    const int r = rows.r0 + t, j = t % MNB;
    wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");      // slot j is there, and the other one has been read
    if (t + 1 < n) load(r + 1, (t + 1) % MNB);
    const bool part = r * MST + MST > count || cache_row(c, r * MST) < whole;
    const char *qb = qs + j * QB;
    const float *zb = zs[j][w];
    // Row tile q's matrix products run in one stream with the exponentials of tile
    // q - 1, so that a wave's vector work executes under its own MFMAs.
    bf16x8 qf[2][NC];
    f32x4 x[2][4];
    float z[2];
    int lim[2] = {0, 0};
    auto fetch = [&](int q) __attribute__((always_inline)) {
#pragma unroll
      for (int jj = 0; jj < NC; ++jj) qf[q & 1][jj] = *(const bf16x8 *)(qb + q * 16 * F::ROWB + qro[jj]);
    };
    auto stream = [&](auto masked) __attribute__((always_inline)) {
      constexpr bool M = decltype(masked)::value;
      fetch(0);
#pragma unroll
      for (int q = 0; q <= NQ; ++q) {
        if (q < NQ - 1) fetch(q + 1);
        if (q < NQ) z[q & 1] = zb[16 * q + lr] * LOG2E;
        if (M && q < NQ) {
          const int m = r * MST + 16 * q + lr;
          lim[q & 1] = m < count ? cache_limit(c, s, cache_row(c, m)) : 0;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (q < NQ && i % (4 / NC) == 0) {
            const int mm = i / (4 / NC), jj = mm / 4, k = mm % 4;
            x[q & 1][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k][jj], qf[q & 1][jj],
                                                                  jj == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : x[q & 1][k], 0, 0, 0);
          }
          if (q > 0) {
            const int p = (q - 1) & 1, k = i / 4, e = i % 4;
            float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[p][k][e], sc, -z[p]));
            if (M) y = kw + 16 * k + 4 * lg + e < lim[p] ? y : 0.f;
            sum[k][e] += y;
            asm volatile("" : "+v"(sum[k][e]));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    if (part)
      stream(std::true_type{});
    else
      stream(std::false_type{});
    __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0): this wave's reads of the slot are done
  }
  // lane lr < 16 of each lane group: key 16 k + 4 lg + e with k = lr / 4, e = lr % 4
  float mine = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = group_sum<16>(sum[k][e]);
      if (lr == 4 * k + e) mine = v;
    }
  const int key = kw + 16 * (lr >> 2) + 4 * lg + (lr & 3);
  if (key >= s.n) return;
  if (a.splits > 1)
    a.part[((int64_t)bh * a.splits + sp) * c.cap + key] = mine;
  else
    mass_store(a, s, b, h, key, mine);
}

// float32: four waves share 32 keys, held in registers, and take every fourth
// tile of 32 rows, read straight from the caches: bound by the matrix instructions (64 cycles each): 2,040 rows over 10,200
// keys, 8 heads of 128, 425 us, 100 TFLOP/s of a library product's 153; 356 rows over 1,500 and 777 keys 11 us, latency.
template <int HD>
__global__ __launch_bounds__(256) void k_cache_mass_f32(CacheMassArgs a) {
  constexpr int KT = 32, NC = HD / 8;
  const CacheArgs &c = a.c;
  const int group = c.heads / c.kvh, nkt = (c.cap + KT - 1) / KT;
  int bh, li;
  cache_block(c, nkt * a.splits, bh, li);
  const int kt = uni(li / a.splits), sp = li - kt * a.splits, b = uni(bh / c.kvh), h = bh - b * c.kvh;
  const CacheSeq s = uniform_seq(c, b);
  const int key0 = kt * KT;
  if (key0 >= s.n) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lg = lane >> 5, count = s.nq * group;
  const MassRows rows(a, s, group, key0, 32, sp);
  const int32_t *tab = c.table + (int64_t)b * c.table_ld;
  f32x4 kf[NC];
  {
    const float *p = (const float *)c.k + slot_row(c, tab, h, min(key0 + lr, s.n - 1)) + 4 * lg;
#pragma unroll
    for (int j = 0; j < NC; ++j) kf[j] = *(const f32x4 *)(p + 8 * j);
  }
  const float sc = LOG2E / sqrtf((float)HD);
  float sum[16] = {};
  for (int r = rows.r0 + w; r < rows.r1; r += 4) {
    const int m = r * 32 + lr, mm = min(m, count - 1), i = cache_row(c, mm), head = h * group + mm - i * group;
    const float *Q = (const float *)a.q + (int64_t)(s.q0 + i) * a.ldq + (int64_t)head * HD + 4 * lg;
    const float z = a.lse[(int64_t)(s.q0 + i) * c.heads + head] * LOG2E;
    const int lim = m < count ? cache_limit(c, s, i) : 0;
    f32x16 x;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const f32x4 qf = *(const f32x4 *)(Q + 8 * j);
#pragma unroll
      for (int d = 0; d < 4; ++d) x = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j][d], qf[d], x, 0, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float p = exp2f(x[e] * sc - z);
      sum[e] += key0 + 8 * (e / 4) + 4 * lg + e % 4 < lim ? p : 0.f;
    }
  }
  __shared__ float ws[4][KT];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float v = group_sum<16>(sum[e]);
    v += __shfl_xor(v, 16, 64);
    if (lr == 0) ws[w][8 * (e / 4) + 4 * lg + e % 4] = v;
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
// Rows per block and key ranges. Lengths are known on the device only; the host
// has their bounds.
//
// Up to 64 rows, and float32: blocks of 16 or 32 rows, and enough ranges to fill
// the compute units; with several sequences half as many again, since some are shorter (eight tokens over 1 to 32,768
// keys, 32 heads on 8 of 128: 87 us, 103 without; 16 over 4,000 keys each, 16 heads of 128: 94, 98 with twice as many; four
// over 100 to 30,000: 40, 50 without and 36 with twice as many). A second launch and its reads
// cost about 5 us: 16 rows and fewer are not cut below 65,536 / hd keys (1,000 keys, 16 heads
// of 64, one row: 10.1 us whole, 13.0 in four), others not below 256, float32 beyond 256 keys not below 128 (its tile
// of 32 keys is 2 us of matrix instructions, 4 at hd 128: one row over 642 keys, 8 heads, 16.5 and 22.9 us with 256, 13.7 and 17.9 so).
// Of hd 128 only up to 32 rows where there is much to read (64 rows, 16 heads, eight sequences of 1,000 keys: 34
// us, 28.6 in blocks of 128 rows; one of 3,456 keys: 19.4 and 20.8).
//
// More rows: blocks of 128 or 256 rows and the number of ranges by estimate: rounds of blocks on
// the compute units, a start and end of 7 us each and a time per tile of 64 keys (measured alone
// on a compute unit: 256 rows 1.03 us at hd 64, 1.4 at hd 128; 128 rows 0.58 and 1.08), then the
// second launch and the scratch written and read. 384 rows over 3,456 keys, 16 heads of 64: 256 rows 27.1 us, 128 rows 23.9;
// 1,024 over 8,192 keys, 16 heads of 128: 77 against 84. Three chunks of 333 rows over 3,456 keys:
// 55 us if half of the ranges are taken to be there, 41 as they fill their bound.
void attn_plan(int dtype, const CacheArgs &c, size_t scratch, int *rpb, int *range, int *splits) {
  const int64_t m = (int64_t)c.max_q * (c.heads / c.kvh);
  // Of several sequences not all ranges that the bounds allow for are there: of few rows each two thirds; else
  // the fewer the less the chunks fill their bound (unlike chunks going with unlike lengths)
  const bool few = dtype == 0 || m <= 32 || (m <= 64 && (c.hd == 64 || (int64_t)c.batch * c.kvh * c.cap < 100000));
  const int64_t cus = std::max(1, device_cus()), most = std::max<int64_t>(1, (int64_t)c.batch * c.max_q);
  const int64_t slots = c.batch == 1 ? cus : few ? cus * 3 / 2 : cus + cus * 7 / 10 * (most - std::min<int64_t>(most, c.rows)) / most;
  auto set = [&](int r, int64_t keys) {
    *rpb = r;
    const int64_t step = r == 128 && c.hd == 64 ? 128 : 64;   // keys that a block works on at a time
    *range = (int)((std::max<int64_t>(keys, 64) + step - 1) / step * step);
    *splits = std::max(1, (c.cap + *range - 1) / *range);
  };
  if (few) {
    const int r = dtype == 1 && m <= 16 ? 16 : 32;
    const int64_t blocks = std::max<int64_t>(1, attn_blocks(r, c));
    const int64_t want = std::max<int64_t>(1, slots / blocks);
    const int64_t least = r == 16 ? 65536 / c.hd : dtype == 1 || c.cap <= 256 ? 256 : 128;
    set(r, std::max(least, (c.cap + want - 1) / want));
  } else {
    const int64_t tiles = (c.cap + 63) / 64;
    double best = 0;
    for (int r = 256; r >= 128; r -= 128) {
      const double tile = c.hd == 128 ? (r == 256 ? 1.4 : 1.08) : (r == 256 ? 1.03 : 0.58);
      const int64_t blocks = std::max<int64_t>(1, attn_blocks(r, c));
      for (int64_t n = 1; n <= 32 && (n == 1 || tiles >= 4 * n); ++n) {
        const double rounds = (double)((blocks * n + slots - 1) / slots);
        double t = rounds * ((double)((tiles + n - 1) / n) * tile + 7.0);
        if (n > 1) t += 5.0 + (double)attn_part_bytes(c, (int)n) * 2 / 4e6;
        if (best == 0 || t < best) {
          best = t;
          set(r, (tiles + n - 1) / n * 64);
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
hipError_t launch_few(const CacheAttnArgs &a, hipStream_t s) {
  constexpr int LDS = 4 * 2 * FSL * Few<HD>::TILE;
  static DeviceOnce once;
  const hipError_t lim = once_on_device(once, [] {
    return hipFuncSetAttribute((const void *)k_cache_attn_few<HD, RT>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  });
  if (lim != hipSuccess) return lim;
  hipLaunchKernelGGL((k_cache_attn_few<HD, RT>), dim3(a.blocks), dim3(256), LDS, s, a);
  return hipGetLastError();
}
template <int HD, bool SMALL, int W, int KG, int KH>
hipError_t launch_many(const CacheAttnArgs &a, hipStream_t s) {
  constexpr int LDS = KG * 2 * NB * KV * Few<HD>::ROWB;
  static DeviceOnce once;
  const hipError_t lim = once_on_device(once, [] {
    return hipFuncSetAttribute((const void *)k_cache_attn_many<HD, SMALL, W, KG, KH>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  });
  if (lim != hipSuccess) return lim;
  hipLaunchKernelGGL((k_cache_attn_many<HD, SMALL, W, KG, KH>), dim3(a.blocks), dim3(64 * W), LDS, s, a);
  return hipGetLastError();
}
template <int HD>
hipError_t launch_bf16(const CacheAttnArgs &a, hipStream_t s) {
  constexpr int W128 = HD == 64 ? 8 : 4, KG = HD == 64 ? 2 : 1;   // of blocks of 128 rows
  const int rpb = a.rpb;
  const bool small = a.c.plog < 6;
  if (rpb == 256) return small ? launch_many<HD, true, 8, 1, 1>(a, s) : launch_many<HD, false, 8, 1, 1>(a, s);
  if constexpr (HD == 128)
    if (rpb == 128 && a.sh.groups > 0) return small ? launch_many<HD, true, 8, 1, 2>(a, s) : launch_many<HD, false, 8, 1, 2>(a, s);
  if (rpb == 128) return small ? launch_many<HD, true, W128, KG, 1>(a, s) : launch_many<HD, false, W128, KG, 1>(a, s);
  return rpb == 16 ? launch_few<HD, 1>(a, s) : launch_few<HD, 2>(a, s);
}

}  // namespace

size_t cache_attn_scratch(int dtype, const CacheArgs &c) {
  int rpb, range, splits;
  attn_plan(dtype, c, ~(size_t)0, &rpb, &range, &splits);
  return splits > 1 ? attn_part_bytes(c, splits) : 0;
}

static hipError_t launch_pass(int dtype, const CacheAttnArgs &a, hipStream_t s) {
  if (dtype == 1) return a.c.hd == 128 ? launch_bf16<128>(a, s) : launch_bf16<64>(a, s);
  const dim3 grid(a.blocks);
  if (a.c.hd == 128)
    hipLaunchKernelGGL((k_cache_attn_f32<128>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_cache_attn_f32<64>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_attention(int dtype, const CacheAttnArgs &in, hipStream_t s) {
  CacheAttnArgs a = in;
  attn_plan(dtype, a.c, a.part ? a.part_bytes : 0, &a.rpb, &a.range, &a.splits);
  a.blocks = attn_grid(a);
  if (a.c.rows <= 0 || a.c.max_q <= 0) return hipSuccess;
  const hipError_t e = launch_pass(dtype, a, s);
  return e != hipSuccess || a.splits <= 1 ? e : launch_combine(dtype, a, false, s);
}

// us per 64 keys in blocks of 16, 32, 128 and 256 rows (alone on a compute unit)
SharedPlan cache_shared_plan(int dtype, const CacheArgs &c, const CacheShared &sh) {
  static const double tile[4][4] = {{0, 1.0, 0, 0}, {0, 2.0, 0, 0}, {0.55, 0.71, 0.58, 1.03}, {0.72, 0.95, 0.95, 1.4}};
  return plan_shared(dtype, c, sh, tile[2 * dtype + (c.hd == 128)]);
}

hipError_t launch_cache_attention_shared(int dtype, const CacheAttnArgs &in, const SharedPlan &p, hipStream_t s) {
  return launch_shared(dtype, in, p, launch_pass, s);
}

static int64_t mass_blocks(int dtype, const CacheArgs &c) {
  const int kt = dtype == 1 ? MKT : 32;
  return (int64_t)c.batch * c.kvh * (((int64_t)c.cap + kt - 1) / kt);
}
static size_t mass_part_bytes(const CacheArgs &c, int splits) {
  return (size_t)c.batch * c.kvh * splits * c.cap * sizeof(float);
}
// Row ranges of at least 256 rows, as many as give every compute unit a block (300 rows over 1,000 keys, 4 heads of 64:
// 11.3 us, 14.5 in two ranges; 600: 13.9 and 12.8)
static int mass_wanted(int dtype, const CacheArgs &c) {
  const int64_t fill = device_cus() / std::max<int64_t>(1, mass_blocks(dtype, c));
  const int64_t most = (int64_t)c.max_q * (c.heads / c.kvh) / 256;
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
      hipLaunchKernelGGL((k_cache_mass_bf16<128>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_cache_mass_bf16<64>), grid, dim3(256), 0, s, a);
  } else {
    if (a.c.hd == 128)
      hipLaunchKernelGGL((k_cache_mass_f32<128>), grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_cache_mass_f32<64>), grid, dim3(256), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits <= 1) return e;
  hipLaunchKernelGGL(k_cache_mass_combine, dim3((a.c.cap + 255) / 256, a.c.kvh, a.c.batch), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace wdc
