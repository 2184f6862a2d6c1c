// Paged key/value cache of a streaming rollout: storing a chunk's keys and
// values (with the per-head norms and the rotation of q and k in the same pass)
// and dropping the keys of least accumulated attention weight. The attention
// over the cache and the accumulation of its weights: cache_attention.hip.
#include "common.h"

#include <algorithm>
#include <type_traits>

namespace wdc {
namespace {

// ---------------------------------------------------------------- append
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 u = *(const bf16x8 *)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)u[e];
  } else {
    const f32x4 u = *(const f32x4 *)p, v = *(const f32x4 *)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = u[e];
      x[4 + e] = v[e];
    }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 u;
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = (__bf16)x[e];
    *(bf16x8 *)p = u;
  } else {
    *(f32x4 *)p = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4 *)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// Eight elements of a head over HD / 8 lanes as e4m3 codes of x 2^-E, with E the smallest exponent, from -117 on, that keeps
// the head's finite elements within 448 2^E (448: the largest code). Returns E + 127. A power of two changes no
// digit of a floating-point code, and from 2^-117 on every value code 2^E is a normal number in bf16 as in float32: what
// reads the cache has the values exactly. The one rounding is to nearest even; infinities and NaN become NaN, and elements
// beyond 240 * 2^120, the largest value of these that is finite, become it.
template <int HD>
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint2 &codes) {
  float big = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(x[e]) < INFINITY ? fabsf(x[e]) : 0.f);
  const uint32_t u = __float_as_uint(group_max<HD / 8>(big));
  const int byte = max((int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), 10);
  const float down = __uint_as_float((uint32_t)(254 - byte) << 23);
  const float most = byte == 247 ? 240.f : 448.f;   // 256 * 2^120 would be an infinity
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = fabsf(x[e]) < INFINITY ? fminf(fmaxf(x[e] * down, -most), most) : NAN;
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
  codes = make_uint2((uint32_t)lo, (uint32_t)hi);
  return (uint32_t)byte;
}

// x -> x / sqrt(mean(x^2) + 1e-6) [* w] over a head, pair (2p, 2p + 1) turned by
// the row's angle of p, in float32, rounded once. A thread takes 8 consecutive
// elements of one head, so a head's sum of squares is one butterfly over HD / 8
// consecutive lanes.
//
// A block takes R rows: their sequence, destination and the HD / 2 cosines and
// sines of each are found once and shared by all heads through LDS. The angle is
// coordinate x frequency in float64 turns, reduced to half a turn before it is
// rounded: far into a long rollout a float32 angle would be off by whole
// fractions of a turn. What that rounding takes off (up to 2^-25 pi, three half steps of a sine) is put back to
// first order.
//
// Bound by memory: 4,080 rows of 16 + 2 x 16 heads of 128 (100 MB) 21.9 us, 4.6 TB/s, where a large copy
// reaches 4.9 (four inputs in turn, more than the last-level cache holds: 25.5 us); blocks of 1 row 22.7 us, of 4
// rows 24.4. Fewer than 1,024 rows take a row a block and split its heads over blocks: one launch of 4 us, most of
// it latency. Codes (84 MB) go a row a block always: 20.8 us, 4.0 TB/s, of two rows 22.4, of which the single bytes of the powers
// cost 0.5.
template <typename T, int HD, int R, bool CODES>
__global__ __launch_bounds__(256) void k_cache_append(CacheAppendArgs a) {
  constexpr int TPH = HD / 8, HALF = HD / 2;
  const CacheArgs &c = a.c;
  __shared__ float2 cs[R][HALF];
  __shared__ int64_t dst[R];             // element offset of (page, kv head 0, slot) in k and v; -1: not stored
  __shared__ int live[R];
  const int tid = threadIdx.x, lane = tid & 63;
  const int row0 = a.first + blockIdx.x * R;
  const int nqk = c.heads + c.kvh, chunks = (nqk + c.kvh) * TPH;
  // chunk j of the rows, asked for one turn ahead, the first before the rows' places are looked up
  float next[R][8];
  auto fetch = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (j < chunks && row0 + r < c.rows) load8((const T *)a.qkv + (int64_t)(row0 + r) * a.ld + 8 * (int64_t)j, next[r]);
  };
  fetch(tid + blockIdx.y * 256);
  if (tid < 64) {
    // row r belongs to the sequence whose number is the count of chunk ends <= r
    int cnt[R] = {};
    for (int e0 = 0; e0 < c.batch; e0 += 64) {
      const int end = e0 + lane < c.batch ? c.q_start[e0 + lane + 1] : 0x7fffffff;
#pragma unroll
      for (int r = 0; r < R; ++r) cnt[r] += __popcll(__ballot(end <= row0 + r));
    }
    int b = cnt[0];
#pragma unroll
    for (int r = 1; r < R; ++r)
      if (lane == r) b = cnt[r];
    if (lane < R) {
      const int row = row0 + lane;
      int64_t d = -1;
      int ok = 0;
      if (row < c.rows && b < c.batch) {
        const CacheSeq s = cache_seq(c, b);
        const int i = row - s.q0, slot = s.start + i;
        ok = i >= 0 && i < s.nq;
        if (ok && slot >= 0) {
          const int e = c.table[(int64_t)b * c.table_ld + (slot >> c.plog)];
          // a chunk's slot on no page of the cache is not stored anywhere
          if (e >= 0 && e < c.pages)
            d = ((((int64_t)e * c.kvh) << c.plog) + (slot & ((1 << c.plog) - 1))) * HD;
        }
      }
      dst[lane] = d;
      live[lane] = !ok ? 0 : a.pos && a.pos[3 * (int64_t)row] >= 0 ? 2 : 1;   // 2: turned
    }
  }
  for (int e = tid; e < R * HALF; e += 256) {
    const int r = e / HALF, p = e % HALF, row = row0 + r;
    float2 v = make_float2(1.f, 0.f);
    if (a.pos && row < c.rows && a.pos[3 * (int64_t)row] >= 0) {
      const int ax = p < a.axis_end[0] ? 0 : p < a.axis_end[1] ? 1 : 2;
      const double turns = (double)a.pos[3 * (int64_t)row + ax] * a.freq[p];
      const double half = 2.0 * (turns - rint(turns));
      float s, k;
      sincospif((float)half, &s, &k);
      const float d = (float)((half - (double)(float)half) * 3.14159265358979323846);
      v = make_float2(k - d * s, s + d * k);
    }
    cs[r][p] = v;
  }
  __syncthreads();
  for (int j = tid + blockIdx.y * 256; j < chunks; j += 256 * gridDim.y) {
    const int h = j / TPH, e8 = 8 * (j % TPH);
    float x[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[r][e] = next[r][e];
    fetch(j + 256 * gridDim.y);
    if (h < nqk) {                       // whole heads, so whole groups of lanes
      const float *w = h < c.heads ? a.qw : a.kw;
      float wt[8];
      if (w) load8(w + e8, wt);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (!live[r]) continue;
        if (a.norm) {
          float sq = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sq += x[r][e] * x[r][e];
          const float inv = 1.f / sqrtf(group_sum<TPH>(sq) * (1.f / HD) + 1e-6f);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[r][e] *= inv;
        }
        if (w)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[r][e] *= wt[e];
        if (CODES && live[r] == 1) continue;     // (turned by nothing an infinity would make its neighbour NaN)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const float2 t = cs[r][e8 / 2 + p];
          const float u0 = x[r][2 * p] * t.x - x[r][2 * p + 1] * t.y, u1 = x[r][2 * p] * t.y + x[r][2 * p + 1] * t.x;
          x[r][2 * p] = u0;
          x[r][2 * p + 1] = u1;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!live[r]) continue;
      if (h < c.heads) {
        store8((T *)a.q + (int64_t)(row0 + r) * a.ldq + (int64_t)h * HD + e8, x[r]);
      } else if (dst[r] >= 0) {
        const int kh = h < nqk ? h - c.heads : h - nqk;
        if constexpr (CODES) {
          const int64_t at = dst[r] / HD + ((int64_t)kh << c.plog);
          uint2 codes;
          const uint32_t byte = quantise8<HD>(x[r], codes);
          *(uint2 *)((uint8_t *)(h < nqk ? c.k : c.v) + at * HD + e8) = codes;
          if (e8 == 0) c.scale[2 * at + (h < nqk ? 0 : 1)] = (uint8_t)byte;
          continue;
        }
        store8((T *)(h < nqk ? c.k : c.v) + dst[r] + (((int64_t)kh << c.plog) * HD) + e8, x[r]);
      }
    }
  }
}

// Rows [a.first, rows) in launches of at most 2^23 blocks (a launch has fewer than 2^32 threads); f(first row, rows)
template <class F>
hipError_t row_launches(int rows, int per_block, F &&f) {
  constexpr int64_t MOST = int64_t(1) << 23;
  for (int64_t first = 0; first < rows; first += MOST * per_block) {
    f((int)first, (int)std::min<int64_t>(rows - first, MOST * per_block));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int HD, bool CODES>
hipError_t append(const CacheAppendArgs &in, hipStream_t s) {
  CacheAppendArgs a = in;
  const int chunks = (a.c.heads + 2 * a.c.kvh) * (HD / 8);
  if (a.c.rows >= 1024 && !CODES)
    return row_launches(a.c.rows, 2, [&](int first, int rows) {
      a.first = first;
      hipLaunchKernelGGL((k_cache_append<T, HD, 2, CODES>), dim3((rows + 1) / 2), dim3(256), 0, s, a);
    });
  const int split = std::min((chunks + 255) / 256, std::max(1, 512 / a.c.rows));
  return row_launches(a.c.rows, 1, [&](int first, int rows) {
    a.first = first;
    hipLaunchKernelGGL((k_cache_append<T, HD, 1, CODES>), dim3(rows, split), dim3(256), 0, s, a);
  });
}

// ---------------------------------------------------------------- read
// Stored rows back in the model dtype: row i of a chunk of q rows over n keys is slot n - q + i. A block takes a row, a thread
// 8 codes at a time. Bound by memory, more so by its writes: 33,660 rows of 2 x 16 heads of 128 (415 MB, two thirds of it
// written) 92.5 us, 4.5 TB/s, where a large copy reaches 4.9; two rows a block 95 to 99 us, four 103, stores past the caches 123.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_cache8_read(Cache8ReadArgs a) {
  constexpr int TPH = HD / 8;
  const CacheArgs &c = a.c;
  __shared__ int64_t src;                // (page, kv head 0, slot); -1: on no page, -2: row of no chunk
  const int tid = threadIdx.x, lane = tid & 63, row = a.first + blockIdx.x;
  if (tid < 64) {
    int b = 0;                           // the count of chunk ends <= row
    for (int e0 = 0; e0 < c.batch; e0 += 64) {
      const int end = e0 + lane < c.batch ? c.q_start[e0 + lane + 1] : 0x7fffffff;
      b += __popcll(__ballot(end <= row));
    }
    if (lane == 0) {
      int64_t d = -2;
      if (row < c.rows && b < c.batch) {
        const CacheSeq s = cache_seq(c, b);
        const int i = row - s.q0, slot = s.start + i;
        if (i >= 0 && i < s.nq) {
          const int e = slot >= 0 ? c.table[(int64_t)b * c.table_ld + (slot >> c.plog)] : -1;
          d = e >= 0 && e < c.pages ? (((int64_t)e * c.kvh) << c.plog) + (slot & ((1 << c.plog) - 1)) : -1;
        }
      }
      src = d;
    }
  }
  __syncthreads();
  const int64_t from = src;
  if (from == -2) return;
  const int per = c.kvh * TPH, first = a.k ? 0 : per, last = a.v ? 2 * per : per;
  for (int j = first + tid + blockIdx.y * 256; j < last; j += 256 * gridDim.y) {
    const bool key = j < per;
    const int jj = key ? j : j - per, h = jj / TPH, e8 = 8 * (jj % TPH);
    uint2 u = make_uint2(0, 0);
    float up = 1.f;
    if (from >= 0) {
      const int64_t at = from + ((int64_t)h << c.plog);
      u = *(const uint2 *)((const uint8_t *)(key ? c.k : c.v) + at * HD + e8);
      up = __uint_as_float((uint32_t)c.scale[2 * at + (key ? 0 : 1)] << 23);
    }
    const uint32_t w[2] = {u.x, u.y};
    float x[8];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[q], up, false);
      const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[q], up, true);
      x[4 * q] = lo[0];
      x[4 * q + 1] = lo[1];
      x[4 * q + 2] = hi[0];
      x[4 * q + 3] = hi[1];
    }
    store8((T *)(key ? a.k : a.v) + (int64_t)row * (key ? a.ldk : a.ldv) + (int64_t)h * HD + e8, x);
  }
}

template <typename T, int HD>
hipError_t read(const Cache8ReadArgs &in, hipStream_t s) {
  Cache8ReadArgs a = in;
  const int chunks = a.c.kvh * (HD / 8) * ((a.k ? 1 : 0) + (a.v ? 1 : 0));
  const int split = std::min((chunks + 255) / 256, std::max(1, 512 / a.c.rows));
  return row_launches(a.c.rows, 1, [&](int first, int rows) {
    a.first = first;
    hipLaunchKernelGGL((k_cache8_read<T, HD>), dim3(rows, split), dim3(256), 0, s, a);
  });
}

// ---------------------------------------------------------------- evict
// Order of the weights as unsigned numbers; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t mass_order(float m) {
  if (m != m) m = -INFINITY;
  const uint32_t u = __float_as_uint(m == 0.f ? 0.f : m);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int EVT = 1024, EVW = EVT / 64;   // threads and waves of a selection block (256 and 4 for short sequences)
constexpr int EVP = 16;                     // parts of a long (sequence, kv head); one wave sums up one part
constexpr int EVK = 8;                      // weights that a thread keeps in registers
constexpr int EVA = 8192;                   // keys that share digit 0 with the threshold, listed as they come
// words of LDS for histograms: copies of one, to spread equal digits over
constexpr int ev_words(int threads) { return threads == EVT ? 4096 : 2048; }
static_assert(EVP == EVW, "a wave per part");
// digits of the order values, from the top: 10, 11 and 11 bits
__device__ __forceinline__ constexpr int ev_shift(int d) { return d == 0 ? 22 : d == 1 ? 11 : 0; }
__device__ __forceinline__ constexpr int ev_bins(int d) { return d == 0 ? 1024 : 2048; }

// Scratch of one (sequence, kv head), in 32-bit words: the number of moves, then moves (to, from); with parts,
// their histograms of digit 0 and cumulated ones of digit 1, the order values of all slots, those that share
// digit 0 with the threshold (part by part, from the part's first slot) and a few words each.
__host__ __device__ inline int64_t evict_words(int moves, int parts, int cap) {
  const int64_t slots = ((int64_t)cap + 3) / 4 * 4;
  return 4 + 2 * (((int64_t)moves + 1) / 2 * 2) + (parts > 1 ? EVP * (1024 + 2048) + 2 * slots + 2 * EVP + 4 : 0);
}

// What one block of the selection works on: slots [s0, s1) of a (sequence, kv head) of n > keep
// keys. STORED: the order values of the weights are read from the scratch (else from the masses).
template <bool STORED, int T>
struct EvictPart {
  const CacheEvictArgs &a;
  int h, b, n, s0, s1, low_len, high_len;
  const int32_t *tab;
  int32_t *list;
  int j0, j1;        // the wave's slots: a contiguous run of them, so that lists in wave order are in slot order
  uint32_t u[EVK];   // order values of slots j0 + 64 i + lane; those of longer runs are read where they are needed
  uint32_t *hist, *from, *order, *alike, *above, *count, *found;
  __device__ __forceinline__ EvictPart(const CacheEvictArgs &a_) : a(a_), h(blockIdx.x), b(blockIdx.z) {
    const CacheArgs &c = a.c;
    n = __builtin_amdgcn_readfirstlane(min(max(c.kv_len[b], 0), c.cap));
    tab = c.table + (int64_t)b * c.table_ld;
    list = a.list + ((int64_t)b * c.kvh + h) * evict_words(a.moves, a.parts, c.cap);
    hist = (uint32_t *)list + 4 + 2 * (((int64_t)a.moves + 1) / 2 * 2);
    from = hist + EVP * ev_bins(0);
    order = from + EVP * ev_bins(1);
    alike = order + ((int64_t)c.cap + 3) / 4 * 4;
    above = alike + ((int64_t)c.cap + 3) / 4 * 4;   // [EVP] keys of a part above the threshold's digit 0
    count = above + EVP;                         // [EVP] keys of a part that share it
    found = count + EVP;                         // the threshold's digit 0, its rank among those that share it, their number
    low_len = (a.keep + a.low - 1) / a.low;
    high_len = a.parts > a.low ? (max(n - a.keep, 0) + a.parts - a.low - 1) / (a.parts - a.low) : 0;
    s0 = bound(blockIdx.y);
    s1 = bound(blockIdx.y + 1);
    const int run = ((s1 - s0 + T - 1) / T) * 64;
    j0 = min(s0 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * run, s1);
    j1 = min(j0 + run, s1);
    if (STORED) {
#pragma unroll
      for (int i = 0; i < EVK; ++i)
        if (j0 + 64 * i < j1) u[i] = read(j0 + 64 * i);
      return;
    }
    // The masses; those of slots below keep go to `out`, if it is not mass itself: most stay, k_evict_move
    // replaces the others.
    float x[EVK];
    int at[EVK];
#pragma unroll
    for (int i = 0; i < EVK; ++i)
      if (j0 + 64 * i < j1) {
        x[i] = weight(j0 + 64 * i, at[i]);
        u[i] = mass_order(x[i]);
      }
    if (a.out == a.mass) return;
#pragma unroll
    for (int i = 0; i < EVK; ++i)
      if (j0 + 64 * i < j1 && at[i] >= 0) a.out[at[i]] = x[i];
    for (int j = j0 + 64 * EVK; j < j1; j += 64) {
      const float y = weight(j, at[0]);
      if (at[0] >= 0) a.out[at[0]] = y;
    }
  }
  // place in the pool of slot j with table entry e (pools hold fewer than 2^31 slots)
  __device__ __forceinline__ int spot(int e, int j) const {
    return ((cache_page(a.c, e) * a.c.kvh + h) << a.c.plog) + (j & ((1 << a.c.plog) - 1));
  }
  // weight of slot first + lane, or of the run's last; at: its place in `out`, -1: none
  __device__ __forceinline__ float weight(int first, int &at) const {
    const int own = first + (int)(threadIdx.x & 63), j = min(own, j1 - 1), e = tab[j >> a.c.plog], x = spot(e, j);
    at = own < min(j1, a.keep) && (unsigned)e < (unsigned)a.c.pages ? x : -1;
    return a.mass[x];
  }
  // its order value
  __device__ __forceinline__ uint32_t read(int first) const {
    int at;
    return STORED ? order[min(first + (int)(threadIdx.x & 63), j1 - 1)] : mass_order(weight(first, at));
  }
  // f(slot, its order value) for the wave's slots, 64 at a time in order; slots >= j1 come along
  template <class F>
  __device__ __forceinline__ void each(F &&f) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < EVK; ++i)
      if (j0 + 64 * i < j1) f(j0 + 64 * i + lane, u[i]);
    for (int j = j0 + 64 * EVK; j < j1; j += 64) f(j + lane, read(j));
  }
  // first slot of part p: parts [0, low) cut [0, keep) evenly, the others [keep, n)
  __device__ __forceinline__ int bound(int p) const {
    if (a.parts == 1) return p ? n : 0;
    return p <= a.low ? min(p * low_len, min(n, a.keep)) : min(a.keep + (p - a.low) * high_len, n);
  }
  // slots that compete: behind the first `sink`, before the last `recent`
  __device__ __forceinline__ bool middle(int j) const { return j >= a.sink && j < n - a.recent; }
};

// hist[d] += 1 for lanes with d >= 0; a lane's place among those with its d (from hist[d] on). Lanes that share the
// first one's d are added up first: of masses that are all alike every lane would add to one word, one
// after the other.
__device__ __forceinline__ uint32_t evict_tally(uint32_t *hist, int d) {
  const int lane = threadIdx.x & 63;
  const uint64_t live = __ballot(d >= 0);
  if (!live) return 0;
  const int first = __builtin_ctzll(live), same = __builtin_amdgcn_readlane(d, first);
  const uint64_t alike = __ballot(d == same);
  uint32_t at = 0;
  if (d >= 0 && (lane == first || d != same)) at = atomicAdd(&hist[d], d == same ? (uint32_t)__popcll(alike) : 1u);
  const uint32_t base = __builtin_amdgcn_readlane(at, first);
  return d == same ? base + __popcll(alike & (lane ? ~0ull >> (64 - lane) : 0ull)) : at;
}

// Histogram of digit d of the block's slots that share the digits found so far, in as many copies as there is room for
template <bool STORED, int T>
__device__ __forceinline__ void evict_count(const EvictPart<STORED, T> &p, uint32_t *hist, int d, uint32_t prefix,
                                            uint32_t known) {
  const int tid = threadIdx.x, copy = (tid >> 6) % (ev_words(T) / ev_bins(d)) * ev_bins(d);
  for (int i = tid; i < ev_words(T); i += T) hist[i] = 0;
  __syncthreads();
  p.each([&](int j, uint32_t u) __attribute__((always_inline)) {
    const bool in = j < p.j1 && p.middle(j) && (u & known) == prefix;
    evict_tally(hist, in ? copy + (int)((u >> ev_shift(d)) & (ev_bins(d) - 1)) : -1);
  });
  __syncthreads();
}

// Sum of x over the threads before this one
template <int T>
__device__ __forceinline__ uint32_t block_before(uint32_t x) {
  __shared__ uint32_t wsum[T / 64];
  const uint32_t incl = (uint32_t)wave_scan((int)x);
  if ((threadIdx.x & 63) == 63) wsum[threadIdx.x >> 6] = incl;
  __syncthreads();
  uint32_t before = incl - x;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) before += i < (int)(threadIdx.x >> 6) ? wsum[i] : 0u;
  return before;
}

// Bin in which the rank-th key from the top lies, and its rank there. Bins go
// from the top: thread t has bins top = bins - 1 - PER t, top - 1, .. with count(0), count(1), .. keys.
// All threads get the results; *size: the keys of that bin.
template <int T, int PER, class F>
__device__ __forceinline__ void evict_pick(F &&count, int top, int rank, int *bin, int *r, int *size) {
  __shared__ int got[3];
  uint32_t mine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) mine += count(i);
  const uint32_t before = block_before<T>(mine);
  if (before < (uint32_t)rank && before + mine >= (uint32_t)rank) {   // one thread
    uint32_t x = rank - before, at = 0, n = 0;
    bool found = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t c = count(i);
      if (!found && x <= c) {
        found = true;
        at = i;
        n = c;
      }
      if (!found) x -= c;
    }
    got[0] = top - (int)at;
    got[1] = (int)x;
    got[2] = (int)n;
  }
  __syncthreads();
  *bin = got[0];
  *r = got[1];
  *size = got[2];
  __syncthreads();
}

// The lists of one part, given the threshold in the digits `known`: slots whose order value is above it in
// them are kept, of the part's `eqn` equal to it those that are among the first `taken` of all (eq0 of them lie in
// parts before); hr holes and mr movers lie in parts before. Each wave takes a contiguous run of slots,
// and counts of runs are added in order, so every list is in slot order.
template <bool STORED, int T>
__device__ __forceinline__ void evict_lists(const EvictPart<STORED, T> &p, uint32_t threshold, uint32_t known, bool any,
                                            int taken, int eq0, int eqn, int hr, int mr) {
  __shared__ int wcnt[3][(T / 64)];
  const CacheEvictArgs &a = p.a;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), keep = a.keep;
  int32_t *idx = a.index ? a.index + ((int64_t)p.b * a.c.kvh + p.h) * keep : nullptr;
  const int j1 = p.j1;
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
  // Kept: above `limit`. Only where some of a part's equal ones stay and others not they have to be numbered.
  // (Order values are at least 0x7fffff, NaN and -inf, so the threshold is not 0.)
  const bool mixed = __builtin_amdgcn_readfirstlane(any && taken > eq0 && taken < eq0 + eqn);
  const uint32_t limit = !any ? ~0u : taken >= eq0 + eqn ? threshold - 1 : threshold | ~known;
  auto equal = [&](int j, uint32_t u) { return j < j1 && p.middle(j) && (u & known) == threshold; };
  if (mixed) {
    int eq = 0;
    p.each([&](int j, uint32_t u) __attribute__((always_inline)) { eq += __popcll(__ballot(equal(j, u))); });
    if (lane == 0) wcnt[0][w] = eq;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < (T / 64); ++i) eq0 += i < w ? wcnt[0][i] : 0;
  }
  // f(slot, kept) in order
  auto kept_each = [&](auto &&f) __attribute__((always_inline)) {
    int er = eq0;
    p.each([&](int j, uint32_t u) __attribute__((always_inline)) {
      bool kept = j < j1 && (!p.middle(j) || u > limit);
      if (mixed) {
        const uint64_t eb = __ballot(equal(j, u));
        kept = kept || (eb >> lane & 1 && er + __popcll(eb & below) < taken);
        er += __popcll(eb);
      }
      f(j, kept);
    });
  };
  int holes = 0, movers = 0;
  kept_each([&](int j, bool kept) __attribute__((always_inline)) {
    holes += __popcll(__ballot(j < j1 && !kept && j < keep));
    movers += __popcll(__ballot(kept && j >= keep));
  });
  if (lane == 0) {
    wcnt[1][w] = holes;
    wcnt[2][w] = movers;
  }
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < (T / 64); ++i) {
    hr += i < w ? wcnt[1][i] : 0;
    mr += i < w ? wcnt[2][i] : 0;
    total += wcnt[1][i];
  }
  if (!STORED && threadIdx.x == 0) p.list[0] = min(total, a.moves);
  kept_each([&](int j, bool kept) __attribute__((always_inline)) {
    const bool hole = j < j1 && !kept && j < keep, mover = kept && j >= keep;
    const uint64_t hb = __ballot(hole), mb = __ballot(mover);
    const int hx = hr + __popcll(hb & below), mx = mr + __popcll(mb & below);
    if (hole && hx < a.moves) p.list[4 + 2 * hx] = j;
    if (mover && mx < a.moves) p.list[5 + 2 * mx] = j;
    if (idx && kept && j < keep) idx[j] = j;
    hr += __popcll(hb);
    mr += __popcll(mb);
  });
}

// A sequence that is short enough: everything stays
template <bool STORED, int T>
__device__ __forceinline__ void evict_none(const EvictPart<STORED, T> &p) {
  const CacheEvictArgs &a = p.a;
  int32_t *idx = a.index ? a.index + ((int64_t)p.b * a.c.kvh + p.h) * a.keep : nullptr;
  const int first = blockIdx.y * T + threadIdx.x, step = gridDim.y * T;
  if (idx) {
    for (int j = first; j < p.n; j += step) idx[j] = j;
    for (int j = p.n + first; j < a.keep; j += step) idx[j] = -1;
  }
  if (first == 0) p.list[0] = 0;
}

// The kept set of one (sequence, kv head). With m = keep - sink - recent places
// for the n - sink - recent keys in between: the m-th largest weight is found digit by
// digit with a histogram each, then the keys above it and the first of those
// equal to it are kept. Kept keys below `keep` stay; hole j below it takes kept key j from above, so
// nothing that is still to be read is written and only those rows move.
//
// One block does it all for short sequences (STAGE -1), of 256 threads for the shortest, whose time is barriers (12
// kv heads, 76 keys: 13.5 us with the moves, 16.6 with 1,024; 2,048 sequences of 100 keys, 16 heads: 172, 752; but four
// of 2,000 keys: 19.3, 17.0). What bounds that form on long ones is
// the instruction rate of one compute unit (67,320 slots: 189 us), so long ones are cut into EVP parts of one
// block each and the steps become launches. 0: order values stored, digit 0 counted. 1: digit 0 of the
// threshold from all parts' counts; the keys that share it listed, those above it counted. 2: the other digits from
// the listed keys of all parts, how many keys of each part are kept, hence the ranks that its lists start
// from, and the lists. Parts do not cross `keep`. Keys listed in stage 1 are few unless most masses are alike:
// more than EVA of them are sorted by digit 1 within their part, with the number of keys from
// each bin on, so that stage 2 reads those of one bin only. 16 heads, 67,320 slots, 61,200 kept: 8.5, 6 and
// 11 us, launches and the latency of a dozen dependent steps (masses over many binades; within one 48 us in all,
// all equal 58). Reading all 16 parts' counts of every digit in every block instead took 15 us more.
template <int STAGE, int T>
__global__ __launch_bounds__(T) void k_evict_select(CacheEvictArgs a) {
  constexpr int EVH = ev_words(T);
  __shared__ uint32_t hist[EVH];
  const EvictPart<(STAGE > 0), T> p(a);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), part = blockIdx.y;
  if (p.n <= a.keep) {
    if (STAGE < 0 || STAGE == 2) evict_none(p);
    return;
  }
  const int m = a.keep - a.sink - a.recent;
  // evict_pick from the LDS histogram of digit d
  auto pick = [&](auto dc, int rank, int *bin, int *r, int *size) __attribute__((always_inline)) {
    constexpr int D = decltype(dc)::value, PER = ev_bins(D) / T;
    const int top = ev_bins(D) - 1 - PER * tid;
    evict_pick<T, PER>([&](int i) {
      uint32_t n = 0;
#pragma unroll
      for (int q = 0; q < EVH; q += ev_bins(D)) n += hist[q + top - i];
      return n;
    }, top, rank, bin, r, size);
  };
  if constexpr (STAGE < 0) {
    uint32_t prefix = 0, known = 0;
    int rank = m, bin, size = m + 1;
    for (int d = 0; d < 3 && m > 0 && size != rank; ++d) {   // until all of a bin are taken
      evict_count(p, hist, d, prefix, known);
      if (d == 0)
        pick(std::integral_constant<int, 0>{}, rank, &bin, &rank, &size);
      else
        pick(std::integral_constant<int, 1>{}, rank, &bin, &rank, &size);   // (digit 2 has as many bins)
      prefix |= (uint32_t)bin << ev_shift(d);
      known |= (uint32_t)(ev_bins(d) - 1) << ev_shift(d);
    }
    evict_lists(p, prefix, known, m > 0, rank, 0, size, 0, 0);
  } else if constexpr (STAGE == 0) {
    if (m == 0) return;
    evict_count(p, hist, 0, 0, 0);
    p.each([&](int j, uint32_t u) __attribute__((always_inline)) {
      if (j < p.j1) p.order[j] = u;
    });
    static_assert(ev_bins(0) == T && T == EVT && EVH == 4 * EVT, "a thread per bin");
    p.hist[part * EVT + tid] = hist[tid] + hist[EVT + tid] + hist[2 * EVT + tid] + hist[3 * EVT + tid];
  } else if constexpr (STAGE == 1) {
    __shared__ uint32_t listed, over;
    if (m == 0) return;
    const int top = EVT - 1 - tid;
    uint32_t sum = 0;
#pragma unroll
    for (int q = 0; q < EVP; ++q) sum += p.hist[q * EVT + top];
    if (tid == 0) listed = over = 0;
    for (int i = tid; i < ev_bins(1); i += EVT) hist[i] = 0;
    int bin, rank, size;
    evict_pick<T, 1>([&](int) { return sum; }, top, m, &bin, &rank, &size);
    if (part == 0 && tid == 0) {
      p.found[0] = (uint32_t)bin << ev_shift(0);
      p.found[1] = (uint32_t)rank;
      p.found[2] = (uint32_t)size;
    }
    auto digit0 = [&](int j, uint32_t u) { return j < p.j1 && p.middle(j) ? (int)(u >> ev_shift(0)) : -1; };
    auto digit1 = [&](int j, uint32_t u) { return digit0(j, u) == bin ? (int)(u >> ev_shift(1)) & (ev_bins(1) - 1) : -1; };
    if (size > EVA) {
      p.each([&](int j, uint32_t u) __attribute__((always_inline)) { evict_tally(hist, digit1(j, u)); });
      __syncthreads();
      const int b1 = ev_bins(1) - 1 - 2 * tid;   // from bins b1 and b1 - 1 on; hist: where they begin in the list
      const uint32_t x = hist[b1], y = hist[b1 - 1], before = block_before<T>(x + y);
      *(uint2 *)(p.from + part * ev_bins(1) + b1 - 1) = make_uint2(before + x + y, before + x);
      hist[b1] = before;
      hist[b1 - 1] = before + x;
      __syncthreads();
    }
    p.each([&](int j, uint32_t u) __attribute__((always_inline)) {
      const int d = digit0(j, u);
      const uint64_t same = __ballot(d == bin), more = __ballot(d > bin);
      uint32_t at = 0;
      if (lane == 0) {
        if (more) atomicAdd(&over, (uint32_t)__popcll(more));
        if (same) at = atomicAdd(&listed, (uint32_t)__popcll(same));
      }
      if (size > EVA)
        at = evict_tally(hist, digit1(j, u));
      else
        at = __builtin_amdgcn_readfirstlane(at) + __popcll(same & (lane ? ~0ull >> (64 - lane) : 0ull));
      if (d == bin) p.alike[p.s0 + at] = u;
    });
    __syncthreads();
    if (tid == 0) {
      p.count[part] = listed;
      p.above[part] = over;
    }
  } else {
    __shared__ int gt[EVP], eq[EVP];
    constexpr int NA = 4;                        // listed keys that a thread keeps in registers
    uint32_t prefix = 0;
    int rank = 0;
    if (m > 0) {
      const uint32_t *al = p.alike + p.bound(w);   // wave w has those of part w
      int more = __builtin_amdgcn_readfirstlane((int)p.count[w]);
      uint32_t x[NA];
      auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
          if (64 * i < more) x[i] = al[min(64 * i + lane, more - 1)];
      };
      load();
      prefix = p.found[0];
      rank = (int)p.found[1];
      const bool sorted = p.found[2] > EVA;
      int up = (int)p.above[w], equal = 0, over = 0, bin, size;
      auto alike = [&](auto &&f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NA; ++i)
          if (64 * i < more) f(x[i], 64 * i + lane < more);
#pragma unroll 8
        for (int i = 64 * NA; i < more; i += 64) f(al[min(i + lane, more - 1)], i + lane < more);
      };
      if (sorted) {                              // total number of keys from each bin on
        uint2 sum = make_uint2(0u, 0u);
#pragma unroll
        for (int q = 0; q < EVP; ++q) {
          const uint2 y = *(const uint2 *)(p.from + q * ev_bins(1) + 2 * tid);
          sum.x += y.x;
          sum.y += y.y;
        }
        *(uint2 *)(hist + 2 * tid) = sum;
        if (tid == 0) hist[ev_bins(1)] = 0;
        __syncthreads();
        const uint32_t next = hist[2 * tid + 2];
        const bool one = sum.y >= (uint32_t)rank && next < (uint32_t)rank, two = sum.x >= (uint32_t)rank && sum.y < (uint32_t)rank;
        if (one || two) {                        // one thread
          gt[0] = 2 * tid + (one ? 1 : 0);
          gt[1] = rank - (int)(one ? next : sum.y);
        }
        __syncthreads();
        bin = gt[0];
        rank = gt[1];
        __syncthreads();
        prefix |= (uint32_t)bin << ev_shift(1);
        const uint32_t *f = p.from + w * ev_bins(1) + bin;
        const int skip = bin + 1 < ev_bins(1) ? __builtin_amdgcn_readfirstlane((int)f[1]) : 0;
        more = __builtin_amdgcn_readfirstlane((int)f[0]) - skip;
        up += skip;
        al += skip;
        load();
      }
#pragma unroll
      for (int d = 1; d < 3; ++d) {
        if (d == 1 && sorted) continue;
        const int copy = w % (EVH / ev_bins(d)) * ev_bins(d);
        const uint32_t known = ~0u << ev_shift(d - 1);
        for (int i = tid; i < EVH; i += EVT) hist[i] = 0;
        __syncthreads();
        alike([&](uint32_t y, bool in) __attribute__((always_inline)) {
          evict_tally(hist, in && (y & known) == prefix ? copy + (int)((y >> ev_shift(d)) & (ev_bins(d) - 1)) : -1);
        });
        __syncthreads();
        pick(std::integral_constant<int, 1>{}, rank, &bin, &rank, &size);
        prefix |= (uint32_t)bin << ev_shift(d);
      }
      alike([&](uint32_t y, bool in) __attribute__((always_inline)) {
        over += in && y > prefix ? 1 : 0;
        equal += in && y == prefix ? 1 : 0;
      });
      up += wave_sum(over);
      equal = wave_sum(equal);
      if (lane == 0) {                           // what the wave's part keeps for sure, and may
        gt[w] = up;
        eq[w] = equal;
      }
    } else if (lane == 0) {
      gt[w] = eq[w] = 0;
    }
    __syncthreads();
    // lane q (of every wave): part q; sums over the parts before it
    const int q = lane % EVP, q0 = p.bound(q), q1 = p.bound(q + 1), my = eq[q];
    static_assert(EVP == 16, "row_scan");
    auto before = [&](int x) { return row_scan(x) - x; };
    const int eq0 = before(my);
    const int fixed = max(0, min(q1, a.sink) - q0) + max(0, q1 - max(q0, p.n - a.recent));
    const int kept = fixed + gt[q] + min(my, max(0, rank - eq0));
    const int holes = q < a.low ? q1 - q0 - kept : 0, movers = q < a.low ? 0 : kept;
    const int hr = before(holes), mr = before(movers);
    if (part == 0 && tid == EVP - 1) p.list[0] = min(hr + holes, a.moves);
    auto of = [&](int x) { return __builtin_amdgcn_readlane(x, part); };
    evict_lists(p, prefix, ~0u, m > 0, rank, of(eq0), of(my), of(hr), of(mr));
  }
}

// The moves that k_evict_select listed. RB bytes of a row: 16 per thread, the
// lanes of a row consecutive; block x takes moves x, x + grid, .. of its (sequence, head).
template <int RB>
__global__ __launch_bounds__(256) void k_evict_move(CacheEvictArgs a) {
  constexpr int TPR = RB / 16, RPB = 256 / TPR;
  const CacheArgs &c = a.c;
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int32_t *list = a.list + ((int64_t)b * c.kvh + h) * evict_words(a.moves, a.parts, c.cap);
  const int32_t *tab = c.table + (int64_t)b * c.table_ld;
  const int cnt = list[0];
  const int pmask = (1 << c.plog) - 1;
  auto at = [&](int j) {
    return (((int64_t)cache_page(c, tab[j >> c.plog]) * c.kvh + h) << c.plog) + (j & pmask);
  };
  if (blockIdx.x == 0 && h == 0 && tid == 0) {
    const int n = min(max(c.kv_len[b], 0), c.cap);
    a.len_out[b] = min(n, a.keep);
  }
  const int e = (tid % TPR) * 16;
  for (int r = blockIdx.x * RPB + tid / TPR; r < cnt; r += gridDim.x * RPB) {
    const int to = list[4 + 2 * r], from = list[5 + 2 * r];
    if (e == 0 && a.index) a.index[((int64_t)b * c.kvh + h) * a.keep + to] = from;
    if ((unsigned)tab[to >> c.plog] >= (unsigned)c.pages) continue;   // a slot on no page of the cache
    const int64_t d = at(to), s = at(from);
    const uint4 kk = *(const uint4 *)((const char *)c.k + s * RB + e), vv = *(const uint4 *)((const char *)c.v + s * RB + e);
    *(uint4 *)((char *)c.k + d * RB + e) = kk;
    *(uint4 *)((char *)c.v + d * RB + e) = vv;
    if (e == 0) a.out[d] = a.mass[s];
  }
}

}  // namespace

hipError_t launch_cache_append(int dtype, const CacheAppendArgs &a, hipStream_t s) {
  if (a.c.rows <= 0) return hipSuccess;
  if (a.c.scale) {
    if (dtype == 1) return a.c.hd == 128 ? append<bf16_t, 128, true>(a, s) : append<bf16_t, 64, true>(a, s);
    return a.c.hd == 128 ? append<float, 128, true>(a, s) : append<float, 64, true>(a, s);
  }
  if (dtype == 1) return a.c.hd == 128 ? append<bf16_t, 128, false>(a, s) : append<bf16_t, 64, false>(a, s);
  return a.c.hd == 128 ? append<float, 128, false>(a, s) : append<float, 64, false>(a, s);
}

hipError_t launch_cache8_read(int dtype, const Cache8ReadArgs &a, hipStream_t s) {
  if (a.c.rows <= 0 || (!a.k && !a.v)) return hipSuccess;
  if (dtype == 1) return a.c.hd == 128 ? read<bf16_t, 128>(a, s) : read<bf16_t, 64>(a, s);
  return a.c.hd == 128 ? read<float, 128>(a, s) : read<float, 64>(a, s);
}

// Moves and parts of a launch over these bounds. One block per (sequence, kv head) for up to 8,192 slots (16 heads: 8,000
// slots 20.8 us, in parts 20.9; 12,000: 31.4 and 22.1), for more where there are more of them, which share the compute
// units (four sequences of 10,000, 8 heads: 31.0 and 34.8; of 16,000, eight of 4 heads: 46.9 and 37.5; twelve of 5,000, 16
// heads: 36.8 and 162), and always where they fill these.
static void evict_plan(CacheEvictArgs &a) {
  a.moves = std::max(0, std::min(a.keep, a.c.cap - a.keep));
  const int heads = a.c.batch * a.c.kvh;
  a.parts = a.c.cap <= 8192 + 256 * std::max(0, heads - 16) || a.moves == 0 || heads >= 256 ? 1 : EVP;
  a.low = a.parts == 1 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(EVP - 1, (int64_t)EVP * a.keep / std::max(1, a.c.cap)));
}

size_t cache_evict_scratch(const CacheArgs &c, int keep) {
  CacheEvictArgs a{};
  a.c = c;
  a.keep = keep;
  evict_plan(a);
  return (size_t)c.batch * c.kvh * (size_t)evict_words(a.moves, a.parts, c.cap) * sizeof(int32_t);
}

hipError_t launch_cache_evict(int dtype, const CacheEvictArgs &in, hipStream_t s) {
  CacheEvictArgs a = in;
  evict_plan(a);
  const dim3 sel(a.c.kvh, a.parts, a.c.batch);   // with 8 kv heads the parts of one share an XCD, and their counts its L2
  if (a.parts == 1) {
    if (a.c.cap <= (a.c.batch * a.c.kvh >= 512 ? 2048 : 1024))
      hipLaunchKernelGGL((k_evict_select<-1, 256>), sel, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL((k_evict_select<-1, EVT>), sel, dim3(EVT), 0, s, a);
  } else {
    hipLaunchKernelGGL((k_evict_select<0, EVT>), sel, dim3(EVT), 0, s, a);
    hipLaunchKernelGGL((k_evict_select<1, EVT>), sel, dim3(EVT), 0, s, a);
    hipLaunchKernelGGL((k_evict_select<2, EVT>), sel, dim3(EVT), 0, s, a);
  }
  const int rb = a.c.hd * (dtype == 1 ? 2 : 4), rpb = 256 / (rb / 16);
  const int per = std::max(1, 2048 / std::max(1, a.c.kvh * a.c.batch));
  const dim3 grid(std::max(1, std::min((a.moves + rpb - 1) / rpb, per)), a.c.kvh, a.c.batch);
  if (rb == 128) hipLaunchKernelGGL((k_evict_move<128>), grid, dim3(256), 0, s, a);
  if (rb == 256) hipLaunchKernelGGL((k_evict_move<256>), grid, dim3(256), 0, s, a);
  if (rb == 512) hipLaunchKernelGGL((k_evict_move<512>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace wdc
