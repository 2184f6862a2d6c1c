// Paged key/value cache of a streaming rollout: storing a chunk's keys and
// values (with the per-head norms and the rotation of q and k in the same pass)
// and dropping the keys of least accumulated attention weight. The attention
// over the cache and the accumulation of its weights: cache_attention.hip.
#include "common.h"

#include <algorithm>

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

// x -> x / sqrt(mean(x^2) + 1e-6) [* w] over a head, pair (2p, 2p + 1) turned by
// the row's angle of p, in float32, rounded once. A thread takes 8 consecutive
// elements of one head, so a head's sum of squares is one butterfly over HD / 8
// consecutive lanes.
//
// A block takes R rows: their sequence, destination and the HD / 2 cosines and
// sines of each are found once and shared by all heads through LDS. The angle is
// coordinate x frequency in float64 turns, reduced to half a turn before it is
// rounded: far into a long rollout a float32 angle would be off by whole
// fractions of a turn.
template <typename T, int HD, int R>
__global__ __launch_bounds__(256) void k_cache_append(CacheAppendArgs a) {
  constexpr int TPH = HD / 8, HALF = HD / 2;
  const CacheArgs &c = a.c;
  __shared__ float2 cs[R][HALF];
  __shared__ int64_t dst[R];             // element offset of (page, kv head 0, slot) in k and v; -1: not stored
  __shared__ int live[R];
  const int tid = threadIdx.x, lane = tid & 63;
  const int row0 = blockIdx.x * R;
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
      live[lane] = ok;
    }
  }
  for (int e = tid; e < R * HALF; e += 256) {
    const int r = e / HALF, p = e % HALF, row = row0 + r;
    float2 v = make_float2(1.f, 0.f);
    if (a.pos && row < c.rows && a.pos[3 * (int64_t)row] >= 0) {
      const int ax = p < a.axis_end[0] ? 0 : p < a.axis_end[1] ? 1 : 2;
      const double turns = (double)a.pos[3 * (int64_t)row + ax] * a.freq[p];
      sincospif((float)(2.0 * (turns - rint(turns))), &v.y, &v.x);
    }
    cs[r][p] = v;
  }
  __syncthreads();
  const int nqk = c.heads + c.kvh, chunks = (nqk + c.kvh) * TPH;
  for (int j = tid + blockIdx.y * 256; j < chunks; j += 256 * gridDim.y) {
    const int h = j / TPH, e8 = 8 * (j % TPH);
    float x[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (live[r]) load8((const T *)a.qkv + (int64_t)(row0 + r) * a.ld + (int64_t)h * HD + e8, x[r]);
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
        store8((T *)(h < nqk ? c.k : c.v) + dst[r] + (((int64_t)kh << c.plog) * HD) + e8, x[r]);
      }
    }
  }
}

template <typename T, int HD>
hipError_t append(const CacheAppendArgs &a, hipStream_t s) {
  const int chunks = (a.c.heads + 2 * a.c.kvh) * (HD / 8);
  if (a.c.rows >= 1024) {
    hipLaunchKernelGGL((k_cache_append<T, HD, 4>), dim3((a.c.rows + 3) / 4), dim3(256), 0, s, a);
  } else {
    const int split = std::min((chunks + 255) / 256, std::max(1, 512 / a.c.rows));
    hipLaunchKernelGGL((k_cache_append<T, HD, 1>), dim3(a.c.rows, split), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------- evict
// Order of the weights as unsigned numbers; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t mass_order(float m) {
  if (m != m) m = -INFINITY;
  const uint32_t u = __float_as_uint(m == 0.f ? 0.f : m);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int EVT = 1024, EVW = EVT / 64;   // threads and waves of a selection block

// The kept set of one (sequence, kv head). With m = keep - sink - recent places
// for the n - sink - recent keys in between: the m-th largest weight is found digit by
// digit (11, 11 and 10 bits, a histogram each), then the keys above it and the
// first of those equal to it are kept. Each wave takes a contiguous run of
// slots; counts of runs are added in order, so every list is in slot order.
// Kept keys below `keep` stay; hole j below it takes kept key j from above, so
// nothing that is still to be read is written and only those rows move.
__global__ __launch_bounds__(EVT) void k_evict_select(CacheEvictArgs a) {
  __shared__ uint32_t hist[2048];
  __shared__ uint32_t wsum[EVW];
  __shared__ int wcnt[3][EVW];
  __shared__ uint32_t sh_prefix;
  __shared__ int sh_rank;
  const CacheArgs &c = a.c;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = min(max(c.kv_len[b], 0), c.cap);
  const int keep = a.keep;
  const int32_t *tab = c.table + (int64_t)b * c.table_ld;
  int32_t *list = a.list + ((int64_t)b * c.kvh + h) * (1 + 2 * (int64_t)a.moves);
  int32_t *idx = a.index ? a.index + ((int64_t)b * c.kvh + h) * keep : nullptr;
  const int pmask = (1 << c.plog) - 1;
  auto at = [&](int j) {
    return (((int64_t)cache_page(c, tab[j >> c.plog]) * c.kvh + h) << c.plog) + (j & pmask);
  };
  // a slot on no page of the cache: read as one of its pages, never written
  auto stored = [&](int j) { return (unsigned)tab[j >> c.plog] < (unsigned)c.pages; };
  if (n <= keep) {
    for (int j = tid; j < n; j += EVT) {
      if (a.out != a.mass && stored(j)) a.out[at(j)] = a.mass[at(j)];
      if (idx) idx[j] = j;
    }
    if (idx)
      for (int j = n + tid; j < keep; j += EVT) idx[j] = -1;
    if (tid == 0) list[0] = 0;
    return;
  }
  const int lo = a.sink, hi = n - a.recent, m = keep - a.sink - a.recent;
  // the m-th largest order value of [lo, hi), and how many of its equals are taken
  uint32_t prefix = 0, known = 0;
  int rank = m;                          // rank among the keys that share the digits found so far
  if (m > 0) {
    const int shifts[3] = {21, 10, 0}, bins[3] = {2048, 2048, 1024};
    for (int d = 0; d < 3; ++d) {
      for (int i = tid; i < bins[d]; i += EVT) hist[i] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += EVT) {
        const uint32_t u = mass_order(a.mass[at(j)]);
        if ((u & known) == prefix) atomicAdd(&hist[(u >> shifts[d]) & (bins[d] - 1)], 1u);
      }
      __syncthreads();
      // bins from the top: thread t holds a pair of them (the last digit: one)
      const int per = bins[d] / EVT, top = bins[d] - 1 - per * tid;
      uint32_t mine = hist[top] + (per > 1 ? hist[top - 1] : 0u), incl = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t t = __shfl_up(incl, o, 64);
        if (lane >= o) incl += t;
      }
      if (lane == 63) wsum[w] = incl;
      __syncthreads();
      uint32_t before = incl - mine;
      for (int i = 0; i < w; ++i) before += wsum[i];
      if (before < (uint32_t)rank && before + mine >= (uint32_t)rank) {   // one thread
        int bin = top, r = rank - (int)before;
        if (per > 1 && (uint32_t)r > hist[top]) {
          r -= (int)hist[top];
          bin = top - 1;
        }
        sh_prefix = prefix | ((uint32_t)bin << shifts[d]);
        sh_rank = r;
      }
      __syncthreads();
      prefix = sh_prefix;
      rank = sh_rank;
      known |= (uint32_t)(bins[d] - 1) << shifts[d];
      __syncthreads();
    }
  }
  // runs of whole 64s per wave over [0, n)
  const int run = ((n + 64 * EVW - 1) / (64 * EVW)) * 64;
  const int j0 = min(w * run, n), j1 = min(j0 + run, n);
  // class of slot j: 2 kept, 1 equal to the threshold, 0 dropped
  auto cls = [&](int j, float x) {
    if (j < lo || j >= hi) return 2;
    if (m == 0) return 0;
    const uint32_t u = mass_order(x);
    return u > prefix ? 2 : u == prefix ? 1 : 0;
  };
  int eq = 0;
  for (int j = j0; j < j1; j += 64) {
    const int jj = j + lane;
    eq += __popcll(__ballot(jj < j1 && cls(jj, a.mass[at(min(jj, n - 1))]) == 1));
  }
  if (lane == 0) wcnt[0][w] = eq;
  __syncthreads();
  int eq0 = 0;
  for (int i = 0; i < w; ++i) eq0 += wcnt[0][i];
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
  int holes = 0, movers = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int er = eq0, hr = holes, mr = movers;   // pass 1: ranks before this run
    for (int j = j0; j < j1; j += 64) {
      const int jj = j + lane;
      const bool in = jj < j1;
      const float x = a.mass[at(min(jj, n - 1))];
      const int cl = in ? cls(jj, x) : 0;
      const uint64_t eb = __ballot(cl == 1);
      const bool kept = cl == 2 || (cl == 1 && er + __popcll(eb & below) < rank);
      er += __popcll(eb);
      const bool hole = in && !kept && jj < keep, mover = in && kept && jj >= keep;
      const uint64_t hb = __ballot(hole), mb = __ballot(mover);
      if (pass == 1) {
        if (hole) {
          const int r = hr + __popcll(hb & below);
          if (r < a.moves) list[1 + 2 * r] = jj;
        }
        if (mover) {
          const int r = mr + __popcll(mb & below);
          if (r < a.moves) list[2 + 2 * r] = jj;
        }
        if (in && kept && jj < keep) {
          if (a.out != a.mass && stored(jj)) a.out[at(jj)] = x;
          if (idx) idx[jj] = jj;
        }
      }
      hr += __popcll(hb);
      mr += __popcll(mb);
    }
    if (pass == 0) {
      if (lane == 0) {
        wcnt[1][w] = hr;
        wcnt[2][w] = mr;
      }
      __syncthreads();
      int total = 0;
      for (int i = 0; i < EVW; ++i) {
        if (i < w) {
          holes += wcnt[1][i];
          movers += wcnt[2][i];
        }
        total += wcnt[1][i];
      }
      if (tid == 0) list[0] = min(total, a.moves);
    }
  }
}

// The moves that k_evict_select listed. RB bytes of a row: 16 per thread, the
// lanes of a row consecutive; block x takes moves x, x + grid, .. of its (sequence, head).
template <int RB>
__global__ __launch_bounds__(256) void k_evict_move(CacheEvictArgs a) {
  constexpr int TPR = RB / 16, RPB = 256 / TPR;
  const CacheArgs &c = a.c;
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int32_t *list = a.list + ((int64_t)b * c.kvh + h) * (1 + 2 * (int64_t)a.moves);
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
    const int to = list[1 + 2 * r], from = list[2 + 2 * r];
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
  if (dtype == 1) return a.c.hd == 128 ? append<bf16_t, 128>(a, s) : append<bf16_t, 64>(a, s);
  return a.c.hd == 128 ? append<float, 128>(a, s) : append<float, 64>(a, s);
}

static int evict_moves(const CacheArgs &c, int keep) { return std::max(0, std::min(keep, c.cap - keep)); }

size_t cache_evict_scratch(const CacheArgs &c, int keep) {
  return (size_t)c.batch * c.kvh * (1 + 2 * (size_t)evict_moves(c, keep)) * sizeof(int32_t);
}

hipError_t launch_cache_evict(int dtype, const CacheEvictArgs &in, hipStream_t s) {
  CacheEvictArgs a = in;
  a.moves = evict_moves(a.c, a.keep);
  hipLaunchKernelGGL(k_evict_select, dim3(a.c.kvh, a.c.batch), dim3(EVT), 0, s, a);
  const int rb = a.c.hd * (dtype == 1 ? 2 : 4), rpb = 256 / (rb / 16);
  const int per = std::max(1, 2048 / std::max(1, a.c.kvh * a.c.batch));
  const dim3 grid(std::max(1, std::min((a.moves + rpb - 1) / rpb, per)), a.c.kvh, a.c.batch);
  if (rb == 128) hipLaunchKernelGGL((k_evict_move<128>), grid, dim3(256), 0, s, a);
  if (rb == 256) hipLaunchKernelGGL((k_evict_move<256>), grid, dim3(256), 0, s, a);
  if (rb == 512) hipLaunchKernelGGL((k_evict_move<512>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace wdc
