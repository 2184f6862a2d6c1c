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
// power of two of an exponent byte
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float((byte & 255u) << 23); }

// ---------------------------------------------------------------- float32
// As over a cache in float32: v_mfma_f32_32x32x2_f32, four waves share 32 rows and take every fourth key
// tile of 32 of the block's range. S^T = K Q^T leaves a lane one row and 16 keys, which O^T = V^T P^T takes one by
// one as its B operand. Codes come straight from the cache, those of K 16 at a time (which dimension a lane
// takes in which step is free as long as K and Q agree: lane group g has [g hd / 2, + hd / 2)).
template <typename T, int HD>
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
  const int t0 = nr > 1 ? sp * (a.range / 32) : 0, t1 = nr > 1 ? min(t0 + a.range / 32, tiles) : tiles;
  const T *Q = (const T *)a.q + (int64_t)(s.q0 + row) * a.ldq + (int64_t)(h * group + mm - row * group) * HD + NC * lg;
  const uint8_t *K = (const uint8_t *)c.k + NC * lg, *V = (const uint8_t *)c.v + NI * lr;
  const float sc = LOG2E / sqrtf((float)HD);
  float qf[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) qf[j] = ld<T>(Q + j) * sc;
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
    for (int e4 = 0; e4 < 4; ++e4) {             // four keys of one page, as a rule
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
  T *O = (T *)a.o + (int64_t)(s.q0 + row) * a.ldo + (int64_t)head * HD + dim0;
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
        st<T>(O + NI * e + i, den == 0.f ? 0.f : y / den);
    }
  if (w != 0 || lg != 0) return;
  if (part_ >= 0) {
    *(float2 *)part_ml(a, at) = make_float2(mx, den);
  } else if (a.lse) {
    a.lse[(int64_t)(s.q0 + row) * c.heads + head] = den == 0.f ? -INFINITY : (mx + log2f(den)) * LN2;
  }
}

// ---------------------------------------------------------------- launches
// Blocks of 32 rows, and enough ranges to fill the compute units
void plan8(int dtype, const CacheArgs &c, size_t scratch, int *rpb, int *range, int *splits) {
  const int64_t slots = std::max(1, device_cus()), blocks = std::max<int64_t>(1, attn_blocks(32, c));
  const int64_t want = std::max<int64_t>(1, slots / blocks);
  const int64_t keys = std::max<int64_t>(256, (c.cap + want - 1) / want);
  *rpb = 32;
  *range = (int)((keys + 63) / 64 * 64);
  *splits = std::max(1, (c.cap + *range - 1) / *range);
  while (*splits > 1 && attn_part_bytes(c, *splits) > scratch) {
    *range = (int)std::min<int64_t>((int64_t)*range * 2, 1 << 30);
    *splits = (c.cap + *range - 1) / *range;
  }
}

template <typename T>
hipError_t launch_t(const CacheAttnArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)(attn_blocks(a.rpb, a.c) * a.splits));
  if (a.c.hd == 128)
    hipLaunchKernelGGL((k_cache8_attn_f32<T, 128>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_cache8_attn_f32<T, 64>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_pass8(int dtype, const CacheAttnArgs &a, hipStream_t s) {
  return dtype == 1 ? launch_t<bf16_t>(a, s) : launch_t<float>(a, s);
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
  a.parts = a.splits;
  if (a.c.rows <= 0 || a.c.max_q <= 0) return hipSuccess;
  const hipError_t e = launch_pass8(dtype, a, s);
  return e != hipSuccess || a.splits <= 1 ? e : launch_combine(dtype, a, s);
}

size_t cache8_shared_scratch(int dtype, const CacheArgs &c, const CacheShared &sh) {
  return shared_part_bytes(c, shared_passes(dtype, c, sh, plan8));
}

hipError_t launch_cache8_attention_shared(int dtype, const CacheAttnArgs &in, hipStream_t s) {
  return launch_shared(dtype, in, plan8, launch_pass8, s);
}

}  // namespace wdc
