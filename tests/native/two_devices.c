/*
 * Shared-past calls whose stream belongs to another device than the current one, with devices of unlike numbers of
 * compute units. This program defines the HIP calls that the library makes on the way (no GPU is used): device 0 has
 * 256 compute units, device 1 has 32, the context's stream belongs to device 1, and launches are only written down.
 *
 * The scratch asked for, the scratch that a call insists on and the launches have to be those of the stream's device,
 * whatever device is current, and the current device has to be what it was.
 */
#include <hip/hip_runtime_api.h>
#include <stdio.h>
#include <string.h>

#include "wdc.h"

static int current, fail, launches, wrong_device;
static unsigned long long grids;
static const int units[2] = {256, 32};
static int the_stream;

hipError_t hipGetDevice(int *d) {
  *d = current;
  return hipSuccess;
}
hipError_t hipSetDevice(int d) {
  current = d;
  return hipSuccess;
}
hipError_t hipStreamGetDevice(hipStream_t s, hipDevice_t *d) {
  *d = s == (hipStream_t)&the_stream;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t a, int d) {
  *v = a == hipDeviceAttributeMultiprocessorCount ? units[d] : 0;
  return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void *f, hipFuncAttribute a, int v) {
  (void)f, (void)a, (void)v;
  return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }

static struct {
  dim3 grid, block;
  size_t lds;
  hipStream_t stream;
} config;                                        /* of the launch under way */
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t s);
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *s);
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t s) {
  config.grid = grid;
  config.block = block;
  config.lds = lds;
  config.stream = s;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *s) {
  *grid = config.grid;
  *block = config.block;
  *lds = config.lds;
  *s = config.stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t lds, hipStream_t s) {
  (void)f, (void)args, (void)lds, (void)s;
  ++launches;
  wrong_device += current != 1;
  grids = grids * 1000003 + ((unsigned long long)grid.x << 24) + (unsigned long long)grid.y * 4096 + block.x;
  return hipSuccess;
}

#define EXPECT(cond)                                             \
  do {                                                           \
    if (!(cond)) {                                               \
      fprintf(stderr, "FAIL line %d: %s\n", __LINE__, #cond);    \
      fail = 1;                                                  \
    }                                                            \
  } while (0)

int main(void) {
  for (int dtype = 0; dtype < 2; ++dtype)
    for (int codes = 0; codes < 2; ++codes) {
      wdc_model_desc d;
      memset(&d, 0, sizeof d);
      d.dtype = dtype;
      d.hidden = 4096;
      d.heads = 32;
      d.head_dim = 128;
      d.mlp_ratio = 4;
      d.lat_c = 16;
      d.lat_f = 1;
      d.lat_h = d.lat_w = 2;
      d.patch_t = 1;
      d.patch_h = d.patch_w = 2;
      d.rope_t = 16;
      d.rope_h = d.rope_w = 56;
      wdc_ctx *ctx = NULL, *near = NULL;
      EXPECT(wdc_create(&d, NULL, (wdc_stream)&the_stream, &ctx) == WDC_OK);
      EXPECT(wdc_create(&d, NULL, NULL, &near) == WDC_OK);
      if (fail) return 1;
      void *p = (void *)(size_t)(1 << 20);
      const wdc_paged_cache cache = {p, p, 10000, 64, 8, 0};
      const wdc_paged_cache8 cache8 = {p, p, p, 10000, 64, 8, 0};
      const wdc_chunks q = {p, p, p, 32, 400, 32, 1, 25000, 0};
      const wdc_prefix pre = {p, p, 1, 24448, 900, 0};
      size_t need[2], other;
      unsigned long long done[2] = {0, 0};
      for (int cur = 0; cur < 2; ++cur) {
        current = cur;
        need[cur] = codes ? wdc_cache8_attention_scratch(ctx, &cache8, &q, &pre)
                          : wdc_cache_attention_shared_scratch(ctx, &cache, &q, &pre);
        EXPECT(current == cur && need[cur] > 0);
      }
      EXPECT(need[0] == need[1]);
      current = 0;                               /* a stream of the current device: its own scratch, another */
      other = codes ? wdc_cache8_attention_scratch(near, &cache8, &q, &pre)
                    : wdc_cache_attention_shared_scratch(near, &cache, &q, &pre);
      EXPECT(other != need[1]);
      for (int cur = 0; cur < 2; ++cur)
        for (int less = 1; less >= 0; --less) {
          const size_t n = need[1] - (size_t)less;
          const int before = launches;
          current = cur;
          grids = 0;
          const wdc_status st =
              codes ? wdc_cache8_attention(ctx, &cache8, &q, &pre, p, 4096, 1, p, 4096, NULL, p, n)
                    : wdc_cache_attention_shared(ctx, &cache, &q, &pre, p, 4096, 1, p, 4096, NULL, p, n);
          EXPECT(st == (less ? WDC_E_WORKSPACE : WDC_OK));
          EXPECT(current == cur);
          EXPECT(less ? launches == before : launches > before);
          done[cur] = grids;
        }
      EXPECT(done[0] == done[1] && wrong_device == 0);
      wdc_destroy(ctx);
      wdc_destroy(near);
    }
  if (!fail) printf("two_devices: ok\n");
  return fail;
}
