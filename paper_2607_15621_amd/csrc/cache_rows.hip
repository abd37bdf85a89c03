// Whole rows of a cache, replaced by packed rows (an fp8 cache's scales found from them) and read back.

#include "common.h"
#include "kernels.h"

namespace fsx {

__device__ __forceinline__ float row_value(const void* p, int f32, int64_t i) {
  return f32 ? ((const float*)p)[i] : bf16_to_f32(((const uint16_t*)p)[i]);
}

// Scale of (agent, layer, head, keys or values): one workgroup.
__global__ __launch_bounds__(256) void k_row_scales(RowsArgs a) {
  __shared__ float red[4];
  const CacheView& cv = a.cv;
  int i = blockIdx.x;
  const int kv = i & 1;
  i >>= 1;
  const int h = i % cv.H, l = i / cv.H % a.layers, b = i / cv.H / a.layers;
  if (a.n[b] == 0) return;
  const void* src = kv ? a.v : a.k;
  float top = 0.f;
  const int64_t total = (int64_t)a.n[b] * cv.Dh;
  for (int64_t e = threadIdx.x; e < total; e += 256) {
    const float x = fabsf(row_value(src, a.rows_f32, (((int64_t)l * a.total + a.src[b] + e / cv.Dh) * cv.H + h) * cv.Dh + e % cv.Dh));
    if (x < INFINITY) top = fmaxf(top, x);
  }
  for (int j = 1; j < 64; j <<= 1) top = fmaxf(top, __shfl_xor(top, j));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float* sc = const_cast<float*>(kv ? cv.v_scale : cv.k_scale);
    sc[cache_scale_index(cv, b, cv.layer + l, h)] = top > 0.f ? fmaxf(top / 448.f * a.headroom, 0x1p-126f) : 1.f;
  }
}

// One element per thread of a packed row <-> its slot.
template <bool READ>
__global__ __launch_bounds__(256) void k_rows(RowsArgs a) {
  const CacheView& cv = a.cv;
  const int64_t A = (int64_t)cv.H * cv.Dh, per_layer = a.prefix[a.B] * A;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= per_layer * a.layers) return;
  const int l = (int)(i / per_layer), ch = (int)(i % cv.Dh), h = (int)(i % A / cv.Dh);
  const int64_t r = i % per_layer / A;
  int b = 0;
  while (r >= a.prefix[b + 1]) ++b;
  const int64_t t = r - a.prefix[b];
  int64_t slot = a.slot[b] + t;
  if (slot >= cv.cap) slot -= cv.cap;
  const int64_t at = cache_head_base(cv, b, cv.layer + l, h) + slot * cv.rs + ch;
  const int64_t row = (((int64_t)l * a.total + a.src[b] + t) * cv.H + h) * cv.Dh + ch;
  for (int kv = 0; kv < 2; ++kv) {
    void* rows = kv ? a.v : a.k;
    void* c = const_cast<void*>(kv ? cv.v : cv.k);
    if (!rows) continue;
    const float sc = cv.dtype == FSX_FP8_E4M3 ? (kv ? cv.v_scale : cv.k_scale)[cache_scale_index(cv, b, cv.layer + l, h)] : 1.f;
    if (READ) {
      const float x = cv.dtype == FSX_FP8_E4M3 ? e4m3_to_f32(((const uint8_t*)c)[at]) * sc
                                               : row_value(c, cv.dtype == FSX_F32, at);
      if (a.rows_f32) ((float*)rows)[row] = x;
      else ((uint16_t*)rows)[row] = f32_to_bf16(x);
    } else {
      const float x = row_value(rows, a.rows_f32, row);
      if (cv.dtype == FSX_FP8_E4M3) ((uint8_t*)c)[at] = (uint8_t)e4m3_encode(x, sc);
      else if (cv.dtype == FSX_BF16) ((uint16_t*)c)[at] = f32_to_bf16(x);
      else ((float*)c)[at] = x;
    }
  }
}

hipError_t launch_replace_rows(const RowsArgs& a, hipStream_t s) {
  const int64_t total = a.prefix[a.B] * a.cv.H * a.cv.Dh * a.layers;
  if (total == 0) return hipSuccess;
  if (a.cv.dtype == FSX_FP8_E4M3)
    hipLaunchKernelGGL(k_row_scales, dim3((unsigned)(2 * a.B * a.layers * a.cv.H)), dim3(256), 0, s, a);
  hipLaunchKernelGGL(k_rows<false>, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_read_rows(const RowsArgs& a, hipStream_t s) {
  const int64_t total = a.prefix[a.B] * a.cv.H * a.cv.Dh * a.layers;
  if (total == 0) return hipSuccess;
  hipLaunchKernelGGL(k_rows<true>, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace fsx
