// Whole rows of a cache, replaced by packed rows (an fp8 cache's scales found from them) and read back.  All of it is memory
// traffic: a row is read once and written once, 16 elements per thread at a time, except that the scales of long rows need a
// pass of their own before the codes.

#include <algorithm>
#include <type_traits>

#include "codes_device.h"
#include "common.h"
#include "kernels.h"

namespace fsx {

// ---------------------------------------------------------------------------------------------------------------
// A workgroup takes a.block rows of one agent in one layer, keys or values, and all heads: packed rows are then read or written
// in one run, a head-major cache in runs of a.block rows per head.  Four 16-element pieces are in flight per thread.
template <int PDT, int CDT, bool READ>
__global__ __launch_bounds__(256) void k_convert_rows(RowsArgs a) {
  const CacheView& cv = a.cv;
  const int lane = threadIdx.x & 63, l = blockIdx.y, kv = blockIdx.z;
  void* rows = kv ? a.v : a.k;
  if (!rows) return;
  // (written from the last rows back: of rows whose scales were found just before, those are still in the memory-side cache)
  const int blk = READ ? (int)blockIdx.x : (int)(gridDim.x - 1 - blockIdx.x);
  const int b = __popcll(__ballot(lane < a.B && a.block_prefix[lane + 1] <= blk));
  const int r0 = (blk - a.block_prefix[b]) * a.block, nr = min(a.block, a.n[b] - r0);
  char* cache = (char*)const_cast<void*>(kv ? cv.v : cv.k);
  const float* scales = CDT == FSX_FP8_E4M3 ? (kv ? cv.v_scale : cv.k_scale) + cache_scale_index(cv, b, cv.layer + l, 0) : nullptr;
  const int64_t base = cache_head_base(cv, b, cv.layer + l, 0), packed = ((int64_t)l * a.total + a.src[b] + r0) * cv.H * cv.Dh;
  const int64_t slot0 = a.slot[b] + r0;
  const int cpr = cv.Dh / 16, total = nr * cv.H * cpr;
  const bool token_major = cv.hs == cv.Dh;
  for (int e0 = threadIdx.x; e0 < total; e0 += 4 * 256) {
    Raw16<READ ? CDT : PDT> in[4];
    int64_t at[4], row[4];
    float sc[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = min(e0 + 256 * u, total - 1), c = e % cpr, i = e / cpr;
      const int h = token_major ? i % cv.H : i / nr, r = token_major ? i / cv.H : i - h * nr;
      int64_t slot = slot0 + r;
      if (slot >= cv.cap) slot -= cv.cap;
      at[u] = base + h * cv.hs + slot * cv.rs + 16 * c;
      row[u] = packed + ((int64_t)r * cv.H + h) * cv.Dh + 16 * c;
      sc[u] = CDT == FSX_FP8_E4M3 ? scales[h] : 1.f;
      if constexpr (READ) in[u] = load_raw<CDT>(cache, at[u]);
      else in[u] = load_raw<PDT>(rows, row[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (e0 + 256 * u >= total) break;
      if constexpr (READ) {
        store_raw<PDT>(rows, row[u], convert<CDT, PDT>(in[u], sc[u]));
      } else {
        // scales of long rows (k_row_tops): 0 where every row is, for which the first rows' workgroup writes 1
        if (CDT == FSX_FP8_E4M3 && sc[u] == 0.f) {
          sc[u] = 1.f;
          const int i = (e0 + 256 * u) / cpr, h = token_major ? i % cv.H : i / nr;
          if (r0 == 0) const_cast<float*>(scales)[h] = 1.f;
        }
        store_raw<CDT>(cache, at[u], convert<PDT, CDT>(in[u], sc[u]));
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------
// A buffer at an address that is the same in every lane, which the compiler does not always see.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_buffer(const void* p, int bytes) {
  const uint64_t u = (uint64_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// An fp8 cache's rows that fit the registers of a workgroup: for one (agent, layer, keys or values, head) after the other it
// holds the rows while it finds their largest magnitude, so they are read once, and as each piece is encoded the next rows'
// piece is sent for in its place.  Thread t keeps pieces t, t + T, .. of 16 bytes.
template <int DT, int T, int U>
__global__ __launch_bounds__(T) void k_replace_held(RowsArgs a) {
  constexpr int ES = DT == FSX_F32 ? 4 : 2, E = 16 / ES;  // elements of a piece
  __shared__ float red[2][T / 64];
  const CacheView& cv = a.cv;
  const int cpr = cv.Dh / E, step = T / cpr;  // pieces of a row; rows apart
  const int total = 2 * cv.H * a.layers * a.B;
  // Offsets of the thread's first piece from the first row, in the packed rows and in the cache; loads past the last row give
  // zeros and stores there are dropped (the buffers end with it).
  const uint32_t c = threadIdx.x % cpr, r0 = threadIdx.x / cpr, none = 0x80000000u;
  const uint32_t from = r0 < (uint32_t)step ? r0 * (uint32_t)(cv.H * cv.Dh * ES) + 16 * c : none;
  const uint32_t to = r0 < (uint32_t)step ? r0 * (uint32_t)cv.rs + E * c : none;
  const uint32_t from_step = (uint32_t)step * (uint32_t)(cv.H * cv.Dh * ES), to_step = (uint32_t)step * (uint32_t)cv.rs;
  struct Item {
    int h, kv, l, b, n;
  };
  auto item = [&](int i) {
    // (the same in every lane, which a division on the vector units hides)
    const int r = __builtin_amdgcn_readfirstlane(i / cv.H), b = __builtin_amdgcn_readfirstlane((r >> 1) / a.layers);
    return Item{i - r * cv.H, r & 1, (r >> 1) - b * a.layers, b, a.n[b]};
  };
  auto next_of = [&](int i) {  // the next one that has rows
    for (i += gridDim.x; i < total && a.n[__builtin_amdgcn_readfirstlane(i / (2 * cv.H * a.layers))] == 0;) i += gridDim.x;
    return i;
  };
  auto source = [&](const Item& it, bool any) {
    char* p = (char*)(it.kv ? a.v : a.k) + (((int64_t)it.l * a.total + a.src[it.b]) * cv.H + it.h) * cv.Dh * ES;
    return uniform_buffer(p, any ? ((it.n - 1) * cv.H + 1) * cv.Dh * ES : 0);
  };
  auto encode = [&](auto ordinary, u32x4_t p, const Scale& sc, __amdgpu_buffer_rsrc_t dst, uint32_t at) {
    constexpr bool ORD = decltype(ordinary)::value;
    if constexpr (DT == FSX_F32) {
      const uint32_t o = encode4<ORD>(__uint_as_float(p.x), __uint_as_float(p.y), __uint_as_float(p.z), __uint_as_float(p.w), sc);
      __builtin_amdgcn_raw_buffer_store_b32(o, dst, at, 0, 0);
    } else {
      const u32x2 o = {encode4<ORD>(__uint_as_float(p.x << 16), __uint_as_float(p.x & 0xFFFF0000u), __uint_as_float(p.y << 16),
                                    __uint_as_float(p.y & 0xFFFF0000u), sc),
                       encode4<ORD>(__uint_as_float(p.z << 16), __uint_as_float(p.z & 0xFFFF0000u), __uint_as_float(p.w << 16),
                                    __uint_as_float(p.w & 0xFFFF0000u), sc)};
      __builtin_amdgcn_raw_buffer_store_b64(o, dst, at, 0, 0);
    }
  };
  u32x4_t x[U];
  int i = next_of((int)blockIdx.x - (int)gridDim.x);
  if (i >= total) return;
  bool held = false;
  for (int turn = 0;; turn ^= 1) {
    const Item it = item(i);
    const auto own = source(it, true);
    if (!held) {
      uint32_t f = from;
#pragma unroll
      for (int u = 0; u < U; ++u, f += from_step) x[u] = __builtin_amdgcn_raw_buffer_load_b128(own, f, 0, 0);
    }
    uint32_t t = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) t = fold_top<DT>(t, make_uint4(x[u].x, x[u].y, x[u].z, x[u].w), false);
    float top = top_value<DT>(t);
    // Rows with elements that are not finite (and, below, tiny scales) take their pieces from memory again, in a short loop.
    const bool finite = top < INFINITY;
    if (!finite) {
      t = 0;
#pragma unroll 1
      for (uint32_t u = 0, f = from; u < U; ++u, f += from_step) {
        const u32x4_t p = __builtin_amdgcn_raw_buffer_load_b128(own, f, 0, 0);
        t = fold_top<DT>(t, make_uint4(p.x, p.y, p.z, p.w), true);
      }
      top = top_value<DT>(t);
    }
    top = rows_max(top);  // over lanes 16 apart, then over the 16
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int v = __builtin_bit_cast(int, top);
      const int o = s == 0 ? __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false)
                           : (s == 1 ? __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, false)
                                     : (s == 2 ? __builtin_amdgcn_update_dpp(0, v, 0x122, 0xF, 0xF, false)
                                               : __builtin_amdgcn_update_dpp(0, v, 0x121, 0xF, 0xF, false)));
      top = fmaxf(top, __builtin_bit_cast(float, o));
    }
    if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = top;
    const bool all_finite = __all(finite);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T / 64; ++j) top = fmaxf(top, red[turn][j]);
    const Scale sc(scale_of(top, a.headroom));
    if (threadIdx.x == 0) const_cast<float*>(it.kv ? cv.v_scale : cv.k_scale)[cache_scale_index(cv, it.b, cv.layer + it.l, it.h)] = sc.s;
    const auto dst = uniform_buffer((const char*)(it.kv ? cv.v : cv.k) + cache_head_base(cv, it.b, cv.layer + it.l, it.h),
                                    (int)((it.n - 1) * cv.rs + cv.Dh));
    i = next_of(i);
    held = all_finite && !__any(sc.tiny);
    uint32_t f = from, at = to;
    if (held) {
      const auto src = source(item(min(i, total - 1)), i < total);  // (none: the loads give zeros)
      // running offsets, hidden from the compiler, which would keep all 2 U of them in registers
      asm volatile("" : "+v"(f), "+v"(at));
#pragma unroll
      for (int u = 0; u < U; ++u, f += from_step, at += to_step) {
        encode(std::true_type{}, x[u], sc, dst, at);
        x[u] = __builtin_amdgcn_raw_buffer_load_b128(src, f, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll 1
      for (int u = 0; u < U; ++u, f += from_step, at += to_step)
        encode(std::false_type{}, __builtin_amdgcn_raw_buffer_load_b128(own, f, 0, 0), sc, dst, at);
    }
    if (i >= total) break;
  }
}

// Longer rows: the scales first, in a pass of their own, so these are read twice (four histories of fp32 rows, 2 layers: 362 us for
// the scales and 460 for the codes, 5.6 TB/s both; layer by layer, in pieces of the memory-side cache's size, 880 in all).  The
// scales start at 0 (k_clear_scales); a workgroup takes a.block rows and 256 pieces of their width, a thread the same piece of
// every row, and raises the scales of its heads (scale_of grows with the magnitude, and a maximum does not depend on the order;
// positive floats compare as their bits).
__global__ __launch_bounds__(256) void k_clear_scales(RowsArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x, H = a.cv.H, b = blockIdx.z, l = blockIdx.y;
  if (i >= 2 * H || a.n[b] == 0) return;
  const_cast<float*>(i < H ? a.cv.k_scale : a.cv.v_scale)[cache_scale_index(a.cv, b, a.cv.layer + l, i % H)] = 0.f;
}

template <int DT>
__global__ __launch_bounds__(256) void k_row_tops(RowsArgs a) {
  constexpr int ES = DT == FSX_F32 ? 4 : 2, E = 16 / ES;
  __shared__ uint32_t tops[256];
  const CacheView& cv = a.cv;
  const int lane = threadIdx.x & 63, cpr = cv.Dh / E, pieces = cv.H * cpr, groups = (pieces + 255) / 256;
  const int l = blockIdx.y / groups, p = blockIdx.y % groups * 256 + threadIdx.x, kv = blockIdx.z;
  const int b = __popcll(__ballot(lane < a.B && a.block_prefix[lane + 1] <= (int)blockIdx.x));
  const int r0 = ((int)blockIdx.x - a.block_prefix[b]) * a.block, nr = min(a.block, a.n[b] - r0);
  const int h0 = blockIdx.y % groups * 256 / cpr;
  tops[threadIdx.x] = 0;
  __syncthreads();
  if (p < pieces) {
    const char* src = (const char*)(kv ? a.v : a.k) + ((int64_t)l * a.total + a.src[b] + r0) * pieces * 16 + (int64_t)p * 16;
    auto largest = [&](bool finite_only) {
      uint32_t t = 0;
      int r = 0;
      for (; r + 8 <= nr; r += 8) {
        uint4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = *reinterpret_cast<const uint4*>(src + (int64_t)(r + u) * pieces * 16);
#pragma unroll
        for (int u = 0; u < 8; ++u) t = fold_top<DT>(t, x[u], finite_only);
      }
      for (; r < nr; ++r) t = fold_top<DT>(t, *reinterpret_cast<const uint4*>(src + (int64_t)r * pieces * 16), finite_only);
      return top_value<DT>(t);
    };
    float top = largest(false);
    if (!(top < INFINITY)) top = largest(true);
    atomicMax(&tops[p / cpr - h0], __float_as_uint(top));
  }
  __syncthreads();
  const int h = h0 + threadIdx.x;
  if (threadIdx.x < 256 / cpr + 2 && h < cv.H && tops[threadIdx.x])
    atomicMax(reinterpret_cast<uint32_t*>(const_cast<float*>(kv ? cv.v_scale : cv.k_scale)) + cache_scale_index(cv, b, cv.layer + l, h),
              __float_as_uint(scale_of(__uint_as_float(tops[threadIdx.x]), a.headroom)));
}

// Rows per workgroup, so that there are about `wgs` workgroups, and the workgroups of the agents before.  A launch holds fewer than
// 2^32 threads, 2^24 workgroups of 256 (one with more runs the rest of its threads by 2^32, without an error), so from 2^27 rows on
// a workgroup takes more of them.
static int plan_blocks(RowsArgs& a, int64_t per_row_wgs, int64_t wgs, int least, int most) {
  const int64_t rows = a.prefix[a.B];
  a.block = (int)std::max({(int64_t)least, std::min<int64_t>(most, rows * per_row_wgs / wgs), (rows >> 23) + 1});
  for (int b = 0; b < a.B; ++b) a.block_prefix[b + 1] = a.block_prefix[b] + (a.n[b] + a.block - 1) / a.block;
  return a.block_prefix[a.B];
}

template <int PDT, bool READ>
static hipError_t launch_convert(RowsArgs a, hipStream_t s) {
  const dim3 grid(plan_blocks(a, 2 * a.layers, 2048, 1, 16), a.layers, 2);
  switch (a.cv.dtype) {
    case FSX_F32: hipLaunchKernelGGL((k_convert_rows<PDT, FSX_F32, READ>), grid, dim3(256), 0, s, a); break;
    case FSX_BF16: hipLaunchKernelGGL((k_convert_rows<PDT, FSX_BF16, READ>), grid, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((k_convert_rows<PDT, FSX_FP8_E4M3, READ>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

template <int DT>
static hipError_t launch_replace(const RowsArgs& a, hipStream_t s) {
  if (a.cv.dtype == FSX_FP8_E4M3) {
    const int n = *std::max_element(a.n, a.n + a.B);
    const int cpr = a.cv.Dh * (DT == FSX_F32 ? 4 : 2) / 16;
    auto held = [&](auto fn, int T, int U, int per_cu) {
      if (cpr > T || (int64_t)n > (int64_t)(T / cpr) * U || (int64_t)(T / cpr) * U * std::max<int64_t>((int64_t)a.cv.H * a.cv.Dh * 4, a.cv.rs) > INT32_MAX)
        return false;
      const int64_t items = (int64_t)2 * a.cv.H * a.layers * a.B;
      hipLaunchKernelGGL(fn, dim3((unsigned)std::min<int64_t>(items, 256 * per_cu)), dim3(T), 0, s, a);
      return true;
    };
    if (held(k_replace_held<DT, 256, 4>, 256, 4, 6) || held(k_replace_held<DT, 512, 8>, 512, 8, 2) ||
        held(k_replace_held<DT, 1024, 16>, 1024, 16, 1))
      return hipGetLastError();
    hipLaunchKernelGGL(k_clear_scales, dim3((2 * a.cv.H + 255) / 256, a.layers, a.B), dim3(256), 0, s, a);
    RowsArgs t = a;
    const int groups = (a.cv.H * cpr + 255) / 256;
    const int blocks = plan_blocks(t, 2 * a.layers * groups, 4096, 8, 64);
    hipLaunchKernelGGL(k_row_tops<DT>, dim3(blocks, a.layers * groups, 2), dim3(256), 0, s, t);
  }
  return launch_convert<DT, false>(a, s);
}

hipError_t launch_replace_rows(const RowsArgs& a, hipStream_t s) {
  return a.rows_f32 ? launch_replace<FSX_F32>(a, s) : launch_replace<FSX_BF16>(a, s);
}

hipError_t launch_read_rows(const RowsArgs& a, hipStream_t s) {
  return a.rows_f32 ? launch_convert<FSX_F32, true>(a, s) : launch_convert<FSX_BF16, true>(a, s);
}

}  // namespace fsx
