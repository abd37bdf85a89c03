// Whole rows of a cache, replaced by packed rows (an fp8 cache's scales found from them) and read back.  All of it is memory
// traffic: a row is read once and written once, 16 elements per thread at a time, except that the scales of long rows need a
// pass of their own before the codes.

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fsx {

// Sixteen elements of packed rows or of a cache, as they lie in memory.
template <int DT>
struct Raw16 {
  static constexpr int N = DT == FSX_F32 ? 4 : (DT == FSX_BF16 ? 2 : 1);  // 16-byte pieces
  uint4 p[N];
};
template <int DT>
__device__ __forceinline__ Raw16<DT> load_raw(const void* base, int64_t at) {
  constexpr int ES = DT == FSX_F32 ? 4 : (DT == FSX_BF16 ? 2 : 1);
  Raw16<DT> r;
#pragma unroll
  for (int i = 0; i < Raw16<DT>::N; ++i) r.p[i] = reinterpret_cast<const uint4*>((const char*)base + at * ES)[i];
  return r;
}
template <int DT>
__device__ __forceinline__ void store_raw(void* base, int64_t at, const Raw16<DT>& r) {
  constexpr int ES = DT == FSX_F32 ? 4 : (DT == FSX_BF16 ? 2 : 1);
#pragma unroll
  for (int i = 0; i < Raw16<DT>::N; ++i) reinterpret_cast<uint4*>((char*)base + at * ES)[i] = r.p[i];
}

// A scale and its reciprocal.  With r the correctly rounded 1 / s, q = x r and e = x - q s (exact in an fma), q + e r is the
// correctly rounded x / s (Markstein, 1990), where nothing underflows: s >= 2^-60 makes sure of that for every quotient that is
// not far below half the smallest code.  Six instructions where the division takes eleven: the 16 agents' rows were bound by
// those.
struct Scale {
  float s, r;
  bool tiny;
  __device__ __forceinline__ explicit Scale(float scale) : s(scale), r(1.0f / scale), tiny(scale < 0x1p-60f) {}
  __device__ __forceinline__ float quotient(float x) const {
    if (tiny) return x / s;
    const float q = __builtin_amdgcn_fmed3f(x * r, -512.0f, 512.0f);  // no element is larger, but for infinities
    return __builtin_copysignf(fmaf(fmaf(-q, s, x), r, q), x);  // (a zero's sign is lost in the sum)
  }
};

// Codes of four elements by the scale, as e4m3_encode gives them.  The instruction rounds to nearest even; of a NaN it drops
// the sign, which is put back.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, const Scale& scale) {
  const float y[4] = {scale.quotient(a), scale.quotient(b), scale.quotient(c), scale.quotient(d)};
  auto clamp = [](float v) { return __builtin_amdgcn_fmed3f(v, -448.0f, 448.0f); };
  uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp(y[0]), clamp(y[1]), 0, false);
  w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp(y[2]), clamp(y[3]), (int)w, true);
  if (__builtin_isunordered(y[0], y[1]) || __builtin_isunordered(y[2], y[3])) {
    const float x[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (y[i] != y[i]) w = (w & ~(0xFFu << 8 * i)) | (0x7Fu | __float_as_uint(x[i]) >> 31 << 7) << 8 * i;
  }
  return w;
}

template <int DT>
__device__ __forceinline__ void to_floats(const Raw16<DT>& r, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < Raw16<DT>::N; ++i) {
    const uint32_t w[4] = {r.p[i].x, r.p[i].y, r.p[i].z, r.p[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == FSX_F32) {
        x[4 * i + j] = __uint_as_float(w[j]);
      } else if constexpr (DT == FSX_BF16) {
        x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
        x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
      } else {
        const f16x2 lo = __builtin_bit_cast(f16x2, e4m3x2_to_f16x2(w[j], false)), hi = __builtin_bit_cast(f16x2, e4m3x2_to_f16x2(w[j], true));
        x[4 * j] = (float)lo[0];
        x[4 * j + 1] = (float)lo[1];
        x[4 * j + 2] = (float)hi[0];
        x[4 * j + 3] = (float)hi[1];
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ Raw16<DT> from_floats(const float (&x)[16], const Scale& scale) {
  Raw16<DT> r;
#pragma unroll
  for (int i = 0; i < Raw16<DT>::N; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == FSX_F32) w[j] = __float_as_uint(x[4 * i + j]);
      else if constexpr (DT == FSX_BF16) w[j] = pack_bf16x2(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
      else w[j] = encode4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3], scale);
    }
    r.p[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return r;
}
// The same elements in another type (a bit copy where the types are the same): cached values times scale, or into a cache by it.
template <int FROM, int TO>
__device__ __forceinline__ Raw16<TO> convert(const Raw16<FROM>& r, float scale) {
  if constexpr (FROM == TO) {
    return r;
  } else {
    float x[16];
    to_floats<FROM>(r, x);
    if constexpr (FROM == FSX_FP8_E4M3)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= scale;
    return from_floats<TO>(x, Scale(scale));
  }
}

// Scale of the largest finite magnitude `top`.
__device__ __forceinline__ float scale_of(float top, float headroom) {
  return top > 0.f ? fmaxf(top / 448.f * headroom, 0x1p-126f) : 1.f;
}

// The larger of `top` and the finite magnitudes of a 16-byte piece.
template <int DT>
__device__ __forceinline__ float piece_top(float top, const uint4& p) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (DT == FSX_F32) {
      const float x = __uint_as_float(w[j] & 0x7FFFFFFFu);
      top = fmaxf(top, x < INFINITY ? x : 0.f);
    } else {
      const float x = __uint_as_float((w[j] << 16) & 0x7FFF0000u), y = __uint_as_float(w[j] & 0x7FFF0000u);
      top = fmaxf(top, x < INFINITY ? x : 0.f);
      top = fmaxf(top, y < INFINITY ? y : 0.f);
    }
  }
  return top;
}

// ---------------------------------------------------------------------------------------------------------------
// A workgroup takes a.block rows of one agent in one layer, keys or values, and all heads: packed rows are then read or written
// in one run, a head-major cache in runs of a.block rows per head.  Four 16-element pieces are in flight per thread.
template <int PDT, int CDT, bool READ>
__global__ __launch_bounds__(256) void k_convert_rows(RowsArgs a) {
  const CacheView& cv = a.cv;
  const int lane = threadIdx.x & 63, l = blockIdx.y, kv = blockIdx.z;
  void* rows = kv ? a.v : a.k;
  if (!rows) return;
  const int b = __popcll(__ballot(lane < a.B && a.block_prefix[lane + 1] <= (int)blockIdx.x));
  const int r0 = ((int)blockIdx.x - a.block_prefix[b]) * a.block, nr = min(a.block, a.n[b] - r0);
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
// An fp8 cache's rows that fit the registers of a workgroup: for one (agent, layer, keys or values, head) after the other it
// holds the rows while it finds their largest magnitude, so they are read once, and as each piece is encoded the next rows'
// piece is sent for in its place.  Thread t keeps pieces t, t + T, .. of 16 bytes.
template <int DT, int T, int U>
__global__ __launch_bounds__(T) void k_replace_held(RowsArgs a) {
  constexpr int ES = DT == FSX_F32 ? 4 : 2, E = 16 / ES;  // elements of a piece
  __shared__ float red[2][T / 64];
  const CacheView& cv = a.cv;
  const int cpr = cv.Dh / E, step = T / cpr;  // pieces of a row; rows apart
  const int c = threadIdx.x % cpr, r0 = threadIdx.x / cpr;
  const uint32_t stride = (uint32_t)(cv.H * cv.Dh * ES);
  const int total = 2 * cv.H * a.layers * a.B;
  struct Item {
    int h, kv, l, b, n;
  };
  auto item = [&](int i) {
    Item x;
    x.h = i % cv.H;
    i /= cv.H;
    x.kv = i & 1;
    i >>= 1;
    x.l = i % a.layers;
    x.b = i / a.layers;
    x.n = a.n[x.b];
    return x;
  };
  auto next_of = [&](int i) {  // the next one that has rows
    for (i += gridDim.x; i < total && a.n[i / (2 * cv.H * a.layers)] == 0;) i += gridDim.x;
    return i;
  };
  uint4 x[U];
  auto load = [&](const Item& it, int u) {  // past the last row: that row again
    const char* src = (const char*)(it.kv ? a.v : a.k) + (((int64_t)it.l * a.total + a.src[it.b]) * cv.H + it.h) * cv.Dh * ES;
    x[u] = *reinterpret_cast<const uint4*>(src + ((uint32_t)min(r0 + step * u, it.n - 1) * stride + 16 * c));
  };
  int i = next_of((int)blockIdx.x - (int)gridDim.x);
  if (i >= total) return;
  Item it = item(i);
#pragma unroll
  for (int u = 0; u < U; ++u) load(it, u);
  for (int turn = 0;; turn ^= 1) {
    float top = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) top = piece_top<DT>(top, x[u]);
    top = rows_max(top);  // over lanes 16 apart, then over the 16
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int t = __builtin_bit_cast(int, top);
      const int o = s == 0 ? __builtin_amdgcn_update_dpp(0, t, 0x128, 0xF, 0xF, false)
                           : (s == 1 ? __builtin_amdgcn_update_dpp(0, t, 0x124, 0xF, 0xF, false)
                                     : (s == 2 ? __builtin_amdgcn_update_dpp(0, t, 0x122, 0xF, 0xF, false)
                                               : __builtin_amdgcn_update_dpp(0, t, 0x121, 0xF, 0xF, false)));
      top = fmaxf(top, __builtin_bit_cast(float, o));
    }
    if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < T / 64; ++j) top = fmaxf(top, red[turn][j]);
    const Scale sc(scale_of(top, a.headroom));
    if (threadIdx.x == 0) const_cast<float*>(it.kv ? cv.v_scale : cv.k_scale)[cache_scale_index(cv, it.b, cv.layer + it.l, it.h)] = sc.s;
    uint8_t* dst = (uint8_t*)const_cast<void*>(it.kv ? cv.v : cv.k) + cache_head_base(cv, it.b, cv.layer + it.l, it.h);
    const int j = next_of(i);
    const bool more = j < total;
    const Item nx = item(more ? j : i);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + step * u;
      const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      uint32_t o[2];
      if constexpr (DT == FSX_F32) {
        o[0] = encode4(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3]), sc);
      } else {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          o[e] = encode4(__uint_as_float(w[2 * e] << 16), __uint_as_float(w[2 * e] & 0xFFFF0000u), __uint_as_float(w[2 * e + 1] << 16),
                         __uint_as_float(w[2 * e + 1] & 0xFFFF0000u), sc);
      }
      if (more) load(nx, u);
      if (r0 < step && r < it.n) {
        if constexpr (DT == FSX_F32) *reinterpret_cast<uint32_t*>(dst + (int64_t)r * cv.rs + E * c) = o[0];
        else *reinterpret_cast<uint2*>(dst + (int64_t)r * cv.rs + E * c) = make_uint2(o[0], o[1]);
      }
    }
    if (!more) break;
    i = j;
    it = nx;
  }
}

// Longer rows: the scales first.  They start at 0 (k_clear_scales); a workgroup takes a.block rows and 256 pieces of their width,
// a thread the same piece of every row, and raises the scales of its heads (scale_of grows with the magnitude, and a maximum
// does not depend on the order; positive floats compare as their bits).
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
    float top = 0.f;
    int r = 0;
    for (; r + 8 <= nr; r += 8) {
      uint4 x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = *reinterpret_cast<const uint4*>(src + (int64_t)(r + u) * pieces * 16);
#pragma unroll
      for (int u = 0; u < 8; ++u) top = piece_top<DT>(top, x[u]);
    }
    for (; r < nr; ++r) top = piece_top<DT>(top, *reinterpret_cast<const uint4*>(src + (int64_t)r * pieces * 16));
    atomicMax(&tops[p / cpr - h0], __float_as_uint(top));
  }
  __syncthreads();
  const int h = h0 + threadIdx.x;
  if (threadIdx.x < 256 / cpr + 2 && h < cv.H && tops[threadIdx.x])
    atomicMax(reinterpret_cast<uint32_t*>(const_cast<float*>(kv ? cv.v_scale : cv.k_scale)) + cache_scale_index(cv, b, cv.layer + l, h),
              __float_as_uint(scale_of(__uint_as_float(tops[threadIdx.x]), a.headroom)));
}

// Rows per workgroup, so that there are about `wgs` workgroups, and the workgroups of the agents before.
static int plan_blocks(RowsArgs& a, int64_t per_row_wgs, int64_t wgs, int least, int most) {
  const int64_t rows = a.prefix[a.B];
  a.block = (int)std::max<int64_t>(least, std::min<int64_t>(most, rows * per_row_wgs / wgs));
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
      if (cpr > T || (int64_t)n > (int64_t)(T / cpr) * U || (int64_t)n * a.cv.H * a.cv.Dh * 4 > INT32_MAX) return false;
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
