// Elements of packed rows and of caches, sixteen at a time, and their E4M3 codes: what the kernels that bring rows into a cache and
// out of it share.
#pragma once

#include "common.h"

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

// A scale and its reciprocal.  With r the correctly rounded 1 / s, q = x r and e = q s - x (exact in an fma), q - e r is the
// correctly rounded x / s (Markstein, 1990), where nothing underflows: s >= 2^-60 makes sure of that for every quotient that is
// not far below half the smallest code.  (Of a zero, this order of signs keeps its own.)  Three instructions where the division
// takes eleven: the 16 agents' rows were bound by those.
struct Scale {
  float s, r;
  bool tiny;
  __device__ __forceinline__ explicit Scale(float scale) : s(scale), r(1.0f / scale), tiny(scale < 0x1p-60f) {}
};

// Codes of four elements by the scale, as e4m3_encode gives them; the instruction rounds to nearest even.
// ORDINARY: the scale is not tiny and the elements are finite, so that none is more than a rounding above 448 scales, which
// needs no clamp.  Otherwise step by step; of a NaN the instruction drops the sign, which is put back.
template <bool ORDINARY>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, const Scale& scale) {
  const float x[4] = {a, b, c, d};
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (ORDINARY) {
      const float q = x[i] * scale.r, e = fmaf(q, scale.s, -x[i]);
      y[i] = fmaf(-e, scale.r, q);
    } else {
      y[i] = __builtin_amdgcn_fmed3f(x[i] / scale.s, -448.0f, 448.0f);
    }
  }
  uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], (int)w, true);
  if (!ORDINARY) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (x[i] != x[i]) w = (w & ~(0xFFu << 8 * i)) | (0x7Fu | __float_as_uint(x[i]) >> 31 << 7) << 8 * i;
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
template <int DT, bool ORDINARY = false>
__device__ __forceinline__ Raw16<DT> from_floats(const float (&x)[16], const Scale& scale) {
  Raw16<DT> r;
#pragma unroll
  for (int i = 0; i < Raw16<DT>::N; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (DT == FSX_F32) w[j] = __float_as_uint(x[4 * i + j]);
      else if constexpr (DT == FSX_BF16) w[j] = pack_bf16x2(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
      else w[j] = encode4<ORDINARY>(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3], scale);
    }
    r.p[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return r;
}

// Scale of the largest finite magnitude `top`.
__device__ __forceinline__ float scale_of(float top, float headroom) {
  return top > 0.f ? fmaxf(top / 448.f * headroom, 0x1p-126f) : 1.f;
}

// Largest magnitude of pieces: fp32, or two bf16 halves side by side, as bits, which positive values compare by.  Pieces are
// folded whatever they hold; where the result is not finite, they are folded again without what is not.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <int DT>
__device__ __forceinline__ uint32_t fold_top(uint32_t top, uint4 p, bool finite_only) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (DT == FSX_F32) {
      uint32_t v = w[j] & 0x7FFFFFFFu;
      if (finite_only && v >= 0x7F800000u) v = 0;
      top = max(top, v);
    } else {
      u16x2 v = __builtin_bit_cast(u16x2, w[j] & 0x7FFF7FFFu);
      if (finite_only) {
        if (v.x >= 0x7F80) v.x = 0;
        if (v.y >= 0x7F80) v.y = 0;
      }
      top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), v));
    }
  }
  return top;
}
template <int DT>
__device__ __forceinline__ float top_value(uint32_t top) {
  return DT == FSX_F32 ? __uint_as_float(top) : __uint_as_float(max(top << 16, top & 0xFFFF0000u));
}

// The same elements in another type (a bit copy where the types are the same): cached values times scale, or into a cache by it.
template <int FROM, int TO>
__device__ __forceinline__ Raw16<TO> convert(const Raw16<FROM>& r, float scale) {
  if constexpr (FROM == TO) {
    return r;
  } else {
    float x[16];
    to_floats<FROM>(r, x);
    const Scale sc(scale);
    if constexpr (FROM == FSX_FP8_E4M3) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] *= scale;
    } else if constexpr (TO == FSX_FP8_E4M3) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < Raw16<FROM>::N; ++i) top = fold_top<FROM>(top, r.p[i], false);
      if (__all(!sc.tiny && top_value<FROM>(top) < INFINITY)) return from_floats<TO, true>(x, sc);
    }
    return from_floats<TO>(x, sc);
  }
}

}  // namespace fsx
