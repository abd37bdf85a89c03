// Rotary positions with several axes: channel pair j of every head is turned by the angle p[axis_j] f_j, p a token's positions
// (a place in a text; the time, height and width of a piece of a frame),
//   y_a = x_a cos t - x_b sin t,   y_b = x_b cos t + x_a sin t.
// The gradient of the rotation is the rotation back.
//
// Bound by memory: every element is read and written once.  The angles of a row are the same for all of its heads, so a workgroup
// computes the sines and cosines of its rows once, into LDS, and then walks over the heads (16,384 bf16 rows of 64 heads x 128, 537 MB:
// 105 us, 5.1 TB/s; a large copy reaches 4.9).
//
// Angles: positions are whole numbers and f_j / 2 pi is given as a fraction of a turn in units of 2^-64 (turns.h), so their product
// modulo 2^64 is the angle's place in its turn, exact but for the fraction's own rounding (2^-65 a step, 2^-34 at position 2^31),
// however far the position: nothing has to be reduced.  The angle is then within an eighth of a turn of a quarter, where Taylor
// polynomials are off by less than 2e-9 (sine to x^9, cosine to x^10); with the roundings on the way a sine or cosine is off by at
// most 2^-22.

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fsx {

// cos and sin of t turns of 2^-64.
__device__ __forceinline__ float2 turn_cos_sin(uint64_t t) {
  const uint32_t u = (uint32_t)((t + 0x80000000u) >> 32);  // rounded to 2^-32
  const uint32_t quarter = (u + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(u - (quarter << 30)) * 1.46291807926715968e-9f;  // 2 pi 2^-32
  const float z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

// V elements of 16 or 32 bits as one access.
template <typename T, int V>
struct __attribute__((aligned(sizeof(T) * V))) Piece {
  T e[V];
};
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return bf16_to_f32(x); }
__device__ __forceinline__ void from_float(float& y, float x) { y = x; }
__device__ __forceinline__ void from_float(uint16_t& y, float x) { y = f32_to_bf16(x); }

// A workgroup takes a.block rows and every gridDim.y-th run of heads.  A thread turns V pairs at a time: two pieces of V elements,
// V apart side by side (adjacent pairs) or a.pairs apart (halves).
template <typename T, int V>
__global__ __launch_bounds__(256) void k_rotary(RotaryArgs a) {
  __shared__ float2 cs[2048];  // [row][pair]; a.block * a.pairs at most
  const int64_t r0 = (int64_t)blockIdx.x * a.block;
  const int nr = (int)min((int64_t)a.block, a.rows - r0), n = a.pairs;
  for (int i = threadIdx.x; i < nr * n; i += 256) {
    const int r = i / n, j = i - r * n;
    const int64_t p = a.pos[a.axis[j] * a.pos_axis + (r0 + r) * a.pos_row];
    float2 t = turn_cos_sin((uint64_t)p * a.turn[j]);
    if (a.inverse) t.y = -t.y;
    cs[i] = t;
  }
  __syncthreads();
  const int ppr = n / V, rest = a.copy_rest ? (a.dim - 2 * n) / V : 0, per_head = ppr + rest;  // pieces of a head
  const int total = nr * a.heads * per_head;
  const T* x = reinterpret_cast<const T*>(a.x) + r0 * a.x_row;
  T* y = reinterpret_cast<T*>(a.y) + r0 * a.y_row;
  for (int e = blockIdx.y * 256 + threadIdx.x; e < total; e += gridDim.y * 256) {
    const int rh = e / per_head, p = e - rh * per_head, r = rh / a.heads, h = rh - r * a.heads;
    const T* xh = x + r * a.x_row + h * a.x_head;
    T* yh = y + r * a.y_row + h * a.y_head;
    if (p >= ppr) {
      const int at = 2 * n + (p - ppr) * V;
      *reinterpret_cast<Piece<T, V>*>(yh + at) = *reinterpret_cast<const Piece<T, V>*>(xh + at);
      continue;
    }
    const int lo = a.adjacent ? 2 * p * V : p * V, hi = a.adjacent ? lo + V : n + lo;
    const Piece<T, V> u = *reinterpret_cast<const Piece<T, V>*>(xh + lo), w = *reinterpret_cast<const Piece<T, V>*>(xh + hi);
    const float2* t = cs + r * n + p * V;
    Piece<T, V> yu, yw;
    if (a.adjacent) {
      auto both = [&](int i) { return i < V ? to_float(u.e[i % V]) : to_float(w.e[i % V]); };
      auto put = [&](int i, float f) { from_float(i < V ? yu.e[i % V] : yw.e[i % V], f); };
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xa = both(2 * j), xb = both(2 * j + 1);
        put(2 * j, fmaf(xa, t[j].x, -xb * t[j].y));
        put(2 * j + 1, fmaf(xb, t[j].x, xa * t[j].y));
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xa = to_float(u.e[j]), xb = to_float(w.e[j]);
        from_float(yu.e[j], fmaf(xa, t[j].x, -xb * t[j].y));
        from_float(yw.e[j], fmaf(xb, t[j].x, xa * t[j].y));
      }
    }
    *reinterpret_cast<Piece<T, V>*>(yh + lo) = yu;
    *reinterpret_cast<Piece<T, V>*>(yh + hi) = yw;
  }
}

hipError_t launch_rotary(RotaryArgs a, hipStream_t s) {
  // the widest piece that the widths, strides and addresses allow.  Pairs that are not a multiple of four go element by element, in 2 or
  // 4 bytes an access: the two halves of a head then begin at different places of their 16 bytes.
  const int es = a.f32 ? 4 : 2;
  const auto fits = [&](int v) {
    const int64_t b = v * es;
    return a.pairs % v == 0 && (!a.copy_rest || (a.dim - 2 * a.pairs) % v == 0) && (uintptr_t)a.x % b == 0 && (uintptr_t)a.y % b == 0 &&
           a.x_row % v == 0 && a.x_head % v == 0 && a.y_row % v == 0 && a.y_head % v == 0;
  };
  const int v = !a.f32 && fits(8) ? 8 : (fits(4) ? 4 : 1);
  const int64_t units = (int64_t)a.heads * (a.pairs + (a.copy_rest ? a.dim - 2 * a.pairs : 0)) / v;  // of a row
  // rows of a workgroup: up to eight pieces for each of its threads, once the rows are many, and as few threads without one in the
  // last turn as may be (16,001 fp32 rows of 15 heads of 40 pairs, 154 MB: 34.6 us with 5 rows, 37.4 with 7)
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>({2048 / units, a.rows / 2048, 2048 / a.pairs}));
  const auto busy = [&](int64_t b) { return (double)(b * units) / ((b * units + 255) / 256 * 256); };
  int64_t best = most;
  for (int64_t b = most; b >= 1 && 2 * b > most; --b)
    if (busy(b) > busy(best) + 0.02) best = b;
  a.block = (int)std::max<int64_t>(best, (a.rows >> 23) + 1);
  const int64_t blocks = (a.rows + a.block - 1) / a.block;
  const dim3 grid((unsigned)blocks, (unsigned)std::max<int64_t>(1, std::min<int64_t>((a.block * units + 255) / 256, 2048 / blocks)));
  const auto fn = a.f32 ? (v == 4 ? k_rotary<float, 4> : k_rotary<float, 1>)
                        : (v == 8 ? k_rotary<uint16_t, 8> : (v == 4 ? k_rotary<uint16_t, 4> : k_rotary<uint16_t, 1>));
  return enqueue(fn, grid, dim3(256), s, a);
}

}  // namespace fsx
