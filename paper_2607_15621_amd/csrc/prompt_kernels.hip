// Attention over whole prompts (Sec. 3.3: a cache rebuilt from scratch): packed sequences of different lengths, causal, with
// grouped heads.
//
// Query t of a sequence with nq new tokens over nk keys sees the keys j <= nk - nq + t; per head
//   O_t = sum_j exp(s_tj) v_j / sum_j exp(s_tj),   s_tj = scale q_t . k_j,   lse_t = log sum_j exp(s_tj).

#include "common.h"
#include "kernels.h"

namespace fsx {

// One wave per (query row, head): 64 keys at a time, one per lane, with the running maximum and sum of the softmax; then a
// lane owns D / 64 output channels.  Masked keys are never read.
template <int D>
__global__ __launch_bounds__(256) void k_prompt_rows(PromptArgs a) {
  __shared__ float sq[4][D];
  __shared__ float sp[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t item = (int64_t)blockIdx.x * 4 + w;
  if (item >= (int64_t)a.row_prefix[a.n_seq] * a.H) return;
  const int r = (int)(item / a.H), h = (int)(item % a.H);
  int s = 0;
  while (r >= a.row_prefix[s + 1]) ++s;
  const int t = r - a.row_prefix[s], seen = a.nk[s] - a.nq[s] + t + 1;
  const int64_t row = a.q0[s] + t;
  for (int c = lane; c < D; c += 64) {
    const int64_t i = row * a.q_row + h * a.q_head + c;
    sq[w][c] = a.q_f32 ? bf16_to_f32(f32_to_bf16(((const float*)a.q)[i])) : bf16_to_f32(((const uint16_t*)a.q)[i]);
  }
  const uint16_t* k = a.k + a.k0[s] * a.k_row + (h / a.G) * a.k_head;
  const uint16_t* v = a.v + a.k0[s] * a.v_row + (h / a.G) * a.v_head;
  float m = -INFINITY, l = 0.f, o[D / 64] = {};
  for (int j0 = 0; j0 < seen; j0 += 64) {
    const int n = min(64, seen - j0);
    float x = -INFINITY;
    if (lane < n) {
      const uint16_t* kr = k + (int64_t)(j0 + lane) * a.k_row;
      float dot = 0.f;
      for (int c = 0; c < D; ++c) dot += sq[w][c] * bf16_to_f32(kr[c]);
      x = dot * a.c;
    }
    float mx = x;
    for (int i = 1; i < 64; i <<= 1) mx = fmaxf(mx, __shfl_xor(mx, i));
    const float mn = fmaxf(m, mx), mz = mn == -INFINITY ? 0.f : mn;
    const float p = lane < n ? exp2f(x - mz) : 0.f, alpha = exp2f(m - mz);
    l = l * alpha + wave_sum(p);
    m = mn;
    sp[w][lane] = p;
    for (int e = 0; e < D / 64; ++e) o[e] *= alpha;
    for (int j = 0; j < n; ++j)
      for (int e = 0; e < D / 64; ++e) o[e] += sp[w][j] * bf16_to_f32(v[(int64_t)(j0 + j) * a.v_row + lane + 64 * e]);
  }
  for (int e = 0; e < D / 64; ++e) {
    const float y = seen > 0 ? o[e] / l : 0.f;
    const int64_t i = row * a.o_row + h * a.o_head + lane + 64 * e;
    if (a.o_f32) ((float*)a.out)[i] = y;
    else ((uint16_t*)a.out)[i] = f32_to_bf16(y);
  }
  if (a.lse && lane == 0) a.lse[row * a.H + h] = seen > 0 ? (m + log2f(l)) / LOG2E : -INFINITY;
}

hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t s) {
  const int64_t items = (int64_t)a.row_prefix[a.n_seq] * a.H;
  if (items == 0) return hipSuccess;
  const dim3 grid((unsigned)((items + 3) / 4));
  if (a.D == 64)
    hipLaunchKernelGGL(k_prompt_rows<64>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k_prompt_rows<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace fsx
