// Attention of one new token over the pages of its sequence, with grouped heads: for every query head
//   O = sum_j exp(s_j) v_j / sum_j exp(s_j),   s_j = scale q . k_j,   lse = log sum_j exp(s_j)   over the sequence's rows j.
//
// Bound by memory: every key and value is read once, for all the query heads that share it, and a token has few of those.  The
// rows of a sequence are cut into parts so that there are workgroups enough; a workgroup takes one part for one key head (and at
// most 16 of its query heads), and k_page_merge puts the parts' states together.
//
// The four waves of a workgroup take tiles of 32 rows in turn, each on its own until the end.  Nothing goes through LDS on the way:
//   S = K Q^T   16x16x32 MFMA, A = 16 rows x 32 channels of keys as loaded (16 bytes of a row per lane), B = the queries; lane l
//   then has the scores of query l % 16 and rows 4 (l / 16) .. + 3 of each half of the tile;
//   O^T += V^T P^T   these registers, rounded to bf16, are the B operand as they stand; of the values a lane loads a piece of
//   channels of the same eight rows (16 lanes take a whole row), and turned over in registers the pieces are the A operand, row
//   r of product c being channel (D / 16) r + c.
// With fewer than 16 query heads the other columns are idle; the products take a small part of the loads' time all the same.

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fsx {

constexpr int PA_WAVES = 4, PA_KEYS = 32, PA_STEP = PA_WAVES * PA_KEYS;  // rows that a workgroup takes at a time

// A state of a part: G x D sums of weighted values, then G maxima (log2 units) and G sums of weights; whole 16-byte pieces.
__host__ __device__ constexpr int64_t part_floats(int G, int D) { return ((int64_t)G * (D + 2) + 3) / 4 * 4; }

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2v;
// Two E4M3 codes as bf16, exact: every E4M3 value is one.
__device__ __forceinline__ uint32_t e4m3x2_to_bf16x2(uint32_t packed, bool word) {
  return word ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(packed, 1.0f, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(packed, 1.0f, false));
}

// Rows of keys and values of a tile, as loaded.
template <int D, bool FP8>
struct PageTile {
  static constexpr int KP = FP8 ? D / 64 : D / 32;                 // 16-byte pieces of a key row per lane
  static constexpr int VW = FP8 ? D / 64 : D / 32;                 // words of a value row per lane
  uint4 k[2][KP];
  uint32_t v[2][4][VW];
  float4 ks[2], vs[2];  // FP8: scales of rows 4 (lane / 16) ..
};

template <int D, bool FP8>
__global__ __launch_bounds__(256, 2) void k_page_attention(PageAttentionArgs a) {
  constexpr int KS = D / 32, NC = D / 16, ES = FP8 ? 1 : 2;  // steps of the first product, products of the second
  using Tile = PageTile<D, FP8>;
  __shared__ float xo[PA_WAVES][16][D + 4];
  __shared__ float xm[PA_WAVES][16], xl[PA_WAVES][16];
  const PagePool& p = a.pool;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;

  // The part: entry e, part x of n, key head hk, query heads h0 .. of it.
  const int blocks = (a.G + 15) / 16;
  const int unit = blockIdx.x, hq = blockIdx.y, hk = hq / blocks, qb = hq - hk * blocks;
  int e = 0;
#pragma unroll
  for (int i = 0; i < PAGE_QUERIES; i += 64) e += __popcll(__ballot(i + lane < a.n && a.prefix[i + lane + 1] <= unit));
  e = __builtin_amdgcn_readfirstlane(e);
  const int x = unit - a.prefix[e], n = a.prefix[e + 1] - a.prefix[e], seq = a.seq[e];
  const int gq = min(16, a.G - 16 * qb), h0 = hk * a.G + 16 * qb;
  const int len = p.len[seq];
  const int per = ((len + n - 1) / n + PA_KEYS - 1) / PA_KEYS * PA_KEYS;  // (in a captured graph the length is not the planned one)
  const int begin = min(x * per, len), end = min(begin + per, len);
  const int32_t* __restrict__ pages = p.table + (int64_t)seq * p.most;

  // queries: channels of step s that the lane's keys hold
  uint4 q[KS];
  {
    const int64_t at = (a.row + e) * a.q_row + (int64_t)(h0 + min(c16, gq - 1)) * a.q_head;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int ch = FP8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
      if (a.q_f32) {
        const float4* f = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + at + ch);
        const float4 u = f[0], v = f[1];
        q[s] = make_uint4(pack_bf16x2(u.x, u.y), pack_bf16x2(u.z, u.w), pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
      } else {
        q[s] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.q) + at + ch);
      }
    }
  }

  const int last_page = max(len - 1, 0) >> p.shift;
  const char* kbase = (const char*)p.k;
  const char* vbase = (const char*)p.v;
  const int lane_k = c16 * D * ES + 16 * g, lane_v = 4 * g * D * ES + c16 * (D / 16) * ES;
  // First element row of the page row that tile row `key` is (past the end: some row that exists).
  const auto row_of = [&](int key) {
    const int page = pages[min(key >> p.shift, last_page)];
    return (((int64_t)a.layer * p.pages + page) * p.Hk + hk) * p.P + (key & (p.P - 1));
  };
  const auto load_k = [&](Tile& t, const int64_t (&row)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* src = kbase + row[h] * (D * ES) + lane_k;
#pragma unroll
      for (int i = 0; i < Tile::KP; ++i) t.k[h][i] = *reinterpret_cast<const uint4*>(src + 64 * i);
      if constexpr (FP8) t.ks[h] = *reinterpret_cast<const float4*>(p.k_scale + row[h] + 4 * g);
    }
  };
  const auto load_v = [&](Tile& t, const int64_t (&row)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* src = vbase + row[h] * (D * ES) + lane_v;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (Tile::VW == 4) {
          const uint4 u = *reinterpret_cast<const uint4*>(src + i * D * ES);
          t.v[h][i][0] = u.x, t.v[h][i][1] = u.y, t.v[h][i][2] = u.z, t.v[h][i][3] = u.w;
        } else if constexpr (Tile::VW == 2) {
          const uint2 u = *reinterpret_cast<const uint2*>(src + i * D * ES);
          t.v[h][i][0] = u.x, t.v[h][i][1] = u.y;
        } else {
          t.v[h][i][0] = *reinterpret_cast<const uint32_t*>(src + i * D * ES);
        }
      }
      if constexpr (FP8) t.vs[h] = *reinterpret_cast<const float4*>(p.v_scale + row[h] + 4 * g);
    }
  };

  f32x4 o[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;  // maximum (log2 units), the same in the four lanes of a query; the lane's share of the sum

  Tile t;
  int key = begin + w * PA_KEYS;
  if (key < end) {
    int64_t row[2] = {row_of(key), row_of(key + 16)};
    load_k(t, row);
    load_v(t, row);
    for (;;) {
      const int next = key + PA_STEP;
      const bool more = next < end;
      int64_t nrow[2] = {row_of(more ? next : key), row_of((more ? next : key) + 16)};
      // scores
      f32x4 s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          uint4 ka;
          if constexpr (FP8) {
            const uint4 u = t.k[h][i / 2];
            const uint32_t lo = i % 2 ? u.z : u.x, hi = i % 2 ? u.w : u.y;
            ka = make_uint4(e4m3x2_to_bf16x2(lo, false), e4m3x2_to_bf16x2(lo, true), e4m3x2_to_bf16x2(hi, false), e4m3x2_to_bf16x2(hi, true));
          } else {
            ka = t.k[h][i];
          }
          s[h] = mfma_bf16(ka, q[i], s[h]);
        }
      }
      float sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sc[i] = s[i / 4][i % 4] * a.c;
        if constexpr (FP8) sc[i] *= reinterpret_cast<const float*>(&t.ks[i / 4])[i % 4];
      }
      if (more) load_k(t, nrow);
      const int left = end - key;  // rows of the tile that count
      if (left < PA_KEYS) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (16 * (i / 4) + 4 * g + i % 4 >= left) sc[i] = -INFINITY;
      }
      // The maximum that the exponents are taken from is raised only where they would pass 2^8, which sums in fp32 and relative
      // roundings do not mind; then it is the same in the lanes of a query.
      float top = vmax3(vmax3(sc[0], sc[1], sc[2]), vmax3(sc[3], sc[4], sc[5]), vmax(sc[6], sc[7]));
      if (__any(top > m + 8.f)) {
        const float now = rows_max(vmax(top, m)), back = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.f : now));
        m = now;
        l *= back;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[c][i] *= back;
      }
      const float mz = m == -INFINITY ? 0.f : m;
      float pr[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        pr[i] = __builtin_amdgcn_exp2f(sc[i] - mz);
        l += pr[i];
        if constexpr (FP8) pr[i] *= reinterpret_cast<const float*>(&t.vs[i / 4])[i % 4];
      }
      if (left < PA_KEYS) {  // whatever lies behind the last row
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (16 * (i / 4) + 4 * g + i % 4 >= left) {
            pr[i] = 0.f;
#pragma unroll
            for (int j = 0; j < Tile::VW; ++j) t.v[i / 4][i % 4][j] = 0;
          }
      }
      const uint4 pb = make_uint4(pack_bf16x2(pr[0], pr[1]), pack_bf16x2(pr[2], pr[3]), pack_bf16x2(pr[4], pr[5]), pack_bf16x2(pr[6], pr[7]));
      // values: product c takes channel c of every lane's piece, eight rows of it
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        uint32_t r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // rows 2 j and 2 j + 1
          const int h = j / 2, i = 2 * (j % 2);
          if constexpr (FP8) {
            // bytes c of two rows side by side, then to bf16
            const uint32_t two = __builtin_amdgcn_perm(t.v[h][i + 1][c / 4], t.v[h][i][c / 4], c % 4 < 2 ? 0x05010400u : 0x07030602u);
            r[j] = e4m3x2_to_bf16x2(two, c % 2);
          } else {
            r[j] = __builtin_amdgcn_perm(t.v[h][i + 1][c / 2], t.v[h][i][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
          }
        }
        o[c] = mfma_bf16(make_uint4(r[0], r[1], r[2], r[3]), pb, o[c]);
      }
      if (!more) break;
      load_v(t, nrow);
      key = next;
    }
  }
  l = rows_sum(l);

  // The waves' states put together.  Lane: query c16, o[c][i]: channel (D / 16) (4 g + i) + c.
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) xo[w][c16][NC * (4 * g + i) + c] = o[c][i];
  if (g == 0) {
    xm[w][c16] = m;
    xl[w][c16] = l;
  }
  __syncthreads();
  // thread: query t / 16, channels D / 16 (t % 16) ..
  const int qi = threadIdx.x >> 4, ch = NC * (threadIdx.x & 15);
  if (qi >= gq) return;
  float mm = xm[0][qi], f[PA_WAVES], ll = 0.f;
#pragma unroll
  for (int i = 1; i < PA_WAVES; ++i) mm = vmax(mm, xm[i][qi]);
  const float mz = mm == -INFINITY ? 0.f : mm;
#pragma unroll
  for (int i = 0; i < PA_WAVES; ++i) {
    f[i] = __builtin_amdgcn_exp2f(xm[i][qi] - mz);
    ll += xl[i][qi] * f[i];
  }
  float r[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    r[c] = 0.f;
#pragma unroll
    for (int i = 0; i < PA_WAVES; ++i) r[c] += xo[i][qi][ch + c] * f[i];
  }
  if (n > 1) {
    float* part = a.part + ((int64_t)unit * gridDim.y * part_floats(min(a.G, 16), D)) + hq * part_floats(min(a.G, 16), D);
#pragma unroll
    for (int c = 0; c < NC; c += 4) *reinterpret_cast<float4*>(part + qi * D + ch + c) = make_float4(r[c], r[c + 1], r[c + 2], r[c + 3]);
    if ((threadIdx.x & 15) == 0) {
      part[min(a.G, 16) * D + qi] = mm;
      part[min(a.G, 16) * (D + 1) + qi] = ll;
    }
    return;
  }
  const float inv = len > 0 ? 1.f / ll : 0.f;
  const int64_t row = a.row + e;
  const int64_t at = row * a.o_row + (int64_t)(h0 + qi) * a.o_head + ch;
#pragma unroll
  for (int c = 0; c < NC; c += 4) {
    if (a.o_f32) {
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at + c) = make_float4(r[c] * inv, r[c + 1] * inv, r[c + 2] * inv, r[c + 3] * inv);
    } else {
      *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + at + c) =
          make_uint2(pack_bf16x2(r[c] * inv, r[c + 1] * inv), pack_bf16x2(r[c + 2] * inv, r[c + 3] * inv));
    }
  }
  if (a.lse && (threadIdx.x & 15) == 0) a.lse[row * a.H + h0 + qi] = (mm + __builtin_amdgcn_logf(ll)) * (1.f / LOG2E);
}

// The parts of one (entry, query head) put together, in their order: D / 4 threads take every PM-th part, then the groups' states.
template <int D>
__global__ __launch_bounds__(256) void k_page_merge(PageAttentionArgs a) {
  constexpr int T = D / 4, GROUPS = 256 / T;
  __shared__ float4 xo[GROUPS][T];
  __shared__ float xl[GROUPS], xm[GROUPS];
  const int e = blockIdx.x, h = blockIdx.y, hk = h / a.G, gi = h - hk * a.G, blocks = (a.G + 15) / 16, rows = min(a.G, 16);
  const int n = a.prefix[e + 1] - a.prefix[e];
  if (n <= 1) return;  // written already
  const int grp = threadIdx.x / T, t = threadIdx.x % T;
  const int64_t step = (int64_t)blocks * (a.H / a.G) * part_floats(rows, D);
  const float* part = a.part + a.prefix[e] * step + (hk * blocks + gi / 16) * part_floats(rows, D);
  const int qi = gi % 16;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](float mc, float lc, float4 v) {
    const float now = fmaxf(m, mc), z = now == -INFINITY ? 0.f : now;
    const float f = __builtin_amdgcn_exp2f(m - z), fc = __builtin_amdgcn_exp2f(mc - z);
    m = now;
    l = l * f + lc * fc;
    o = make_float4(o.x * f + v.x * fc, o.y * f + v.y * fc, o.z * f + v.z * fc, o.w * f + v.w * fc);
  };
  for (int x0 = grp; x0 < n; x0 += 4 * GROUPS) {
    float mc[4], lc[4];
    float4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float* s = part + min(x0 + u * GROUPS, n - 1) * step;
      v[u] = reinterpret_cast<const float4*>(s + qi * D)[t];
      mc[u] = s[rows * D + qi];
      lc[u] = s[rows * (D + 1) + qi];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (x0 + u * GROUPS < n) add(mc[u], lc[u], v[u]);
  }
  xo[grp][t] = o;
  if (t == 0) {
    xm[grp] = m;
    xl[grp] = l;
  }
  __syncthreads();
  if (grp) return;
#pragma unroll
  for (int i = 1; i < GROUPS; ++i) add(xm[i], xl[i], xo[i][t]);
  const float inv = a.pool.len[a.seq[e]] > 0 ? 1.f / l : 0.f;
  const int64_t row = a.row + e, at = row * a.o_row + (int64_t)h * a.o_head + 4 * t;
  if (a.o_f32) *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + at) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
  if (a.lse && t == 0) a.lse[row * a.H + h] = (m + __builtin_amdgcn_logf(l)) * (1.f / LOG2E);
}

int64_t plan_page_attention(const PagePool& p, int H, int n, const int32_t* seqs, const int32_t* host_len, int64_t workspace_bytes,
                            std::vector<int32_t>& parts) {
  constexpr int64_t WGS = 2048;
  const int G = H / p.Hk, units = p.Hk * ((G + 15) / 16);
  const int64_t state = 4 * units * part_floats(std::min(G, 16), p.D);  // bytes of a part, all heads
  int64_t rows = 0;
  for (int i = 0; i < n; ++i) rows += host_len[seqs[i]];
  int64_t chunk = std::max<int64_t>(PA_STEP, (rows * units / WGS + PA_STEP - 1) / PA_STEP * PA_STEP), need = 0;
  parts.resize(n);
  for (;; chunk *= 2) {
    need = 0;
    int64_t split = 0;
    for (int i = 0; i < n; ++i) {
      parts[i] = (int32_t)std::max<int64_t>(1, (host_len[seqs[i]] + chunk - 1) / chunk);
      need += parts[i];
      split += parts[i] > 1;
    }
    need = split ? need * state : 0;
    if (need <= workspace_bytes) return need;
  }
}

hipError_t launch_page_attention(PageAttentionArgs a, int n, const int32_t* seqs, const std::vector<int32_t>& parts, hipStream_t s) {
  const PagePool& p = a.pool;
  const int blocks = (a.G + 15) / 16, rows = std::min(a.G, 16);
  for (int i = 0; i < n;) {
    a.n = std::min(PAGE_QUERIES, n - i);
    a.row = i;
    a.prefix[0] = 0;
    bool split = false;
    for (int j = 0; j < a.n; ++j) {
      a.seq[j] = seqs[i + j];
      a.prefix[j + 1] = a.prefix[j] + parts[i + j];
      split |= parts[i + j] > 1;
    }
    const dim3 grid(a.prefix[a.n], p.Hk * blocks), merge(a.n, a.H);
    const auto fn = p.D == 64 ? (p.fp8 ? k_page_attention<64, true> : k_page_attention<64, false>)
                              : (p.fp8 ? k_page_attention<128, true> : k_page_attention<128, false>);
    hipLaunchKernelGGL(fn, grid, dim3(256), 0, s, a);
    if (split) {
      if (p.D == 64) hipLaunchKernelGGL(k_page_merge<64>, merge, dim3(256), 0, s, a);
      else hipLaunchKernelGGL(k_page_merge<128>, merge, dim3(256), 0, s, a);
    }
    a.part += (int64_t)a.prefix[a.n] * p.Hk * blocks * part_floats(rows, p.D);
    i += a.n;
  }
  return hipGetLastError();
}

}  // namespace fsx
