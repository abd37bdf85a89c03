// Pages of a pool: the device's copy of the sequences' lists, pages copied as forked sequences diverge, rows that close up when a
// sequence keeps some of them, and packed rows written into pages.  All of it is memory traffic.

#include <algorithm>

#include "codes_device.h"
#include "common.h"
#include "kernels.h"

namespace fsx {

// First element of row r of a page, for one head of a layer; and the scale of that row.
__device__ __forceinline__ int64_t page_row(const PagePool& p, int layer, int page, int h, int r) {
  return (((int64_t)layer * p.pages + page) * p.Hk + h) * p.P + r;
}

// ---------------------------------------------------------------------------------------------------------------
// A workgroup for each run of entries, and one for each copied page, layer and head.
__global__ __launch_bounds__(256) void k_page_update(PageUpdateArgs a) {
  const PagePool& p = a.pool;
  if ((int)blockIdx.x < a.n_runs) {
    const PageRun r = a.runs[blockIdx.x];
    int32_t* to = a.table + (int64_t)r.seq * p.most + r.at;
    const int32_t* from = p.table + (int64_t)~r.first * p.most + r.at;
    for (int i = threadIdx.x; i < r.count; i += 256) to[i] = r.first < 0 ? from[i] : r.first + i;
    if (a.len && threadIdx.x == 0) a.len[r.seq] = r.len;
    return;
  }
  const int i = blockIdx.x - a.n_runs, n = a.n_copies, lh = i / n;  // a page's copies side by side
  const PageCopy c = a.copies[i - lh * n];
  const int layer = lh / p.Hk, h = lh - layer * p.Hk;
  const int64_t from = page_row(p, layer, c.from, h, 0), to = page_row(p, layer, c.to, h, 0);
  const int es = p.fp8 ? 1 : 2, pieces = c.rows * p.D * es / 16;
  const auto copy = [&](void* base) {
    const u32x4_t* src = reinterpret_cast<const u32x4_t*>((const char*)base + from * p.D * es);
    u32x4_t* dst = reinterpret_cast<u32x4_t*>((char*)base + to * p.D * es);
    for (int e0 = threadIdx.x; e0 < pieces; e0 += 4 * 256) {
      u32x4_t x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = src[min(e0 + 256 * u, pieces - 1)];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (e0 + 256 * u < pieces) dst[e0 + 256 * u] = x[u];
    }
  };
  copy(p.k);
  copy(p.v);
  if (p.fp8)
    for (int e = threadIdx.x; e < c.rows; e += 256) {
      p.k_scale[to + e] = p.k_scale[from + e];
      p.v_scale[to + e] = p.v_scale[from + e];
    }
}

hipError_t launch_page_update(const PagePool& pool, int32_t* table, int32_t* len, const std::vector<PageRun>& runs,
                              const std::vector<PageCopy>& copies, hipStream_t s) {
  PageUpdateArgs a;
  a.pool = pool;
  a.table = table;
  a.len = len;
  for (size_t r = 0, c = 0; r < runs.size() || c < copies.size();) {
    a.n_runs = (int)std::min<size_t>(PAGE_RUNS, runs.size() - r);
    a.n_copies = (int)std::min<size_t>(PAGE_COPIES, copies.size() - c);
    std::copy_n(runs.begin() + r, a.n_runs, a.runs);
    std::copy_n(copies.begin() + c, a.n_copies, a.copies);
    r += a.n_runs;
    c += a.n_copies;
    hipLaunchKernelGGL(k_page_update, dim3(a.n_runs + a.n_copies * pool.layers * pool.Hk), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------------------------
// Rows that close up, in place where the sequence has its pages alone.  A workgroup takes one head of one layer, keys or values, of
// a sequence from its first row that is written to its last: no row moves up, so the rows that a stretch of the outcome overwrites
// come from that stretch or have been read before, and a stretch is read whole before it is written.
__global__ __launch_bounds__(256) void k_page_move(PageMoveArgs a) {
  __shared__ PageRange ranges[PAGE_RANGES];
  const PagePool& p = a.pool;
  const PageMove m = a.moves[blockIdx.y];
  for (int i = threadIdx.x; i < m.n_ranges; i += 256) ranges[i] = a.ranges[m.range + i];
  __syncthreads();
  const int lh = blockIdx.x >> 1, kv = blockIdx.x & 1, layer = lh / p.Hk, h = lh - layer * p.Hk;
  const int es = p.fp8 ? 1 : 2, ppr = p.D * es / 16;  // pieces of a row
  char* base = (char*)(kv ? p.v : p.k);
  float* scales = kv ? p.v_scale : p.k_scale;
  const int32_t* from = p.table + (int64_t)m.seq * p.most;
  const int32_t* to = a.to_table + (int64_t)m.seq * p.most;
  const auto source = [&](int i) {
    int lo = 0;
    for (int n = m.n_ranges; n > 1;) {  // the last range that begins at or before row i
      const int half = n >> 1;
      if (ranges[lo + half].count <= i) lo += half;
      n -= half;
    }
    const int r = i - ranges[lo].count + ranges[lo].first;
    return page_row(p, layer, from[r >> p.shift], h, r & (p.P - 1));
  };
  const auto target = [&](int i) { return page_row(p, layer, to[i >> p.shift], h, i & (p.P - 1)); };
  constexpr int U = 4;
  const int stretch = U * 256 / ppr;  // rows; 256 at most
  for (int i0 = m.start; i0 < m.rows; i0 += stretch) {
    const int n = min(stretch, m.rows - i0) * ppr;
    u32x4_t x[U];
    float sc = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = min((int)threadIdx.x + 256 * u, n - 1), i = e / ppr;
      x[u] = *reinterpret_cast<const u32x4_t*>(base + source(i0 + i) * p.D * es + 16 * (e - i * ppr));
    }
    const bool scaled = p.fp8 && (int)threadIdx.x < min(stretch, m.rows - i0);
    if (scaled) sc = scales[source(i0 + threadIdx.x)];
    vm_wait_all();  // (a barrier alone does not wait for loads)
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = (int)threadIdx.x + 256 * u, i = e / ppr;
      if (e < n) *reinterpret_cast<u32x4_t*>(base + target(i0 + i) * p.D * es + 16 * (e - i * ppr)) = x[u];
    }
    if (scaled) scales[target(i0 + threadIdx.x)] = sc;
  }
}

hipError_t launch_page_move(const PagePool& pool, const int32_t* to_table, const std::vector<PageMove>& moves,
                            const std::vector<PageRange>& ranges, hipStream_t s) {
  PageMoveArgs a;
  a.pool = pool;
  a.to_table = to_table;
  for (size_t i = 0; i < moves.size();) {
    int n_ranges = 0;
    for (a.n_moves = 0; i < moves.size() && a.n_moves < PAGE_MOVES && n_ranges + moves[i].n_ranges <= PAGE_RANGES; ++i) {
      PageMove m = moves[i];
      int32_t rows = 0;
      for (int r = 0; r < m.n_ranges; ++r) {
        const PageRange& x = ranges[m.range + r];
        a.ranges[n_ranges + r] = {x.first, rows};
        rows += x.count;
      }
      m.range = n_ranges;
      n_ranges += m.n_ranges;
      a.moves[a.n_moves++] = m;
    }
    hipLaunchKernelGGL(k_page_move, dim3(2 * pool.layers * pool.Hk, a.n_moves), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------------------------
// Packed rows into the last rows of their sequences.  A workgroup takes a.block rows of one sequence in one layer, keys or values,
// and all heads; a thread 16 elements of a head's row at a time, so that the threads of a row (4 or 8) find its scale by exchange
// and each element is read once.
template <int PDT, int CDT>
__global__ __launch_bounds__(256) void k_page_write(PageWriteArgs a) {
  const PagePool& p = a.pool;
  const int lane = threadIdx.x & 63, l = blockIdx.y, kv = blockIdx.z, blk = blockIdx.x;
  int s = 0;
#pragma unroll
  for (int i = 0; i < PAGE_WRITES; i += 64) s += __popcll(__ballot(i + lane < a.n && a.block_prefix[i + lane + 1] <= blk));
  const int r0 = (blk - a.block_prefix[s]) * a.block, nr = min(a.block, a.rows[s] - r0), seq = a.seq[s];
  const int first = p.len[seq] - a.rows[s] + r0;  // row of the sequence
  const int32_t* pages = p.table + (int64_t)seq * p.most;
  const char* rows = (const char*)(kv ? a.v : a.k);
  const int64_t row_step = kv ? a.v_row : a.k_row, head_step = kv ? a.v_head : a.k_head;
  const int64_t packed = l * (kv ? a.v_layer : a.k_layer) + (a.start[s] + r0) * row_step;
  char* cache = (char*)(kv ? p.v : p.k);
  float* scales = kv ? p.v_scale : p.k_scale;
  const int cpr = p.D / 16, total = nr * p.Hk * cpr;
  for (int e0 = threadIdx.x; e0 < total; e0 += 4 * 256) {
    Raw16<PDT> in[4];
    int64_t at[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      // (past the end: the last row again, by whole rows)
      const int e = e0 + 256 * u < total ? e0 + 256 * u : total - cpr + e0 % cpr;
      const int c = e % cpr, i = e / cpr, r = i / p.Hk, h = i - r * p.Hk, row = max(first + r, 0);
      in[u] = load_raw<PDT>(rows, packed + r * row_step + h * head_step + 16 * c);
      at[u] = page_row(p, a.layer + l, pages[row >> p.shift], h, row & (p.P - 1));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = e0 + 256 * u, c = e % cpr;
      float scale = 1.f;
      if constexpr (CDT == FSX_FP8_E4M3) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < Raw16<PDT>::N; ++i) t = fold_top<PDT>(t, in[u].p[i], false);
        float top = top_value<PDT>(t);
        if (!(top < INFINITY)) {
          t = 0;
#pragma unroll
          for (int i = 0; i < Raw16<PDT>::N; ++i) t = fold_top<PDT>(t, in[u].p[i], true);
          top = top_value<PDT>(t);
        }
        // over the 4 or 8 threads of the row: lane ^ 1, lane ^ 2, then the mirrored lane of eight
        const auto other = [](float f, auto ctrl) {
          return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, f), decltype(ctrl)::value, 0xF, 0xF, false));
        };
        top = fmaxf(top, other(top, std::integral_constant<int, 0xB1>{}));
        top = fmaxf(top, other(top, std::integral_constant<int, 0x4E>{}));
        if (cpr == 8) top = fmaxf(top, other(top, std::integral_constant<int, 0x141>{}));
        scale = scale_of(top, 1.f);
      }
      const auto out = convert<PDT, CDT>(in[u], scale);
      if (e < total && first + (e / cpr) / p.Hk >= 0) {
        store_raw<CDT>(cache, at[u] * p.D + 16 * c, out);
        if (CDT == FSX_FP8_E4M3 && c == 0) scales[at[u]] = scale;
      }
    }
  }
}

hipError_t launch_page_write(PageWriteArgs a, int n, const int32_t* seqs, const int64_t* start, const int64_t* rows, hipStream_t s) {
  const PagePool& p = a.pool;
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += rows[i];
  // rows of a workgroup: four pieces for every thread, once there are workgroups enough
  const int64_t full = std::max<int64_t>(1, 4 * 256 / (p.Hk * (p.D / 16)));
  a.block = (int)std::max<int64_t>({1, std::min<int64_t>(full, total * a.n_layers * 2 / 2048), (total >> 23) + 1});
  for (int i = 0; i < n;) {
    a.n = 0;
    a.block_prefix[0] = 0;
    for (; i < n && a.n < PAGE_WRITES; ++i) {
      if (!rows[i]) continue;
      a.seq[a.n] = seqs[i];
      a.start[a.n] = start[i];
      a.rows[a.n] = (int32_t)rows[i];
      a.block_prefix[a.n + 1] = a.block_prefix[a.n] + (int)((rows[i] + a.block - 1) / a.block);
      ++a.n;
    }
    if (!a.n) break;
    const dim3 grid(a.block_prefix[a.n], a.n_layers, 2);
    const auto fn = a.rows_f32 ? (p.fp8 ? k_page_write<FSX_F32, FSX_FP8_E4M3> : k_page_write<FSX_F32, FSX_BF16>)
                               : (p.fp8 ? k_page_write<FSX_BF16, FSX_FP8_E4M3> : k_page_write<FSX_BF16, FSX_BF16>);
    hipLaunchKernelGGL(fn, grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace fsx
