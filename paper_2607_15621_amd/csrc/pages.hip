// Pages of a pool: the device's copy of the sequences' lists, pages copied as forked sequences diverge, rows that close up when a
// sequence keeps some of them, and packed rows written into pages.  All of it is memory traffic.

#include <algorithm>
#include <type_traits>

#include "codes_device.h"
#include "common.h"
#include "kernels.h"

namespace fsx {

// First element of row r of a page, for one head of a layer; and the scale of that row.
__device__ __forceinline__ int64_t page_row(const PagePool& p, int layer, int page, int h, int r) {
  return (((int64_t)layer * p.pages + page) * p.Hk + h) * p.P + r;
}

// ---------------------------------------------------------------------------------------------------------------
// A workgroup for each run of entries, and one for each copied page, layer, head, and keys or values; it reads the page's rows once
// for up to four copies (16 copies of 43 bf16 rows, 32 layers of 8 heads of 128 channels, 96 MB: 18 us, 5.4 TB/s, mostly written; 23
// with a read for every copy).
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
  const int i = blockIdx.x - a.n_runs, kv = i & 1, n = a.n_copies, lh = (i >> 1) / n;
  const PageCopies& c = a.copies[(i >> 1) - lh * n];
  const int layer = lh / p.Hk, h = lh - layer * p.Hk, targets = c.n;
  const int es = p.fp8 ? 1 : 2, pieces = c.rows * p.D * es / 16;
  const int64_t from = page_row(p, layer, c.from, h, 0);
  char* base = (char*)(kv ? p.v : p.k);
  int64_t to[PAGE_TARGETS];
#pragma unroll
  for (int t = 0; t < PAGE_TARGETS; ++t) to[t] = page_row(p, layer, c.to[t], h, 0);
  const u32x4_t* src = reinterpret_cast<const u32x4_t*>(base + from * p.D * es);
  for (int e0 = threadIdx.x; e0 < pieces; e0 += 4 * 256) {
    u32x4_t x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = src[min(e0 + 256 * u, pieces - 1)];
#pragma unroll
    for (int t = 0; t < PAGE_TARGETS; ++t) {
      if (t >= targets) break;
      u32x4_t* dst = reinterpret_cast<u32x4_t*>(base + to[t] * p.D * es);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (e0 + 256 * u < pieces) dst[e0 + 256 * u] = x[u];
    }
  }
  if (p.fp8) {
    float* scales = kv ? p.v_scale : p.k_scale;
    for (int e = threadIdx.x; e < c.rows; e += 256)
      for (int t = 0; t < targets; ++t) scales[page_row(p, layer, c.to[t], h, e)] = scales[from + e];
  }
}

hipError_t launch_page_update(const PagePool& pool, int32_t* table, int32_t* len, const std::vector<PageRun>& runs,
                              const std::vector<PageCopy>& copies, hipStream_t s) {
  PageUpdateArgs a{};
  a.pool = pool;
  a.table = table;
  a.len = len;
  for (size_t r = 0, c = 0; r < runs.size() || c < copies.size();) {
    a.n_runs = (int)std::min<size_t>(PAGE_RUNS, runs.size() - r);
    std::copy_n(runs.begin() + r, a.n_runs, a.runs);
    r += a.n_runs;
    for (a.n_copies = 0; c < copies.size(); ++c) {
      PageCopies* last = a.n_copies ? &a.copies[a.n_copies - 1] : nullptr;
      if (last && last->from == copies[c].from && last->rows == copies[c].rows && last->n < PAGE_TARGETS) {
        last->to[last->n++] = copies[c].to;
      } else {
        if (a.n_copies == PAGE_COPIES) break;
        a.copies[a.n_copies++] = {copies[c].from, copies[c].rows, 1, {copies[c].to}};
      }
    }
    const hipError_t e = enqueue(k_page_update, dim3(a.n_runs + 2 * a.n_copies * pool.layers * pool.Hk), dim3(256), s, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------------------------------------------------------
// Rows that close up, in place where the sequence has its pages alone.  A workgroup takes one head of one layer, keys or values (or
// some of their channels), of a sequence from its first row that is written to its last: no row moves up, so the rows that a stretch
// of the outcome overwrites come from that stretch or have been read before.  A stretch is read whole before it is written, and the
// next one is on its way by then (16 sequences of 1,024 bf16 rows, 560 of them moved, 4 layers of 8 heads of 128 channels, 294 MB: 48
// us, 6.1 TB/s, some of it from the memory-side cache; 80 with the pages looked up when they are needed, 84 with one stretch at a time).
__global__ __launch_bounds__(256) void k_page_move(PageMoveArgs a) {
  __shared__ PageRange ranges[PAGE_RANGES];
  const PagePool& p = a.pool;
  const PageMove m = a.moves[blockIdx.y];
  if (a.len && blockIdx.x == 0 && threadIdx.x == 0) a.len[m.seq] = m.rows;  // (not read here)
  for (int i = threadIdx.x; i < m.n_ranges; i += 256) ranges[i] = a.ranges[m.range + i];
  __syncthreads();
  const int unit = blockIdx.x / a.split, part = blockIdx.x - unit * a.split;
  const int lh = unit >> 1, kv = unit & 1, layer = lh / p.Hk, h = lh - layer * p.Hk;
  const int es = p.fp8 ? 1 : 2, ppr = p.D * es / 16 / a.split;  // pieces of a row: 4, 8 or 16
  char* base = (char*)(kv ? p.v : p.k) + part * ppr * 16;
  float* scales = p.fp8 && part == 0 ? (kv ? p.v_scale : p.k_scale) : nullptr;
  const int32_t* from = p.table + (int64_t)m.seq * p.most;
  const int32_t* to = a.to_table + (int64_t)m.seq * p.most;
  const auto source = [&](int i) {  // the row that becomes row i
    int lo = 0;
    for (int n = m.n_ranges; n > 1;) {  // the last range that begins at or before row i
      const int half = n >> 1;
      if (ranges[lo + half].count <= i) lo += half;
      n -= half;
    }
    return i - ranges[lo].count + ranges[lo].first;
  };
  const auto place = [&](int page, int row) { return page_row(p, layer, page, h, row & (p.P - 1)); };
  constexpr int U = 4;
  const int stretch = U * 256 / ppr, shift = __builtin_ctz(ppr);  // rows; 256 at most
  // Where a stretch's pieces come from and go to is looked up two stretches ahead: loads come back in order, so pages looked up
  // behind the rows under way would come when those have.
  struct Pages {
    int row[U], from[U], to[U], scale_row, scale_from, scale_to;
  };
  struct Stretch {
    u32x4_t x[U];
    int to[U], scale_to;
    float scale;
  };
  const auto look_up = [&](Pages& g, int i0) {
    const int n = min(stretch, m.rows - i0) * ppr;
    if (n <= 0) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + (min((int)threadIdx.x + 256 * u, n - 1) >> shift);
      g.row[u] = source(i);
      g.from[u] = from[g.row[u] >> p.shift];
      g.to[u] = to[i >> p.shift];
    }
    if (scales) {
      const int i = i0 + min((int)threadIdx.x, (n >> shift) - 1);
      g.scale_row = source(i);
      g.scale_from = from[g.scale_row >> p.shift];
      g.scale_to = to[i >> p.shift];
    }
  };
  const auto load = [&](Stretch& s, const Pages& g, int i0) {
    const int n = min(stretch, m.rows - i0) * ppr;
    if (n <= 0) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = min((int)threadIdx.x + 256 * u, n - 1);
      s.x[u] = *reinterpret_cast<const u32x4_t*>(base + place(g.from[u], g.row[u]) * p.D * es + 16 * (e & (ppr - 1)));
      s.to[u] = g.to[u];
    }
    if (scales) {
      s.scale = scales[place(g.scale_from, g.scale_row)];
      s.scale_to = g.scale_to;
    }
  };
  const auto store = [&](Stretch& s, int i0) {
    // all of the stretch is read: this wave's part has arrived (the registers are needed here), and so have the others'
    asm volatile("" : "+v"(s.x[0]), "+v"(s.x[1]), "+v"(s.x[2]), "+v"(s.x[3]), "+v"(s.scale)::"memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int n = min(stretch, m.rows - i0) * ppr;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = (int)threadIdx.x + 256 * u;
      if (e < n) *reinterpret_cast<u32x4_t*>(base + place(s.to[u], i0 + (e >> shift)) * p.D * es + 16 * (e & (ppr - 1))) = s.x[u];
    }
    if (scales && (int)threadIdx.x < n >> shift) scales[place(s.scale_to, i0 + (int)threadIdx.x)] = s.scale;
  };
  Pages g[2];
  Stretch s[2];
  s[0].scale = s[1].scale = 0.f;
  look_up(g[0], m.start);
  look_up(g[1], m.start + stretch);
  load(s[0], g[0], m.start);
  for (int i0 = m.start; i0 < m.rows; i0 += 2 * stretch) {
    const int i1 = i0 + stretch, i2 = i1 + stretch;
    look_up(g[0], i2);
    load(s[1], g[1], i1);
    store(s[0], i0);
    if (i1 >= m.rows) break;
    look_up(g[1], i2 + stretch);
    load(s[0], g[0], i2);
    store(s[1], i1);
  }
}

hipError_t launch_page_move(const PagePool& pool, const int32_t* to_table, int32_t* len, const std::vector<PageMove>& moves,
                            const std::vector<PageRange>& ranges, hipStream_t s) {
  PageMoveArgs a{};
  a.pool = pool;
  a.to_table = to_table;
  a.len = len;
  // Channels shared out where sequences, layers and heads are few: four workgroups for each CU, or pieces of 64 bytes of a row.
  const int64_t units = (int64_t)2 * pool.layers * pool.Hk * moves.size();
  const int most = pool.D * (pool.fp8 ? 1 : 2) / 64;
  for (a.split = 1; a.split < most && units * a.split < 1024;) a.split *= 2;
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
    const hipError_t e = enqueue(k_page_move, dim3(2 * pool.layers * pool.Hk * a.split, a.n_moves), dim3(256), s, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------------------------------------------------------
// Packed rows into the last rows of their sequences.  A workgroup takes a.block rows of one sequence in one layer, keys or values,
// and all heads; a thread 16 bytes of a cached row at a time.  The threads of an fp8 row (4 or 8) find its scale by exchange, so each
// element is read once.  16 prompts of 1,024 bf16 rows into fp8 pages, 32 heads of 128 channels, 407 MB: 87 us, 4.7 TB/s (a large
// copy: 4.9).
template <int PDT>
struct Raw8 {
  uint4 p[PDT == FSX_F32 ? 2 : 1];
};
template <int PDT, int E>
using RawRows = std::conditional_t<E == 16, Raw16<PDT>, Raw8<PDT>>;
template <int PDT, int E>
__device__ __forceinline__ RawRows<PDT, E> load_rows(const void* base, int64_t at) {
  RawRows<PDT, E> r;
  const uint4* src = reinterpret_cast<const uint4*>((const char*)base + at * (PDT == FSX_F32 ? 4 : 2));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(r) / 16); ++i) r.p[i] = src[i];
  return r;
}
__device__ __forceinline__ uint4 to_bf16(const Raw8<FSX_BF16>& r) { return r.p[0]; }
__device__ __forceinline__ uint4 to_bf16(const Raw8<FSX_F32>& r) {
  const uint4 a = r.p[0], b = r.p[1];
  return make_uint4(pack_bf16x2(__uint_as_float(a.x), __uint_as_float(a.y)), pack_bf16x2(__uint_as_float(a.z), __uint_as_float(a.w)),
                    pack_bf16x2(__uint_as_float(b.x), __uint_as_float(b.y)), pack_bf16x2(__uint_as_float(b.z), __uint_as_float(b.w)));
}

template <int PDT, int CDT>
__global__ __launch_bounds__(256) void k_page_write(PageWriteArgs a) {
  const PagePool& p = a.pool;
  const int lane = threadIdx.x & 63, l = blockIdx.y, kv = blockIdx.z, blk = blockIdx.x;
  // the entry, its arguments in one round trip, a value per lane
  static_assert(PAGE_WRITES == 128, "two entries for each lane");
  const int prefix[2] = {a.block_prefix[lane + 1], a.block_prefix[64 + lane + 1]}, seqs[2] = {a.seq[lane], a.seq[64 + lane]};
  const int counts[2] = {a.rows[lane], a.rows[64 + lane]};
  const int64_t starts[2] = {a.start[lane], a.start[64 + lane]};
  const int s = __popcll(__ballot(lane < a.n && prefix[0] <= blk)) + __popcll(__ballot(64 + lane < a.n && prefix[1] <= blk));
  const auto of = [&](const int (&v)[2], int i) {
    return i < 64 ? __builtin_amdgcn_readlane(v[0], i) : __builtin_amdgcn_readlane(v[1], i - 64);
  };
  const int low[2] = {(int)starts[0], (int)starts[1]}, high[2] = {(int)(starts[0] >> 32), (int)(starts[1] >> 32)};
  const int64_t start = (int64_t)of(high, s) << 32 | (uint32_t)of(low, s);
  const int seq = of(seqs, s), count = of(counts, s), r0 = (blk - (s ? of(prefix, s - 1) : 0)) * a.block, nr = min(a.block, count - r0);
  const int first = p.len[seq] - count + r0;  // row of the sequence
  const int32_t* pages = p.table + (int64_t)seq * p.most;
  const char* rows = (const char*)(kv ? a.v : a.k);
  const int64_t row_step = kv ? a.v_row : a.k_row, head_step = kv ? a.v_head : a.k_head;
  const int64_t packed = l * (kv ? a.v_layer : a.k_layer) + (start + r0) * row_step;
  const int64_t layer_row = (int64_t)(a.layer + l) * p.pages * p.Hk * p.P;
  char* cache = (char*)(kv ? p.v : p.k);
  float* scales = kv ? p.v_scale : p.k_scale;
  constexpr int E = CDT == FSX_BF16 ? 8 : 16, U = 4;  // elements of 16 bytes; pieces under way
  // The thread's piece of a head's row, and its (row, head), which moves on by `heads` of them at a time.
  const int cpr = p.D / E, c = threadIdx.x & (cpr - 1), heads = 256 / cpr, dr = heads / p.Hk, dh = heads - dr * p.Hk;
  int r = (int)threadIdx.x / cpr / p.Hk, h = (int)threadIdx.x / cpr - r * p.Hk;
  while (r < nr) {
    RawRows<PDT, E> in[U];
    int64_t at[U];
    bool valid[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(r, nr - 1), row = max(first + i, 0);
      in[u] = load_rows<PDT, E>(rows, packed + i * row_step + h * head_step + E * c);
      at[u] = layer_row + (int64_t)pages[row >> p.shift] * (p.Hk * p.P) + h * p.P + (row & (p.P - 1));
      valid[u] = r < nr && first + i >= 0;
      r += dr, h += dh;
      if (h >= p.Hk) h -= p.Hk, ++r;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (CDT == FSX_BF16) {
        if (valid[u]) *reinterpret_cast<uint4*>((uint16_t*)cache + at[u] * p.D + E * c) = to_bf16(in[u]);
      } else {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < Raw16<PDT>::N; ++i) t = fold_top<PDT>(t, in[u].p[i], false);
        float top = top_value<PDT>(t);
        const bool finite = top < INFINITY;
        if (!finite) {
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
        const Scale scale(scale_of(top, 1.f));
        float x[16];
        to_floats<PDT>(in[u], x);
        const auto out = __all(finite && !scale.tiny) ? from_floats<CDT, true>(x, scale) : from_floats<CDT>(x, scale);
        if (valid[u]) {
          store_raw<CDT>(cache, at[u] * p.D + 16 * c, out);
          if (c == 0) scales[at[u]] = scale.s;
        }
      }
    }
  }
}

hipError_t launch_page_write(PageWriteArgs a, int n, const int32_t* seqs, const int64_t* start, const int64_t* rows, hipStream_t s) {
  const PagePool& p = a.pool;
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += rows[i];
  // rows of a workgroup: four pieces for every thread, once there are two workgroups for each CU (15,000 rows of 4 heads of 64 channels,
  // uneven sequences, into fp8 pages: 10 us, with eight for each 15)
  const int64_t full = std::max<int64_t>(1, 4 * 256 / (p.Hk * (p.D / (p.fp8 ? 16 : 8))));
  a.block = (int)std::max<int64_t>({1, std::min<int64_t>(full, total * a.n_layers * 2 / 512), (total >> 23) + 1});
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
    const hipError_t e = enqueue(fn, grid, dim3(256), s, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fsx
