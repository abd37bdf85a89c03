// C ABI of the rotary positions and of the pages: argument checks, the handle with its lists on host and device, and the launches.
// See include/fsx.h for the contract of every entry point.

#include <array>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "extents.h"
#include "kernels.h"
#include "turns.h"

using namespace fsx;

// The caller's memory: keys, values and, fp8, their scales (otherwise empty, at 0).
static std::array<Extent, 4> pool_memory(const fsx_pages_cfg& cfg) {
  const int64_t rows = (int64_t)cfg.n_layers * cfg.n_pages * cfg.n_kv_heads * cfg.page_rows;
  const bool fp8 = cfg.dtype == FSX_FP8_E4M3;
  const int64_t bytes = rows * cfg.head_dim * (fp8 ? 1 : 2), scales = fp8 ? 4 * rows : 0;
  return {block(cfg.k, bytes), block(cfg.v, bytes), block(fp8 ? cfg.k_scale : nullptr, scales), block(fp8 ? cfg.v_scale : nullptr, scales)};
}

struct fsx_pages {
  fsx_pages_cfg cfg{};
  int device = 0;
  PageLists lists;
  int32_t* table = nullptr;  // device [max_seqs][max_seq_pages]
  int32_t* next = nullptr;   // device: lists that rows move to
  int32_t* len = nullptr;    // device [max_seqs]
  bool failed = false;       // the device's lists may not be the host's
  explicit fsx_pages(const fsx_pages_cfg& c) : cfg(c), lists(c.n_pages, c.max_seqs, c.max_seq_pages, c.page_rows) {}
  ~fsx_pages() {
    // (a handle may be given back while some stream is captured; the free itself is no part of that)
    hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
    const bool swapped = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
    (void)hipFree(table);
    if (swapped) (void)hipThreadExchangeStreamCaptureMode(&mode);
  }
  std::array<Extent, 4> memory() const { return pool_memory(cfg); }
  PagePool pool() const {
    int shift = 0;
    while (1 << shift < cfg.page_rows) ++shift;
    return {cfg.k, cfg.v, cfg.k_scale, cfg.v_scale, table, len, cfg.n_layers, cfg.n_pages, cfg.n_kv_heads, cfg.page_rows, shift,
            cfg.head_dim, cfg.dtype == FSX_FP8_E4M3, cfg.max_seq_pages};
  }
};

namespace {

int bad(const std::string& msg) { return set_error(FSX_E_INVALID, msg); }
int done() { return set_error(FSX_OK, ""); }
// (reported here, so it does not stay behind as the thread's last error)
int hip_error(const char* what, hipError_t e) {
  (void)hipGetLastError();
  return set_error(FSX_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// No exception crosses the boundary.
template <class F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return set_error(FSX_E_OOM, "out of host memory");
  } catch (...) {
    return set_error(FSX_E_INVALID, "unexpected error");
  }
}

// A handle that can be used, on its own device.
int check_handle(const fsx_pages* h) {
  if (!h) return bad("pages is NULL");
  if (h->failed) return set_error(FSX_E_HIP, "an earlier call of this handle failed on the device");
  int device = 0;
  const hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return hip_error("hipGetDevice", e);
  if (device != h->device) return bad("the handle belongs to device " + std::to_string(h->device) + ", not to the current one");
  return FSX_OK;
}

// What the calls that change lists check alike.
int check_change(const fsx_pages* h, int32_t n, const void* a, const void* b, void* stream) {
  if (const int rc = check_handle(h)) return rc;
  if (n < 0 || n > h->cfg.max_seqs) return bad("n must be in 0..max_seqs");
  if (n > 0 && (!a || !b)) return bad("the sequences' host arrays must be non-NULL");
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  const hipError_t e = hipStreamIsCapturing((hipStream_t)stream, &status);
  if (e != hipSuccess) return hip_error("hipStreamIsCapturing", e);
  if (status != hipStreamCaptureStatusNone)
    return set_error(FSX_E_UNSUPPORTED, "lists cannot be changed inside a captured graph: change them before its replay");
  return FSX_OK;
}

int enqueued(fsx_pages* h, hipError_t e) {
  if (e == hipSuccess) return done();
  h->failed = true;
  return hip_error("the lists' kernels", e);
}

int check_rotary(const fsx_rotary_desc* d) {
  if (!d) return bad("desc is NULL");
  if (d->dtype != FSX_BF16 && d->dtype != FSX_F32) return set_error(FSX_E_UNSUPPORTED, "x and y must be BF16 or F32");
  if (d->n_heads < 1 || d->n_heads > 4096) return bad("n_heads must be in 1..4096");
  if (d->head_dim < 2 || d->head_dim > 1024) return bad("head_dim must be in 2..1024");
  if (d->n_pairs < 1 || d->n_pairs > ROTARY_PAIRS || 2 * d->n_pairs > d->head_dim)
    return bad("n_pairs must be in 1..128, at most head_dim / 2");
  if (d->layout != FSX_ROTARY_HALVES && d->layout != FSX_ROTARY_ADJACENT) return bad("layout must be one of FSX_ROTARY_*");
  if (d->n_axes < 1 || d->n_axes > 256) return bad("n_axes must be in 1..256");
  if (d->inverse != 0 && d->inverse != 1) return bad("inverse must be 0 or 1");
  if (!d->axis || !d->freq) return bad("axis and freq must be non-NULL host arrays");
  for (int j = 0; j < d->n_pairs; ++j) {
    if (d->axis[j] < 0 || d->axis[j] >= d->n_axes) return bad("axis of pair " + std::to_string(j) + " outside 0..n_axes-1");
    if (!(std::fabs(d->freq[j]) <= 0x1p20)) return bad("freq of pair " + std::to_string(j) + " must be at most 2^20");
  }
  for (const int64_t s : {d->x_row, d->x_head, d->y_row, d->y_head, d->pos_axis, d->pos_row})
    if (s < 0 || s > (int64_t)1 << 30) return bad("strides must be in 0..2^30 elements");
  return FSX_OK;
}

// Elements from the first to behind the last of rows of heads.
int64_t extent(int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t dim) {
  return (rows - 1) * row + (heads - 1) * head + dim;
}

// What the attention reads of its descriptor.
int check_attention(const fsx_pages* h, const fsx_prompt_desc* d, int32_t n, const int32_t* seqs) {
  if (!d) return bad("desc is NULL");
  const fsx_pages_cfg& c = h->cfg;
  if (d->n_kv_heads != c.n_kv_heads || d->head_dim != c.head_dim) return bad("n_kv_heads and head_dim must be the pool's");
  if (d->n_heads < 1 || d->n_heads > 4096 || d->n_heads % c.n_kv_heads) return bad("n_heads must be in 1..4096, a multiple of n_kv_heads");
  if ((d->q_dtype != FSX_BF16 && d->q_dtype != FSX_F32) || (d->out_dtype != FSX_BF16 && d->out_dtype != FSX_F32))
    return set_error(FSX_E_UNSUPPORTED, "q and out must be BF16 or F32");
  if (!(d->scale >= 0.f) || d->scale > 1e30f) return bad("scale must be positive, or 0 for 1 / sqrt(head_dim)");
  if (n < 1 || n > 65536) return bad("n must be in 1..65536");
  if (!seqs) return bad("seqs must be a non-NULL host array");
  for (int i = 0; i < n; ++i)
    if (seqs[i] < 0 || seqs[i] >= c.max_seqs) return bad("sequence " + std::to_string(seqs[i]) + " outside 0..max_seqs-1");
  return FSX_OK;
}

}  // namespace

extern "C" int fsx_rotary_rows(const fsx_rotary_desc* d, const void* x, void* y, const int32_t* positions, int64_t n_rows,
                               void* stream) {
  return guarded([&]() -> int {
    if (const int rc = check_rotary(d)) return rc;
    if (n_rows < 0) return bad("n_rows must be >= 0");
    if (n_rows > 1 << 26) return set_error(FSX_E_UNSUPPORTED, "more than 2^26 rows");
    if (n_rows == 0) return done();
    if (!x || !y || !positions) return bad("x, y and positions must be non-NULL");
    const uintptr_t es = d->dtype == FSX_F32 ? 4 : 2;
    if ((uintptr_t)x % es || (uintptr_t)y % es || (uintptr_t)positions % 4) return bad("x, y and positions must be aligned to their elements");
    const int64_t H = d->n_heads, D = d->head_dim;
    if (!apart({0, n_rows, d->y_row, H, d->y_head, D})) return bad("rows and heads of y overlap");
    if (x == y ? (d->x_row != d->y_row && n_rows > 1) || (d->x_head != d->y_head && H > 1) : false)
      return bad("x and y in the same place must have the same strides");
    if (x != y) {
      const uintptr_t xe = (uintptr_t)x + es * extent(n_rows, d->x_row, H, d->x_head, D);
      const uintptr_t ye = (uintptr_t)y + es * extent(n_rows, d->y_row, H, d->y_head, D);
      if ((uintptr_t)x < ye && (uintptr_t)y < xe) {
        // the heads of one may lie between those of the other, in rows of the same length
        const int64_t row = d->x_row, wx = (H - 1) * d->x_head + D, wy = (H - 1) * d->y_head + D;
        const int64_t to = ((int64_t)((uintptr_t)y - (uintptr_t)x) / (int64_t)es), at = row ? (to % row + row) % row : 0;
        const bool whole = ((uintptr_t)y - (uintptr_t)x) % es == 0;
        if (!whole || row != d->y_row || row < wx || row < wy || at < wx || at + wy > row) return bad("x and y overlap");
      }
    }
    // positions that a pair's axis reads (an axis of its own for every pair, at most)
    const int64_t es8 = (int64_t)es, at = (int64_t)(uintptr_t)positions;
    const Extent rotated{(int64_t)(uintptr_t)y, n_rows, d->y_row * es8, H, d->y_head * es8, D * es8};
    for (int j = 0; j < d->n_pairs; ++j)
      if (j == 0 || d->axis[j] != d->axis[j - 1])
        if (meet({at + 4 * d->axis[j] * d->pos_axis, n_rows, 4 * d->pos_row, 1, 0, 4}, rotated)) return bad("positions and y overlap");
    RotaryArgs a{};
    a.x = x; a.y = y; a.pos = positions;
    a.x_row = d->x_row; a.x_head = d->x_head; a.y_row = d->y_row; a.y_head = d->y_head;
    a.pos_axis = d->pos_axis; a.pos_row = d->pos_row;
    a.rows = n_rows; a.heads = d->n_heads; a.dim = d->head_dim; a.pairs = d->n_pairs;
    a.f32 = d->dtype == FSX_F32; a.adjacent = d->layout == FSX_ROTARY_ADJACENT; a.inverse = d->inverse;
    a.copy_rest = x != y && 2 * d->n_pairs < d->head_dim;
    for (int j = 0; j < d->n_pairs; ++j) {
      a.turn[j] = turn_per_step(d->freq[j]);
      a.axis[j] = (uint8_t)d->axis[j];
    }
    const hipError_t e = launch_rotary(a, (hipStream_t)stream);
    return e == hipSuccess ? done() : hip_error("the rotation's kernel", e);
  });
}

extern "C" int fsx_pages_create(const fsx_pages_cfg* c, void* stream, fsx_pages** out) {
  if (!out) return bad("out is NULL");
  *out = nullptr;
  return guarded([&]() -> int {
    if (!c) return bad("cfg is NULL");
    if (c->dtype != FSX_BF16 && c->dtype != FSX_FP8_E4M3) return set_error(FSX_E_UNSUPPORTED, "pages must be BF16 or FP8_E4M3");
    if (c->n_layers < 1 || c->n_layers > 1024) return bad("n_layers must be in 1..1024");
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return bad("n_kv_heads must be in 1..1024");
    if (c->n_layers * c->n_kv_heads > 1 << 16) return set_error(FSX_E_UNSUPPORTED, "n_layers * n_kv_heads beyond 2^16");
    if (c->head_dim != 64 && c->head_dim != 128) return set_error(FSX_E_UNSUPPORTED, "head_dim must be 64 or 128");
    if (c->page_rows < 16 || c->page_rows > 256 || (c->page_rows & (c->page_rows - 1)))
      return bad("page_rows must be 16, 32, 64, 128 or 256");
    if (c->n_pages < 1) return bad("n_pages must be at least 1");
    if ((__int128)c->n_layers * c->n_pages * c->n_kv_heads * c->page_rows > (__int128)1 << 48) return bad("a pool beyond 2^48 rows");
    if (c->max_seqs < 1 || c->max_seqs > 65536) return bad("max_seqs must be in 1..65536");
    if (c->max_seq_pages < 1 || (int64_t)c->max_seq_pages * c->page_rows > 1 << 28 || (int64_t)c->max_seqs * c->max_seq_pages > 1 << 28)
      return bad("max_seq_pages must be at least 1, times page_rows and times max_seqs at most 2^28");
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return bad("k and v must be non-NULL and 16-byte aligned");
    if (c->dtype == FSX_FP8_E4M3 && (!c->k_scale || !c->v_scale || !aligned16(c->k_scale) || !aligned16(c->v_scale)))
      return bad("fp8 pages need k_scale and v_scale, 16-byte aligned");
    // Keys and values are moved by workgroups of their own: in one place, one would read what the other has moved already.
    const auto memory = pool_memory(*c);
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < i; ++j)
        if (meet(memory[i], memory[j])) return bad("k, v, k_scale and v_scale must not overlap");
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    hipError_t e = hipStreamIsCapturing((hipStream_t)stream, &status);
    if (e != hipSuccess) return hip_error("hipStreamIsCapturing", e);
    if (status != hipStreamCaptureStatusNone) return set_error(FSX_E_UNSUPPORTED, "pages cannot be created inside a captured graph");
    auto* h = new fsx_pages(*c);
    const size_t entries = ((size_t)c->max_seqs * c->max_seq_pages + 63) / 64 * 64, bytes = 4 * (2 * entries + ((size_t)c->max_seqs + 63) / 64 * 64);
    e = hipGetDevice(&h->device);
    if (e == hipSuccess) e = hipMalloc((void**)&h->table, bytes);
    if (e == hipErrorOutOfMemory) {
      (void)hipGetLastError();
      delete h;
      return set_error(FSX_E_OOM, "no device memory for the lists");
    }
    if (e == hipSuccess) e = launch_fill_zero(h->table, bytes, (hipStream_t)stream);
    if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
    if (e != hipSuccess) {
      delete h;
      return hip_error("fsx_pages_create", e);
    }
    h->next = h->table + entries;
    h->len = h->next + entries;
    *out = h;
    return done();
  });
}

extern "C" void fsx_pages_destroy(fsx_pages* h) { delete h; }

extern "C" int fsx_pages_extend(fsx_pages* h, int32_t n, const int32_t* seqs, const int32_t* rows, void* stream) {
  return guarded([&]() -> int {
    if (const int rc = check_change(h, n, seqs, rows, stream)) return rc;
    if (const int rc = h->lists.extend(n, seqs, rows)) return set_error(rc, h->lists.error);
    return enqueued(h, launch_page_update(h->pool(), h->table, h->len, h->lists.runs, h->lists.copies, (hipStream_t)stream));
  });
}

extern "C" int fsx_pages_fork(fsx_pages* h, int32_t n, const int32_t* src, const int32_t* dst, const int32_t* rows, void* stream) {
  return guarded([&]() -> int {
    if (const int rc = check_change(h, n, src, dst, stream)) return rc;
    if (const int rc = h->lists.fork(n, src, dst, rows)) return set_error(rc, h->lists.error);
    return enqueued(h, launch_page_update(h->pool(), h->table, h->len, h->lists.runs, {}, (hipStream_t)stream));
  });
}

extern "C" int fsx_pages_keep(fsx_pages* h, int32_t n, const int32_t* seqs, const int32_t* n_ranges, const int32_t* first,
                              const int32_t* count, void* stream) {
  return guarded([&]() -> int {
    if (const int rc = check_change(h, n, seqs, n_ranges, stream)) return rc;
    for (int i = 0; i < n; ++i) {
      if (n_ranges[i] > PAGE_RANGES) return set_error(FSX_E_UNSUPPORTED, "more than 256 ranges of a sequence");
      if (n_ranges[i] > 0 && (!first || !count)) return bad("first and count must be non-NULL host arrays");
    }
    PageLists& l = h->lists;
    if (const int rc = l.keep(n, seqs, n_ranges, first, count)) return set_error(rc, l.error);
    const hipStream_t s = (hipStream_t)stream;
    const PagePool pool = h->pool();
    // Where pages are replaced, the rows move by both lists before the new one becomes the sequence's; elsewhere the lists stay, and
    // the lengths are set with the rows.
    const bool in_place = l.before.empty();
    hipError_t e = in_place ? hipSuccess : launch_page_update(pool, h->next, nullptr, l.before, {}, s);
    if (e == hipSuccess) e = launch_page_move(pool, in_place ? h->table : h->next, in_place ? h->len : nullptr, l.moves, l.ranges, s);
    if (in_place) {
      size_t m = 0, left = 0;
      for (const PageRun& r : l.runs) {
        if (m < l.moves.size() && l.moves[m].seq == r.seq) ++m;
        else l.runs[left++] = r;
      }
      l.runs.resize(left);
    }
    if (e == hipSuccess) e = launch_page_update(pool, h->table, h->len, l.runs, {}, s);
    return enqueued(h, e);
  });
}

extern "C" int fsx_pages_free(fsx_pages* h, int32_t n, const int32_t* seqs, void* stream) {
  return guarded([&]() -> int {
    if (const int rc = check_change(h, n, seqs, seqs, stream)) return rc;
    if (const int rc = h->lists.free(n, seqs)) return set_error(rc, h->lists.error);
    return enqueued(h, launch_page_update(h->pool(), h->table, h->len, h->lists.runs, {}, (hipStream_t)stream));
  });
}

extern "C" int fsx_pages_tables(const fsx_pages* h, int32_t* len, int32_t* table, int64_t* free_pages) {
  if (!h) return bad("pages is NULL");
  const PageLists& l = h->lists;
  if (len) std::copy(l.len.begin(), l.len.end(), len);
  if (table) std::copy(l.table.begin(), l.table.end(), table);
  if (free_pages) *free_pages = l.n_free;
  return done();
}

extern "C" int fsx_pages_write(fsx_pages* h, const fsx_pages_rows* d, const void* k_rows, const void* v_rows, int32_t n,
                               const int32_t* seqs, const int64_t* row_start, const int64_t* row_len, void* stream) {
  return guarded([&]() -> int {
    if (const int rc = check_handle(h)) return rc;
    if (!d) return bad("desc is NULL");
    const fsx_pages_cfg& c = h->cfg;
    if (d->rows_dtype != FSX_BF16 && d->rows_dtype != FSX_F32) return bad("rows must be BF16 or F32");
    if (d->layer < 0 || d->n_layers < 1 || d->layer > c.n_layers - d->n_layers) return bad("layers outside 0..n_layers-1 of the pages");
    if (d->total_rows < 0 || d->total_rows > (int64_t)1 << 40) return bad("total_rows must be in 0..2^40");
    for (const int64_t s : {d->k_layer, d->k_row, d->k_head, d->v_layer, d->v_row, d->v_head})
      if (s < 0 || s % 8 || s > (int64_t)1 << 50) return bad("strides must be non-negative multiples of 8 elements");
    for (const int64_t s : {d->k_row, d->v_row})
      if ((__int128)s * d->total_rows > (__int128)1 << 60) return bad("strides beyond 2^60 elements in all");
    if (n < 0 || n > c.max_seqs) return bad("n must be in 0..max_seqs");
    if (n > 0 && (!seqs || !row_start || !row_len)) return bad("seqs, row_start and row_len must be non-NULL host arrays");
    if (const int rc = h->lists.check(n, seqs)) return set_error(rc, h->lists.error);
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
      const auto who = [&] { return "sequence " + std::to_string(seqs[i]); };
      if (row_len[i] < 0 || row_len[i] > h->lists.len[seqs[i]])
        return bad(who() + " has " + std::to_string(h->lists.len[seqs[i]]) + " rows, not " + std::to_string(row_len[i]));
      if (row_start[i] < 0 || row_start[i] > d->total_rows - row_len[i]) return bad("packed rows of " + who() + " outside 0..total_rows-1");
      if (!h->lists.writable(seqs[i], row_len[i])) return bad("rows of " + who() + " lie in a page that another sequence has too: extend it first");
      total += row_len[i];
    }
    if (total == 0) return done();
    if (total > (int64_t)1 << 31) return set_error(FSX_E_UNSUPPORTED, "more than 2^31 rows");
    if (!k_rows || !v_rows || !aligned16(k_rows) || !aligned16(v_rows)) return bad("k_rows and v_rows must be non-NULL and 16-byte aligned");
    // rows that lie in the pool themselves, its scales among it, would be read and written at once
    const int64_t es = d->rows_dtype == FSX_F32 ? 4 : 2;
    const auto meets = [&](const void* rows, int64_t layer, int64_t row, int64_t head) {
      const __int128 n = (__int128)(d->n_layers - 1) * layer + (__int128)(d->total_rows - 1) * row + (__int128)(c.n_kv_heads - 1) * head + c.head_dim;
      const __int128 from = (__int128)(uintptr_t)rows, to = from + n * es;
      for (const Extent& x : h->memory())
        if (from < x.end() && x.at < to) return true;
      return false;
    };
    if (meets(k_rows, d->k_layer, d->k_row, d->k_head) || meets(v_rows, d->v_layer, d->v_row, d->v_head))
      return bad("k_rows and v_rows must not lie in the pool");
    PageWriteArgs a{};
    a.pool = h->pool();
    a.k = k_rows; a.v = v_rows;
    a.k_layer = d->k_layer; a.k_row = d->k_row; a.k_head = d->k_head;
    a.v_layer = d->v_layer; a.v_row = d->v_row; a.v_head = d->v_head;
    a.rows_f32 = d->rows_dtype == FSX_F32; a.layer = d->layer; a.n_layers = d->n_layers;
    const hipError_t e = launch_page_write(a, n, seqs, row_start, row_len, (hipStream_t)stream);
    return e == hipSuccess ? done() : hip_error("the rows' kernel", e);
  });
}

extern "C" int fsx_pages_attention_workspace(const fsx_pages* h, const fsx_prompt_desc* d, int32_t n, const int32_t* seqs,
                                             int64_t* bytes) {
  if (!bytes) return bad("bytes is NULL");
  *bytes = 0;
  return guarded([&]() -> int {
    if (!h) return bad("pages is NULL");
    if (const int rc = check_attention(h, d, n, seqs)) return rc;
    PagePlan plan;
    plan_page_attention(h->pool(), h->lists, d->n_heads, n, seqs, INT64_MAX, plan);
    *bytes = plan.bytes;
    return done();
  });
}

extern "C" int fsx_pages_attention(fsx_pages* h, const fsx_prompt_desc* d, int32_t layer, const void* q, void* out, float* lse,
                                   int32_t n, const int32_t* seqs, void* workspace, int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (const int rc = check_handle(h)) return rc;
    if (const int rc = check_attention(h, d, n, seqs)) return rc;
    if (layer < 0 || layer >= h->cfg.n_layers) return bad("layer outside 0..n_layers-1 of the pages");
    if (d->q_rows < n || d->q_rows > (int64_t)1 << 40) return bad("q_rows must be in n..2^40");
    for (const int64_t s : {d->q_row, d->q_head, d->out_row, d->out_head})
      if (s < 0 || s % 8 || s > (int64_t)1 << 40) return bad("strides must be non-negative multiples of 8 elements, at most 2^40");
    if (!apart({0, n, d->out_row, d->n_heads, d->out_head, d->head_dim})) return bad("rows and heads of out overlap");
    if (!q || !out || !aligned16(q) || !aligned16(out)) return bad("q and out must be non-NULL and 16-byte aligned");
    if (workspace_bytes < 0 || (workspace_bytes > 0 && !workspace) || !aligned16(workspace))
      return bad("workspace must be 16-byte aligned, of workspace_bytes >= 0 bytes");
    // Workgroups end one after the other: what some write must not be what others have still to read, or written by two.
    const auto rows = [&](const void* p, int32_t dtype, int64_t row, int64_t head) {
      const int64_t es = dtype == FSX_F32 ? 4 : 2;
      return Extent{(int64_t)(uintptr_t)p, n, row * es, d->n_heads, head * es, d->head_dim * es};
    };
    const Extent writes[] = {rows(out, d->out_dtype, d->out_row, d->out_head), block(lse, (int64_t)4 * n * d->n_heads), block(workspace, workspace_bytes)};
    const char* names[] = {"out", "lse", "workspace"};
    for (int i = 0; i < 3; ++i) {
      if (!(i == 0 || (i == 1 ? lse != nullptr : workspace_bytes > 0))) continue;
      if (meet(rows(q, d->q_dtype, d->q_row, d->q_head), writes[i])) return bad(std::string(names[i]) + " must not overlap q");
      for (const Extent& x : h->memory())
        if (meet(x, writes[i])) return bad(std::string(names[i]) + " must not lie in the pool");
      for (int j = 0; j < i; ++j)
        if ((j == 0 || lse) && meet(writes[i], writes[j])) return bad(std::string(names[i]) + " must not overlap " + names[j]);
    }
    PageAttentionArgs a{};
    a.pool = h->pool();
    a.q = q; a.out = out; a.lse = lse; a.part = (float*)workspace;
    a.q_row = d->q_row; a.q_head = d->q_head; a.o_row = d->out_row; a.o_head = d->out_head;
    a.H = d->n_heads; a.G = d->n_heads / h->cfg.n_kv_heads; a.layer = layer;
    a.q_f32 = d->q_dtype == FSX_F32; a.o_f32 = d->out_dtype == FSX_F32;
    a.c = (d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->head_dim)) * 1.4426950408889634f;
    PagePlan plan;
    plan_page_attention(a.pool, h->lists, a.H, n, seqs, workspace_bytes, plan);
    const hipError_t e = launch_page_attention(a, seqs, plan, (hipStream_t)stream);
    return e == hipSuccess ? done() : hip_error("the attention's kernels", e);
  });
}
