// Host-visible launch interface of the expert-tick kernels (internal to libfsx).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>
#include <vector>

#include "../../include/fsx.h"
#include "head_device.h"
#include "page_lists.h"

namespace fsx {

// Sets the calling thread's message of fsx_last_error ("" clears it) and returns code.
int set_error(int code, const std::string& msg);

// Enqueues a kernel and returns the launch's own status: hipGetLastError would take an error that other code of the thread met and
// left there for one of this launch.
template <class... P, class... A>
hipError_t enqueue(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t s, const A&... a) {
  return [&](const P&... p) {
    void* args[] = {const_cast<void*>(static_cast<const void*>(&p))...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, args, 0, s);
  }(a...);
}

// Per-forward description of the agents, passed by value in kernel arguments.
struct TickParams {
  int32_t B, S, T, M;                         // agents, tokens per agent, pooled tokens, rows = B*S
  int32_t n_tt;                               // ceil(S / 16): query tiles per (agent, head)
  int32_t chunk_rows;                         // per-phase path: cache rows per attention work item
  int32_t n_items;                            // per-phase path: attention work items
  // per-phase path, query tiles that share rows (k_attention_tiles): groups of att_qg query tiles (0 groups: one wave per
  // item instead), the longest group's chunks, whether a group spans the agents of a shared cache, and their ring start
  int32_t att_groups, att_qg, att_chunks, att_shared;
  int64_t att_start;
  int32_t Mp;                                 // M rounded up to 8: rows of tile-major activations
  int32_t Ms;                                 // M rounded up to 32: rows of the sums of squares
  int64_t pos[FSX_MAX_BATCH];                 // rotary position of token 0
  int64_t start[FSX_MAX_BATCH];               // ring slot of the oldest valid row
  int32_t len[FSX_MAX_BATCH];                 // valid cache rows
  int32_t chunk_prefix[FSX_MAX_BATCH + 1];    // per-phase path: chunks before agent b (plan_chunks; at least one each)
  // tick kernel attention: agents in the order order[0..B-1]; the k-th weighs seg_w[k] work tiles per head
  // (its 32-row cache tiles, then the 32-row tiles of the expert's own rows), seg_p[k] = seg_w[0] + ... +
  // seg_w[k-1]; partial-state slots of XCD X
  // are X * slot_x .. X * slot_x + slot_x - 1
  int32_t order[FSX_MAX_BATCH];
  int32_t seg_w[FSX_MAX_BATCH];
  int32_t seg_p[FSX_MAX_BATCH + 1];
  int32_t slot_x;
  // tick kernel: row blocks of every residual column tile in the cross-XCD reductions (pieces; see reduce_piece)
  int32_t rblk;
};

// Cache view of one layer.  Element offset of (agent b, layer l, head h, ring slot j, channel c):
// b * bs + l * H * cap * Dh + h * hs + j * rs + c, with (hs, rs) = (cap * Dh, Dh) for a head-major cache and
// (Dh, H * Dh) for a token-major one; bs = n_layers * H * cap * Dh, or 0 when every agent reads the same rings
// (a shared cache).  fp8 scale of (b, l, h): [b * sbs + l * H + h], sbs = n_layers * H or 0.
struct CacheView {
  const void* k;     // base of the whole cache tensor
  const void* v;
  const float* k_scale;  // fp8 only: [batch][n_layers][H] ([1][n_layers][H] when shared)
  const float* v_scale;
  int64_t cap;           // ring rows
  int64_t hs;            // elements between the rows of two heads of one slot
  int64_t rs;            // elements between two ring slots of one head
  int64_t bs;            // elements between the rings of two agents (0: shared)
  int32_t sbs;           // scales between two agents (0: shared)
  int32_t n_layers;
  int32_t layer;
  int32_t dtype;         // fsx_dtype
  int32_t H, Dh;
};
// Element offset of row slot 0 of (agent b, layer l, head h).
__host__ __device__ inline int64_t cache_head_base(const CacheView& cv, int b, int l, int h) {
  return (int64_t)b * cv.bs + (int64_t)l * cv.H * cv.cap * cv.Dh + (int64_t)h * cv.hs;
}
__host__ __device__ inline int64_t cache_scale_index(const CacheView& cv, int b, int l, int h) {
  return (int64_t)b * cv.sbs + (int64_t)l * cv.H + h;
}

// ------------------------------------------------------------------ packing (create time)
enum PackKind { PACK_PLAIN = 0, PACK_ROPE_PAIRS = 1, PACK_SWIGLU_PAIRS = 2 };
hipError_t launch_pack(const uint16_t* a, const uint16_t* b, int N, int K, int kind, int param, const float* gain,
                       void* dst, hipStream_t s);

// ------------------------------------------------------------------ fused-path phases
struct FastWeights {
  const uint4* wqkv;   // packed [3A][d]  (q, k rows paired for rotary)
  const uint4* wo;     // packed [d][A]
  const uint4* wgu;    // packed [2F][d]  (gate/up rows paired)
  const uint4* wd;     // packed [d][F]
  const float* attn_norm;
  const float* ffn_norm;
};

struct Workspace {
  float* h;          // [M][d] residual stream
  uint16_t* xb;      // [M][max(d, ...)] bf16 normalised input of the next projection
  float* q;          // [M][A] rotated, pre-scaled queries
  uint16_t* kself;   // [M][A] bf16 rotated keys of the expert tokens
  uint16_t* vself;   // [M][A] bf16 values of the expert tokens
  uint16_t* attn;    // [M][A] bf16 attention output
  uint16_t* z;       // [M][F] bf16 SwiGLU output
  float* part;       // [ksplit][M][d] split-K partial sums
  // partial attention states, 16 * Dh and 32 floats per item: unnormalised outputs, running maxima (log2 units) and sums (the
  // tick kernel: [16][Dh] and [16][2]; the phases: in the order of store_state)
  float* att_o;
  float* att_ml;
  float* rope;       // [M][Dh/2][2] cos, sin
  float* ss;         // [M][d/512] per-chunk sums of squares (wide rows)
  float* rs;         // [M] RMSNorm scale of each row (wide rows)
  uint32_t* rcnt;    // [M] chunks of the row reduced so far (wide rows; zero between launches)
  uint32_t* acnt;    // [B*H*n_tt] attention chunks finished (zero between launches)
};

struct Dims {
  int d, H, Dh, A, F, n_layers, n_out;
  float eps, rope_base;
  int head_kind;  // 0: mean over the expert tokens + linear; 1: two-layer head over the waypoint queries
};

// Rows wide enough (the backbone's width) that the per-phase reductions split them into chunks of RN_CHUNK columns,
// one workgroup each, and leave the RMSNorm scale to the next projection.
constexpr int RN_CHUNK = 512;
__host__ __device__ inline bool wide_rows(const Dims& dm) { return dm.d >= 4 * RN_CHUNK && dm.d % RN_CHUNK == 0; }

// packed: agents of different lengths, their rows by tp.chunk_prefix.
hipError_t launch_embed(const void* tokens, int tok_dtype, const float* g0, const TickParams& tp, const Dims& dm,
                        const Workspace& ws, hipStream_t s, bool packed = false);
// after_reduction: xb comes from a reduction (not from the embedding); for wide rows it is then unscaled and the
// projection applies the RMSNorm row scales from the chunk sums of squares.
hipError_t launch_gemm_qkv(const FastWeights& w, const TickParams& tp, const Dims& dm, const Workspace& ws,
                           hipStream_t s, bool after_reduction);
constexpr int ATT_Q = 6;  // query tiles of a workgroup that share their rows at most
// The attention of every (agent, head), its work items (tp.chunk_prefix, tp.n_items) merged.
hipError_t launch_attention(const CacheView& cv, const TickParams& tp, const Dims& dm, const Workspace& ws,
                            hipStream_t s, bool causal = false);
// Split-K ranges (at most 8) of the output and down projections over M rows.
int gemm_split(int M, int N, int K);
hipError_t launch_gemm_o(const FastWeights& w, const TickParams& tp, const Dims& dm, const Workspace& ws,
                         int ksplit, hipStream_t s);
hipError_t launch_gemm_gu(const FastWeights& w, const TickParams& tp, const Dims& dm, const Workspace& ws,
                          hipStream_t s);
hipError_t launch_gemm_down(const FastWeights& w, const TickParams& tp, const Dims& dm, const Workspace& ws,
                            int ksplit, hipStream_t s);
// With rows_into, the same launch also stores the layer's new rows (ws.kself / ws.vself, B agents x S tokens) into ring
// slots (start + len + t) mod capacity of cache layer rows_into->layer (after the attention has read the old rows).
hipError_t launch_reduce_norm(const TickParams& tp, const Dims& dm, const Workspace& ws, int ksplit,
                              const float* gain, float* hidden_layer, hipStream_t s, const CacheView* rows_into = nullptr);
hipError_t launch_head(const TickParams& tp, const Dims& dm, const Workspace& ws, const float* final_norm,
                       const void* head_w, int head_dtype, float* waypoints, hipStream_t s);
// The two-layer query head of every agent from a row-major residual h [M][d] (both per-op paths).
hipError_t launch_query_head(const float* h, const TickParams& tp, const Dims& dm, const float* final_norm,
                             const QueryHead& qh, float* waypoints, hipStream_t s);

// ------------------------------------------------------------------ persistent tick kernel
// The tick kernel splits every layer over the chip's XCDs the way a tensor-parallel layer is split over
// devices: XCD X owns a contiguous range of heads and of FFN columns.  Buffers marked "per XCD" hold one
// replica per XCD rank (at most NXMAX); those indexed by head or FFN unit are written and read by one XCD only;
// the residual and its bf16 copies are written once (each piece by one workgroup) and read by every XCD.
constexpr int NXMAX = 16;
constexpr int NXR = 8;      // XCDs the cross-XCD reductions read at most (the XCD count of gfx950 parts)
constexpr int FPAD = 16;     // flags are 64-bit stamps, one per 128-byte line (index * FPAD)
constexpr int XFLAGS = 512;  // flag slots per XCD of the per-XCD flag arrays

struct TickArgs {
  const char* wbase;   // packed weights of layer 0; layers follow back to back (see layer_w)
  const float* final_norm;
  const void* head_w;
  int head_dtype;
  QueryHead qhead;     // head kind 1
  int tok_dtype;
  const void* tokens;
  CacheView cv;
  float* waypoints;
  float* hidden;       // optional caller buffer [n_layers][M][d]
  uint64_t* reg;       // [grid] registration words: epoch << 8 | hardware XCD id
  // written by the owner of each piece, read by every XCD
  float* hres;         // residual stream, tile-major [d/16 column tiles][Mp rows][16 columns]
  uint16_t* xb_mid;    // [Mp][d] bf16 copy of the residual after attention (input of the FFN)
  uint16_t* xb_out;    // [Mp][d] bf16 copy of the residual after the FFN (input of the next layer)
  float* ssq_mid;      // [d/16][Ms] per-tile sums of squares
  float* ssq_out;
  // per XCD
  float* rope;         // [M][Dh/2][2] cos, sin
  int64_t x_stride_r;  // floats between replicas of rope
  // by head / FFN unit
  float* q;            // [M][A] rotated, pre-scaled queries
  uint16_t* kself;     // [M][A]
  uint16_t* vself;     // [M][A]
  uint16_t* attn;      // [M][A]
  uint16_t* z;         // [Mp][F] SwiGLU output
  float* att_o;        // [slot * n_tt + query tile][16][Dh] partial attention states
  float* att_ml;       // [slot * n_tt + query tile][16][2]
  // crossing XCDs: stamped 8-byte words (payload in the low half, stamp in the high half)
  uint64_t* po;        // [NXMAX][d/16][Mp][16] output-projection partials
  uint64_t* pd;        // [NXMAX][d/16][Mp][16] down-projection partials
  // flags (stamps), each in its own 128-byte line: element [i] lives at f[i * FPAD]
  uint64_t* f_rope;    // [NXMAX][XFLAGS] by workgroup slot
  uint64_t* f_out;     // [XFLAGS] by residual piece (column tile * rblk + row block)
  uint64_t* f_mid;     // [XFLAGS] by residual piece
  uint64_t* f_q;       // [3A/16][row blocks of 80 rows]
  uint64_t* f_attn;    // [B*H][n_tt] per query tile
  uint64_t* f_rng;     // [slot] partial states written
  uint64_t* f_z;       // [F/8][row blocks of 80 rows]
  uint64_t* status;
  uint64_t epoch;
  uint64_t timeout_ticks;  // real-time counter ticks (100 MHz)
  uint64_t* trace;         // optional: [grid][trace_events(n_layers)] real-time stamps per workgroup
};

// per workgroup: start, after the embedding, 16 events per layer (5 phase ends, then 11 sub-phase marks), end
__host__ __device__ inline int trace_events(int n_layers) { return 2 + 16 * n_layers + 1; }

hipError_t tick_occupancy(int kt, int* blocks_per_cu);
hipError_t launch_tick(const TickArgs& a, const TickParams& tp, const Dims& dm, int grid, hipStream_t s);
// Hardware XCD id of every workgroup of a one-workgroup-per-CU launch (create-time placement check).
hipError_t probe_xcds(uint32_t* dev_out, int grid, hipStream_t s);

// Zero `bytes` (a multiple of 256) at p with a kernel.
hipError_t launch_fill_zero(void* p, size_t bytes, hipStream_t s);

// ------------------------------------------------------------------ measurement helper
// One read-only pass over `bytes` (a multiple of 16) of buf; mode 0 register loads, 1 direct loads into LDS;
// sink: DEVICE [1024] uint32 checksum words.
hipError_t launch_probe_read(const void* buf, int64_t bytes, int mode, uint32_t* sink, hipStream_t s);

// ------------------------------------------------------------------ cache append
hipError_t launch_append(const fsx_cache_desc& c, const void* k_rows, const void* v_rows, int n_rows,
                         const int64_t* dst_first_slot /* host [batch] */, hipStream_t s);
// bf16 / fp32 rows (rows_dtype) encoded into an fp8 cache with its existing scales.
hipError_t launch_append_quantize(const fsx_cache_desc& c, const void* k_rows, const void* v_rows, int rows_dtype,
                                  int n_rows, const int64_t* dst_first_slot, hipStream_t s);

// ------------------------------------------------------------------ whole prompts
// Packed sequences of the prompt attention, longest keys first, by value in kernel arguments.
struct PromptArgs {
  const void* q;
  const uint16_t* k;
  const uint16_t* v;
  void* out;
  float* lse;           // [q_rows][H] or NULL
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;  // elements
  int32_t H, G, D;      // query heads, query heads per key head, head width
  int32_t q_f32, o_f32;
  int32_t kernel;       // FSX_PROMPT_*
  float c;              // scores in log2 units = c * q.k
  int32_t n_seq;
  int64_t q0[FSX_MAX_BATCH], k0[FSX_MAX_BATCH];
  int32_t nq[FSX_MAX_BATCH], nk[FSX_MAX_BATCH];
  int32_t item_prefix[FSX_MAX_BATCH + 1];  // workgroups of the sequences before
  // keys in chunks (few rows)
  float* part;           // states of the workgroups
  int32_t chunk;         // tiles of a chunk
  int32_t n_split[FSX_MAX_BATCH], merge_prefix[FSX_MAX_BATCH + 1];
};
// Whether the keys are walked in chunks, and how; the bytes of workspace that the plan uses, at most workspace_bytes.
bool plan_prompt(PromptArgs& a, int64_t workspace_bytes, int64_t* need);
hipError_t launch_prompt_attention(PromptArgs a, void* workspace, int64_t workspace_bytes, hipStream_t s);

// ------------------------------------------------------------------ cache rows replaced and read
// Rows of one agent: packed rows src .. src + n - 1 of every layer <-> ring slots (slot + i) mod cap.
struct RowsArgs {
  CacheView cv;          // layer: the first one; scales of a cache that is replaced are written
  void* k;               // packed rows [layers][total][H][Dh], or NULL
  void* v;
  int32_t rows_f32;      // packed rows are fp32, else bf16
  int32_t layers, B;
  int64_t total;
  float headroom;
  int64_t src[FSX_MAX_BATCH], slot[FSX_MAX_BATCH];
  int32_t n[FSX_MAX_BATCH];
  int64_t prefix[FSX_MAX_BATCH + 1];  // rows of the agents before
  int32_t block;                      // rows of a workgroup, and workgroups of the agents before
  int32_t block_prefix[FSX_MAX_BATCH + 1];
};
hipError_t launch_replace_rows(const RowsArgs& a, hipStream_t s);
hipError_t launch_read_rows(const RowsArgs& a, hipStream_t s);

// ------------------------------------------------------------------ rotary positions
constexpr int ROTARY_PAIRS = 128;
struct RotaryArgs {
  const void* x;
  void* y;
  const int32_t* pos;
  int64_t x_row, x_head, y_row, y_head, pos_axis, pos_row;  // elements
  int64_t rows;
  int32_t heads, dim, pairs, f32, adjacent, inverse;
  int32_t copy_rest;                // channels past the pairs are copied (y is not x)
  int32_t block;                    // rows of a workgroup
  uint64_t turn[ROTARY_PAIRS];      // turns per step of the pair's axis, mod 1, in units of 2^-64
  uint8_t axis[ROTARY_PAIRS];
};
hipError_t launch_rotary(RotaryArgs a, hipStream_t s);

// ------------------------------------------------------------------ pages
// A pool of pages [layers][pages][Hk][P][D] and, on the device, every sequence's list [sequences][most] and length.
struct PagePool {
  void* k;
  void* v;
  float* k_scale;  // [layers][pages][Hk][P], fp8 only
  float* v_scale;
  const int32_t* table;
  const int32_t* len;
  int32_t layers, pages, Hk, P, shift, D, fp8, most;  // P = 1 << shift
};
// Entries of lists and lengths, and pages copied, up to four copies of one page side by side.
constexpr int PAGE_RUNS = 80, PAGE_COPIES = 64, PAGE_TARGETS = 4;
struct PageCopies {
  int32_t from, rows, n, to[PAGE_TARGETS];
};
struct PageUpdateArgs {
  PagePool pool;
  int32_t* table;  // written; copied entries come from pool.table
  int32_t* len;    // NULL: lengths stay
  int32_t n_runs, n_copies;
  PageRun runs[PAGE_RUNS];
  PageCopies copies[PAGE_COPIES];
};
static_assert(sizeof(PageUpdateArgs) <= 4096, "kernel arguments");
hipError_t launch_page_update(const PagePool& pool, int32_t* table, int32_t* len, const std::vector<PageRun>& runs,
                              const std::vector<PageCopy>& copies, hipStream_t s);
// Rows that close up: row i of the outcome, from `start` on, is row i - to + first of the last range with to <= i.
constexpr int PAGE_MOVES = 64, PAGE_RANGES = 256;
struct PageMoveArgs {
  PagePool pool;
  const int32_t* to_table;
  int32_t* len;            // lengths of the sequences that move, or NULL
  int32_t n_moves, split;  // workgroups that share a row's channels
  PageMove moves[PAGE_MOVES];
  PageRange ranges[PAGE_RANGES];  // count: the first row's place in the outcome
};
hipError_t launch_page_move(const PagePool& pool, const int32_t* to_table, int32_t* len, const std::vector<PageMove>& moves,
                            const std::vector<PageRange>& ranges, hipStream_t s);
// Packed rows into the last rows of sequences.
constexpr int PAGE_WRITES = 128;
struct PageWriteArgs {
  PagePool pool;
  const void* k;
  const void* v;
  int64_t k_layer, k_row, k_head, v_layer, v_row, v_head;  // elements
  int32_t rows_f32, layer, n_layers;
  int32_t n, block;      // entries; rows of a workgroup
  int64_t start[PAGE_WRITES];
  int32_t seq[PAGE_WRITES], rows[PAGE_WRITES], block_prefix[PAGE_WRITES + 1];
};
hipError_t launch_page_write(PageWriteArgs a, int n, const int32_t* seqs, const int64_t* start, const int64_t* rows, hipStream_t s);
// One new token of every entry's sequence over its pages.  Entries whose sequences share their first pages are neighbours; the rows
// of those pages, `base` of them, are read for a tile of such entries at a time.
constexpr int PAGE_QUERIES = 128;
struct PageAttentionArgs {
  PagePool pool;
  const void* q;
  void* out;
  float* lse;            // [n][H] or NULL
  float* part;           // states of the workgroups
  int64_t q_row, q_head, o_row, o_head;  // elements
  int32_t H, G, layer, q_f32, o_f32;
  float c;               // scores in log2 units = c * q.k
  int32_t n, n_tiles;
  // Steps of 32 rows, and some for each stretch's start: those of the tiles, `tiled` of them, then those of the entries.  A workgroup
  // takes `per` of them, whatever they belong to, or (each) at most `per` of one tile or entry, the tiles' tiled_parts stretches first.
  int32_t per, each, tiled, total, tiled_parts;
  int32_t seq[PAGE_QUERIES], base[PAGE_QUERIES];
  uint16_t row[PAGE_QUERIES];
  int32_t all[PAGE_QUERIES + 1];                                      // parts of the split entries before, shared rows' too
  int32_t steps[PAGE_QUERIES + 1], parts[PAGE_QUERIES + 1];           // steps, and stretches, before the entries' own
  uint8_t tile[PAGE_QUERIES / 2], members[PAGE_QUERIES / 2];          // first entries of the tiles, and how many
  int32_t tile_steps[PAGE_QUERIES / 2 + 1], tile_parts[PAGE_QUERIES / 2 + 1];  // before the tiles
};
static_assert(sizeof(PageAttentionArgs) <= 4096, "kernel arguments");
// How a call is shared out.
struct PagePlan {
  struct Entry {
    int32_t index, base;        // row of q; rows that a tile reads
    int32_t steps, own, shared; // steps of the others; parts of them, and of the tile's
    int states() const { return own + shared > 1 ? own + shared : 0; }  // that are put together
  };
  struct Tile {
    int32_t first, members;
  };
  struct Launch {
    int32_t first, n, first_tile, n_tiles, per, each, extra, workgroups, parts;  // extra: steps added to every stretch
  };
  std::vector<Entry> entries;
  std::vector<Tile> tiles;
  std::vector<Launch> launches;
  bool wide = false;   // workgroups of eight waves
  int64_t bytes = 0;   // of workspace
};
void plan_page_attention(const PagePool& pool, const PageLists& lists, int H, int n, const int32_t* seqs, int64_t workspace_bytes,
                         PagePlan& plan);
hipError_t launch_page_attention(PageAttentionArgs a, const int32_t* seqs, const PagePlan& plan, hipStream_t s);

// ------------------------------------------------------------------ simple per-op path (any dtype)
struct GenericWeights {
  const void* wq; const void* wk; const void* wv; const void* wo;
  const void* wg; const void* wu; const void* wd;
  const float* attn_norm; const float* ffn_norm;
};
struct GenericWorkspace {
  float* h; float* q; float* k; float* v; float* attn; float* g; float* rope;
};
hipError_t generic_tick(const GenericWeights* layers, const float* final_norm, const void* head_w,
                        const QueryHead& qhead, int wdtype,
                        const void* tokens, const CacheView& cv0, const TickParams& tp, const Dims& dm,
                        const GenericWorkspace& ws, float* waypoints, float* hidden, hipStream_t s);

}  // namespace fsx
