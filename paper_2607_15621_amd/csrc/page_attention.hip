// Attention of one new token over the pages of its sequence, with grouped heads: for every query head
//   O = sum_j exp(s_j) v_j / sum_j exp(s_j),   s_j = scale q . k_j,   lse = log sum_j exp(s_j)   over the sequence's rows j.
//
// Bound by memory: every key and value is read once, for all the query heads that share it, and a token has few of those.  The
// rows of all sequences, one after the other, are cut into even shares for the workgroups, one for each CU; a workgroup takes one key
// head (and at most 16 of its query heads), and k_page_merge puts the states of a sequence's parts together.  Pages that several
// sequences share (forks of one history) are read once for as many of them as the 16 columns of a product hold.
// 64 histories of 501 to 14,928 rows (2.03 GB; 32 query heads over 8 key heads of 128 channels, bf16, as everywhere below where nothing
// else is said): 336 us, 6.0 TB/s, which is what a plain read reaches; one of 100,003 rows 76 us, 5.4 TB/s, 16 of 301 to 7,936 55 us, 4.9
// TB/s, of which 5 us are the merge and 3 the way to the first keys (arguments, length, list).
//
// The waves of a workgroup take tiles of 32 rows in turn, each on its own until the end.  Nothing goes through LDS on the way:
//   S = K Q^T   16x16x32 MFMA, A = 16 rows x 32 channels of keys as loaded (16 bytes of a row per lane), B = the queries; lane l
//   then has the scores of query l % 16 and rows 4 (l / 16) .. + 3 of each half of the tile;
//   O^T += V^T P^T   these registers, rounded to bf16, are the B operand as they stand; of the values a lane loads a piece of
//   channels of the same eight rows (16 lanes take a whole row), and turned over in registers the pieces are the A operand, row
//   r of product c being channel (D / 16) r + c.
// With fewer than 16 query heads the other columns are idle; the products take a small part of the loads' time all the same.

#include <algorithm>
#include <cstring>
#include <numeric>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace fsx {

constexpr int PA_KEYS = 32;     // rows that a wave takes at a time
// Steps that a stretch's start and end are worth, where a workgroup takes one after the other: as part of its length, in even shares (64
// sequences of 1 to 7,300 rows, as many of one length as of twice that, 24 heads over 8: 58.8 us without and 50.6 with it; 2 and 4: 55.0
// and 52.9, 10: 50.0).
constexpr int PA_START = 8;
constexpr int PA_SHARED = 128;  // shared rows that are worth a tile

// Columns of a workgroup: 16, or 32 for groups of more query heads, which would read the keys twice (16 histories of 900 rows, 8
// key heads, 160 query heads: 17.7 us instead of 22.2; a single key head and 20 query heads, little enough to be read twice: 12.4 and
// 11.5).
__host__ __device__ constexpr int columns(int G) { return G > 16 ? 32 : 16; }

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

template <int D, bool FP8, int WAVES, int CT>
__global__ __launch_bounds__(64 * WAVES, WAVES == 8 || CT == 1 ? 2 : 1) void k_page_attention(PageAttentionArgs a) {
  constexpr int KS = D / 32, NC = D / 16, ES = FP8 ? 1 : 2;  // steps of the first product, products of the second
  constexpr int STEP = WAVES * PA_KEYS, W = 16 * CT;  // rows at a time; columns
  using Tile = PageTile<D, FP8>;
  // Lists and lengths.  Nothing writes them while this runs: said so (constant memory), they are read by scalar loads.  As vector
  // loads they came behind the values under way, and every tile waited for both.
  typedef const __attribute__((address_space(4))) int32_t* list_t;
  __shared__ float xo[WAVES][W][D + 4];
  __shared__ float xm[WAVES][W], xl[WAVES][W];
  const PagePool& p = a.pool;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
  const int blocks = (a.G + W - 1) / W;
  // Stretch by stretch, the longest first, where each is a workgroup; otherwise head by head (us, the other way round: 64 of 17 to 1,466
  // fp8 rows behind 2,051 shared ones, 32 heads over 32, 100 instead of 82; 64 of 501 to 14,928 and 16 of 301 to 7,936 rows no different).
  const int hq = a.each ? blockIdx.x : blockIdx.y, index = a.each ? blockIdx.y : blockIdx.x;
  const int hk = hq / blocks, qb = hq - hk * blocks, h0 = hk * a.G + W * qb, rows = min(a.G, W);
  const list_t lens = (list_t)p.len;

  // The arguments are cold in every launch, a microsecond away: what may be needed of them comes in one round trip, a value per
  // lane, and is looked up by lane.
  struct Column {
    int lo, hi;
    __device__ __forceinline__ int before(int i) const {  // how many are at most i
      return __popcll(__ballot(lo <= i)) + __popcll(__ballot(hi <= i));
    }
    __device__ __forceinline__ int at(int i) const {
      return i < 64 ? __builtin_amdgcn_readlane(lo, i) : __builtin_amdgcn_readlane(hi, i - 64);
    }
    __device__ __forceinline__ int start(int i, int first) const { return i == 0 ? first : at(i - 1); }
  };
  const auto column = [&](const auto& v, int index, int n) {
    const int x = v[index], y = v[64 + index];
    return Column{lane < n ? x : INT32_MAX, 64 + lane < n ? y : INT32_MAX};
  };
  const char* kbase = (const char*)p.k;
  const char* vbase = (const char*)p.v;
  const int64_t layer_row = ((int64_t)a.layer * p.pages * p.Hk + hk) * p.P;
  const uint32_t lane_k = c16 * D * ES + 16 * g, lane_v = 4 * g * D * ES + c16 * (D / 16) * ES, lane_s = 4 * g;
  const auto load_k = [&](Tile& t, const int64_t (&row)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* src = kbase + row[h] * (D * ES) + lane_k;
#pragma unroll
      for (int i = 0; i < Tile::KP; ++i) t.k[h][i] = *reinterpret_cast<const uint4*>(src + 64 * i);
      if constexpr (FP8) t.ks[h] = *reinterpret_cast<const float4*>(p.k_scale + row[h] + lane_s);
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
      if constexpr (FP8) t.vs[h] = *reinterpret_cast<const float4*>(p.v_scale + row[h] + lane_s);
    }
  };

  int at = a.each ? 0 : index * a.per, until = a.each ? 1 : min(at + a.per, a.total);  // the workgroup's steps
  while (at < until) {
    // The stretch: of the rows of entry e from base on, or of those that a tile's members e .. e + members - 1 share.
    int e, from, to, base, seq0, members = 1;
    bool shared;
    {
      int here = lane;
      asm volatile("" : "+v"(here));  // (looked up again for the next stretch: kept, they are a dozen registers)
      const Column steps = column(a.steps, here + 1, a.n), parts = column(a.parts, here + 1, a.n);
      const Column seqs = column(a.seq, here, a.n), bases = column(a.base, here, a.n);
      Column tile_steps{INT32_MAX, INT32_MAX}, tile_parts = tile_steps, tile = tile_steps;
      if (a.n_tiles) {
        const int x = a.tile_steps[here + 1], y = a.tile_parts[here + 1];
        tile.lo = a.tile[here] | a.members[here] << 8;
        if (lane < a.n_tiles) tile_steps.lo = x, tile_parts.lo = y;
      }
      const int i = a.each ? index : at;
      shared = i < (a.each ? a.tiled_parts : a.tiled);
      int before;  // stretches before, of all
      if (shared) {
        const int t = (a.each ? tile_parts : tile_steps).before(i), x = tile.at(t);
        e = x & 255, members = x >> 8, from = tile_steps.start(t, 0), to = tile_steps.at(t), before = tile_parts.start(t, 0);
      } else {
        e = (a.each ? parts : steps).before(i);
        from = steps.start(e, a.tiled), to = steps.at(e), before = parts.start(e, a.tiled_parts);
      }
      if (a.each) {
        at = from + (i - before) * a.per;
        until = min(to, at + a.per);
      }
      base = bases.at(e), seq0 = seqs.at(e);
    }
    const int cut = min(to, until), part = a.each ? (at - from) / a.per : at / a.per - from / a.per;
    const int width = shared ? a.G : min(W, a.G - W * qb);  // columns of an entry
    // The thread's column of the outcome (of the first 16; more are one entry's): an entry, and where its state goes.
    const int ch = NC * (threadIdx.x & 15), en = e + min((int)(threadIdx.x >> 4) / width, members - 1);
    const int n_parts = a.all[en + 1] - a.all[en], out_row = a.row[en];
    const int slot = a.all[en] + part + (shared ? a.parts[en + 1] - a.parts[en] : 0);  // parts of its own rows, then of the shared
    // The lane's columns: queries of the channels that its keys have in step s.  Fp32 queries are rounded to bf16 (by 2^-8 of
    // each at most), as the attention over whole prompts rounds them: a token's scores are the same in both, and no key has more bits.
    uint4 q[CT][KS];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int col = 16 * ct + c16;
      const int64_t at_q = a.row[e + min(col / width, members - 1)] * a.q_row + (int64_t)(h0 + col % width) * a.q_head;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int c = FP8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
        if (a.q_f32) {
          const float4* f = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + at_q + c);
          const float4 u = f[0], v = f[1];
          q[ct][s] = make_uint4(pack_bf16x2(u.x, u.y), pack_bf16x2(u.z, u.w), pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
        } else {
          q[ct][s] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.q) + at_q + c);
        }
      }
    }
    // The pages of the first tile as planned come along with the length (entries of a list are pages that exist, also behind its end).
    list_t pages = (list_t)(p.table + (int64_t)seq0 * p.most);
    const int first_key = (shared ? 0 : base) + (at - from + w) * PA_KEYS;
    const int guess0 = min(first_key >> p.shift, p.most - 1), guess1 = min((first_key + 16) >> p.shift, p.most - 1);
    const int page0 = pages[guess0], page1 = pages[guess1], len0 = lens[seq0];
    // Its steps as planned, its start among them, are at - from .. cut - from of to - from; of the rows that are found (in a captured
    // graph not those that were planned) it takes the same share.
    const int total = shared ? base : max(len0 - base, 0), found = (total + PA_KEYS - 1) / PA_KEYS;
    const auto share = [&](int step) {
      return step == 0 || found == to - from ? step : (step == to - from ? found : (int)((int64_t)step * found / (to - from)));
    };
    const int begin = (shared ? 0 : base) + share(at - from) * PA_KEYS;
    const int stop = min(begin + (share(cut - from) - share(at - from)) * PA_KEYS, (shared ? 0 : base) + total);

    // Whether the members of the tile still share these pages (since a graph was captured, their lists may have changed); if not,
    // each takes a round of its own.
    int rounds = 1;
    if (shared) {
      const int first = begin >> p.shift, count = stop > begin ? ((stop - 1) >> p.shift) - first + 1 : 0;
      bool same = true;
      for (int i = threadIdx.x; i < count * members; i += 64 * WAVES) {
        const int j = i / members, s = a.seq[e + i - j * members];
        same &= p.len[s] >= base && p.table[(int64_t)s * p.most + first + j] == p.table[(int64_t)seq0 * p.most + first + j];
      }
      rounds = __builtin_amdgcn_readfirstlane(__syncthreads_and(same) ? 1 : members);
    }

    for (int round = 0; round < rounds; ++round) {
      const int seq = round ? a.seq[e + round] : seq0, len = round ? lens[seq] : len0, end = min(stop, len);
      if (round) pages = (list_t)(p.table + (int64_t)seq * p.most);
      const int last_page = max(len - 1, 0) >> p.shift;
      // First element row of the page row that tile row `key` is (past the end: some row that exists).
      const auto row_in = [&](int page, int key) { return layer_row + (int64_t)page * (p.Hk * p.P) + (key & (p.P - 1)); };
      const auto row_of = [&](int key) { return row_in(pages[min(key >> p.shift, last_page)], key); };
      f32x4 o[CT][NC];
      float m[CT], l[CT];  // maximum (log2 units), the same in the four lanes of a query; the lane's share of the sum
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        m[ct] = -INFINITY, l[ct] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[ct][c] = f32x4{0.f, 0.f, 0.f, 0.f};
      }

      Tile t;
      int key = begin + w * PA_KEYS;
      int64_t next[2];  // rows of the tile after, looked up a tile ahead of its loads
      // A tile: while it is computed, the next one's keys are loaded in place of its keys and, behind it, values in place of its values.
      // The last is another copy of the code: loads under a condition would be waited for as if they had been left out.
      const auto compute = [&](auto more) {
        constexpr bool MORE = decltype(more)::value;
        // scores
        f32x4 s[CT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) s[ct][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            uint4 ka;
            if constexpr (FP8) {
              const uint4 u = t.k[h][i / 2];
              const uint32_t lo = i % 2 ? u.z : u.x, hi = i % 2 ? u.w : u.y;
              ka = make_uint4(e4m3x2_to_bf16x2(lo, false), e4m3x2_to_bf16x2(lo, true), e4m3x2_to_bf16x2(hi, false),
                              e4m3x2_to_bf16x2(hi, true));
            } else {
              ka = t.k[h][i];
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) s[ct][h] = mfma_bf16(ka, q[ct][i], s[ct][h]);
          }
        }
        float sc[CT][8];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            sc[ct][i] = s[ct][i / 4][i % 4] * a.c;
            if constexpr (FP8) sc[ct][i] *= reinterpret_cast<const float*>(&t.ks[i / 4])[i % 4];
          }
        if constexpr (MORE) load_k(t, next);
        const int left = MORE ? PA_KEYS : end - key;  // rows of the tile that count: all of them, but for the last of the wave's
        uint4 pb[CT], pl[CT];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          if (left < PA_KEYS) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (16 * (i / 4) + 4 * g + i % 4 >= left) sc[ct][i] = -INFINITY;
          }
          // The maximum that the exponents are taken from is raised only where they would pass 2^8, which sums in fp32 and relative
          // roundings do not mind; then it is the same in the lanes of a query.
          const float(&x)[8] = sc[ct];
          float top = vmax3(vmax3(x[0], x[1], x[2]), vmax3(x[3], x[4], x[5]), vmax(x[6], x[7]));
          if (__any(top > m[ct] + 8.f)) {
            const float now = rows_max(vmax(top, m[ct])), back = __builtin_amdgcn_exp2f(m[ct] - (now == -INFINITY ? 0.f : now));
            m[ct] = now;
            l[ct] *= back;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[ct][c][i] *= back;
          }
          const float mz = m[ct] == -INFINITY ? 0.f : m[ct];
          float pr[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            pr[i] = __builtin_amdgcn_exp2f(x[i] - mz);
            l[ct] += pr[i];
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
          // The weights as two bf16 values: their upper halves, and what those leave out, rounded (2^-15 of a weight is lost; a second
          // product costs nothing next to the loads).  The second one is kept above zero where the weight is, by 2^-24 of it: an
          // infinite value times zero, or a negative rest, would be NaN.  Of weights below 2^-109 that is no bf16 value any more: the
          // rest is then the least there is, 2^-133.  (Fp8 values are finite or NaN.)
          const auto upper = [&](int i) {
            return __builtin_amdgcn_perm(__float_as_uint(pr[i + 1]), __float_as_uint(pr[i]), 0x07060302u);
          };
          const auto rest = [&](int i) {
            const auto left_out = [](float w) {
              const float x = fmaf(w, 0x1p-24f, w - __uint_as_float(__float_as_uint(w) & 0xFFFF0000u));
              if constexpr (FP8) return x;
              else return vmax(x, fminf(w, 0x1p-133f));
            };
            return pack_bf16x2(left_out(pr[i]), left_out(pr[i + 1]));
          };
          pb[ct] = make_uint4(upper(0), upper(2), upper(4), upper(6));
          pl[ct] = make_uint4(rest(0), rest(2), rest(4), rest(6));
        }
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
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            o[ct][c] = mfma_bf16(make_uint4(r[0], r[1], r[2], r[3]), pb[ct], o[ct][c]);
            o[ct][c] = mfma_bf16(make_uint4(r[0], r[1], r[2], r[3]), pl[ct], o[ct][c]);
          }
        }
        if constexpr (MORE) {
          load_v(t, next);
          __builtin_amdgcn_sched_barrier(0);  // (not to be one with the first tile's loads, at the head of the loop)
        }
      };
      if (key < end) {
        const bool planned = round == 0 && key == first_key && ((key + 16) >> p.shift) <= last_page;
        next[0] = planned ? row_in(page0, key) : row_of(key);
        next[1] = planned ? row_in(page1, key + 16) : row_of(key + 16);
        load_k(t, next);
        load_v(t, next);
        next[0] = row_of(key + STEP), next[1] = row_of(key + STEP + 16);
        if (key + STEP < end) {
          do {
            compute(std::true_type{});
            key += STEP;
            next[0] = row_of(key + STEP), next[1] = row_of(key + STEP + 16);
          } while (key + STEP < end);
        }
        compute(std::false_type{});
      }

      // The waves' states put together.  Lane: query c16 of a column tile, o[c][i]: channel (D / 16) (4 g + i) + c.
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const float sum = rows_sum(l[ct]);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) xo[w][16 * ct + c16][NC * (4 * g + i) + c] = o[ct][c][i];
        if (g == 0) {
          xm[w][16 * ct + c16] = m[ct];
          xl[w][16 * ct + c16] = sum;
        }
      }
      __syncthreads();
      // thread: column t / 16 of a column tile, channels D / 16 (t % 16) ..
      for (int qi = threadIdx.x >> 4; qi < min(W, width * members); qi += 4 * WAVES) {
        const int member = qi / width, gi = qi - member * width;
        if (rounds > 1 && member != round) continue;
        float mm = xm[0][qi], f[WAVES], ll = 0.f;
#pragma unroll
        for (int i = 1; i < WAVES; ++i) mm = vmax(mm, xm[i][qi]);
        const float mz = mm == -INFINITY ? 0.f : mm;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
          f[i] = __builtin_amdgcn_exp2f(xm[i][qi] - mz);
          ll += xl[i][qi] * f[i];
        }
        float r[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          r[c] = 0.f;
#pragma unroll
          for (int i = 0; i < WAVES; ++i) r[c] += xo[i][qi][ch + c] * f[i];
        }
        if (n_parts > 1) {
          float* state = a.part + ((int64_t)slot * (p.Hk * blocks) + hq) * part_floats(rows, D);
#pragma unroll
          for (int c = 0; c < NC; c += 4)
            *reinterpret_cast<float4*>(state + gi * D + ch + c) = make_float4(r[c], r[c + 1], r[c + 2], r[c + 3]);
          if ((threadIdx.x & 15) == 0) {
            state[rows * D + gi] = mm;
            state[rows * (D + 1) + gi] = ll;
          }
        } else {
          const float inv = len > 0 ? 1.f / ll : 0.f;
          const int64_t to_out = out_row * a.o_row + (int64_t)(h0 + gi) * a.o_head + ch;
#pragma unroll
          for (int c = 0; c < NC; c += 4) {
            if (a.o_f32) {
              *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + to_out + c) =
                  make_float4(r[c] * inv, r[c + 1] * inv, r[c + 2] * inv, r[c + 3] * inv);
            } else {
              *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + to_out + c) =
                  make_uint2(pack_bf16x2(r[c] * inv, r[c + 1] * inv), pack_bf16x2(r[c + 2] * inv, r[c + 3] * inv));
            }
          }
          if (a.lse && (threadIdx.x & 15) == 0)
            a.lse[(int64_t)out_row * a.H + h0 + gi] = (mm + __builtin_amdgcn_logf(ll)) * (1.f / LOG2E);
        }
      }
      if (round + 1 < rounds || cut < until) __syncthreads();  // the exchange is free again
    }
    at = cut;
  }
}

// The parts of one (entry, query head) put together: groups of D / 4 threads take every GROUPS-th part each, then the first the groups'
// states.  What counts is the round trips to other XCDs' memory, so where a sequence has many parts there are four times the groups
// (five sequences, the longest of 36,830 rows in 288 parts, 4 heads over 1: 15.9 us in all instead of 19.1).
template <int D, int THREADS>
__global__ __launch_bounds__(THREADS) void k_page_merge(PageAttentionArgs a) {
  constexpr int T = D / 4, GROUPS = THREADS / T, AT_ONCE = 4;
  __shared__ float4 xo[GROUPS][T];
  __shared__ float xl[GROUPS], xm[GROUPS];
  const int e = blockIdx.x, h = blockIdx.y, hk = h / a.G, gi = h - hk * a.G;
  const int W = columns(a.G), blocks = (a.G + W - 1) / W, rows = min(a.G, W);
  const int n = a.all[e + 1] - a.all[e];
  if (n <= 1) return;  // written already
  const int grp = threadIdx.x / T, t = threadIdx.x % T;
  const int64_t step = (int64_t)blocks * (a.H / a.G) * part_floats(rows, D);
  const float* part = a.part + a.all[e] * step + (hk * blocks + gi / W) * part_floats(rows, D);
  const int qi = gi % W;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto raise = [&](float to) {  // the maximum; what the exponents are taken from
    const float z = to == -INFINITY ? 0.f : to, f = __builtin_amdgcn_exp2f(m - z);
    m = to;
    l *= f;
    o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
    return z;
  };
  const auto add = [&](float mc, float lc, float4 v, float z) {
    const float f = __builtin_amdgcn_exp2f(mc - z);
    l += lc * f;
    o = make_float4(o.x + v.x * f, o.y + v.y * f, o.z + v.z * f, o.w + v.w * f);
  };
  for (int x0 = grp; x0 < n; x0 += AT_ONCE * GROUPS) {
    float mc[AT_ONCE], lc[AT_ONCE], now = m;
    float4 v[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const float* s = part + min(x0 + u * GROUPS, n - 1) * step;
      v[u] = reinterpret_cast<const float4*>(s + qi * D)[t];
      mc[u] = s[rows * D + qi];
      lc[u] = s[rows * (D + 1) + qi];
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
      if (x0 + u * GROUPS < n) now = fmaxf(now, mc[u]);
    const float z = raise(now);
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
      if (x0 + u * GROUPS < n) add(mc[u], lc[u], v[u], z);
  }
  xo[grp][t] = o;
  if (t == 0) {
    xm[grp] = m;
    xl[grp] = l;
  }
  __syncthreads();
  if (grp) return;
  float now = m;
#pragma unroll 8
  for (int i = 1; i < GROUPS; ++i) now = fmaxf(now, xm[i]);
  const float z = raise(now);
#pragma unroll 8
  for (int i = 1; i < GROUPS; ++i) add(xm[i], xl[i], xo[i][t], z);
  const float inv = a.pool.len[a.seq[e]] > 0 ? 1.f / l : 0.f;
  const int64_t row = a.row[e], at = row * a.o_row + (int64_t)h * a.o_head + 4 * t;
  const float4 r = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  if (a.o_f32) *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = r;
  else *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + at) = make_uint2(pack_bf16x2(r.x, r.y), pack_bf16x2(r.z, r.w));
  if (a.lse && t == 0) a.lse[row * a.H + h] = (m + __builtin_amdgcn_logf(l)) * (1.f / LOG2E);
}

// Sequences that share whole pages from their first on, as groups of neighbours, where several of them fit a tile's columns.
static void share_pages(const PageLists& lists, const int32_t* seqs, int per_tile, PagePlan& plan) {
  std::vector<PagePlan::Entry>& es = plan.entries;
  const auto list = [&](const PagePlan::Entry& x) { return &lists.table[(size_t)seqs[x.index] * lists.most]; };
  const auto whole = [&](const PagePlan::Entry& x) { return lists.len[seqs[x.index]] / lists.P; };
  // (a sequence named twice shares with itself)
  const auto key = [&](const PagePlan::Entry& x) { return whole(x) > 0 ? list(x)[0] : -1; };
  std::stable_sort(es.begin(), es.end(), [&](const auto& x, const auto& y) { return key(x) < key(y); });
  const auto longer = [&](const PagePlan::Entry& x, const PagePlan::Entry& y) { return lists.len[seqs[x.index]] > lists.len[seqs[y.index]]; };
  for (size_t i = 0, e; i < es.size(); i = e) {
    for (e = i + 1; e < es.size() && key(es[e]) == key(es[i]);) ++e;
    if (key(es[i]) < 0) continue;
    while (e - i > 1) {
      // pages that each has in common with the first; the group, the most in common first, that saves the most reading
      for (size_t j = i; j < e; ++j) {
        const int most = std::min(whole(es[i]), whole(es[j]));
        const int32_t *u = list(es[i]), *v = list(es[j]);
        int n = u == v ? most : 0;
        while (n + 64 <= most && !memcmp(u + n, v + n, 64 * sizeof(int32_t))) n += 64;
        while (n < most && u[n] == v[n]) ++n;
        es[j].base = n;
      }
      std::stable_sort(es.begin() + i, es.begin() + e, [](const auto& x, const auto& y) { return x.base > y.base; });
      size_t k = 2;
      for (size_t j = 3; j <= e - i; ++j)
        if ((int64_t)es[i + j - 1].base * (j - 1) > (int64_t)es[i + k - 1].base * (k - 1)) k = j;
      const int rows = es[i + k - 1].base * lists.P;
      const size_t in = rows < PA_SHARED ? 0 : (k % per_tile == 1 ? k - 1 : k);  // (a tile of one saves nothing)
      for (size_t j = 0; j < k; ++j) es[i + j].base = j < in ? rows : 0;
      std::stable_sort(es.begin() + i, es.begin() + i + in, longer);
      for (size_t j = 0; j < in; j += per_tile) plan.tiles.push_back({(int32_t)(i + j), (int32_t)std::min<size_t>(per_tile, in - j)});
      i += k;
    }
    for (; i < e; ++i) es[i].base = 0;
  }
}

void plan_page_attention(const PagePool& p, const PageLists& lists, int H, int n, const int32_t* seqs, int64_t workspace_bytes,
                         PagePlan& plan) {
  constexpr int64_t CUS = 256;
  const int G = H / p.Hk, W = columns(G), units = p.Hk * ((G + W - 1) / W);
  const int64_t state = 4 * units * part_floats(std::min(G, W), p.D);  // bytes of a part, all heads
  plan.entries.resize(n);
  bool shared = false;
  int longest = 0;
  for (int i = 0; i < n; ++i) {
    const int32_t s = seqs[i], len = lists.len[s];
    plan.entries[i] = {i, 0, 0, 1, 0};
    shared |= len >= lists.P && lists.ref[lists.table[(size_t)s * lists.most]] > 1;
    longest = std::max(longest, len);
  }
  if (shared && G <= 8 && n > 1) share_pages(lists, seqs, 16 / G, plan);
  // Short sequences that do not fill the chip: no parts, in workgroups of eight waves, and one launch.  us with and without, 32 heads
  // over 8: one sequence of 300 rows 8.5 and 10.6, of 1,000 14.3 and 10.4, 16 of 500 10.9 and 13.5, of 1,000 16.2 and 17.9; 64 of
  // 1,000 53 and 49, 200 of 600 107 and 95.
  const int64_t all = (int64_t)n * units;
  plan.wide = plan.tiles.empty() && all < 2 * CUS && longest <= (4 * all >= CUS ? 1024 : 512);
  const auto steps = [](int64_t rows) { return (int)((rows + PA_KEYS - 1) / PA_KEYS); };
  for (auto& x : plan.entries) x.steps = std::max(1, steps(lists.len[seqs[x.index]] - x.base));
  // The launches, the members of a tile together.
  for (int i = 0, tile = 0; i < n;) {
    int m = std::min(PAGE_QUERIES, n - i), end = tile;
    const int tiles = (int)plan.tiles.size();
    while (end < tiles && plan.tiles[end].first + plan.tiles[end].members <= i + m) ++end;
    if (end < tiles && plan.tiles[end].first < i + m) m = plan.tiles[end].first - i;
    plan.launches.push_back({i, m, tile, end - tile, 1, 1, 0, m, 0});
    i += m;
    tile = end;
  }
  const auto whole = [&] {  // a workgroup for each entry and key head
    plan.bytes = 0;
    for (auto& x : plan.entries) x.own = 1, x.shared = 0;
    for (auto& l : plan.launches) l.per = 1 << 30, l.each = 1, l.extra = 0, l.workgroups = l.n, l.parts = 0;
  };
  if (plan.wide) return whole();
  // As many steps for every workgroup, at least four (one for each wave), so that all of them run at once and end together; a
  // workgroup's steps may begin in one sequence and end in another.  Where those stretches are many and short, their starts and ends
  // weigh more than an even share: then each is a workgroup of its own.  us, the one and the other: 64 histories of 501 to 14,928 rows
  // (32 heads over 8) 338 and 374, 16 of 301 to 7,936 55 and 71; 64 of 17 to 1,466 fp8 rows behind 2,051 shared ones (32 over 32) 109
  // and 82, one of 60,000 and 63 of 10 (32 over 32) 187 and 171.  So too where a share is short, with two workgroups for each CU if there
  // are several sequences: 16 of 301 to 1,051 (32 over 8) 15.3 instead of 17.3, 16 of 1,500 fp8 rows 16.3 instead of 19.1, five of 300
  // to 5,000 15.2 instead of 17.2.  Otherwise more workgroups than CUs cost: 16 of 301 to 7,936 58 instead of 55, one of 100,003 79
  // instead of 76.
  const auto cut = [&](int64_t workgroups, bool apart) {
    int64_t most = 0;
    for (auto& l : plan.launches) {
      int64_t total = 0, stretches = l.n_tiles + l.n;
      for (int t = 0; t < l.n_tiles; ++t) total += steps(plan.entries[plan.tiles[l.first_tile + t].first].base);
      for (int j = 0; j < l.n; ++j) total += plan.entries[l.first + j].steps;
      const bool few = total < 48 * workgroups;
      l.each = apart || few || (stretches > 3 * workgroups && total < (p.fp8 ? 128 : 64) * stretches);
      l.extra = l.each ? 0 : PA_START;
      total += stretches * l.extra;
      const int64_t share = few && l.n > 1 ? 2 * workgroups : workgroups;
      l.per = (int)std::max<int64_t>(4, (total + share - 1) / share);
      l.workgroups = (int)((total + l.per - 1) / l.per);
      const auto parts = [&](int64_t at, int64_t count) {
        return (int)(l.each ? (count + l.per - 1) / l.per : (at + count - 1) / l.per - at / l.per + 1);
      };
      int64_t at = 0;
      stretches = l.parts = 0;
      for (int t = 0; t < l.n_tiles; ++t) {
        const auto& x = plan.tiles[l.first_tile + t];
        const int count = steps(plan.entries[x.first].base) + l.extra, m = parts(at, count);
        for (int j = 0; j < x.members; ++j) plan.entries[x.first + j].shared = m;
        stretches += m;
        at += count;
      }
      for (int j = 0; j < l.n; ++j) {
        auto& x = plan.entries[l.first + j];
        x.own = parts(at, x.steps + l.extra);
        stretches += x.own;
        l.parts += x.states();
        at += x.steps + l.extra;
      }
      if (l.each) l.workgroups = (int)stretches;
      most += l.parts;
    }
    plan.bytes = most * state;
  };
  const int64_t full = std::max<int64_t>(1, CUS / units);
  // With less workspace than that, even shares of up to a quarter fewer workgroups, then longer parts, but none of several sequences: at
  // the least a workgroup for each.  us (32 heads over 8 of 128 channels, bf16) with nine tenths of the workspace, and where parts come
  // apart at once, in half the workgroups: 64 of 501 to 14,928 rows 337 and 374, 16 of 301 to 7,936 56 and 63, one of 100,003 76 and 87.
  const auto fits = [&](int64_t workgroups, bool apart) {
    cut(workgroups, apart);
    return plan.bytes <= workspace_bytes;
  };
  bool done = fits(full, false);
  if (!done && workspace_bytes >= 2 * state) {  // (what is split has two parts at least)
    for (int64_t w = full - 1; !done && 4 * w >= 3 * full; w -= std::max<int64_t>(1, full / 16)) done = fits(w, false);
    // fewer by as many as there are parts too many, were all of them the workgroups': never too few, so again until it fits
    for (int64_t w = std::max<int64_t>(1, 3 * full / 4); !done && w >= 1;) {
      done = fits(w, true);
      if (!done) w = std::min(w - 1, (int64_t)((double)w * workspace_bytes / plan.bytes));
    }
  }
  if (!done) {
    plan.tiles.clear();
    for (auto& x : plan.entries) x.base = 0;
    for (auto& l : plan.launches) l.first_tile = l.n_tiles = 0;
    for (auto& x : plan.entries) x.steps = std::max(1, steps(lists.len[seqs[x.index]]));
    whole();
  }
  for (const auto& l : plan.launches)
    if (l.each && !l.n_tiles)
      std::stable_sort(plan.entries.begin() + l.first, plan.entries.begin() + l.first + l.n,
                       [](const auto& x, const auto& y) { return x.steps > y.steps; });
}

hipError_t launch_page_attention(PageAttentionArgs a, const int32_t* seqs, const PagePlan& plan, hipStream_t s) {
  const PagePool& p = a.pool;
  const int W = columns(a.G), blocks = (a.G + W - 1) / W, rows = std::min(a.G, W);
  for (const auto& l : plan.launches) {
    a.n = l.n;
    a.n_tiles = l.n_tiles;
    a.per = l.per;
    a.each = l.each;
    a.all[0] = a.tile_steps[0] = a.tile_parts[0] = 0;
    for (int t = 0; t < l.n_tiles; ++t) {
      const PagePlan::Tile& x = plan.tiles[l.first_tile + t];
      a.tile[t] = (uint8_t)(x.first - l.first);
      a.members[t] = (uint8_t)x.members;
      a.tile_steps[t + 1] = a.tile_steps[t] + (plan.entries[x.first].base + PA_KEYS - 1) / PA_KEYS + l.extra;
      a.tile_parts[t + 1] = a.tile_parts[t] + plan.entries[x.first].shared;
    }
    a.steps[0] = a.tiled = a.tile_steps[l.n_tiles];
    a.parts[0] = a.tiled_parts = a.tile_parts[l.n_tiles];
    int most = 0;  // parts of an entry
    for (int j = 0; j < l.n; ++j) {
      const PagePlan::Entry& x = plan.entries[l.first + j];
      a.seq[j] = seqs[x.index];
      a.row[j] = (uint16_t)x.index;
      a.base[j] = x.base;
      a.steps[j + 1] = a.steps[j] + x.steps + l.extra;
      a.parts[j + 1] = a.parts[j] + x.own;
      a.all[j + 1] = a.all[j] + x.states();
      most = std::max(most, x.own + x.shared);
    }
    a.total = a.steps[l.n];
    const dim3 grid(l.each ? p.Hk * blocks : l.workgroups, l.each ? l.workgroups : p.Hk * blocks), merge(l.n, a.H);
    const auto launch = [&](auto ct) {
      constexpr int CT = decltype(ct)::value;
      if (plan.wide) {
        const auto fn = p.D == 64 ? (p.fp8 ? k_page_attention<64, true, 8, CT> : k_page_attention<64, false, 8, CT>)
                                  : (p.fp8 ? k_page_attention<128, true, 8, CT> : k_page_attention<128, false, 8, CT>);
        return enqueue(fn, grid, dim3(512), s, a);
      } else {
        const auto fn = p.D == 64 ? (p.fp8 ? k_page_attention<64, true, 4, CT> : k_page_attention<64, false, 4, CT>)
                                  : (p.fp8 ? k_page_attention<128, true, 4, CT> : k_page_attention<128, false, 4, CT>);
        return enqueue(fn, grid, dim3(256), s, a);
      }
    };
    hipError_t e = W == 32 ? launch(std::integral_constant<int, 2>{}) : launch(std::integral_constant<int, 1>{});
    if (e == hipSuccess && l.parts) {
      const auto fn = p.D == 64 ? (most > 32 ? k_page_merge<64, 1024> : k_page_merge<64, 256>)
                                : (most > 32 ? k_page_merge<128, 1024> : k_page_merge<128, 256>);
      e = enqueue(fn, merge, dim3(most > 32 ? 1024 : 256), s, a);
    }
    if (e != hipSuccess) return e;
    a.part += (int64_t)l.parts * p.Hk * blocks * part_floats(rows, p.D);
  }
  return hipSuccess;
}

}  // namespace fsx
