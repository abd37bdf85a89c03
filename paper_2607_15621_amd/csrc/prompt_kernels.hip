// Attention over whole prompts (Sec. 3.3: a cache rebuilt from scratch): packed sequences of different lengths, causal, with
// grouped heads.
//
// Query t of a sequence with nq new tokens over nk keys sees the keys j <= nk - nq + t; per head
//   O_t = sum_j exp(s_tj) v_j / sum_j exp(s_tj),   s_tj = scale q_t . k_j,   lse_t = log sum_j exp(s_tj).

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fsx {

// The rows of a (sequence, key head) are its tokens' query heads of that key head, token by token: row r is token r / G, head
// r % G of the group, so all query heads that share keys read them from one tile.
//
// A wave takes 32 rows and walks over the keys in tiles that direct loads bring into LDS ahead of it; the waves of a workgroup share
// them.  Everything is held transposed, a query per lane column:
//   S^T = K Q^T   32x32x16 MFMA, A = 32 keys x 16 channels from LDS, B = the wave's queries, kept in registers;
//   a lane then has 16 of 32 keys' scores of one query (lane l and l ^ 32 share query l % 32), so maximum and sum are lane
//   operations and one exchange of halves;
//   O^T += V^T P^T   the scores' registers, rounded to bf16, are the B operand as they stand (slots 0-3 of lane half g: keys
//   4g .. 4g + 3, slots 4-7: 8 + 4g ..); A = V^T in the same order of keys by transposing LDS reads.
constexpr int PT_KEYS = 64;

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ f32x16 mfma32_bf16(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Four values down a column: lane i of 16 gets column i of the 4 rows x 16 columns of 16 bits whose 8-byte pieces the lanes
// point at (row i / 4, columns 4 (i % 4) ..).
__device__ __forceinline__ uint2 lds_column4(const char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p)));
}

// Where 16-byte piece p of a tile's row lies: in row-piece p ^ k_turn (keys) or p ^ v_turn (values), so that the reads of a column
// of rows are spread over the banks.  With the pieces in order the reads of 32 rows took 16 times (values: twice) as long.  Reads
// of keys, and of values 64 channels wide, meet no bank twice; a read of values 128 wide takes four rows and four pieces at once,
// of which rows 0 and 1, and 2 and 3, share banks: four cycles instead of two (SQ_LDS_BANK_CONFLICT: 2 per such read).
template <int D>
__device__ __forceinline__ int k_turn(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D>
__device__ __forceinline__ int v_turn(int row) { return D == 128 ? 2 * (row & 7) : 2 * (row & 3); }

// The sequence of item i (items of sequence s being prefix[s] .. prefix[s + 1] - 1) and the item's place in it.  One sequence
// per lane: a round trip for all of it; loaded by sequence they were two or three more, a microsecond each, the arguments being
// cold in every launch (one row of 16 sequences, up to 8k keys: 64.6 -> 61.8 us; four of 64 over long histories 46.6 -> 44.4).
struct PromptSeq {
  int place, nq, nk, n_split, first_item;
  int64_t q0, k0;
  __device__ __forceinline__ PromptSeq(const PromptArgs& a, const int32_t* prefix, int i, int lane) {
    static_assert(FSX_MAX_BATCH == WAVE, "a sequence per lane");
    const int at = prefix[lane], end = prefix[lane + 1], items = a.item_prefix[lane], q = a.nq[lane], k = a.nk[lane], n = a.n_split[lane];
    const int64_t qs = a.q0[lane], ks = a.k0[lane];
    const int s = __popcll(__ballot(lane < a.n_seq && end <= i));
    auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, s); };
    auto pick64 = [&](int64_t v) { return (int64_t)((uint64_t)(uint32_t)pick((int)(v >> 32)) << 32 | (uint32_t)pick((int)v)); };
    place = i - pick(at);
    nq = pick(q);
    nk = pick(k);
    n_split = pick(n);
    first_item = pick(items);
    q0 = pick64(qs);
    k0 = pick64(ks);
  }
};

// max / sum with lane l ^ 32
__device__ __forceinline__ float half_max(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return vmax(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// 32 queries' running state: O^T block b, register i: channel 32 b + 8 (i / 4) + 4 (lane / 32) + i % 4 of query lane % 32;
// m: maximum in log2 units, l: the lane's share of the sum.
template <int D>
struct PromptState {
  f32x16 o[D / 32];
  float m, l;
};

// The wave's queries as the B operand: step s, lane l: channels 16 s + 8 (l / 32) .. + 7 of query l % 32.  Where they come in fp32
// they are rounded to bf16 (at most 2^-8 of each, as the keys that they meet were: fp32 matrix instructions run at a sixteenth of
// the rate).
template <int D>
__device__ __forceinline__ void load_queries(const PromptArgs& a, int64_t at, int half, uint4 (&qf)[D / 16]) {
  if (a.q_f32) {
    const float* q = (const float*)a.q + at + 8 * half;
    float4 x[D / 8];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) x[i] = *reinterpret_cast<const float4*>(q + 16 * (i / 2) + 4 * (i % 2));
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      qf[s] = make_uint4(pack_bf16x2(x[2 * s].x, x[2 * s].y), pack_bf16x2(x[2 * s].z, x[2 * s].w),
                         pack_bf16x2(x[2 * s + 1].x, x[2 * s + 1].y), pack_bf16x2(x[2 * s + 1].z, x[2 * s + 1].w));
  } else {
    const uint16_t* q = (const uint16_t*)a.q + at + 8 * half;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) qf[s] = *reinterpret_cast<const uint4*>(q + 16 * s);
  }
}

// Block b of the output row (query lane % 32), scaled by inv.
__device__ __forceinline__ void store_block(const PromptArgs& a, const f32x16& o, int b, int64_t at, bool valid, float inv, int half) {
#pragma unroll
  for (int g = 0; g < 4; g += 2) {  // channels 32 b + 8 g .. + 15
    if (a.o_f32) {
      if (valid)
#pragma unroll
        for (int e = g; e < g + 2; ++e)
          *reinterpret_cast<float4*>((float*)a.out + at + 32 * b + 8 * e + 4 * half) =
              make_float4(o[4 * e] * inv, o[4 * e + 1] * inv, o[4 * e + 2] * inv, o[4 * e + 3] * inv);
      continue;
    }
    uint32_t x[2][2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int w = 0; w < 2; ++w) x[e][w] = pack_bf16x2(o[4 * (g + e) + 2 * w] * inv, o[4 * (g + e) + 2 * w + 1] * inv);
    // eight channels in a row for each half after the exchange
    const auto r0 = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
    const auto r1 = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
    if (valid)
      *reinterpret_cast<uint4*>((uint16_t*)a.out + at + 32 * b + 8 * (g + half)) = make_uint4(r0[0], r1[0], r0[1], r1[1]);
  }
}

// The value is computed here: neither the products nor the vector work that make it may move to the other side of a barrier,
// which to the compiler concerns memory alone.
__device__ __forceinline__ void here(f32x16& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void here(uint4& x) {
  u32x4_t y = __builtin_bit_cast(u32x4_t, x);
  asm volatile("" : "+v"(y));
  x = __builtin_bit_cast(uint4, y);
}

// S^T of a tile of 32 KB keys, in LDS at kt.
template <int D, int KB>
__device__ __forceinline__ void tile_scores(const char* kt, const uint4 (&qf)[D / 16], int lane, f32x16 (&s)[KB]) {
  constexpr int KS = D / 16, AHEAD = 4;  // the reads run ahead of the products
  const int half = lane >> 5, row = lane & 31;
  uint4 kf[KB * KS];
  auto load_k = [&](int i) {
    const int b = i / KS, k = i % KS;
    kf[i] = *reinterpret_cast<const uint4*>(kt + (32 * b + row) * 2 * D + 16 * ((2 * k + half) ^ k_turn<D>(row)));
  };
#pragma unroll
  for (int b = 0; b < KB; ++b) s[b] = f32x16{};
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load_k(i);
#pragma unroll
  for (int i = 0; i < KB * KS; i += 2) {
    if (i + AHEAD < KB * KS) load_k(i + AHEAD);
    if (i + AHEAD + 1 < KB * KS) load_k(i + AHEAD + 1);
    __builtin_amdgcn_sched_barrier(0);
    s[i / KS] = mfma32_bf16(kf[i], qf[i % KS], s[i / KS]);
    s[(i + 1) / KS] = mfma32_bf16(kf[i + 1], qf[(i + 1) % KS], s[(i + 1) / KS]);
  }
}

// The tile's probabilities (B operand of the second product) from its scores, and the state's maximum and sum.  lim: the last
// key (counted from the tile's first) that the lane's query sees; masked: whether some query does not see all of them.  between(i)
// runs after the exponentials of the i-th 16-key step.
// The probabilities are rounded to bf16, at most 2^-8 of each, for a second product on the bf16 matrix instructions (fp32 ones run
// at a sixteenth of the rate); their sum is taken before the rounding, in fp32.
// The maximum that the exponents are taken from is raised only where they would pass 2^8 (sums in fp32 and relative roundings do not
// mind), so the exponentials need not wait for the tile's own maximum; a tile that raises it does them again.
template <int D, int KB, class Between>
__device__ __forceinline__ void tile_softmax(f32x16 (&s)[KB], float c, int lim, bool masked, int half, PromptState<D>& st, uint4 (&pf)[2 * KB],
                                             Between between) {
  if (masked) {
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 32 * b + 8 * (i / 4) + 4 * half + i % 4 <= lim ? s[b][i] : -INFINITY;
  }
  float ps[4];
  auto probabilities = [&](float mz, int k) {
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[k / 2][8 * (k % 2) + i], c, -mz));
#pragma unroll
    for (int i = 0; i < 4; ++i) ps[i] = k == 0 ? p[i] + p[i + 4] : ps[i] + (p[i] + p[i + 4]);
    pf[k] = make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
  };
  float mx[4];
#pragma unroll
  for (int k = 0; k < 2 * KB; ++k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = s[k / 2][8 * (k % 2) + 2 * i], y = s[k / 2][8 * (k % 2) + 2 * i + 1];
      mx[i] = k == 0 ? vmax(x, y) : vmax3(mx[i], x, y);
    }
    probabilities(st.m == -INFINITY ? 0.f : st.m, k);
    between(k);
  }
  const float top = half_max(vmax3(vmax(mx[0], mx[1]), mx[2], mx[3])) * c;
  if (__any(top > st.m + 8.f)) {
    const float mn = fmaxf(st.m, top), alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - mn);
    st.m = mn;
    st.l *= alpha;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[b][i] *= alpha;
#pragma unroll
    for (int k = 0; k < 2 * KB; ++k) probabilities(mn == -INFINITY ? 0.f : mn, k);
  }
  st.l += (ps[0] + ps[1]) + (ps[2] + ps[3]);
}

// O^T += V^T P^T of a tile, its values in LDS at vt.
template <int D, int KB>
__device__ __forceinline__ void tile_values(const char* vt, const uint4 (&pf)[2 * KB], int lane, PromptState<D>& st) {
  // V^T of 16 keys x 32 channels: group lane / 16 reads the 4 keys of its half, channels 16 ((lane / 16) % 2) ..
  const int vr = 4 * (lane >> 5) + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  uint4 vf[2 * KB][D / 32];
  auto load_v = [&](int k) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
      const int r0 = 16 * k + vr, r1 = r0 + 8;
      const uint2 lo = lds_column4(vt + r0 * 2 * D + 16 * ((4 * b + vc) ^ v_turn<D>(r0)) + 8 * (lane & 1));
      const uint2 hi = lds_column4(vt + r1 * 2 * D + 16 * ((4 * b + vc) ^ v_turn<D>(r1)) + 8 * (lane & 1));
      vf[k][b] = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  };
  load_v(0);
#pragma unroll
  for (int k = 0; k < 2 * KB; ++k) {
    if (k + 1 < 2 * KB) load_v(k + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < D / 32; ++b) st.o[b] = mfma32_bf16(vf[k][b], pf[k], st.o[b]);
  }
}

template <int D, int KB>
__device__ __forceinline__ void add_tile(const char* kt, const char* vt, const uint4 (&qf)[D / 16], float c, int lim, bool masked,
                                         int lane, PromptState<D>& st) {
  f32x16 s[KB];
  uint4 pf[2 * KB];
  // (the products first where another wave of the SIMD could take its vector work in between: 16 prompts of 1,024 tokens 213 us
  // without, 202 with)
  __builtin_amdgcn_s_setprio(1);
  tile_scores<D, KB>(kt, qf, lane, s);
  __builtin_amdgcn_s_setprio(0);
  tile_softmax<D, KB>(s, c, lim, masked, lane >> 5, st, pf, [](int) {});
  __builtin_amdgcn_s_setprio(1);
  tile_values<D, KB>(vt, pf, lane, st);
  __builtin_amdgcn_s_setprio(0);
}

// Values that are not finite, in keys that some of the queries do not see: a product with the weight 0 would make NaN of them.
// They are met only after an output turned out not finite; the tiles are then run again with such values set to zero, and
// first[kind][channel] is the first key with a NaN, +infinity or -infinity there, to be added to the queries that see it.
template <int D>
__device__ __forceinline__ void take_out_nonfinite(char* vt, int rows, int n_keys, int k0, int* first, int tid, int threads) {
  constexpr int RB = 2 * D;
  for (int i = tid; i < rows * (RB / 16); i += threads) {
    const int r = i / (RB / 16), ch = 8 * ((i % (RB / 16)) ^ v_turn<D>(r));
    uint16_t* p = reinterpret_cast<uint16_t*>(vt + 16 * i);
    for (int e = 0; e < 8; ++e) {
      const uint16_t x = p[e];
      if ((x & 0x7F80) != 0x7F80) continue;
      p[e] = 0;
      if (r < n_keys) atomicMin(first + (x & 0x7F ? 0 : 1 + (x >> 15)) * D + ch + e, k0 + r);
    }
  }
}
template <int D>
__device__ __forceinline__ void put_back_nonfinite(PromptState<D>& st, const int* first, int lim, int half) {
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int ch = 32 * b + 8 * (i / 4) + 4 * half + i % 4;
      const float bad[3] = {NAN, INFINITY, -INFINITY};
#pragma unroll
      for (int kind = 0; kind < 3; ++kind)
        if (first[kind * D + ch] <= lim) st.o[b][i] += bad[kind];
    }
}
template <int D>
__device__ __forceinline__ bool all_finite(const PromptState<D>& st) {
  float z = 0.f;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) z = fmaf(st.o[b][i], 0.f, z);
  return z == 0.f;
}
template <int D>
__device__ __forceinline__ void clear_state(PromptState<D>& st) {
#pragma unroll
  for (int b = 0; b < D / 32; ++b) st.o[b] = f32x16{};
  st.m = -INFINITY;
  st.l = 0.f;
}

// A wave's 32 rows r0 .. of (sequence s, key head hk), one per lane column; past the last row, that row again, not valid.
struct PromptRows {
  int64_t row;  // row of q, out and lse
  int h, lim;   // query head; last key seen
  bool valid;
  int first, last;  // least and largest last key of the wave's rows (none: INT32_MAX, -1)
  __device__ __forceinline__ PromptRows(const PromptArgs& a, const PromptSeq& s, int hk, int r0, int lane) {
    const int rows = s.nq * a.G, off = s.nk - s.nq, r = r0 + (lane & 31), rc = min(r, rows - 1), t = rc / a.G;
    valid = r < rows;
    row = s.q0 + t;
    h = hk * a.G + rc - t * a.G;
    lim = off + t;
    first = r0 < rows ? off + r0 / a.G : INT32_MAX;
    last = r0 < rows ? off + (min(r0 + 32, rows) - 1) / a.G : -1;
  }
};

// Every wave of the workgroup has got here; memory operations stay on their side.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// Direct load of 16 bytes per lane from base + at (bytes) to LDS at lds + 16 lane.  In assembly, so that the compiler does not
// take every LDS read that might meet it for one that has to wait: the waits are the kernel's own (vm_wait_all, then meet).
// (m0 is named, so that a value of the compiler's own is not thought to outlast the statement; that it is a reserved register is
// what the warning would say.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16(const void* base, uint32_t at, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(at), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// Four waves take 128 rows and walk over the keys in step, one tile ahead; two such workgroups share a CU (three with heads of 64
// channels: 16 prompts of 1,024 tokens 119 us with two, 105 with three, 145 with four, which spill in the main loop; here 9 and,
// with 128 channels, 13 registers spill on the way through the second run over the tiles), and one starts or ends while the other
// computes.
// Bound: no unit is full.  16 prompts of 1,024 tokens (208 us at 2.07 GHz): matrix units 32 % of the cycles, LDS reads 24 %, a third
// of those in bank conflicts of the values; a wave spends 30 % of its cycles waiting to issue.  What is left is the chain of a
// tile (scores, softmax, values), which two waves per SIMD cover in part, and the start and end of workgroups.  In k_prompt_turns
// (matrix units 56 %, LDS 42 %) the longest prompt took 1,210 us instead of 1,890 without LDS reads and tile loads.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_prompt_tiles(PromptArgs a) {
  constexpr int NW = 4, RB = 2 * D, TILE = PT_KEYS * RB, RPI = 1024 / RB, NI = PT_KEYS / RPI / NW;  // rows and loads per wave's load
  __shared__ __align__(1024) char kt[2 * TILE], vt[2 * TILE];
  __shared__ int again, first_bad[3 * D];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const PromptSeq s(a, a.item_prefix, blockIdx.x, lane);
  const int in_seq = s.place, Hk = a.H / a.G;
  const int nk = s.nk, rows = s.nq * a.G, tiles = (rows + NW * 32 - 1) / (NW * 32);
  const int rt = __builtin_amdgcn_readfirstlane(in_seq / Hk), hk = in_seq - rt * Hk;
  const int r0 = (tiles - 1 - rt) * NW * 32;  // the rows with the most keys first
  const int off = nk - s.nq, n_tiles = __builtin_amdgcn_readfirstlane(max(0, (off + (min(r0 + NW * 32, rows) - 1) / a.G + PT_KEYS) / PT_KEYS));
  if (threadIdx.x == 0) again = 0;

  const int lr = lane / (RB / 16), lp = lane % (RB / 16);
  const uint16_t* kbase = a.k + s.k0 * a.k_row + hk * a.k_head;
  const uint16_t* vbase = a.v + s.k0 * a.v_row + hk * a.v_head;
  const uint32_t kl = lds_address(kt), vl = lds_address(vt);
  // the lane's piece of a load, the same in all of a wave's loads
  const uint32_t kp = 16 * (lp ^ k_turn<D>(w * RPI + lr)), vp = 16 * (lp ^ v_turn<D>(w * RPI + lr));
  const uint32_t kat = (uint32_t)lr * (uint32_t)a.k_row * 2 + kp, vat = (uint32_t)lr * (uint32_t)a.v_row * 2 + vp;
  auto load = [&](int j, int n, uint32_t t, const uint16_t* base, int64_t stride, uint32_t at, uint32_t piece) {
    const int i = w + NW * n, r = j * PT_KEYS + i * RPI;
    if (r + RPI <= nk) {
      dma16(base + r * stride, at, t + i * 1024);
    } else {  // past the last key: that key again
      const int r1 = min(r, nk - 1);
      dma16(base + r1 * stride, (uint32_t)min(lr, nk - 1 - r1) * (uint32_t)stride * 2 + piece, t + i * 1024);
    }
  };
  auto issue = [&](int j, int buf) {
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      load(j, n, kl + buf * TILE, kbase, a.k_row, kat, kp);
      load(j, n, vl + buf * TILE, vbase, a.v_row, vat, vp);
    }
  };
  if (n_tiles > 0) issue(0, 0);
  const PromptRows pr(a, s, hk, r0 + 32 * w, lane);
  uint4 qf[D / 16];
  load_queries<D>(a, pr.row * a.q_row + pr.h * a.q_head, half, qf);
  PromptState<D> st;
  clear_state(st);
  for (int j = 0; j < n_tiles; ++j) {
    const int k0 = j * PT_KEYS, buf = j & 1;
    vm_wait_all();
    meet();  // tile j has landed, and every wave is done with the tile before
    if (j + 1 < n_tiles) issue(j + 1, buf ^ 1);
    if (k0 <= pr.last) add_tile<D, 2>(kt + buf * TILE, vt + buf * TILE, qf, a.c, pr.lim - k0, k0 + PT_KEYS - 1 > pr.first, lane, st);
  }
  __syncthreads();
  if (!__all(all_finite(st))) again = 1;
  __syncthreads();
  if (again) {
    for (int i = threadIdx.x; i < 3 * D; i += NW * 64) first_bad[i] = INT32_MAX;
    clear_state(st);
    for (int j = 0; j < n_tiles; ++j) {
      const int k0 = j * PT_KEYS;
      __syncthreads();
      issue(j, 0);
      vm_wait_all();
      __syncthreads();
      if (k0 + PT_KEYS - 1 > off + r0 / a.G) take_out_nonfinite<D>(vt, PT_KEYS, nk - k0, k0, first_bad, threadIdx.x, NW * 64);
      __syncthreads();
      add_tile<D, 2>(kt, vt, qf, a.c, pr.lim - k0, true, lane, st);
    }
    put_back_nonfinite(st, first_bad, pr.lim, half);
  }
  const float l = half_sum(st.l), inv = pr.lim >= 0 ? 1.f / l : 0.f;
  const int64_t at = pr.row * a.o_row + pr.h * a.o_head;
#pragma unroll
  for (int b = 0; b < D / 32; ++b) store_block(a, st.o[b], b, at, pr.valid, inv, half);
  if (a.lse && pr.valid && half == 0)
    a.lse[pr.row * a.H + pr.h] = pr.lim >= 0 ? (st.m + __builtin_amdgcn_logf(l)) * (1.f / LOG2E) : -INFINITY;
}

// Long prompts with heads of 128 channels.  A workgroup of eight waves, two per SIMD, takes 256 rows; the waves work in turns,
// a barrier between the turns: while waves 0-3 run matrix instructions (the scores of tile j + 1, then the values of tile j),
// waves 4-7 run the softmax of tile j on the vector units, and the other way round.
// Waves 0-3 run softmax j in turn 2 j and the products in turn 2 j + 1, waves 4-7 one turn later.  V(j) is read in turns 2 j + 1
// and 2 j + 2, K(j) in turns 2 j - 1 and 2 j (its first pieces one turn before that, ahead of the barrier).
// Loads go out during a wave's softmax: V(j + 1) and K(j + 3) for waves 0-3 (turn 2 j), V(j + 2) and K(j + 4) for waves 4-7 (turn
// 2 j + 1), over V(j - 2), K(j - 1), V(j - 1) and K(j) of three and four buffers; a wave waits for its own before it sends for the
// next two turns later, and the barrier of that turn makes them known to all: V(j + 1) after turn 2 j + 2, K(j + 3) likewise.
__global__ __launch_bounds__(512, 2) void k_prompt_turns(PromptArgs a) {
  constexpr int D = 128, NW = 8, RB = 2 * D, TILE = PT_KEYS * RB, RPI = 1024 / RB, NI = PT_KEYS / RPI / NW;  // rows and loads per wave's load
  constexpr int KS = D / 16, NV = D / 32, KAHEAD = 8;
  __shared__ __align__(1024) char kt[4 * TILE], vt[3 * TILE];
  __shared__ int again, first_bad[3 * D];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const bool second = w >= NW / 2;
  const PromptSeq s(a, a.item_prefix, blockIdx.x, lane);
  const int in_seq = s.place, Hk = a.H / a.G;
  const int nk = s.nk, rows = s.nq * a.G, tiles = (rows + NW * 32 - 1) / (NW * 32);
  const int hk = in_seq % Hk, r0 = (tiles - 1 - in_seq / Hk) * NW * 32;  // the rows with the most keys first
  const PromptRows pr(a, s, hk, r0 + 32 * w, lane);
  const int off = nk - s.nq, n_tiles = max(0, (off + (min(r0 + NW * 32, rows) - 1) / a.G + PT_KEYS) / PT_KEYS);
  if (threadIdx.x == 0) again = 0;

  const int lr = lane / (RB / 16), lp = lane % (RB / 16);
  const uint16_t* kbase = a.k + s.k0 * a.k_row + hk * a.k_head;
  const uint16_t* vbase = a.v + s.k0 * a.v_row + hk * a.v_head;
  const uint32_t kl = lds_address(kt), vl = lds_address(vt);
  // the lane's piece of a load, the same in all of a wave's loads
  const uint32_t kp = 16 * (lp ^ k_turn<D>(w * RPI + lr)), vp = 16 * (lp ^ v_turn<D>(w * RPI + lr));
  const uint32_t kat = (uint32_t)lr * (uint32_t)a.k_row * 2 + kp, vat = (uint32_t)lr * (uint32_t)a.v_row * 2 + vp;
  auto load = [&](int j, int n, uint32_t t, const uint16_t* base, int64_t stride, uint32_t at, uint32_t piece) {
    const int i = w + NW * n, r = j * PT_KEYS + i * RPI;
    if (r + RPI <= nk) {
      dma16(base + r * stride, at, t + i * 1024);
    } else {  // past the last key: that key again
      const int r1 = min(r, nk - 1);
      dma16(base + r1 * stride, (uint32_t)min(lr, nk - 1 - r1) * (uint32_t)stride * 2 + piece, t + i * 1024);
    }
  };
  auto load_keys = [&](int j, int n) { load(j, n, kl + (j & 3) * TILE, kbase, a.k_row, kat, kp); };
  auto load_vals = [&](int j, int n, int buf) { load(j, n, vl + buf * TILE, vbase, a.v_row, vat, vp); };
  auto load_tile = [&](int jk, int jv, int buf) {  // all of a wave's loads of K(jk) and V(jv)
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      if (jk < n_tiles) load_keys(jk, n);
      if (jv < n_tiles) load_vals(jv, n, buf);
    }
  };

  load_tile(0, 0, 0);
  load_tile(1, second ? 1 : n_tiles, 1);
  load_tile(2, n_tiles, 0);
  if (second) load_tile(3, n_tiles, 0);
  uint4 qf[KS];
  load_queries<D>(a, pr.row * a.q_row + pr.h * a.q_head, half, qf);

  // the lane's pieces of K (A operand of the scores, see tile_scores) and V (of the values, see tile_values) in a tile
  const int krow = lane & 31;
  const uint32_t kread = krow * RB + 16 * (half ^ k_turn<D>(krow));
  const int vr = 4 * half + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  uint32_t vread[NV];
#pragma unroll
  for (int b = 0; b < NV; ++b) vread[b] = vr * RB + 16 * ((4 * b + vc) ^ v_turn<D>(vr)) + 8 * (lane & 1);

  f32x16 sc[2];
  PromptState<D> st;
  clear_state(st);
  uint4 kf[2 * KS], pf[4], vf[4][NV];
  auto load_k = [&](int i, uint32_t t) {  // the tile's two blocks of keys in turn
    kf[i] = *reinterpret_cast<const uint4*>(kt + ((t + kread) ^ (32 * (i >> 1))) + (i & 1) * 32 * RB);
  };
  auto load_v = [&](int k, uint32_t t) {
#pragma unroll
    for (int b = 0; b < NV; ++b) {
      const uint2 lo = lds_column4(vt + t + vread[b] + 16 * k * RB), hi = lds_column4(vt + t + vread[b] + (16 * k + 8) * RB);
      vf[k][b] = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  };
  auto scores = [&](uint32_t t, bool values, uint32_t tv) {  // the first KAHEAD keys' pieces are in kf
#pragma unroll
    for (int i = 0; i < 2 * KS; i += 2) {
      if (i + KAHEAD < 2 * KS) {
        load_k(i + KAHEAD, t);
        load_k(i + KAHEAD + 1, t);
      }
      if (values && i == 2 * KS - KAHEAD / 2 - 2) load_v(0, tv);
      if (values && i == 2 * KS - 2) load_v(1, tv);
      __builtin_amdgcn_sched_barrier(0);
      sc[0] = i == 0 ? mfma32_bf16(kf[i], qf[i / 2], f32x16{}) : mfma32_bf16(kf[i], qf[i / 2], sc[0]);
      sc[1] = i == 0 ? mfma32_bf16(kf[i + 1], qf[i / 2], f32x16{}) : mfma32_bf16(kf[i + 1], qf[i / 2], sc[1]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  vm_wait_all();
  __syncthreads();
  if (n_tiles > 0) {
#pragma unroll
    for (int i = 0; i < KAHEAD; ++i) load_k(i, 0);
    scores(0, false, 0);
    here(sc[0]);
    here(sc[1]);
  }
  meet();
  if (second) meet();
  const int jv = second ? 2 : 1, jk = second ? 4 : 3;  // tiles ahead
  int vb = 0, vn = second ? 2 : 1;                     // buffers of V(j) and V(j + jv)
  for (int j = 0; j < n_tiles; ++j) {
    const int k0 = j * PT_KEYS;
    const uint32_t tk = ((j + 1) & 3) * TILE, tv = vb * TILE;
    vm_wait_all();
    tile_softmax<D, 2>(sc, a.c, pr.lim - k0, k0 + PT_KEYS - 1 > pr.first, half, st, pf, [&](int k) {
      if (k >= 2 * NI) return;
      if (k & 1) {
        if (j + jk < n_tiles) load_keys(j + jk, k >> 1);
      } else {
        if (j + jv < n_tiles) load_vals(j + jv, k >> 1, vn);
      }
    });
#pragma unroll
    for (int k = 0; k < 4; ++k) here(pf[k]);
    asm volatile("" : "+v"(st.l));
#pragma unroll
    for (int i = 0; i < KAHEAD; ++i) load_k(i, tk);
    meet();
    __builtin_amdgcn_s_setprio(1);
    scores(tk, true, tv);
    here(sc[0]);
    here(sc[1]);
#pragma unroll
    for (int b = 0; b < NV; ++b) here(st.o[b]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k + 2 < 4) load_v(k + 2, tv);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < NV; ++b) st.o[b] = mfma32_bf16(vf[k][b], pf[k], st.o[b]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int b = 0; b < NV; ++b) here(st.o[b]);
    __builtin_amdgcn_s_setprio(0);
    meet();
    vb = vb == 2 ? 0 : vb + 1;
    vn = vn == 2 ? 0 : vn + 1;
  }
  if (!second) meet();
  if (!__all(all_finite(st))) again = 1;
  __syncthreads();
  if (again) {
    for (int i = threadIdx.x; i < 3 * D; i += NW * 64) first_bad[i] = INT32_MAX;
    clear_state(st);
    for (int j = 0; j < n_tiles; ++j) {
      const int k0 = j * PT_KEYS;
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NI; ++n) {
        load(j, n, kl, kbase, a.k_row, kat, kp);
        load_vals(j, n, 0);
      }
      vm_wait_all();
      __syncthreads();
      if (k0 + PT_KEYS - 1 > off + r0 / a.G) take_out_nonfinite<D>(vt, PT_KEYS, nk - k0, k0, first_bad, threadIdx.x, NW * 64);
      __syncthreads();
      add_tile<D, 2>(kt, vt, qf, a.c, pr.lim - k0, true, lane, st);
    }
  }
  if (again) put_back_nonfinite(st, first_bad, pr.lim, half);
  const float l = half_sum(st.l), inv = pr.lim >= 0 ? 1.f / l : 0.f;
  const int64_t at = pr.row * a.o_row + pr.h * a.o_head;
#pragma unroll
  for (int b = 0; b < D / 32; ++b) store_block(a, st.o[b], b, at, pr.valid, inv, half);
  if (a.lse && pr.valid && half == 0)
    a.lse[pr.row * a.H + pr.h] = pr.lim >= 0 ? (st.m + __builtin_amdgcn_logf(l)) * (1.f / LOG2E) : -INFINITY;
}

// =====================================================================================================
// Few rows: a workgroup takes 32 rows and `chunk` tiles of 32 keys, which its two waves share out, each with its own two
// buffers in LDS and no barrier; at the end they merge their states.  (Two workgroups of two waves fit a CU and start and end
// apart: 64 new rows of four vehicles 54 us with four waves, 48 with two, 51 with one.)  Where the keys are in several chunks,
// the workgroups' states (of rows that exist) go to the workspace (16-byte piece p of lane l of block b at float4 (4 b + p) 64
// + l, then maxima and sums), and k_prompt_merge puts them together in the order of the chunks.
// =====================================================================================================
constexpr int PS_WAVES = 2, PS_KEYS = 32;

template <int D>
__host__ __device__ constexpr int part_floats() { return 32 * D + 64; }

template <int D>
__global__ __launch_bounds__(PS_WAVES * 64, 1) void k_prompt_split(PromptArgs a) {
  constexpr int RB = 2 * D, TILE = PS_KEYS * RB, RPI = 1024 / RB, NI = PS_KEYS / RPI;
  __shared__ __align__(1024) char kb0[PS_WAVES][TILE], kb1[PS_WAVES][TILE], vb0[PS_WAVES][TILE], vb1[PS_WAVES][TILE];
  __shared__ int first_bad[PS_WAVES][3 * D];
  __shared__ float sm[PS_WAVES][32], sl[PS_WAVES][32];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const PromptSeq s(a, a.item_prefix, blockIdx.x, lane);
  const int Hk = a.H / a.G, nk = s.nk, rows = s.nq * a.G, n_rt = (rows + 31) / 32;
  int i = s.place;
  const int hk = i % Hk;
  i /= Hk;
  const int r0 = 32 * (n_rt - 1 - i % n_rt), split = i / n_rt;
  const PromptRows pr(a, s, hk, r0, lane);
  const int n_tiles = max(0, (pr.last + PS_KEYS) / PS_KEYS), t0 = split * a.chunk, t1 = min(t0 + a.chunk, n_tiles);
  if (split > 0 && t0 >= t1) return;  // the merge takes as many chunks as these rows have
  uint4 qf[D / 16];
  load_queries<D>(a, pr.row * a.q_row + pr.h * a.q_head, half, qf);

  const int lr = lane / (RB / 16), lp = lane % (RB / 16);
  const uint16_t* kbase = a.k + s.k0 * a.k_row + hk * a.k_head;
  const uint16_t* vbase = a.v + s.k0 * a.v_row + hk * a.v_head;
  auto issue = [&](int j, char* kt, char* vt) {
#pragma unroll
    for (int n = 0; n < NI; ++n) {
      const int tr = n * RPI + lr;
      const int64_t key = min(j * PS_KEYS + tr, nk - 1);
      load_lds16(kbase + key * a.k_row + 8 * (lp ^ k_turn<D>(tr)), kt + n * 1024);
      load_lds16(vbase + key * a.v_row + 8 * (lp ^ v_turn<D>(tr)), vt + n * 1024);
    }
  };
  PromptState<D> st;
  clear_state(st);
  auto add = [&](int j, const char* kt, const char* vt) {
    add_tile<D, 1>(kt, vt, qf, a.c, pr.lim - j * PS_KEYS, j * PS_KEYS + PS_KEYS - 1 > pr.first, lane, st);
  };
  // One tile ahead; past the last tile the loads repeat it (from the L2), so that a wait for a fixed number of loads is one for
  // the tile at hand.
  if (int j = t0 + w; j < t1) {
    issue(j, kb0[w], vb0[w]);
    for (;;) {
      issue(j + PS_WAVES < t1 ? j + PS_WAVES : j, kb1[w], vb1[w]);
      vm_wait_below_c<2 * NI>();
      add(j, kb0[w], vb0[w]);
      if ((j += PS_WAVES) >= t1) break;
      issue(j + PS_WAVES < t1 ? j + PS_WAVES : j, kb0[w], vb0[w]);
      vm_wait_below_c<2 * NI>();
      add(j, kb1[w], vb1[w]);
      if ((j += PS_WAVES) >= t1) break;
    }
    vm_wait_all();
  }
  if (!__all(all_finite(st))) {
    for (int e = lane; e < 3 * D; e += 64) first_bad[w][e] = INT32_MAX;
    clear_state(st);
    for (int j = t0 + w; j < t1; j += PS_WAVES) {
      issue(j, kb0[w], vb0[w]);
      vm_wait_all();
      if (j * PS_KEYS + PS_KEYS - 1 > pr.first)
        take_out_nonfinite<D>(vb0[w], PS_KEYS, nk - j * PS_KEYS, j * PS_KEYS, first_bad[w], lane, 64);
      add(j, kb0[w], vb0[w]);
    }
    put_back_nonfinite(st, first_bad[w], pr.lim, half);
  }
  // the waves' states, merged: wave b takes block b of the output
  const float lw = half_sum(st.l);
  __syncthreads();
  auto exchange = [&](int x) { return reinterpret_cast<float4*>(x == 0 ? kb0[0] : (x == 1 ? kb1[0] : (x == 2 ? vb0[0] : vb1[0]))); };
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int p = 0; p < 4; ++p)
      exchange(w)[(4 * b + p) * 64 + lane] =
          make_float4(st.o[b][4 * p], st.o[b][4 * p + 1], st.o[b][4 * p + 2], st.o[b][4 * p + 3]);
  if (half == 0) {
    sm[w][lane] = st.m;
    sl[w][lane] = lw;
  }
  __syncthreads();
  const int q = lane & 31;
  float m = -INFINITY, l = 0.f, f[PS_WAVES];
#pragma unroll
  for (int x = 0; x < PS_WAVES; ++x) m = fmaxf(m, sm[x][q]);
#pragma unroll
  for (int x = 0; x < PS_WAVES; ++x) {
    f[x] = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(sm[x][q] - m);
    l += sl[x][q] * f[x];
  }
  const bool whole = s.n_split == 1;
  const float inv = pr.lim >= 0 ? 1.f / l : 0.f;
  float* part = a.part + (int64_t)blockIdx.x * part_floats<D>();
#pragma unroll
  for (int b = w; b < D / 32; b += PS_WAVES) {
    f32x16 o{};
#pragma unroll
    for (int x = 0; x < PS_WAVES; ++x)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const float4 v = exchange(x)[(4 * b + p) * 64 + lane];
        o[4 * p] += v.x * f[x];
        o[4 * p + 1] += v.y * f[x];
        o[4 * p + 2] += v.z * f[x];
        o[4 * p + 3] += v.w * f[x];
      }
    if (whole) {
      store_block(a, o, b, pr.row * a.o_row + pr.h * a.o_head, pr.valid, inv, half);
    } else if (pr.valid) {
#pragma unroll
      for (int p = 0; p < 4; ++p)
        reinterpret_cast<float4*>(part)[(4 * b + p) * 64 + lane] = make_float4(o[4 * p], o[4 * p + 1], o[4 * p + 2], o[4 * p + 3]);
    }
  }
  if (w != 0) return;
  if (!whole && pr.valid) part[32 * D + lane] = half ? l : m;
  if (whole && a.lse && pr.valid && half == 0)
    a.lse[pr.row * a.H + pr.h] = pr.lim >= 0 ? (m + __builtin_amdgcn_logf(l)) * (1.f / LOG2E) : -INFINITY;
}

// The chunks' states of 32 rows put together.  PM_GROUPS groups of waves, a block of 32 channels per wave, take every
// PM_GROUPS-th chunk (the states come from other XCDs' memory, so what counts is how many loads are under way), then the first
// group puts the groups' states together through LDS.
constexpr int PM_GROUPS = 4;

template <int D>
__global__ __launch_bounds__(2 * D * PM_GROUPS) void k_prompt_merge(PromptArgs a) {
  constexpr int NB = D / 32;
  __shared__ float4 xo[PM_GROUPS - 1][NB][4][64];
  __shared__ float xm[PM_GROUPS - 1][32], xl[PM_GROUPS - 1][32];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, q = lane & 31;
  const int blk = w % NB, group = w / NB;
  const PromptSeq s(a, a.merge_prefix, blockIdx.x, lane);
  const int Hk = a.H / a.G, n_rt = (s.nq * a.G + 31) / 32, i = s.place, hk = i % Hk;
  const PromptRows pr(a, s, hk, 32 * (n_rt - 1 - i / Hk), lane);
  const int n_tiles = max(0, (pr.last + PS_KEYS) / PS_KEYS), n = max(1, (n_tiles + a.chunk - 1) / a.chunk);
  const float* part = a.part + (int64_t)(s.first_item + i) * part_floats<D>();
  const int64_t step = (int64_t)n_rt * Hk * part_floats<D>();
  float m = -INFINITY, l = 0.f;
  f32x16 o{};
  auto add = [&](float mc, float lc, const float4 (&v)[4], float mz) {
    const float f = __builtin_amdgcn_exp2f(mc - mz);
    l += lc * f;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      o[4 * p] += v[p].x * f;
      o[4 * p + 1] += v[p].y * f;
      o[4 * p + 2] += v[p].z * f;
      o[4 * p + 3] += v[p].w * f;
    }
  };
  auto raise = [&](float to) {  // the maximum; what the exponents are taken from
    const float mz = to == -INFINITY ? 0.f : to, back = __builtin_amdgcn_exp2f(m - mz);
    m = to;
    l *= back;
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] *= back;
    return mz;
  };
  constexpr int AT_ONCE = 4;  // chunks of a wave whose loads are under way
  if (pr.valid)  // (states of rows that do not exist were not written)
    for (int c0 = group; c0 < n; c0 += AT_ONCE * PM_GROUPS) {
      float mc[AT_ONCE], lc[AT_ONCE];
      float4 v[AT_ONCE][4];
#pragma unroll
      for (int c = 0; c < AT_ONCE; ++c) {
        const float* x = part + min(c0 + c * PM_GROUPS, n - 1) * step;
        mc[c] = x[32 * D + q];
        lc[c] = x[32 * D + 32 + q];
#pragma unroll
        for (int p = 0; p < 4; ++p) v[c][p] = reinterpret_cast<const float4*>(x)[(4 * blk + p) * 64 + lane];
      }
      float mn = m;
#pragma unroll
      for (int c = 0; c < AT_ONCE; ++c) mn = c0 + c * PM_GROUPS < n ? fmaxf(mn, mc[c]) : mn;
      const float mz = raise(mn);
#pragma unroll
      for (int c = 0; c < AT_ONCE; ++c)
        if (c0 + c * PM_GROUPS < n) add(mc[c], lc[c], v[c], mz);
    }
  if (group > 0) {
#pragma unroll
    for (int p = 0; p < 4; ++p) xo[group - 1][blk][p][lane] = make_float4(o[4 * p], o[4 * p + 1], o[4 * p + 2], o[4 * p + 3]);
    if (blk == 0 && half == 0) {
      xm[group - 1][q] = m;
      xl[group - 1][q] = l;
    }
  }
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int g = 0; g < PM_GROUPS - 1; ++g) {
    const float mc = xm[g][q], mz = raise(fmaxf(m, mc));
    const float4 v[4] = {xo[g][blk][0][lane], xo[g][blk][1][lane], xo[g][blk][2][lane], xo[g][blk][3][lane]};
    add(mc, xl[g][q], v, mz);
  }
  const float inv = pr.lim >= 0 ? 1.f / l : 0.f;
  store_block(a, o, blk, pr.row * a.o_row + pr.h * a.o_head, pr.valid, inv, half);
  if (a.lse && pr.valid && half == 0 && blk == 0)
    a.lse[pr.row * a.H + pr.h] = pr.lim >= 0 ? (m + __builtin_amdgcn_logf(l)) * (1.f / LOG2E) : -INFINITY;
}

// Whether the keys of the prompts (on average over their work) are many enough for the waves' turns to be worth the longer start
// and end of their workgroups.  us with and without: 16 prompts of 1,024 tokens 229 and 202, four of 2,048 174 and 166, two of
// 4,096 (32 heads over 8) 272 and 275, one of 8,000 477 and 497, one of 16,001 1,850 and 1,910.  With heads of 64 channels, whose
// products are half as long, never: two prompts of 4,096 179 and 170.
static bool long_prompts(const PromptArgs& a) {
  double work = 0, keys = 0;
  for (int i = 0; i < a.n_seq; ++i) {
    const double w = (double)a.nq[i] * a.nk[i];
    work += w;
    keys += w * a.nk[i];
  }
  return a.D == 128 && keys >= 4096 * work;
}

// Which kernel, and in how many chunks, by what either would take on the chip's 256 CUs (us, measured):
//   the row tiles: 128 rows to a workgroup, two workgroups per CU, 5 to start and end and 2.2 per tile of 64 keys where all CUs are
//   at work (1.5 for a few);
//   the chunks: two workgroups per CU, 5 to start and end and, for each pair of tiles of 32 keys, 1, and 4 more to put chunks
//   together; the last workgroups leave part of the chip idle for a share of their time;
//   either at least its keys' way from memory, 4.5 TB/s, which the work overlaps in part.
// Measured, chunks and row tiles, 32 heads over 8: one prompt of 1,024 tokens 28 and 29, of 2,048 77 and 55, two of 1,500 93 and
// 50, 64 of 300 268 and 125, 16 of 100 23 and 14, 128 new rows of four sequences over 2,000 keys 36 and 48, 256 of two over
// 4,000 63 and 88, 512 of two over 3,000 88 and 69; 32 heads over 32: one prompt of 512 15 and 17, of 768 20 and 23, of 1,024 27
// and 29, 64 new rows of four over 640 to 4,096 46 and 86; heads of 64 channels: 24 prompts of 31 to 698 33 and 24, 130 new rows
// of eight over 5,000 128 and 92.  (Four prompts of 224, 17 and 13, it takes for chunks.)
bool plan_prompt(PromptArgs& a, int64_t workspace_bytes, int64_t* need) {
  constexpr int SLOTS = 512;
  const int Hk = a.H / a.G;
  const int64_t part = 4 * (32 * a.D + 64);
  const double width = a.D == 128 ? 1.0 : 0.5;  // of a tile's work
  *need = 0;
  double tiles = 0, longest = 0, steps = 0, keys = 0;
  int t_max = 1;
  for (int i = 0; i < a.n_seq; ++i) {
    const int64_t r = (int64_t)a.nq[i] * a.G, wide = (r + 127) / 128, n_rt = (r + 31) / 32;
    const double seen = a.nk[i] - 0.5 * std::min(a.nq[i], a.nk[i]);  // keys of a row, on average
    tiles += (double)Hk * wide * (5 + 2.2 * width * (seen / PT_KEYS + 1));
    longest = std::max(longest, 8 + 1.5 * width * (a.nk[i] / PT_KEYS + 1));
    steps += (double)Hk * n_rt * (seen / PS_KEYS + 1);
    keys += (double)Hk * a.nk[i];
    t_max = std::max(t_max, (a.nk[i] + PS_KEYS - 1) / PS_KEYS);
  }
  const double memory = keys * a.D * 4 / 4.5e6;
  tiles = std::max(tiles / SLOTS, longest);
  tiles = std::max(tiles, memory) + 0.35 * std::min(tiles, memory);
  const double per_wave = steps / (SLOTS * PS_WAVES), shared_step = std::max(width, memory / per_wave);
  double best = INFINITY;
  for (const int k : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {  // chunks of the longest keys
    const int chunk = std::max(2 * PS_WAVES, (t_max + k - 1) / k);
    int64_t items = 0, merges = 0;
    for (int i = 0; i < a.n_seq; ++i) {
      const int n_rt = (int)(((int64_t)a.nq[i] * a.G + 31) / 32), n = std::max(1, ((a.nk[i] + PS_KEYS - 1) / PS_KEYS + chunk - 1) / chunk);
      items += (int64_t)n_rt * Hk * n;
      if (n > 1) merges += (int64_t)n_rt * Hk;
    }
    const bool split = merges > 0;
    // (a launch holds fewer than 2^32 threads)
    if (items > UINT32_MAX / (PS_WAVES * 64) || merges > UINT32_MAX / (2 * a.D * PM_GROUPS) || (split && items * part > workspace_bytes)) break;
    const double rounds = std::max(1.0, (double)items / SLOTS), pair = (double)chunk / PS_WAVES;
    const double work = 5 * rounds + width * (rounds > 1 ? std::max(per_wave, pair) : pair);
    const double tail = rounds > 1 ? 0.15 * pair : 0.4 * std::max(0.0, pair - steps / items / PS_WAVES);
    const double cost = std::max(memory, work) + 0.35 * std::min(memory, work) + tail * shared_step + (split ? 4 : 0);
    if (cost >= best) continue;
    best = cost;
    a.chunk = chunk;
    *need = split ? items * part : 0;
  }
  if (a.kernel == FSX_PROMPT_AUTO ? tiles <= best : a.kernel != FSX_PROMPT_CHUNKS) {
    *need = 0;
    return false;
  }
  for (int i = 0; i < a.n_seq; ++i) {
    const int n_rt = (int)(((int64_t)a.nq[i] * a.G + 31) / 32);
    a.n_split[i] = std::max(1, ((a.nk[i] + PS_KEYS - 1) / PS_KEYS + a.chunk - 1) / a.chunk);
    a.item_prefix[i + 1] = a.item_prefix[i] + n_rt * Hk * a.n_split[i];
    a.merge_prefix[i + 1] = a.merge_prefix[i] + (a.n_split[i] > 1 ? n_rt * Hk : 0);
  }
  return true;
}

hipError_t launch_prompt_attention(PromptArgs a, void* workspace, int64_t workspace_bytes, hipStream_t s) {
  if (a.n_seq == 0) return hipSuccess;
  int64_t need = 0;
  if (plan_prompt(a, workspace_bytes, &need)) {
    a.part = (float*)workspace;
    const dim3 grid(a.item_prefix[a.n_seq]), merge(a.merge_prefix[a.n_seq]);
    if (a.D == 64) {
      hipLaunchKernelGGL(k_prompt_split<64>, grid, dim3(PS_WAVES * 64), 0, s, a);
      if (merge.x) hipLaunchKernelGGL(k_prompt_merge<64>, merge, dim3(128 * PM_GROUPS), 0, s, a);
    } else {
      hipLaunchKernelGGL(k_prompt_split<128>, grid, dim3(PS_WAVES * 64), 0, s, a);
      if (merge.x) hipLaunchKernelGGL(k_prompt_merge<128>, merge, dim3(256 * PM_GROUPS), 0, s, a);
    }
    return hipGetLastError();
  }
  const bool turns = a.kernel == FSX_PROMPT_AUTO ? long_prompts(a) : a.kernel == FSX_PROMPT_TURNS;
  const int rows = turns ? 256 : 128;
  for (int i = 0; i < a.n_seq; ++i)
    a.item_prefix[i + 1] = a.item_prefix[i] + (int)(((int64_t)a.nq[i] * a.G + rows - 1) / rows) * (a.H / a.G);
  const dim3 grid(a.item_prefix[a.n_seq]), block(2 * rows);
  const auto fn = turns ? k_prompt_turns : (a.D == 64 ? k_prompt_tiles<64> : k_prompt_tiles<128>);
  hipLaunchKernelGGL(fn, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace fsx
