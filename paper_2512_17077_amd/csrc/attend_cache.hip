// Reuse-phase attention over a KV cache held in 8 bits (cache_kernels.hip), bf16 queries and outputs, fp32 softmax state and
// accumulators.  Two uses, one kernel:
//   Lists    every query head attends over its own kept rows (Section 2.3 Eq. 4 restricted to the kept set of Section 4.5);
//   !Lists   every head attends over the first k_b rows of its sequence (no lists: single tokens of an autoregressive
//            model, or a block over everything).  The query heads of a group then read the same rows, so a tile's 32
//            columns are (query, head of the group) pairs of one KV head and the rows are read once per group.
//
// With scores z_ij = scale * q_i . k_j (in units of log 2) an output is sum_j 2^(z_ij - m_i) v_j / sum_j 2^(z_ij - m_i), in one
// pass over the rows with the running maximum m_i and sum; parts of a list that different waves or workgroups have seen are
// joined by weighting them with 2^(m_part - m).  A code times its scale is a bf16 value exactly, so the arithmetic is that of a
// bf16 cache: probabilities are rounded to bf16 for the matrix cores (the sum adds the rounded ones, so that weights still sum to
// one), outputs once at the end.  Against 64 bits the outputs are off by 1.7e-3 (relative, over all outputs; 256 to 8000 rows), with
// probabilities in fp32 by 1.6e-3 to 1.7e-3: that is the rounding of the outputs.  The two differ from each other by 6e-4 to 1e-3.
//
// What bounds it: the rows, each read once (a block of 32 queries does 64 operations per byte of them, the matrix cores
// could do 350 meanwhile).  Gathered rows of 128 bytes, counted once per list and with the call's start and end in the time, come at
// 3.6 to 4.0 TB/s where lists are taken whole (28 % of sixteen sequences of 512 to 4096 positions, 32 heads: 79 MB in 22.1 us; 30 to
// 50 % of forty: 288 MB in 72.5), at 4.5 in pieces (half of sixteen of 8192: 537 MB in 120) and where the heads of a group find each
// other's rows in the L2 (the forty over 8 KV heads: 63.8 us); rows in order at 6.7.  A workgroup
// alone gets through a row of K and V in 7 ns, which decides where there are few lists.  So:
//   - A workgroup of four waves walks one list or piece of one (or of four heads, see kSide).  Each wave has a span of 32-row
//     tiles of its own and LDS that no other wave touches, so the walk needs no workgroup barrier.
//   - A tile's rows are fetched one tile ahead at head_dim 128, two at 64, into registers.  (Two ahead at 128: 24.6 us against
//     23.4 on sixteen ragged lists, 32 heads; the registers are better spent on operands.)
//   - K goes into LDS as codes and is converted on its way into the matrix cores (half the LDS traffic of converting before);
//     there a lane's 16 bytes are 16 elements of one row, and the queries, which stay in registers, are fetched in that
//     order.  V, which is read transposed, 16 bits at a time, is converted first.  The conversion applies the scale.
//   - Scales are bytes, one per tile row and tensor: lane l fetches that of K row l (V: row l - 32) with the tile.  K's are wanted
//     by the lanes of that column in both halves (one exchange of halves), V's by the lane that converts the row (a lane exchange).
//   - All of a tile's operands are asked for at once, V's before the softmax that stands between.
// Measured (MI355X): sixteen lists of 5 to 50 % of 512 to 4096 positions, 32 heads x 128, 32 queries: 23.4 us; one layer of 32 heads,
// 256 of 1024 positions: 5.8; single tokens of 32 sequences of 4000 to 8192, 32 heads over 8 x 128 (379 MB): 67.2, 5.6 TB/s.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "attend_sparse.h"

namespace dllm {

constexpr int kWaves = 4;
constexpr int kMaxListRows = 2048;   // kept rows of a list that one workgroup walks at most (their ids lie in LDS)

// 16 codes -> 16 bf16 values, in order
__device__ __forceinline__ void widen_codes(v4u x, float unit, v4u& lo, v4u& hi) {
  uint32_t y[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[e], unit, false));
    y[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[e], unit, true));
  }
  lo = v4u{y[0], y[1], y[2], y[3]};
  hi = v4u{y[4], y[5], y[6], y[7]};
}

// A lane converts 16 codes of a V row into two 16-byte chunks of bf16 and lays them half a row apart, so that lanes side by side
// write chunks side by side (next to each other they would use every other bank only).  The accumulators have that order, too: this is
// the chunk of head_dim that stands at chunk `at` of a V tile's row.
template <int D>
__device__ __forceinline__ int placed(int at) { return at < D / 16 ? 2 * at : 2 * (at - D / 16) + 1; }

// Byte offset of 16-byte chunk `cc` of `row` in a tile of codes, permuted so that lanes with neighbouring rows read one
// chunk of each from different banks.
template <int D>
__device__ __forceinline__ int codes_off(int row, int cc) {
  return row * D + ((cc ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4);
}

// What a workgroup takes of one sequence: rows c0 .. c1-1 of its list, one of `parts` segments of it.
struct Segment {
  int b, k0, kb, c0, c1, parts, q0, nq, kv0;
};

// sequence that list position r belongs to: the last one with cu_k[b] <= r among those that keep something
__device__ __forceinline__ int sequence_at(const int32_t* __restrict__ cu_k, int batch, int r, int lane) {
  int lo = 0, n = batch;   // it lies in lo .. lo+n-1
  while (n > 1) {
    const int step = (n + 63) / 64;
    const bool below = lane * step < n && cu_k[lo + lane * step] <= r;
    const int at = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(below) | 1ull);   // cu_k does not decrease
    lo += at * step;
    n = min(step, n - at * step);
  }
  return lo;
}

// Order in which lists that are taken whole are started.  Two workgroups are resident per compute unit, and workgroup i shares
// its unit with workgroup i + 256 (measured: see below), so where all lists are resident but not one per unit, the longest are
// left alone and the others folded, shortest with longest: with pairs = lists beyond 256, the first `pairs` places go to the
// shortest, in rising order, the next to the longest, and those that come second are in falling order.  32 heads x 128, lists of
// 5 to 50 % of 512 to 4096 positions, mean over six draws, as they come / longest first / folded: 9 sequences 18.2 / 19.5 / 17.4
// us, 12 24.6 / 23.6 / 20.4, 14 27.8 / 26.1 / 22.1, 16 28.9 / 27.7 / 25.2.  With more lists than are resident, longest first: 20
// sequences 35.8 / 32.3.
enum : int { kAsTheyCome = 0, kLongestFirst = 1, kFolded = 2 };
constexpr int kUnits = 256;   // compute units

// Heads side by side (HW): in pieces without lists a workgroup's four waves can take a piece of four neighbouring KV heads, each
// wave one of them and all of the piece, instead of a quarter of the piece of one head.  The rows of four heads lie side by side
// in memory, and asked for together they come faster (reading alone, 8 heads x 128 codes: 6.7 TB/s against 5.6 to 6.0), and no
// merge of the waves is left.  But a wave then has four times as many tiles one after the other.  8 heads x 128, single tokens, a
// head per workgroup / four: 32 sequences of 4000 to 8192 72.8 / 67.2 us, 12 36.6 / 33.0, one of 8000 (pieces of 128, the least)
// 10.9 / 11.9; 4 heads, 8 of 3000 to 8000 (160) 17.9 / 16.4; 16 heads x 64, 40 of 1000 to 5000 (896) 63.3 / 56.1, 4 x 64, 30 of
// 1000 to 8000 (288) 22.1 / 22.6.  So from pieces of 160 rows on at head_dim 128, 512 at 64, and up to four column tiles (which
// read the rows again, from the caches: 24 sequences of 500 to 4000, 16 queries of 32 heads over 8, 53.4 / 49.7; 4 of 512
// queries, 32 heads, 204 / 216).
constexpr int kSide = 4;

// Rows are shared out in pieces (Pieces): the lists of one head, laid end to end as cu_k has them, are cut every `piece` rows, and
// a workgroup takes one piece of one head, whatever sequences it holds.  So all workgroups have the same work however long
// the lists are, and those that a cut goes through are merged by a second launch.  Otherwise a workgroup takes one list whole.
// HW: KV heads per workgroup (see kSide).
template <int D, bool Lists, bool Pieces, int HW, int VS>
__global__ __launch_bounds__(kWaves * 64, 2) void attend_cache_kernel(
    const uint16_t* __restrict__ q, CacheView c, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_kv,
    const int32_t* __restrict__ idx, const int32_t* __restrict__ cu_k, int32_t total_k, uint16_t* __restrict__ o,
    float* __restrict__ po, float2* __restrict__ pml, int32_t piece, int order,
    Shape s DLLM_CHECK_PARAM) {
  DLLM_CHECK_EXIT();
  constexpr int CC = D / 16;            // 16-byte chunks of a row of codes
  constexpr int DV = D / VS, CV = CC / VS;   // elements and 16-byte chunks of a V row that this workgroup takes
  constexpr int KTILEB = kTile * D, VTILEB = kTile * 2 * DV;   // K lies in LDS as codes, V as bf16
  constexpr int NLD = kTile * CC / 64;  // 16-byte loads of K per lane and tile
  constexpr int NLV = NLD / VS;         // ... of V
  constexpr int NDB = DV / 32;
  constexpr int NT = D / 16;            // matrix-core steps along head_dim
  constexpr int W = kWaves;
  constexpr int SP = W / HW;            // waves per head, each with a span of the rows
  static_assert(W % HW == 0 && (HW == 1 || (Pieces && !Lists)), "heads side by side: in pieces without lists only");
  constexpr int MAXT = kMaxListRows / kTile / W;
  constexpr int kDepth = D == 128 ? 1 : 2;   // tiles in flight per wave
  constexpr int kMl = Lists ? MAXT * kTile : 64;

  constexpr int WAVEB = KTILEB + VTILEB > NDB * 4096 ? KTILEB + VTILEB : NDB * 4096;
  __shared__ __attribute__((aligned(16))) char lds[W][WAVEB];   // per wave: K tile, V tile; its accumulators at the merge
  __shared__ int sm_rows[W][kMl];   // kept-row ids of each wave's tiles; (m, l) at the merge

  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int col = lane & 31, hf = lane >> 5;
  constexpr bool kHeadsFirst = Lists || !Pieces;
  int unit = kHeadsFirst ? blockIdx.x : blockIdx.y, px = kHeadsFirst ? blockIdx.y : blockIdx.x;
  if constexpr (kHeadsFirst && (D == 64 || Lists)) {
    // Heads that share memory go to one XCD and its L2 (workgroup i runs on XCD i % 8): the lists of the query heads of one KV
    // head, and the two heads whose 64-byte rows share a 128-byte line.  Of 8 * share workgroups in a row, every eighth belongs
    // to one set.  Lists of 5 to 50 % of 512 to 4096, sixteen sequences, 32 heads over 8 x 128 25.4 -> 24.0 us, 40 sequences of
    // 30 to 50 % 69.2 -> 60.7.
    const uint32_t n = gridDim.x, at = blockIdx.x + n * blockIdx.y;
    const uint32_t share = (Lists ? s.group : 1) * (D == 64 && s.hkv % 2 == 0 ? 2 : 1);
    if (share > 1 && (at / (8 * share) + 1) * (8 * share) <= n * gridDim.y) {
      const uint32_t set = at / (8 * share) * 8 + at % 8, sets = n / share;
      px = int(set / sets);
      unit = int(share * (set % sets) + at / 8 % share);
    }
  }
  const int g = Lists ? unit / s.group : unit * HW + wave / SP;   // KV head of this wave
  const int h0 = Lists ? unit : g * s.group;                      // its first query head
  const int heads = Lists ? 1 : s.group;
  const int span = wave % SP;
  // VS: workgroups that share a list's columns of V, where there are units to spare.  One unit gets 36 GB/s of gathered rows,
  // with eight waves no more than with four, so that each takes all of K and its part of V, and needs no merge: lists of 256 /
  // 512 / 1024 rows, 32 heads x 128, alone 7.14 / 9.45 / 14.1 us, in four 5.72 / 7.22 / 10.7; four of 276 to 994 in two 13.0 ->
  // 11.3; single tokens of two sequences of 847 and 738, 8 KV heads, in four 12.1 -> 8.7.  (Two workgroups per unit: 11.3 ->
  // 17.3.)
  const int part = VS > 1 ? int(blockIdx.z) % VS : 0;   // of V's columns
  const int qt0 = VS > 1 ? int(blockIdx.z) / VS : blockIdx.z, qt_step = gridDim.z / VS;   // column tiles
  // column x of a sequence: query x / heads, head h0 + x % heads
  auto query_of = [&](int x) { return Lists ? x : int(uint32_t(x) / uint32_t(heads)); };
  auto clear = [&](int q0, int nq) {   // nothing kept: defined as zeros
    constexpr int RL = D / 2;   // lanes per row of the output, two elements each (a sequence may have 2^31 elements and more)
    for (int x = span * (64 / RL) + lane / RL; x < nq * heads; x += SP * (64 / RL)) {
      const int i = query_of(x);
      *reinterpret_cast<uint32_t*>(o + (int64_t(q0 + i) * s.hq + h0 + (x - i * heads)) * D + lane % RL * 2) = 0;
    }
  };

  Segment sg;
  int end = 0;   // list position behind this piece
  [[maybe_unused]] BatchInfo bi;
  [[maybe_unused]] const bool small = s.batch <= kRankBatch;   // (lane i holds sequence i's offsets)
  // the first sequence from b on that keeps something, and what of it lies in this piece
  auto enter = [&](int b) {
    if (small) {
      const uint64_t some = __builtin_amdgcn_ballot_w64(lane < s.batch && lane >= b && bi.kb > 0);
      b = some ? __builtin_ctzll(some) : s.batch - 1;
      sg.k0 = __builtin_amdgcn_readlane(bi.ko0, b);
      sg.kb = __builtin_amdgcn_readlane(bi.kb, b);
      sg.q0 = __builtin_amdgcn_readlane(bi.q0, b);
      sg.nq = __builtin_amdgcn_readlane(bi.nq, b);
      sg.kv0 = __builtin_amdgcn_readlane(bi.kv0, b);
    } else {
      while (b < s.batch - 1 && cu_k[b + 1] == cu_k[b]) ++b;
      sg.k0 = cu_k[b];
      sg.kb = cu_k[b + 1] - sg.k0;
      sg.q0 = cu_q[b];
      sg.nq = cu_q[b + 1] - sg.q0;
      sg.kv0 = cu_kv[b];
    }
    const int k1 = sg.k0 + sg.kb, fp = int(uint32_t(sg.k0) / uint32_t(piece));
    sg.b = b;
    sg.c0 = max(px * piece, sg.k0) - sg.k0;
    sg.c1 = min(end, k1) - sg.k0;
    sg.parts = sg.kb > 0 ? int(uint32_t(k1 - 1) / uint32_t(piece)) - fp + 1 : 1;
  };
  if constexpr (Pieces) {
    const int first = int(min(int64_t(px) * piece, int64_t(INT32_MAX)));   // (the grid may have a few more than there are pieces)
    int b = 0;
    if (small) {
      bi = load_batch(cu_q, cu_kv, cu_k, s.batch, lane, false);
      end = __builtin_amdgcn_readlane(bi.ko0 + bi.kb, s.batch - 1);
      const uint64_t behind = __builtin_amdgcn_ballot_w64(lane < s.batch && bi.ko0 + bi.kb > first);
      b = behind ? __builtin_ctzll(behind) : 0;
    } else {
      end = cu_k[s.batch];
      b = sequence_at(cu_k, s.batch, first, lane);
    }
    if (px == 0 && blockIdx.z == 0) {
      if (small) {
        for (uint64_t none = __builtin_amdgcn_ballot_w64(lane < s.batch && bi.kb == 0); none != 0; none &= none - 1) {
          const int i = __builtin_ctzll(none);
          clear(__builtin_amdgcn_readlane(bi.q0, i), __builtin_amdgcn_readlane(bi.nq, i));
        }
      } else {
        for (int i = 0; i < s.batch; ++i)
          if (cu_k[i + 1] == cu_k[i]) clear(cu_q[i], cu_q[i + 1] - cu_q[i]);
      }
    }
    if (first >= end) return;
    end = int(min(int64_t(first) + piece, int64_t(end)));
    enter(b);
  } else {
    int place_of = px;
    if (order == kFolded) {
      const int first_round = (kUnits + int(gridDim.x) - 1) / int(gridDim.x), pairs = s.batch - first_round;
      place_of = px < pairs ? s.batch - 1 - px : px - pairs;
    }
    const SeqInfo si = sequence_of_slot(cu_q, cu_kv, cu_k, s.batch, place_of, lane, order != kAsTheyCome);
    if (si.kb == 0) {
      if (qt0 == 0 && part == 0) clear(si.q0, si.nq);
      return;
    }
    sg = {si.b, si.ko0, si.kb, 0, Lists ? min(si.kb, kMaxListRows) : si.kb, 1, si.q0, si.nq, si.kv0};
  }

  char* ktile = lds[wave];
  char* vtile = lds[wave] + KTILEB;
  const int koff = codes_off<D>(col, hf);   // K operand: chunks 2u + hf of row col
  VtAddr<DV> vt;
  vt.init(lane);
  const uint32_t coff = uint32_t(lane) % CC * 16;
  const uint32_t voff = uint32_t(lane) % CV * 16 + part * DV;
  const uint32_t pitch = uint32_t(c.tok);   // a sequence's rows span < 4 GiB (checked on the host)
  const float zscale = s.scale * kLog2e;
  auto opaque = [](int x) {
    asm volatile("" : "+v"(x));
    return x;
  };

  for (;;) {   // segments of the piece
    const int ncols = sg.nq * heads;
    const uint8_t* kbase = c.k + int64_t(sg.kv0) * c.tok + int64_t(g) * c.head;
    const uint8_t* vbase = c.v + int64_t(sg.kv0) * c.tok + int64_t(g) * c.head;
    const uint8_t* sbase = (hf == 0 ? c.ks : c.vs) + g * c.scale_head + scale_slot(sg.kv0, sg.b, c.shift);
    const int32_t* __restrict__ rows = idx + int64_t(h0) * total_k + sg.k0;
    const int c0 = sg.c0, c1 = sg.c1;
    const int ntiles = c1 > c0 ? (c1 - c0 + kTile - 1) / kTile : 0;
    // a wave's tiles are neighbours: it walks a span of its own
    const int t0 = ntiles * span / SP, mine = ntiles * (span + 1) / SP - t0;

    for (int qt = qt0; ntiles > 0 && qt * 32 < ncols; qt += qt_step) {
      float m_used = -FLT_MAX, lsum = 0.0f;
      f32x16 acc[NDB];
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = 0.0f;

      int* my_rows = sm_rows[wave];
      if constexpr (Lists) {   // ids of this wave's tiles (positions past the end repeat the last row, which is masked)
#pragma unroll
        for (int jj = 0; jj < MAXT / 2; ++jj) {
          const int p = jj * 64 + lane;
          const int t = min(c0 + (t0 + (p >> 5)) * kTile + (p & 31), c1 - 1);
          my_rows[p] = rows[t];
        }
      }
      // The queries stay in registers: this lane's column, in the order in which the lane's half of a K row comes (operand t of the
      // products: elements 16 * (t - t % 2 + hf) + 8 * (t % 2) ..)
      v4u qx[NT];
      {
        const int x = min(qt * 32 + col, ncols - 1);   // past the last column: that one again, never stored
        const int qi = query_of(x);
        const uint16_t* qp = q + int64_t(sg.q0 + qi) * s.q_tok + int64_t(h0 + (x - qi * heads)) * s.q_head + 16 * hf;
#pragma unroll
        for (int t = 0; t < NT; ++t) qx[t] = *reinterpret_cast<const v4u*>(qp + 16 * (t & ~1) + 8 * (t & 1));
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

      v4u kr[kDepth][NLD], vr[kDepth][NLV];
      uint32_t sc[kDepth];
      // row `r` (0 .. 31) of the wave's j-th tile
      auto row_of = [&](int j, int r) {
        return Lists ? my_rows[j * kTile + r] : min(c0 + (t0 + j) * kTile + r, c1 - 1);
      };
      auto fetch = [&](v4u (&kx)[NLD], v4u (&vx)[NLV], uint32_t& sx, int j) {
        const uint32_t lane_o = opaque(lane);
        sx = sbase[uint32_t(row_of(j, lane_o & 31)) >> c.shift];
#pragma unroll
        for (int i = 0; i < NLD; ++i) {
          const uint32_t off = __umul24(uint32_t(row_of(j, (i * 64 + lane_o) / CC)), pitch) + coff;
          kx[i] = load_once(kbase + off);
          if constexpr (VS == 1) vx[i] = load_once(vbase + off);
        }
        if constexpr (VS > 1) {
#pragma unroll
          for (int i = 0; i < NLV; ++i)
            vx[i] = load_once(vbase + __umul24(uint32_t(row_of(j, (i * 64 + lane_o) / CV)), pitch) + voff);
        }
      };
#pragma unroll
      for (int d = 0; d < kDepth; ++d)
        if (d < mine) fetch(kr[d], vr[d], sc[d], d);
      for (int j0 = 0; j0 < mine; j0 += kDepth) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
          const int j = j0 + d, tile = t0 + j;
          if (j < mine) {
            VtAddr<DV> vtr;
            vtr.base[0] = opaque(vt.base[0]);
            vtr.base[1] = opaque(vt.base[1]);
            const uint32_t lane_o = opaque(lane);
            const u32x2 both = __builtin_amdgcn_permlane32_swap(sc[d], sc[d], false, false);
            const float ku = scale_of(both[0]);   // of K row col, in both halves
#pragma unroll
            for (int i = 0; i < NLD; ++i) {
              const uint32_t f = i * 64 + lane_o;
              *reinterpret_cast<v4u*>(ktile + codes_off<D>(f / CC, f % CC)) = kr[d][i];
              if (i >= NLV) continue;
              const uint32_t r = f / CV, cc = f % CV;
              const float vu = scale_of(uint32_t(__builtin_amdgcn_ds_bpermute(int(r * 4 + 128), int(sc[d]))));
              v4u lo, hi;
              widen_codes(vr[d][i], vu, lo, hi);
              *reinterpret_cast<v4u*>(vtile + tile_off<DV>(r, cc)) = lo;
              *reinterpret_cast<v4u*>(vtile + tile_off<DV>(r, cc + CV)) = hi;
            }
            if (j + kDepth < mine) fetch(kr[d], vr[d], sc[d], j + kDepth);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            // every operand is asked for at once, V's before the softmax that stands between
            v4u kx[NT / 2], vx[2][NDB];
            const int ko = opaque(koff);
#pragma unroll
            for (int u = 0; u < NT / 2; ++u) kx[u] = *reinterpret_cast<const v4u*>(ktile + (ko ^ (u << 5)));
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int db = 0; db < NDB; ++db) {
                const v2u lo = lds_read_tr16(vtile + vtr.off(0, db) + 16 * u * 2 * DV);
                const v2u hi = lds_read_tr16(vtile + vtr.off(1, db) + 16 * u * 2 * DV);
                vx[u][db] = v4u{lo.x, lo.y, hi.x, hi.y};
              }
            f32x16 st;
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] = 0.0f;
#pragma unroll
            for (int u = 0; u < NT / 2; ++u) {
              v4u lo, hi;
              widen_codes(kx[u], ku, lo, hi);
              st = mfma_bf16(lo, qx[2 * u], st);
              st = mfma_bf16(hi, qx[2 * u + 1], st);
            }
            v4u pb[2];
            softmax_step(st, hf, c1 - (c0 + tile * kTile), zscale, m_used, lsum, acc, pb);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int db = 0; db < NDB; ++db) acc[db] = mfma_bf16(vx[u][db], pb[u], acc[db]);
            __builtin_amdgcn_wave_barrier();
          }
        }
      }

      // ---- what this wave's columns come to, merged over the waves of its head through LDS that only they have used
      const float l = sum_across_halves(lsum);
      const int x = qt * 32 + col;
      const int qi = query_of(x);
      const int64_t row = int64_t(sg.q0 + qi) * s.hq + h0 + (x - qi * heads);
      // elements 4 * u .. of the columns' output (u in the accumulators' order), times l_all
      auto store = [&](int u, float4 a, float m_all, float l_all, float inv) {
        const int at = part * DV + placed<DV>(u) * 8 + 4 * hf;
        if (x >= ncols) return;
        if (!Pieces || sg.parts == 1) {
          *reinterpret_cast<v2u*>(o + row * D + at) = v2u{cvt_pk_bf16(a.x * inv, a.y * inv), cvt_pk_bf16(a.z * inv, a.w * inv)};
        } else {
          // (pieces and sequences only ever go up along a head's lists, so px + b numbers the segments)
          const int64_t slot = (int64_t(px + sg.b) * s.max_q + qi) * s.hq + h0 + (x - qi * heads);
          *reinterpret_cast<float4*>(po + slot * D + at) = a;
          if (u == 0 && hf == 0) pml[slot] = make_float2(m_all, l_all);
        }
      };
      if constexpr (SP == 1) {
        const float inv = 1.0f / l;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4)
            store(db * 4 + i4, make_float4(acc[db][4 * i4 + 0], acc[db][4 * i4 + 1], acc[db][4 * i4 + 2], acc[db][4 * i4 + 3]),
                  m_used, l, inv);
      } else {
        float* sm_ml = reinterpret_cast<float*>(&sm_rows[0][0]);   // [wave][m: 32 | l: 32], row stride kMl
        if (hf == 0) {
          sm_ml[wave * kMl + col] = m_used;
          sm_ml[wave * kMl + 32 + col] = l;
        }
        float4* mrg = reinterpret_cast<float4*>(&lds[0][0]);
        constexpr int kMrgWave = WAVEB / 16;
        static_assert(NDB * 4 * 64 <= kMrgWave, "a wave's accumulators fit its tile buffers");
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4)
            mrg[wave * kMrgWave + (db * 4 + i4) * 64 + lane] =
                make_float4(acc[db][4 * i4 + 0], acc[db][4 * i4 + 1], acc[db][4 * i4 + 2], acc[db][4 * i4 + 3]);
        __syncthreads();
        constexpr int NU = NDB * 4 / SP;
        static_assert(NDB * 4 % SP == 0, "the waves split the output evenly");
        const int w0 = wave - span;
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < SP; ++w) m_all = fmaxf(m_all, sm_ml[(w0 + w) * kMl + col]);
        float f[SP];
        float l_all = 0.0f;
#pragma unroll
        for (int w = 0; w < SP; ++w) {
          f[w] = __builtin_amdgcn_exp2f(sm_ml[(w0 + w) * kMl + col] - m_all);   // 0 for a wave that saw no tile
          l_all += sm_ml[(w0 + w) * kMl + 32 + col] * f[w];
        }
        const float inv = 1.0f / l_all;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
          const int u = span * NU + n;
          float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int w = 0; w < SP; ++w) {
            const float4 y = mrg[(w0 + w) * kMrgWave + u * 64 + lane];
            a.x += y.x * f[w]; a.y += y.y * f[w]; a.z += y.z * f[w]; a.w += y.w * f[w];
          }
          store(u, a, m_all, l_all, inv);
        }
        __syncthreads();   // merge space becomes tile space again
      }
    }
    if constexpr (!Pieces) break;
    else {
      if (sg.k0 + sg.c1 >= end) break;
      enter(sg.b + 1);   // (there is one: the piece goes on)
    }
  }
}

// Merges the parts of every list that a cut went through: one thread per four output elements, the parts of four pieces asked
// for at once, and PG groups of threads that share out the parts of a row where there are many (few rows, then).
template <int D, int PG>
__global__ __launch_bounds__(256) void merge_pieces_kernel(const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k,
                                                           const float* __restrict__ po, const float2* __restrict__ pml,
                                                           uint16_t* __restrict__ o, int32_t piece, Shape s DLLM_CHECK_PARAM) {
  DLLM_CHECK_EXIT();
  constexpr int TPR = D / 4, ROWS = 256 / TPR / PG;   // threads per output row and group, rows per workgroup and turn
  __shared__ float4 sm_a[PG > 1 ? 256 : 1];
  __shared__ float2 sm_ml[PG > 1 ? 256 : 1];
  const int b = blockIdx.y;
  const int k0 = cu_k[b], k1 = cu_k[b + 1], q0 = cu_q[b], n = (cu_q[b + 1] - q0) * s.hq;
  const int fp = int(uint32_t(k0) / uint32_t(piece)), parts = k1 > k0 ? int(uint32_t(k1 - 1) / uint32_t(piece)) - fp + 1 : 0;
  if (parts <= 1) return;
  const int sub = threadIdx.x % TPR, pg = threadIdx.x / TPR % PG;
  const int64_t pitch = int64_t(s.max_q) * s.hq;   // slot of part p: base + row + p * pitch
  const int64_t base = (int64_t(fp) + b) * pitch;
  for (int i0 = blockIdx.x * ROWS; i0 < n; i0 += gridDim.x * ROWS) {
    const int i = i0 + int(threadIdx.x) / (TPR * PG);
    const int64_t row = min(i, n - 1);
    float m_all = -INFINITY, l_all = 0.0f;
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int p0 = 4 * pg; p0 < parts; p0 += 4 * PG) {
      float2 ml[4];
      float4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {   // past the last part: that part again, with no weight
        const int64_t slot = base + row + min(p0 + u, parts - 1) * pitch;
        ml[u] = pml[slot];
        x[u] = *reinterpret_cast<const float4*>(po + slot * D + sub * 4);
      }
      float m_new = m_all;
#pragma unroll
      for (int u = 0; u < 4; ++u) m_new = fmaxf(m_new, ml[u].x);
      const float old = __builtin_amdgcn_exp2f(m_all - m_new);   // first round: exp2(-inf) = 0
      l_all *= old;
      a.x *= old; a.y *= old; a.z *= old; a.w *= old;
      m_all = m_new;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float w = p0 + u < parts ? __builtin_amdgcn_exp2f(ml[u].x - m_all) : 0.0f;
        l_all += ml[u].y * w;
        a.x += x[u].x * w; a.y += x[u].y * w; a.z += x[u].z * w; a.w += x[u].w * w;
      }
    }
    if constexpr (PG > 1) {
      sm_a[threadIdx.x] = a;
      sm_ml[threadIdx.x] = make_float2(m_all, l_all);
      __syncthreads();
      const int first = threadIdx.x - pg * TPR;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < PG; ++w) m = fmaxf(m, sm_ml[first + w * TPR].x);
      a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      l_all = 0.0f;
#pragma unroll
      for (int w = 0; w < PG; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm_ml[first + w * TPR].x - m);   // 0 for a group without parts
        const float4 y = sm_a[first + w * TPR];
        l_all += sm_ml[first + w * TPR].y * f;
        a.x += y.x * f; a.y += y.y * f; a.z += y.z * f; a.w += y.w * f;
      }
      __syncthreads();
    }
    if (i < n && pg == 0) {
      const float inv = 1.0f / l_all;
      *reinterpret_cast<v2u*>(o + (int64_t(q0) * s.hq + row) * D + sub * 4) =
          v2u{cvt_pk_bf16(a.x * inv, a.y * inv), cvt_pk_bf16(a.z * inv, a.w * inv)};
    }
  }
}

// How a call's rows are shared out: in pieces of `piece` rows, or (0) a list per workgroup.
struct CachePlan {
  int32_t piece, n_pieces;   // per head
  int32_t side;              // KV heads per workgroup
  int32_t v_split;           // workgroups that share the columns of V
  int64_t groups;            // workgroups that share the column tiles of a sequence
  int order;
};
// Pieces are cut for one workgroup per compute unit at head_dim 128, two at 64.
static int64_t pieces_per_head(const Shape& s, int64_t units) {
  return std::max<int64_t>(1, (s.d == 128 ? kUnits : 2 * kUnits) / units);
}
// Lists whole or in pieces: the less of two sums, in us, from these measurements.
//   A workgroup alone on its unit takes 7.0 ns per row (head_dim 64: 4.6, whole lists in order 6.0; with half of V 0.78 of that,
//   with a quarter 0.72), two on one unit 0.7 of their sum; where there are more than two, every one takes 4.5 us beside its
//   rows. The card reads gathered rows at 4.9 TB/s (the rates at the top of the file are lower: they count what a call needs beside
//   its rows), rows in order at 5.0, at 6.2 with heads side by side, at 4.2 where every list
//   is a workgroup's own (3.5 where two share V's columns; 64-byte rows two thirds of all that; it includes starting and
//   draining). Without lists every column tile reads the rows again, from the caches, in pieces at 6.6 TB/s. Pieces cost a second
//   launch and its latencies (3.3), what is written and read again (2.75 TB/s, without lists 3.5), and for the further sequences
//   that a piece reaches into 1.4 each with lists, in the mean, 2.5 without, in the piece that has most.
// One sequence of 8000 rows, single tokens, 32 heads over 8 x 128: whole 66.7, in pieces 10.4; of 2000 rows 15.5 / 9.4; 32 of
// 4000 to 8192 79.2 / 67.2; 16 of 1000 12.2 / 17.4; 40 of 100 to 1000 16.1 / 19.4; lists of 32 heads x 128, one of 4096 rows 25.9
// / 14.5, of 1024 10.7 / 10.0, of 256 5.7 / 9.5; four of 276 to 994 11.3 / 16.9; sixteen of 5 to 50 % of 512 to 4096 23.3 / 36.3.
// Over 700 batches, 1 to 40 sequences of 128 to 8192, the choice is 0.3 % above the better one in the mean, 43 % at most (single
// tokens of 25 sequences of 3440, 4 heads x 64, 25.7 against 18.0).
static bool better_in_pieces(const Shape& s, bool lists, int64_t heads, int64_t cols, int64_t tiles, int64_t max_k, int64_t total_k,
                             int64_t piece, int64_t side, int32_t v_split) {
  const double row_us = s.d == 128 ? 7.0e-3 : 4.6e-3, units = double(heads * tiles), n = double((total_k + piece - 1) / piece);
  const double read = double(total_k) * heads * 2 * s.d / (lists ? 4.9e6 : 5.0e6) * (s.d == 128 ? 1.0 : 1.5);
  const double whole_row_us = lists || s.d == 128 ? row_us : 6.0e-3, wgs = units * s.batch;
  double whole = max_k * whole_row_us * (v_split == 4 ? 0.72 : v_split == 2 ? 0.78 : 1.0);
  if (wgs > kUnits) whole = std::max(whole, total_k * units / kUnits * row_us * 0.7);
  whole = std::max(whole, lists ? read : read * 1.2 * tiles * (v_split == 2 ? 1.2 : 1.0));
  if (!lists && wgs > 2 * kUnits) whole = std::max(whole, wgs / (2 * kUnits) * (4.5 + double(total_k) / s.batch * row_us * 1.4));
  double cut = piece * side * row_us;
  if (units / side * n > kUnits) cut *= s.d == 128 ? 1.4 : 1.3;
  cut = std::max(cut, !lists && tiles > 1 ? read * tiles * 5.0 / 6.6 : side > 1 ? read * 5.0 / 6.2 : read) + 3.3;
  if (s.batch > 1) cut += lists ? 1.4 * (s.batch - 1) / n : 2.5 * std::max(1.0, (s.batch - 1) / n);
  cut += std::min(n + s.batch, 2 * n) * units * std::min<int64_t>(32, cols) * s.d * 8 / (lists ? 2.75e6 : 3.5e6);
  return cut < whole;
}
// Where there are many column tiles, as many workgroups as fill the card four times share them out, so that units that get short
// lists take more of them: 32 heads x 128, 5 to 50 % of 500 to 4000 positions, once / four times, longest first: 8 sequences of
// 128 queries 53.4 / 42.6 us, of 256 101.7 / 77.3, 4 of 1024 182 / 136.
static int64_t column_groups(int64_t wgs, int64_t tiles) {
  return std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(tiles, 65535), 8 * kUnits / std::max<int64_t>(1, wgs)));
}
// Workgroups that share V's columns where lists are whole (see attend_cache_kernel): as many as leave no unit two of them.
static int32_t v_split_of(const Shape& s, int64_t wgs) {
  return s.d == 128 && 4 * wgs <= kUnits ? 4 : 2 * wgs <= kUnits ? 2 : 1;
}
static CachePlan plan_attend_cached(const Shape& s, bool lists, int32_t max_k, int64_t total_k) {
  CachePlan p{};
  total_k = std::min<int64_t>(total_k, int64_t(s.batch) * max_k);
  const int64_t heads = lists ? s.hq : s.hkv, cols = lists ? s.max_q : int64_t(s.max_q) * s.group;
  const int64_t tiles = std::max<int64_t>(1, (cols + 31) / 32), units = heads * tiles, resident = 2 * kUnits;
  const int32_t v_split = v_split_of(s, heads * s.batch * column_groups(heads * s.batch, tiles));
  p.side = 1;
  if (max_k > 0) {
    auto piece_for = [&](int64_t side) {
      const int64_t n = pieces_per_head(s, units / side), share = (total_k + n - 1) / n;
      return std::max<int64_t>(128, (share + 31) / 32 * 32);
    };
    int64_t piece = piece_for(1);
    if (!lists && s.hkv % kSide == 0 && tiles <= 4 && piece_for(kSide) >= (s.d == 128 ? 160 : 512)) {
      p.side = kSide;
      piece = piece_for(kSide);
    }
    // (the ids of a list's rows lie in LDS: no workgroup takes more than kMaxListRows of them, whole or in pieces)
    bool cut = lists && max_k > kMaxListRows;
    if (!cut && !(lists && piece > kMaxListRows))
      cut = better_in_pieces(s, lists, heads, cols, tiles, max_k, total_k, piece, p.side, v_split);
    if (lists) piece = std::min<int64_t>(piece, kMaxListRows);
    if (cut) {
      p.piece = int32_t(std::min<int64_t>(piece, INT32_MAX));
      p.n_pieces = int32_t((total_k + p.piece - 1) / p.piece);
    }
  }
  const int64_t wgs = p.piece ? heads / p.side * p.n_pieces : heads * s.batch;
  p.groups = column_groups(wgs, tiles);
  p.v_split = p.piece ? 1 : v_split;
  if (!p.piece && s.batch <= kRankBatch) {
    if (wgs * p.groups > resident) p.order = kLongestFirst;
    else if (wgs > kUnits && p.groups == 1) p.order = kFolded;
  }
  return p;
}
int32_t attend_cached_piece(const Shape& s, bool lists, int32_t max_k, int32_t total_k) {
  return plan_attend_cached(s, lists, max_k, total_k).piece;
}
static size_t partial_slots(const Shape& s, int64_t n_pieces) {
  return size_t(n_pieces + s.batch) * size_t(s.max_q) * size_t(s.hq);
}

size_t attend_cached_workspace(const Shape& s, int32_t max_k) {
  if (max_k == 0 || s.max_q == 0) return 0;
  const int64_t tiles = (int64_t(s.max_q) + 31) / 32, group_tiles = (int64_t(s.max_q) * s.group + 31) / 32;
  const int64_t side = s.hkv % kSide == 0 && group_tiles <= 4 ? kSide : 1;
  int64_t n = std::max(pieces_per_head(s, s.hq * tiles), pieces_per_head(s, s.hkv / side * group_tiles));
  if (max_k > kMaxListRows) n = std::max<int64_t>(n, (int64_t(s.batch) * max_k + kMaxListRows - 1) / kMaxListRows);
  const size_t slots = partial_slots(s, n);
  return align256(slots * s.d * sizeof(float)) + align256(slots * sizeof(float2));
}

hipError_t launch_attend_cached(const Shape& s, const CacheView& c, int32_t max_k, const void* q, const int32_t* cu_q,
                                const int32_t* cu_kv, const int32_t* idx, const int32_t* cu_k, int32_t total_k, void* o, void* ws,
                                hipStream_t st) {
  if (s.max_q == 0) return hipSuccess;   // no sequence has a query: nothing to write
  const bool lists = idx != nullptr;
  const CachePlan p = plan_attend_cached(s, lists, max_k, total_k);
  float* po = static_cast<float*>(ws);
  float2* pml = reinterpret_cast<float2*>(static_cast<char*>(ws) + align256(partial_slots(s, p.n_pieces) * s.d * sizeof(float)));
  const uint16_t* qh = static_cast<const uint16_t*>(q);
  uint16_t* oh = static_cast<uint16_t*>(o);
  // Without lists the heads of one piece run on one XCD if the number of pieces is a multiple of eight: their rows lie side by side.
  const unsigned heads = lists ? s.hq : p.piece ? s.hkv / p.side : s.hkv;
  const unsigned parts = !p.piece ? s.batch : lists || p.n_pieces < 8 ? p.n_pieces : (p.n_pieces + 7) / 8 * 8;
  auto launch = [&](auto kernel, bool heads_first) {
    const dim3 grid(heads_first ? heads : parts, heads_first ? parts : heads, unsigned(p.groups * p.v_split));
    kernel<<<grid, kWaves * 64, 0, st>>>(qh, c, cu_q, cu_kv, idx, cu_k, total_k, oh, po, pml, p.piece, p.order, s DLLM_CHECK_PASS);
  };
  auto with_d = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (p.piece) {
      if (lists) launch(attend_cache_kernel<D, true, true, 1, 1>, true);
      else if (p.side == kSide) launch(attend_cache_kernel<D, false, true, kSide, 1>, false);
      else launch(attend_cache_kernel<D, false, true, 1, 1>, false);
    } else {
      auto whole = [&](auto vs) {
        if (lists) launch(attend_cache_kernel<D, true, false, 1, decltype(vs)::value>, true);
        else launch(attend_cache_kernel<D, false, false, 1, decltype(vs)::value>, true);
      };
      if (p.v_split == D / 32) whole(std::integral_constant<int, D / 32>{});
      else if (p.v_split == 2) whole(std::integral_constant<int, 2>{});
      else whole(std::integral_constant<int, 1>{});
    }
  };
  if (s.d == 128) with_d(std::integral_constant<int, 128>{});
  else with_d(std::integral_constant<int, 64>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.piece) return e;
  auto merge = [&](auto kernel, int rows_per_wg) {
    const int64_t wgs = (int64_t(s.max_q) * s.hq + rows_per_wg - 1) / rows_per_wg;
    const dim3 grid(unsigned(std::min<int64_t>(wgs, std::max<int64_t>(4, 4096 / s.batch))), s.batch);
    kernel<<<grid, 256, 0, st>>>(cu_q, cu_k, po, pml, oh, p.piece, s DLLM_CHECK_PASS);
  };
  const bool many = (int64_t(max_k) + p.piece - 1) / p.piece + 1 > 8;   // parts of the longest list
  if (s.d == 128) {
    if (many) merge(merge_pieces_kernel<128, 8>, 1);
    else merge(merge_pieces_kernel<128, 1>, 8);
  } else {
    if (many) merge(merge_pieces_kernel<64, 8>, 2);
    else merge(merge_pieces_kernel<64, 1>, 16);
  }
  return hipGetLastError();
}

}  // namespace dllm
