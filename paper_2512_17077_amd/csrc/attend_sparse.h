// What the attention kernels over kept rows share (bf16 rows: attend_sparse_bf16.hip; rows of an 8-bit cache:
// attend_cache.hip): the batch's offsets in one workgroup, and the online softmax of one 32-row tile.
#pragma once
#include "attn_tile.h"

namespace dllm {

constexpr int kTile = 32;             // kept rows per wave tile
constexpr int kRankBatch = 64;        // batches up to this size are walked longest kept list first

// Per-sequence offsets a workgroup needs, fetched for the whole (small) batch in one round of
// loads: lane i holds sequence i's entries, and the chosen sequence's are read back by lane index.
struct SeqInfo {
  int b, ko0, kb, q0, nq, kv0;
};

// The batch's offsets as one workgroup holds them: lane i holds sequence i's entries and its rank in
// descending order of kept rows (ties: lower sequence first); every workgroup derives the same order
// from cu_k.  Batches of more than kRankBatch sequences are not ranked and read their entries per use.
struct BatchInfo {
  int ko0, kb, q0, nq, kv0, rank;
};
__device__ __forceinline__ BatchInfo load_batch(const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_kv,
                                                const int32_t* __restrict__ cu_k, int batch, int lane, bool ranked) {
  BatchInfo bi = {0, 0, 0, 0, 0, 0};
  if (batch > kRankBatch) return bi;
  const int i = lane < batch ? lane : batch - 1;
  bi.ko0 = cu_k[i]; bi.kb = cu_k[i + 1] - bi.ko0;
  bi.q0 = cu_q[i]; bi.nq = cu_q[i + 1] - bi.q0;
  bi.kv0 = cu_kv[i];
  if (ranked) {   // (rank_longest_first's longer code, skipped, still cost one layer's call 0.2 of 15 us)
    const int mine = lane < batch ? bi.kb : -1;
    int rank = 0;
    for (int j = 0; j < batch; ++j) {
      const int other = __builtin_amdgcn_readlane(mine, j);
      rank += (other > mine) || (other == mine && j < lane);
    }
    bi.rank = rank;
  }
  return bi;
}

// Sequence handled by slot z.  With `ranked` set (small batches whose workgroups do not all fit on the
// chip at once, or that are shared out by length) it is the z-th in descending order of kept rows, so
// the longest lists start first and the short ones fill the compute units that free up.
__device__ __forceinline__ SeqInfo sequence_of_slot(const BatchInfo& bi, const int32_t* __restrict__ cu_q,
                                                    const int32_t* __restrict__ cu_kv,
                                                    const int32_t* __restrict__ cu_k, int batch, int z, int lane,
                                                    bool ranked) {
  SeqInfo si;
  if (batch > kRankBatch) {
    si.b = z;
    si.ko0 = cu_k[z]; si.kb = cu_k[z + 1] - si.ko0;
    si.q0 = cu_q[z]; si.nq = cu_q[z + 1] - si.q0;
    si.kv0 = cu_kv[z];
    return si;
  }
  int b = z;
  if (ranked) b = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < batch && bi.rank == z));
  si.b = b;
  si.ko0 = __builtin_amdgcn_readlane(bi.ko0, b);
  si.kb = __builtin_amdgcn_readlane(bi.kb, b);
  si.q0 = __builtin_amdgcn_readlane(bi.q0, b);
  si.nq = __builtin_amdgcn_readlane(bi.nq, b);
  si.kv0 = __builtin_amdgcn_readlane(bi.kv0, b);
  return si;
}
__device__ __forceinline__ SeqInfo sequence_of_slot(const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_kv,
                                                    const int32_t* __restrict__ cu_k, int batch, int z, int lane,
                                                    bool ranked) {
  return sequence_of_slot(load_batch(cu_q, cu_kv, cu_k, batch, lane, ranked), cu_q, cu_kv, cu_k, batch, z, lane,
                          ranked);
}

// Online softmax of one 32-key tile: S^T (rows: keys, columns: queries) becomes the bf16 operand P^T of the product with V^T; the
// running maximum and sum of this lane's column, and the accumulators where the maximum is raised, follow.  Keys from
// nvalid on count nothing.
template <int NDB>
__device__ __forceinline__ void softmax_step(f32x16 st, int hf, int nvalid, float zscale, float& m_used, float& lsum,
                                             f32x16 (&acc)[NDB], v4u (&pb)[2]) {
  if (nvalid < kTile) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = 8 * (i / 4) + 4 * hf + (i % 4);
      if (key >= nvalid) st[i] = -INFINITY;
    }
  }
  float tmax = -INFINITY;
#pragma unroll
  for (int i = 0; i < 16; i += 2) tmax = fmaxf(fmaxf(tmax, st[i]), st[i + 1]);
  tmax = max_across_halves(tmax) * zscale;   // zscale >= 0
  if (__builtin_amdgcn_ballot_w64(tmax > m_used + kLazyGrowth) != 0) {
    const float m_new = fmaxf(m_used, tmax);
    const float alpha = __builtin_amdgcn_exp2f(m_used - m_new);   // first tile: exp2 of the lowest number, 0
    m_used = m_new;
    lsum *= alpha;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[db][i] *= alpha;
  }
  const float neg_m = -m_used;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    uint32_t w[4];
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[8 * u + 2 * jj], zscale, neg_m));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(st[8 * u + 2 * jj + 1], zscale, neg_m));
      w[jj] = cvt_pk_bf16(p0, p1);
      lsum = add_pair_bf16(w[jj], lsum);
    }
    pb[u] = v4u{w[0], w[1], w[2], w[3]};
  }
}

}  // namespace dllm
