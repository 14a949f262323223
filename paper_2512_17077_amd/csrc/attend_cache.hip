// Reuse-phase attention over a KV cache held in 8 bits (cache_kernels.hip), bf16 queries and outputs, fp32 softmax state and
// accumulators.  Two uses, one kernel:
//   Lists    every query head attends over its own kept rows (Section 2.3 Eq. 4 restricted to the kept set of Section 4.5);
//   !Lists   every head attends over the first k_b rows of its sequence (no lists: single tokens of an autoregressive
//            model, or a block over everything).  The query heads of a group then read the same rows, so a tile's 32
//            columns are (query, head of the group) pairs of one KV head and the rows are read once per group.
//
// The step is bound by HBM, with half the bytes of the bf16 kernels (attend_sparse_bf16.hip), whose structure it keeps: a
// workgroup of four waves walks one chunk of one list, each wave its own 32-row tiles without a workgroup barrier, and
// what decides is how many rows are in flight.  A tile of codes takes half the registers of a bf16 tile, so a wave keeps
// kDepth tiles ahead.  Codes are converted on their way from the registers to the wave's LDS tile: code * 2^e is a bf16
// value exactly (one conversion instruction per two, which applies the scale too), so from there on the arithmetic is that
// of a bf16 cache, and so is its precision: probabilities are rounded to bf16 for the product with V, outputs once at the end.
// Scales are bytes, one per row of a tile and tensor: lane l fetches that of K row l % 32 (V: lanes 32 to 63) together with
// the rows, and the lanes that convert a row get it by a lane exchange.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "attend_sparse.h"

namespace dllm {

constexpr int kWaves = 4;
constexpr int kMaxChunkRows = 2048;   // kept rows of a list that one workgroup walks at most (their ids lie in LDS)

typedef __attribute__((ext_vector_type(2))) __bf16 bf2;

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

// QG: a sequence's column tiles are shared out to several workgroups (blockIdx.z counts sequences, then groups of tiles)
template <int D, bool Lists, bool QG>
__global__ __launch_bounds__(kWaves * 64, 2) void attend_cache_kernel(
    const uint16_t* __restrict__ q, CacheView c, const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_kv,
    const int32_t* __restrict__ idx, const int32_t* __restrict__ cu_k, int32_t total_k, uint16_t* __restrict__ o,
    float* __restrict__ po, float* __restrict__ pm, float* __restrict__ pl, int32_t chunk_rows, int ranked,
    Shape s DLLM_CHECK_PARAM) {
  DLLM_CHECK_EXIT();
  constexpr int CH = D / 8;             // 16-byte chunks of a bf16 row
  constexpr int CC = D / 16;            // ... of a row of codes
  constexpr int TILEB = kTile * 2 * D;
  constexpr int NLD = kTile * CC / 64;  // 16-byte loads per lane, tile and tensor
  constexpr int NDB = D / 32;
  constexpr int W = kWaves;
  constexpr int MAXT = kMaxChunkRows / (W * kTile);
  constexpr int kDepth = D == 128 ? 2 : 4;   // tiles in flight per wave
  constexpr int kMl = Lists ? MAXT * kTile : 64;

  __shared__ __attribute__((aligned(16))) char lds[W][2 * TILEB];   // per wave: K tile, V tile; merge space afterwards
  __shared__ __attribute__((aligned(16))) char qtile[TILEB];
  __shared__ int sm_rows[W][kMl];   // kept-row ids of each wave's tiles; (m, l) at the merge

  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int col = lane & 31, hf = lane >> 5;
  const int chunk = blockIdx.x;
  int slot = blockIdx.z, qt0 = 0, qstep = 1;
  if constexpr (QG) {
    qt0 = slot / s.batch;
    slot -= qt0 * s.batch;
    qstep = int(gridDim.z) / s.batch;
  }
  const SeqInfo si = sequence_of_slot(cu_q, cu_kv, cu_k, s.batch, slot, lane, ranked != 0);
  const int kb = si.kb, q0 = si.q0, nq = si.nq, kv0 = si.kv0;
  const ChunkGeom cg = chunk_geom(kb, chunk_rows);
  const int c0 = chunk * cg.rows;
  if (c0 >= kb && !(chunk == 0 && kb == 0)) return;
  const int c1 = min(kb, c0 + cg.rows);
  const int h0 = Lists ? int(blockIdx.y) : int(blockIdx.y) * s.group;   // first query head
  const int g = Lists ? h0 / s.group : int(blockIdx.y);
  const int heads = Lists ? 1 : s.group;
  const int ncols = nq * heads;
  if (qt0 * 32 >= ncols) return;
  // column x of this workgroup: query x / heads, head h0 + x % heads
  auto query_of = [&](int x) { return Lists ? x : int(uint32_t(x) / uint32_t(heads)); };
  if (kb == 0) {   // nothing kept: defined as zeros
    if (qt0 == 0)
      for (int e = threadIdx.x; e < ncols * D; e += W * 64) {
        const int x = e / D, i = query_of(x);
        o[(int64_t(q0 + i) * s.hq + h0 + (x - i * heads)) * D + e % D] = 0;
      }
    return;
  }

  const int32_t* __restrict__ rows = idx + int64_t(h0) * total_k + si.ko0;
  const uint8_t* kbase = c.k + int64_t(kv0) * c.tok + int64_t(g) * c.head;
  const uint8_t* vbase = c.v + int64_t(kv0) * c.tok + int64_t(g) * c.head;
  const int64_t scale0 = g * c.scale_head + scale_slot(kv0, si.b, c.shift);
  const uint8_t* sbase = (hf == 0 ? c.ks : c.vs) + scale0;
  const uint32_t pitch = uint32_t(c.tok);   // a sequence's rows span < 4 GiB (checked on the host)
  const float zscale = s.scale * kLog2e;
  const int ntiles = (c1 - c0 + kTile - 1) / kTile;
  char* ktile = lds[wave];
  char* vtile = lds[wave] + TILEB;
  KAddr<D> ka;
  ka.init(lane);
  VtAddr<D> vt;
  vt.init(lane);
  const uint32_t coff = (lane % CC) * 16;
  auto opaque = [](int x) {
    asm volatile("" : "+v"(x));
    return x;
  };

  for (int qt = qt0; qt * 32 < ncols; qt += qstep) {
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
        const int t = min(c0 + (wave + (p >> 5) * W) * kTile + (p & 31), c1 - 1);
        my_rows[p] = rows[t];
      }
    }
    constexpr int NQL = (kTile * CH + W * 64 - 1) / (W * 64);
    v4u qx[NQL];
#pragma unroll
    for (int i = 0; i < NQL; ++i) {
      const int f = i * W * 64 + threadIdx.x, r = f / CH, x = qt * 32 + r;
      qx[i] = v4u{0u, 0u, 0u, 0u};
      if (r < kTile && x < ncols) {
        const int qi = query_of(x);
        qx[i] = *reinterpret_cast<const v4u*>(q + int64_t(q0 + qi) * s.q_tok + int64_t(h0 + (x - qi * heads)) * s.q_head +
                                              (f % CH) * 8);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

    v4u kr[kDepth][NLD], vr[kDepth][NLD];
    uint32_t sc[kDepth];
    // row `r` (0 .. 31) of the wave's j-th tile
    auto row_of = [&](int j, int r) {
      return Lists ? my_rows[j * kTile + r] : min(c0 + (wave + j * W) * kTile + r, c1 - 1);
    };
    auto fetch = [&](v4u (&kx)[NLD], v4u (&vx)[NLD], uint32_t& sx, int j) {
      sx = sbase[uint32_t(row_of(j, col)) >> c.shift];
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const uint32_t off = __umul24(uint32_t(row_of(j, (i * 64 + lane) / CC)), pitch) + coff;
        kx[i] = load_once(kbase + off);
        vx[i] = load_once(vbase + off);
      }
    };
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
      if (wave + d * W < ntiles) fetch(kr[d], vr[d], sc[d], d);
#pragma unroll
    for (int i = 0; i < NQL; ++i) {
      const int f = i * W * 64 + threadIdx.x, r = f / CH;
      if (r < kTile) *reinterpret_cast<v4u*>(qtile + tile_off<D>(r, f % CH)) = qx[i];
    }
    __syncthreads();   // the queries are in place
    for (int j0 = 0; wave + j0 * W < ntiles; j0 += kDepth) {
#pragma unroll
      for (int d = 0; d < kDepth; ++d) {
        const int j = j0 + d, tile = wave + j * W;
        if (tile < ntiles) {
          KAddr<D> kar;
          kar.base = opaque(ka.base);
          VtAddr<D> vtr;
          vtr.base[0] = opaque(vt.base[0]);
          vtr.base[1] = opaque(vt.base[1]);
          const int lane_o = opaque(lane);
#pragma unroll
          for (int i = 0; i < NLD; ++i) {
            const int f = i * 64 + lane_o, r = f / CC, cc = f % CC;
            const float ku = scale_of(uint32_t(__builtin_amdgcn_ds_bpermute(r * 4, int(sc[d]))));
            const float vu = scale_of(uint32_t(__builtin_amdgcn_ds_bpermute(r * 4 + 128, int(sc[d]))));
            v4u lo, hi;
            widen_codes(kr[d][i], ku, lo, hi);
            *reinterpret_cast<v4u*>(ktile + tile_off<D>(r, 2 * cc)) = lo;
            *reinterpret_cast<v4u*>(ktile + tile_off<D>(r, 2 * cc + 1)) = hi;
            widen_codes(vr[d][i], vu, lo, hi);
            *reinterpret_cast<v4u*>(vtile + tile_off<D>(r, 2 * cc)) = lo;
            *reinterpret_cast<v4u*>(vtile + tile_off<D>(r, 2 * cc + 1)) = hi;
          }
          if (tile + kDepth * W < ntiles) fetch(kr[d], vr[d], sc[d], j + kDepth);
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
          sparse_tile_math<D>(ktile, vtile, qtile, kar, vtr, hf, c1 - (c0 + tile * kTile), zscale, m_used, lsum, acc);
          __builtin_amdgcn_wave_barrier();
        }
      }
    }

    // ---- merge the waves' (m, l, O^T) through LDS that only they have used (as in attend_sparse_bf16_kernel)
    const float l = sum_across_halves(lsum);
    float* sm_ml = reinterpret_cast<float*>(&sm_rows[0][0]);   // [wave][m: 32 | l: 32], row stride kMl
    if (hf == 0) {
      sm_ml[wave * kMl + col] = m_used;
      sm_ml[wave * kMl + 32 + col] = l;
    }
    float4* mrg = reinterpret_cast<float4*>(&lds[0][0]);
    constexpr int kMrgWave = 2 * TILEB / 16;
    static_assert(NDB * 4 * 64 <= kMrgWave, "a wave's accumulators fit its tile buffers");
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4)
        mrg[wave * kMrgWave + (db * 4 + i4) * 64 + lane] =
            make_float4(acc[db][4 * i4 + 0], acc[db][4 * i4 + 1], acc[db][4 * i4 + 2], acc[db][4 * i4 + 3]);
    __syncthreads();
    {
      constexpr int PARTS = W / NDB, NQ4 = 4 / PARTS;
      static_assert(W % NDB == 0 && 4 % PARTS == 0, "the waves split the output evenly");
      const int db = wave % NDB, i4_0 = (wave / NDB) * NQ4;
      float m_all = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) m_all = fmaxf(m_all, sm_ml[w * kMl + col]);
      float f[W];
      float l_all = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        f[w] = __builtin_amdgcn_exp2f(sm_ml[w * kMl + col] - m_all);   // 0 for a wave that saw no tile
        l_all += sm_ml[w * kMl + 32 + col] * f[w];
      }
      const int x = qt * 32 + col;
      const int qi = query_of(x);
      const int64_t row = int64_t(q0 + qi) * s.hq + h0 + (x - qi * heads);
      const float inv = 1.0f / l_all;
#pragma unroll
      for (int n = 0; n < NQ4; ++n) {
        float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const float4 y = mrg[w * kMrgWave + (db * 4 + i4_0 + n) * 64 + lane];
          a.x += y.x * f[w]; a.y += y.y * f[w]; a.z += y.z * f[w]; a.w += y.w * f[w];
        }
        const int at = db * 32 + 8 * (i4_0 + n) + 4 * hf;
        if (x < ncols) {
          if (cg.n == 1) {
            *reinterpret_cast<v2u*>(o + row * D + at) = v2u{cvt_pk_bf16(a.x * inv, a.y * inv), cvt_pk_bf16(a.z * inv, a.w * inv)};
          } else {
            const int64_t part = int64_t(chunk) * s.total_q * s.hq + row;
            *reinterpret_cast<float4*>(po + part * D + at) = a;
            if (n == 0 && wave == 0 && hf == 0) { pm[part] = m_all; pl[part] = l_all; }
          }
        }
      }
    }
    if ((qt + qstep) * 32 < ncols) __syncthreads();   // merge space becomes tile space again
  }
}

// How a call's rows are shared out over the compute units (see plan_attend, whose sums these are with this kernel's rates).
static AttendPlan plan_attend_cached(const Shape& s, bool lists, int32_t max_k) {
  AttendPlan p{};
  p.chunk_rows = max_k > 0 ? max_k : 1;
  p.n_chunks = 1;
  p.max_k = max_k;
  p.v_split = 1;
  if (max_k > 0) {
    const int64_t heads = lists ? s.hq : s.hkv, cols = lists ? s.max_q : int64_t(s.max_q) * s.group;
    const int64_t units = int64_t(s.batch) * heads * std::max<int64_t>(1, (cols + 31) / 32);
    int64_t n = std::max<int64_t>(1, 512 / std::max<int64_t>(1, units));
    n = std::max<int64_t>(1, std::min<int64_t>(n, max_k / 256));
    p.chunk_rows = int32_t(((max_k + n - 1) / n + 127) / 128 * 128);
    if (lists) p.chunk_rows = std::min(p.chunk_rows, kMaxChunkRows);
    p.n_chunks = int32_t((int64_t(max_k) + p.chunk_rows - 1) / p.chunk_rows);
  }
  if (p.n_chunks > 1) {
    const size_t slots = size_t(p.n_chunks) * size_t(s.total_q) * size_t(s.hq);
    p.off_po = 0;
    p.off_pm = align256(slots * s.d * sizeof(float));
    p.off_pl = p.off_pm + align256(slots * sizeof(float));
    p.bytes = p.off_pl + align256(slots * sizeof(float));
  }
  return p;
}

size_t attend_cached_workspace(const Shape& s, int32_t max_k) {
  return std::max(plan_attend_cached(s, true, max_k).bytes, plan_attend_cached(s, false, max_k).bytes);
}

hipError_t launch_attend_cached(const Shape& s, const CacheView& c, int32_t max_k, const void* q, const int32_t* cu_q,
                                const int32_t* cu_kv, const int32_t* idx, const int32_t* cu_k, int32_t total_k, void* o, void* ws,
                                hipStream_t st) {
  if (s.max_q == 0) return hipSuccess;   // no sequence has a query: nothing to write
  const AttendPlan p = plan_attend_cached(s, idx != nullptr, max_k);
  char* w = static_cast<char*>(ws);
  float* po = p.n_chunks > 1 ? reinterpret_cast<float*>(w + p.off_po) : nullptr;
  float* pm = p.n_chunks > 1 ? reinterpret_cast<float*>(w + p.off_pm) : nullptr;
  float* pl = p.n_chunks > 1 ? reinterpret_cast<float*>(w + p.off_pl) : nullptr;
  const uint16_t* qh = static_cast<const uint16_t*>(q);
  uint16_t* oh = static_cast<uint16_t*>(o);
  const bool lists = idx != nullptr;
  const int64_t heads = lists ? s.hq : s.hkv, cols = lists ? s.max_q : int64_t(s.max_q) * s.group;
  const int64_t units = int64_t(p.n_chunks) * heads * s.batch, tiles = (cols + 31) / 32;
  const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(tiles, 65535 / s.batch), 512 / units));
  const dim3 grid(p.n_chunks, unsigned(heads), unsigned(s.batch * groups));
  const int ranked = units * groups > 512 ? 1 : 0;
  auto launch = [&](auto kernel) {
    kernel<<<grid, kWaves * 64, 0, st>>>(qh, c, cu_q, cu_kv, idx, cu_k, total_k, oh, po, pm, pl, p.chunk_rows, ranked,
                                         s DLLM_CHECK_PASS);
  };
  auto with_d = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (lists) {
      if (groups > 1) launch(attend_cache_kernel<D, true, true>);
      else launch(attend_cache_kernel<D, true, false>);
    } else {
      if (groups > 1) launch(attend_cache_kernel<D, false, true>);
      else launch(attend_cache_kernel<D, false, false>);
    }
  };
  if (s.d == 128) with_d(std::integral_constant<int, 128>{});
  else with_d(std::integral_constant<int, 64>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_chunks <= 1) return e;
  return launch_merge_chunks(s, p, cu_q, cu_k, nullptr, po, pm, pl, oh, st);
}

}  // namespace dllm
