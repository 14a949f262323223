// The 8-bit KV cache: rows are quantised as they are written, and read back.
//
// An element is stored as an e4m3 code (sign, 4 exponent bits, 3 fraction bits, largest value 448), and a block of T
// tokens of one sequence and KV head shares a scale u, K and V apart: x stands as x^ = code * u.  u is a power of two,
//     u = 2^e with the least e such that  max |x| over the block <= 448 * 2^e,
// stored as the byte e + 127.  A code is floating point itself: its relative error, 2^-4 at most, is the same wherever
// between 224 and 448 the largest code lies, so a finer scale would only add up to one binade of tiny values; and with a
// power of two x / u and code * u are exact, x^ is a bf16 value as it stands (selection and attention convert codes to
// bf16 or fp32 without a rounding), and rows that stay in a block whose scale grows move to the new one without a second
// rounding (but where they fall below 2^-6 * u).
//
// Both kernels only move data: bytes in and out decide.  One wave takes one block of one head of K or of V, so that the maximum
// needs no workgroup barrier and all rows of the block are in flight at once; the four waves of a workgroup take neighbouring
// heads, whose rows are neighbours in memory.  Measured (MI355X, 32 heads x 128, a plain copy 5.2 TB/s): 16 sequences of 512 to
// 4096 rows written from bf16, 847 MB in and out, 146 us, 5.8 TB/s; 8 of 2048 read back, 403 MB, 70 us, 5.7 TB/s; a block of 32
// rows 5.5 us, the time of a launch.
#include <type_traits>

#include "common.h"

namespace dllm {

constexpr int kCacheWaves = 4;
constexpr uint32_t kLeastScale = 32;    // 2^-95: the least code, 2^-9 of it, is a normal fp32 number
constexpr uint32_t kMostScale = 246;    // 2^119: 448 of it is representable
constexpr uint32_t kMostStored = 0x7f600000u;   // 448 * 2^119, as fp32 bits

typedef __attribute__((ext_vector_type(2))) short s16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) float f2;

// What a wave works on: block `blk` of sequence b, KV head g, of K or V; rows lo .. hi-1 of the sequence are moved.
struct CacheJob {
  bool none;
  bool is_v;
  int g, kv0, L, first, lo, hi;   // first: the block's first row; lo, hi: the moved rows of this block
  int64_t row0;                   // of the moved rows' tensor: its row for sequence position 0
  int64_t slot;
};
__device__ __forceinline__ CacheJob cache_job(const Shape& s, const CacheView& c, const RowRange& r,
                                              const int32_t* __restrict__ cu_kv, int groups) {
  CacheJob j;
  const int b = blockIdx.y;
  const int part = int(blockIdx.x) % groups, nth = int(blockIdx.x) / groups;
  const int unit = part * kCacheWaves + __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));   // K heads, then V heads
  j.kv0 = cu_kv[b];
  j.L = cu_kv[b + 1] - j.kv0;
  int at = 0, n = j.L;
  j.row0 = j.kv0;
  if (r.cu_rows != nullptr) {
    const int c0 = r.cu_rows[b];
    n = r.cu_rows[b + 1] - c0;
    at = r.at != nullptr ? r.at[b] : j.L - n;
    j.row0 = int64_t(c0) - at;
  }
  const int lo = max(at, 0), hi = int(min(int64_t(at) + n, int64_t(j.L)));   // rows outside the sequence are left out
  const int blk = (lo >> c.shift) + nth;
  j.first = blk << c.shift;
  j.lo = max(lo, j.first);
  j.hi = int(min(int64_t(hi), int64_t(j.first) + (1 << c.shift)));
  j.none = unit >= 2 * s.hkv || n <= 0 || j.lo >= j.hi;
  j.is_v = unit >= s.hkv;
  j.g = j.is_v ? unit - s.hkv : unit;
  j.slot = j.g * c.scale_head + scale_slot(j.kv0, b, c.shift) + blk;
  return j;
}

// Largest of x over the wave, the same in all lanes: the steps of wave_inclusive_sum, with the maximum (a lane without a source
// adds zero, the least).
template <int Ctrl, int RowMask>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  return max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), Ctrl, RowMask, 0xf, false)));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = dpp_max<0x111, 0xf>(x);
  x = dpp_max<0x112, 0xf>(x);
  x = dpp_max<0x114, 0xf>(x);
  x = dpp_max<0x118, 0xf>(x);
  x = dpp_max<0x142, 0xa>(x);
  x = dpp_max<0x143, 0xc>(x);
  return uint32_t(__builtin_amdgcn_readlane(int(x), 63));
}
// the larger of the two halves' magnitudes, kept in both halves of `most`
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t most, uint32_t x) {
  const u16x2 m = __builtin_elementwise_max(__builtin_bit_cast(u16x2, most), __builtin_bit_cast(u16x2, x & 0x7fff7fffu));
  return __builtin_bit_cast(uint32_t, m);
}
// byte of the least 2^e with value <= 448 * 2^e; `bits`: a finite fp32 number's, sign cleared
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  if (bits == 0) return 0;
  const int c = int(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return uint32_t(min(max(c, int(kLeastScale)), int(kMostScale)));
}
// one value in e4m3; NaN and infinities become NaN, what stands above 448 becomes 448
__device__ __forceinline__ uint32_t encode_any(float x, float inv) {
  const uint32_t bits = __float_as_uint(x);
  const uint32_t sign = (bits >> 24) & 0x80u;
  if ((bits & 0x7fffffffu) >= 0x7f800000u) return sign | 0x7fu;
  const float y = fminf(fabsf(x) * inv, 448.0f);
  return sign | (uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false)) & 0xffu);
}

// ES: bytes per element of the rows (2 = bf16, 4 = fp32); T: tokens per scale
template <int ES, int D, int T>
__global__ __launch_bounds__(kCacheWaves * 64) void cache_write_kernel(const char* __restrict__ k, const char* __restrict__ v,
                                                                     const int32_t* __restrict__ cu_kv, int groups,
                                                                     RowRange r, CacheView c, Shape s DLLM_CHECK_PARAM) {
  DLLM_CHECK_EXIT();
  constexpr int CH = D * ES / 16;         // 16-byte chunks of a source row
  constexpr int NLD = T * CH / 64;        // of the block, per lane
  static_assert(NLD >= 1 && T * CH % 64 == 0, "whole loads");
  const CacheJob j = cache_job(s, c, r, cu_kv, groups);
  if (j.none) return;
  const int lane = threadIdx.x & 63, chunk = lane % CH;
  const char* src = (j.is_v ? v : k) + (j.row0 * s.kv_tok + int64_t(j.g) * s.kv_head) * ES + chunk * 16;
  uint8_t* scale = (j.is_v ? c.vs : c.ks) + j.slot;
  uint8_t* dst = (j.is_v ? c.v : c.k) + int64_t(j.kv0) * c.tok + int64_t(j.g) * c.head;
  const int64_t pitch = s.kv_tok * ES;
  const int block_end = min(j.first + T, j.L);
  const bool keeps = j.lo > j.first || j.hi < block_end;   // rows of this block stay as they are
  const uint32_t old = keeps ? *scale : 0u;

  v4u x[NLD];
#pragma unroll
  for (int i = 0; i < NLD; ++i) {
    const int row = j.first + (i * 64 + lane) / CH;
    x[i] = load_once(src + min(max(row, j.lo), j.hi - 1) * pitch);   // outside: a row of the block again, never stored
  }
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < NLD; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (ES == 2) most = max_abs_bf16x2(most, x[i][e]);
      else most = max(most, x[i][e] & 0x7fffffffu);
    }
  if constexpr (ES == 2) most = max(most << 16, most & 0xffff0000u);
  most = wave_max(most);
  const bool any = most > kMostStored;   // infinities, NaN or more than the format holds: one value at a time
  if (any) {
    most = 0;
#pragma unroll
    for (int i = 0; i < NLD; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t a = ES == 2 ? (x[i][e] << 16) & 0x7fffffffu : x[i][e] & 0x7fffffffu, b = x[i][e] & 0x7fff0000u;
        if (a < 0x7f800000u) most = max(most, a);
        if (ES == 2 && b < 0x7f800000u) most = max(most, b);
      }
    most = wave_max(most);
  }
  const uint32_t code = max(scale_byte(most), old);
  const float unit = scale_of(max(code, 1u));   // byte 0: zeros only
  const float inv = __uint_as_float((254u - min(code, 253u)) << 23);

#pragma unroll
  for (int i = 0; i < NLD; ++i) {
    const int row = j.first + (i * 64 + lane) / CH;
    uint32_t w[ES == 2 ? 2 : 1];
    if (!any) {
      // (by way of fp32: the instruction that takes pairs of bf16 rounds the lower one as if the bits below its half step were zero)
      auto four = [&](float x0, float x1, float x2, float x3) {
        s16x2 p = {0, 0};
        p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, x0, x1, unit, false);
        p = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(p, x2, x3, unit, true);
        return __builtin_bit_cast(uint32_t, p);
      };
      if constexpr (ES == 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          w[h] = four(bf16_lo(x[i][2 * h]), bf16_hi(x[i][2 * h]), bf16_lo(x[i][2 * h + 1]), bf16_hi(x[i][2 * h + 1]));
      } else {
        w[0] = four(__uint_as_float(x[i].x), __uint_as_float(x[i].y), __uint_as_float(x[i].z), __uint_as_float(x[i].w));
      }
    } else {
#pragma unroll
      for (int h = 0; h < (ES == 2 ? 2 : 1); ++h) {
        w[h] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float f;
          if constexpr (ES == 2) f = e % 2 ? bf16_hi(x[i][2 * h + e / 2]) : bf16_lo(x[i][2 * h + e / 2]);
          else f = __uint_as_float(x[i][e]);
          w[h] |= encode_any(f, inv) << (8 * e);
        }
      }
    }
    if (row >= j.lo && row < j.hi) {
      uint8_t* p = dst + row * c.tok + chunk * (16 / ES);
      if constexpr (ES == 2) *reinterpret_cast<v2u*>(p) = v2u{w[0], w[1]};
      else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
  }
  // rows that stay move to the larger scale: one step of 2^(old - code), rounded where a code falls below 2^-6
  if (keeps && code > old) {
    const float step = code - old < 127u ? __uint_as_float((127u - (code - old)) << 23) : 0.0f;
    constexpr int CC = D / 16;   // 16-byte chunks of a row of codes
    for (int i = lane; i < T * CC; i += 64) {
      const int row = j.first + i / CC;
      if (row >= block_end || (row >= j.lo && row < j.hi)) continue;
      v4u* p = reinterpret_cast<v4u*>(dst + row * c.tok + (i % CC) * 16);
      v4u y = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(int(y[e]), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(int(y[e]), true);
        int z = __builtin_amdgcn_cvt_pk_fp8_f32(a.x * step, a.y * step, 0, false);
        z = __builtin_amdgcn_cvt_pk_fp8_f32(b.x * step, b.y * step, z, true);
        y[e] = uint32_t(z);
      }
      *p = y;
    }
  }
  if (lane == 0) *scale = uint8_t(code);
}

template <int ES, int D, int T>
__global__ __launch_bounds__(kCacheWaves * 64) void cache_read_kernel(char* __restrict__ k, char* __restrict__ v,
                                                                    const int32_t* __restrict__ cu_kv, int groups, RowRange r,
                                                                    CacheView c, Shape s DLLM_CHECK_PARAM) {
  DLLM_CHECK_EXIT();
  constexpr int CH = D * ES / 16, NLD = T * CH / 64;   // as in cache_write_kernel: a lane's chunk of 16 bytes is 16 / ES codes
  const CacheJob j = cache_job(s, c, r, cu_kv, groups);
  if (j.none) return;
  const int lane = threadIdx.x & 63, chunk = lane % CH;
  char* dst = (j.is_v ? v : k) + (j.row0 * s.kv_tok + int64_t(j.g) * s.kv_head) * ES + chunk * 16;
  const uint8_t* src = (j.is_v ? c.v : c.k) + int64_t(j.kv0) * c.tok + int64_t(j.g) * c.head + chunk * (16 / ES);
  const float unit = scale_of((j.is_v ? c.vs : c.ks)[j.slot]);
  const int64_t pitch = s.kv_tok * ES;
  typedef __attribute__((ext_vector_type(ES == 2 ? 2 : 1))) uint32_t words;
  words x[NLD];
#pragma unroll
  for (int i = 0; i < NLD; ++i) {
    const int row = j.first + (i * 64 + lane) / CH;
    x[i] = __builtin_nontemporal_load(reinterpret_cast<const words*>(src + min(max(row, j.lo), j.hi - 1) * c.tok));
  }
#pragma unroll
  for (int i = 0; i < NLD; ++i) {
    const int row = j.first + (i * 64 + lane) / CH;
    v4u y;
    if constexpr (ES == 2) {
      y.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i][0], unit, false));
      y.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i][0], unit, true));
      y.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i][1], unit, false));
      y.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i][1], unit, true));
    } else {
      const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x[i][0], unit, false);
      const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x[i][0], unit, true);
      y = v4u{__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y)};
    }
    if (row >= j.lo && row < j.hi) *reinterpret_cast<v4u*>(dst + row * pitch) = y;
  }
}

namespace {
// f(integral_constant ES, D, T) for the call's element size, head_dim and tokens per scale
template <typename F>
void for_cache_shape(const Shape& s, dllm_dtype dt, int shift, F f) {
  auto with_t = [&](auto es, auto d) {
    if (shift == 4) f(es, d, std::integral_constant<int, 16>{});
    else if (shift == 5) f(es, d, std::integral_constant<int, 32>{});
    else f(es, d, std::integral_constant<int, 64>{});
  };
  auto with_d = [&](auto es) {
    if (s.d == 128) with_t(es, std::integral_constant<int, 128>{});
    else with_t(es, std::integral_constant<int, 64>{});
  };
  if (dt == DLLM_BF16) with_d(std::integral_constant<int, 2>{});
  else with_d(std::integral_constant<int, 4>{});
}
// blocks that max_rows rows at any place can touch
int64_t most_blocks(const Shape& s, const CacheView& c, const RowRange& r) {
  const int t = 1 << c.shift;
  return r.cu_rows == nullptr ? (int64_t(s.max_kv) + t - 1) / t : (int64_t(r.max_rows) + t - 2) / t + 1;
}
}  // namespace

hipError_t launch_cache_write(const Shape& s, dllm_dtype dt, const CacheView& c, const RowRange& r, const void* k, const void* v,
                              const int32_t* cu_kv, hipStream_t st) {
  const int groups = (2 * s.hkv + kCacheWaves - 1) / kCacheWaves;
  const dim3 grid(unsigned(most_blocks(s, c, r) * groups), s.batch);
  const char *kc = static_cast<const char*>(k), *vc = static_cast<const char*>(v);
  for_cache_shape(s, dt, c.shift, [&](auto es, auto d, auto t) {
    cache_write_kernel<decltype(es)::value, decltype(d)::value, decltype(t)::value>
        <<<grid, kCacheWaves * 64, 0, st>>>(kc, vc, cu_kv, groups, r, c, s DLLM_CHECK_PASS);
  });
  return hipGetLastError();
}

hipError_t launch_cache_read(const Shape& s, dllm_dtype dt, const CacheView& c, const RowRange& r, void* k, void* v,
                             const int32_t* cu_kv, hipStream_t st) {
  const int groups = (2 * s.hkv + kCacheWaves - 1) / kCacheWaves;
  const dim3 grid(unsigned(most_blocks(s, c, r) * groups), s.batch);
  char *kc = static_cast<char*>(k), *vc = static_cast<char*>(v);
  for_cache_shape(s, dt, c.shift, [&](auto es, auto d, auto t) {
    cache_read_kernel<decltype(es)::value, decltype(d)::value, decltype(t)::value>
        <<<grid, kCacheWaves * 64, 0, st>>>(kc, vc, cu_kv, groups, r, c, s DLLM_CHECK_PASS);
  });
  return hipGetLastError();
}

}  // namespace dllm
