// Device helpers of the 8-bit paged cache: checked request descriptors, e4m3
// conversion and power-of-two scales.
#pragma once

#include <cuda_fp16.h>

#include "vc_common.cuh"

namespace vc {
namespace kv8 {

// Request r of a step: its first packed row, rows and tokens.
struct Req8 {
  int row0, m, len;
};

// Reads and checks request r.  A length outside the block table is clamped, a
// request whose rows do not lie in order in [0, n_rows] counts as empty.
// `status` is any word (here as below; NULL: what is wrong is skipped silently).
__device__ __forceinline__ Req8 load_req(const vc_kv8_step& s, int page, int r, int32_t* status) {
  Req8 q;
  q.row0 = __ldg(s.row_start + r);
  const int next = __ldg(s.row_start + r + 1);
  q.len = __ldg(s.seq_lens + r);
  q.m = next - q.row0;
  if (q.row0 < 0 || next < q.row0 || next > s.n_rows) {
    if (status) set_status(status, VC_ERR_DEVICE_INDEX);
    q.row0 = q.m = 0;
  }
  const int cap = s.max_pages * page;
  if (q.len < 0 || q.len > cap) {
    if (status) set_status(status, VC_ERR_DEVICE_INDEX);
    q.len = min(max(q.len, 0), cap);
  }
  return q;
}

// Page j of request r, or -1 (status set) where the block table holds no page.
__device__ __forceinline__ int load_page(const vc_kv8_step& s, int n_pages, int r, int j, int32_t* status) {
  const int p = __ldg(s.block_table + (int64_t)r * s.max_pages + j);
  if (p >= 0 && p < n_pages) return p;
  if (status) set_status(status, VC_ERR_DEVICE_INDEX);
  return -1;
}

// e4m3 pair -> two fp16 numbers (exact; the NaN codes give NaN).
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t pair) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)pair));
  return h;
}

// Two fp32 numbers, |x| <= 448 or NaN, -> e4m3 pair (x in the low byte), to
// nearest even.
__device__ __forceinline__ uint32_t f32x2_to_e4m3x2(float x, float y) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
  return r;
}

// Two fp32 numbers of any size, or NaN, -> e5m2 pair, to nearest even.
__device__ __forceinline__ uint32_t f32x2_to_e5m2x2(float x, float y) {
  unsigned short r;
  asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
  return r;
}

// The least power of two s = 2^e, e >= -126, with amax <= 448 s; 0 for 0.
// 448 = 1.75 * 2^8, so e is amax's exponent minus 8, or minus 7 where its
// mantissa is above 1.75 (below 2^-126 the clamp decides).
__device__ __forceinline__ float pow2_scale(float amax) {
  if (amax == 0.f) return 0.f;
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127 - ((b & 0x7fffffu) > 0x600000u ? 7 : 8);
  return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
}

// 1 / s for a scale s > 0 (2^-126 .. 2^120, so the reciprocal is normal); 1 for 0.
__device__ __forceinline__ float pow2_inverse(float s) {
  return s == 0.f ? 1.f : __uint_as_float((254u << 23) - __float_as_uint(s));
}

// log2 of a scale; of 0 (a page of zeros, whose contribution does not depend on it) the least.
__device__ __forceinline__ float scale_log2(float s) { return fmaxf((float)(int)(__float_as_uint(s) >> 23) - 127.f, -126.f); }

// 2^e, -126 <= e <= 127; and for an e in [-250, 254] as two such factors.
__device__ __forceinline__ float pow2_bits(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ float2 pow2_factors(int e) { return make_float2(pow2_bits(e >> 1), pow2_bits(e - (e >> 1))); }

// A value that is NaN spoils the sums of rows that see it and no others.  A product
// takes 0 * NaN for a row that does not, so where a tile has tokens that some of the
// unit's rows do not see, NaN codes of V count as 0 and the first such token is
// noted; at the segment's end the rows that see it look their dimensions up.
constexpr int kNoNan = 0x7fffffff;
// 0xff in each byte that is a NaN code
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu); }
// Which of the N dimensions from `col` on (a multiple of 4) are NaN in V of any of
// the request's tokens [from, to): bit i for dimension col + i.
template <int N>
__device__ __forceinline__ uint32_t nan_dims(const vc_kv8& c, const vc_kv8_step& s, int r, int g, int from, int to,
                                          int col) {
  uint32_t found = 0;
#pragma unroll 1
  for (int t = from; t < to; ++t) {
    const int p = load_page(s, c.n_pages, r, t / c.page, nullptr);
    if (p < 0) continue;
    const uint32_t* codes = reinterpret_cast<const uint32_t*>(
        static_cast<const uint8_t*>(c.V_codes) + (((int64_t)p * c.Hkv + g) * c.page + t % c.page) * c.d + col);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint32_t m = nan_codes(__ldg(codes + i));
      found |= ((m & 1u) | (m >> 7 & 2u) | (m >> 14 & 4u) | (m >> 21 & 8u)) << (4 * i);
    }
  }
  return found;
}

}  // namespace kv8
}  // namespace vc
