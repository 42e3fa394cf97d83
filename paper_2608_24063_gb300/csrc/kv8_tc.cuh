// What the tcgen05 attention kernels over the 8-bit cache share: descriptors, MMAs
// issued by a whole warp, codes expanded to fp16 tiles, and the join of a split
// unit's pieces.
#pragma once

#include "kernels.h"
#include "kv8.cuh"
#include "tc_common.cuh"

namespace vc {
namespace kv8 {

using namespace tc;

// Least exponent that a page's scale gives P's factor: below it P is 0 in fp16 anyway, and
// the row's sum is still read off P.
constexpr float kLeastShare = -80.f;

constexpr uint32_t kBlk = 128 * 128;            // 128 rows x 128 bytes (64 fp16 columns)

// Instruction descriptors, D fp32: kind::f16 with A, B fp16, both K-major or B
// MN-major; kind::f8f6f4 with A e4m3 or e5m2 and B e4m3, both K-major.
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t M, uint32_t N) {
  return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
__host__ __device__ constexpr uint32_t idesc_f16_bmn(uint32_t M, uint32_t N) {
  return (1u << 4) | (1u << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
__host__ __device__ constexpr uint32_t idesc_e4m3(uint32_t M, uint32_t N) {
  return (1u << 4) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
__host__ __device__ constexpr uint32_t idesc_e5m2_e4m3(uint32_t M, uint32_t N) { return idesc_e4m3(M, N) | (1u << 7); }

// Descriptor of a K-major tile of 8-bit rows of D bytes: 128-byte swizzle
// (8-row groups 1024 bytes apart) or, at D = 64, 64-byte swizzle (512).
template <int D>
__device__ __forceinline__ uint64_t desc_codes(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)1 << 16;
  d |= (uint64_t)((8 * D) >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)(D == 128 ? 2 : 4) << 61;
  return d;
}
// Byte offset of 8-byte piece c of row r in such a tile.
template <int D>
__device__ __forceinline__ uint32_t code_piece(int r, int c) {
  const int ch = D == 128 ? (c >> 1) ^ (r & 7) : (c >> 1) ^ ((r >> 1) & 3);
  return (uint32_t)(r * D + ch * 16 + (c & 1) * 8);
}

// The issuing warp runs as a whole and each instruction elects its lane: then
// descriptors and addresses are warp-uniform values, and an MMA is issued every 7
// to 15 clocks.  Issued from a branch of one thread, each takes 50 to 60 (and a
// lone one is seen done after 274 clocks instead of 130): as long as it runs.
//
// D[tmem] (+)= A[smem] * B[smem]^T, 8-bit operands.
__device__ __forceinline__ void mma_f8_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_f16_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem].
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Arrive on bar once every MMA issued so far has completed (the same elected lane).
__device__ __forceinline__ void mma_commit_elected(uint64_t* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
      : "memory");
}

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// what half2_bits(lo, hi) lost, as fp16 numbers again
__device__ __forceinline__ uint32_t half2_rest(float lo, float hi, uint32_t bits) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&bits));
  return half2_bits(lo - f.x, hi - f.y);
}

// Eight query values (|z| < 256, or NaN for what is not finite) as the sum of an e4m3
// and an e5m2 number each.  A bf16 number has 8 significant bits, an e4m3 number 4: its
// rounding leaves at most 8 units of the last bit, which 3 bits hold.  So the sum is
// exact from 2^-6 on, where e4m3 still has its 4 bits; below, a rest of at most 2^-10 is
// off by up to 2^-14.
__device__ __forceinline__ void split8(const float (&z)[8], uint2& top, uint2& rest) {
  uint32_t t[2], r[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    float y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = fabsf(z[4 * e + k]) <= 448.f ? z[4 * e + k] : __uint_as_float(0x7fffffffu);
    const uint32_t p0 = f32x2_to_e4m3x2(y[0], y[1]), p1 = f32x2_to_e4m3x2(y[2], y[3]);
    const uint32_t h0 = e4m3x2_to_f16x2(p0), h1 = e4m3x2_to_f16x2(p1);
    const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&h0));
    const float2 f1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
    t[e] = p0 | p1 << 16;
    r[e] = f32x2_to_e5m2x2(y[0] - f0.x, y[1] - f0.y) | f32x2_to_e5m2x2(y[2] - f1.x, y[3] - f1.y) << 16;
  }
  top = make_uint2(t[0], t[1]);
  rest = make_uint2(r[0], r[1]);
}

// Sixteen codes as fp16 numbers (exact): 32 bytes of row `row`, column chunk c
// (16 columns) of a tile: the two 16-byte pieces are written in an order that
// keeps the eight lanes of a row on different banks.
__device__ __forceinline__ void expand16(uint8_t* tile, int row, int c, const uint4& w) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = e4m3x2_to_f16x2(x[i]);
    y[2 * i + 1] = e4m3x2_to_f16x2(x[i] >> 16);
  }
  uint8_t* base = tile + (c >> 2) * kBlk + row * 128;
  const int ch = 2 * (c & 3), r7 = row & 7;
  const uint4 lo = make_uint4(y[0], y[1], y[2], y[3]), hi = make_uint4(y[4], y[5], y[6], y[7]);
  const bool swap = (c & 4) != 0;
  *reinterpret_cast<uint4*>(base + (((ch + swap) ^ r7) << 4)) = swap ? hi : lo;
  *reinterpret_cast<uint4*>(base + (((ch + !swap) ^ r7) << 4)) = swap ? lo : hi;
}

// Takes the NaN codes out of y; whether there was one.
__device__ __forceinline__ bool drop_nan(uint4& y) {
  const uint32_t n[4] = {nan_codes(y.x), nan_codes(y.y), nan_codes(y.z), nan_codes(y.w)};
  y.x &= ~n[0]; y.y &= ~n[1]; y.z &= ~n[2]; y.w &= ~n[3];
  return (n[0] | n[1] | n[2] | n[3]) != 0u;
}

// The references of a row's softmax, log2 units.  x is a score, v the log2 of its page's V
// scale.  m follows the largest x and r + m the largest x + v, both of what the row sees,
// and each may be passed by `slack` before it rises.  m is a score and r a whole number, so
// that the probability 1 of a dominant token is not rounded.  P = 2^(x + v - m - r + const) multiplies the codes as
// they are: a page's scale enters with its tokens' probabilities, so a row's fixed point is
// set by its largest contribution and by nothing that it does not see or that has no weight.
struct RowRefs {
  float m, r, l;
  __device__ __forceinline__ void clear() {
    m = r = -INFINITY;
    l = 0.f;
  }
  // b: largest x of each 16-token group; whether O's reference moves (O times g then)
  __device__ __forceinline__ bool raise(const float (&b)[8], const float* vlog, float slack, float& g) {
    const float tx = fmax3(fmax3(b[0], b[1], b[2]), fmax3(b[3], b[4], b[5]), fmaxf(b[6], b[7]));
    float was = r;
    if (tx > m + slack) {
      l *= ex2(m - tx);                         // 0 on the first
      was -= tx - m;
      m = tx;
    }
    const float4 v0 = *reinterpret_cast<const float4*>(vlog), v1 = *reinterpret_cast<const float4*>(vlog + 4);
    const float mr = base();
    const float ty = fmax3(fmax3(b[0] - mr + v0.x, b[1] - mr + v0.y, b[2] - mr + v0.z),
                           fmax3(b[3] - mr + v0.w, b[4] - mr + v1.x, b[5] - mr + v1.y),
                           fmaxf(b[6] - mr + v1.z, b[7] - mr + v1.w));
    const float up = ty > was + slack ? ceilf(ty) : floorf(was);
    g = was == up ? 1.f : ex2(was - up);
    r = up;
    return up != was;
  }
  __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.f : m; }
  __device__ __forceinline__ float value_base() const { return r == -INFINITY ? 0.f : r; }
};

// 1 / a row's sum; 0 where it saw no token, NaN stays.
__device__ __forceinline__ float inverse_of(float L) { return L > 0.f ? 1.f / L : (L == L ? 0.f : L); }

// Adds up the pieces of a split unit's 128-row tile `x` of `tiles`, called by
// four warps: a warp takes a quarter of the columns of 32 rows, a lane a row, and
// has the values of kJoin pieces in flight at once (8 KV heads over 8192 tokens,
// 19 pieces a unit: 256 rows 156 -> 53 us, 64 rows 65 -> 32 us against a row a
// thread and a piece at a time).  Pieces lie as [block, end of it][tile]: (max,
// sum) of its rows, and outputs [four columns][row].  put(row, column, 16
// unscaled outputs, max, sum).
template <int D, typename Put>
__device__ __forceinline__ void join_pieces(const Kv8AttnArgs& a, int first, int final, int tiles, int x, int rows,
                                            Put put) {
  constexpr int kJoin = 3, kCols = D / 16;      // kCols: float4 a row of a warp
  const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
  for (int r0 = 0; r0 < rows; r0 += 32) {
    const int row = r0 + lane;
    const bool live = row < rows;
    float4 y[kCols];
#pragma unroll
    for (int q = 0; q < kCols; ++q) y[q] = make_float4(0.f, 0.f, 0.f, 0.f);
    float M = -INFINITY, L = 0.f;
    for (int b0 = first; b0 <= final; b0 += kJoin) {
      float2 ml[kJoin];
      float4 z[kJoin][kCols];
#pragma unroll
      for (int n = 0; n < kJoin; ++n) {
        const int b = b0 + n;
        const int64_t tile = (2 * (int64_t)b + (b == first ? 1 : 0)) * tiles + x;
        const bool on = live && b <= final;
        ml[n] = on ? __ldcg(&a.part_ml[tile * 128 + row]) : make_float2(-INFINITY, 0.f);
        const float4* src = reinterpret_cast<const float4*>(a.part_o + tile * 128 * D) + warp * kCols * 128 + row;
#pragma unroll
        for (int q = 0; q < kCols; ++q) z[n][q] = on ? __ldcg(src + q * 128) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      float top = M;
#pragma unroll
      for (int n = 0; n < kJoin; ++n) top = fmaxf(top, ml[n].x);
      const float g = M == -INFINITY ? 1.f : ex2(M - top);
      M = top;
      L *= g;
#pragma unroll
      for (int q = 0; q < kCols; ++q) {
        y[q].x *= g; y[q].y *= g; y[q].z *= g; y[q].w *= g;
      }
#pragma unroll
      for (int n = 0; n < kJoin; ++n) {
        const float wt = ml[n].x == -INFINITY ? 1.f : ex2(ml[n].x - M);
        L = fmaf(ml[n].y, wt, L);
#pragma unroll
        for (int q = 0; q < kCols; ++q) {
          y[q].x = fmaf(z[n][q].x, wt, y[q].x);
          y[q].y = fmaf(z[n][q].y, wt, y[q].y);
          y[q].z = fmaf(z[n][q].z, wt, y[q].z);
          y[q].w = fmaf(z[n][q].w, wt, y[q].w);
        }
      }
    }
    if (!live) continue;
#pragma unroll
    for (int p = 0; p < kCols / 4; ++p) {
      float o[16];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        o[4 * q] = y[4 * p + q].x; o[4 * q + 1] = y[4 * p + q].y;
        o[4 * q + 2] = y[4 * p + q].z; o[4 * q + 3] = y[4 * p + q].w;
      }
      put(row, warp * kCols * 4 + p * 16, o, M, L);
    }
  }
}

}  // namespace kv8
}  // namespace vc
