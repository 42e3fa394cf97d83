// What the mma.sync kernels over the 8-bit cache share: the product, fp16 parts and a
// warp's query fragments.
#pragma once

#include "kv8.cuh"
#include "kv8_sched.cuh"

namespace vc {
namespace kv8 {

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// what pack_f16(lo, hi) lost, as fp16 numbers again
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t packed) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&packed));
  return pack_f16(lo - f.x, hi - f.y);
}

// The warp's query fragments, normalised (lane (gid, tig): row 8 n + gid of the
// unit, dimensions tig * D/4 ...), and the power of two of rows 8 n + 2 tig, + 1.
// TOKENS: rows that are no tokens (more rows than tokens) count as 0.
template <typename T, int D, int NQ, int NP, bool TOKENS = false>
__device__ __forceinline__ void load_q(const T* q, int64_t q_stride, const Unit& u, int G,
                                       uint32_t (&f)[NP][NQ][D / 16][2], float (&qs)[NQ][2]) {
  constexpr int DPT = D / 4;                    // dimensions of a thread
  const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int rho = u.rt * 8 * NQ + 8 * n + gid;
    float x[DPT];
    float amax = 0.f;
    if (rho < u.q.m * G && (!TOKENS || rho >= (u.q.m - u.q.len) * G)) {
      const int i = rho / G, j = rho - i * G;
      const T* src = q + (int64_t)(u.q.row0 + i) * q_stride + (int64_t)(u.g * G + j) * D + tig * DPT;
#pragma unroll
      for (int e = 0; e < DPT; e += 4) {
        const float4 v = load4(src + e);
        x[e] = v.x; x[e + 1] = v.y; x[e + 2] = v.z; x[e + 3] = v.w;
      }
#pragma unroll
      for (int e = 0; e < DPT; ++e) amax = fmaxf(amax, fabsf(x[e]));
    } else {
#pragma unroll
      for (int e = 0; e < DPT; ++e) x[e] = 0.f;
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const uint32_t ex = __float_as_uint(amax) & 0x7f800000u;
    // 2^-126 at least, so that it and its inverse are normal; a row that is not finite as it is
    const float p2 = ex == 0x7f800000u ? 1.f : __uint_as_float(max(ex, 15u << 23) - (14u << 23));
    const float inv = pow2_inverse(p2);
    qs[n][0] = __shfl_sync(0xffffffffu, p2, 8 * tig);
    qs[n][1] = __shfl_sync(0xffffffffu, p2, 8 * tig + 4);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {             // k = 2 tig, + 1 and 2 tig + 8, + 9
        const float a0 = x[4 * s + 2 * h] * inv, a1 = x[4 * s + 2 * h + 1] * inv;
        f[0][n][s][h] = pack_f16(a0, a1);
        if (NP == 2) f[NP - 1][n][s][h] = pack_rest(a0, a1, f[0][n][s][h]);
      }
    }
  }
}

}  // namespace kv8
}  // namespace vc
