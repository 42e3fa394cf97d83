// Device helpers of the rotary positions: eight values of a head as they lie in
// memory, and the angles of a row.
#pragma once

#include "kernels.h"
#include "vc_common.cuh"

namespace vc {
namespace rope {

// Eight values as they lie in memory.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t x[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(x[i] << 16);
        v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(w[i].x); v[4 * i + 1] = __uint_as_float(w[i].y);
        v[4 * i + 2] = __uint_as_float(w[i].z); v[4 * i + 3] = __uint_as_float(w[i].w);
      }
    }
  }
};
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) = pack8(v);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// Cosine and sine of frequency i at row `row`: the phase is an integer (rope.cu).
__device__ __forceinline__ float2 angle(const RopeArgs& a, int i, int64_t row) {
  const int32_t pos = __ldg(a.positions + (int64_t)a.axis[i] * a.n_rows + row);
  const uint64_t phase = (uint64_t)(int64_t)pos * a.freq[i];
  const float turn = (float)(int32_t)(phase >> 32) * 0x1p-31f;    // half turns in [-1, 1)
  float s, c;
  sincospif(turn, &s, &c);
  return make_float2(c, a.inverse ? -s : s);
}

// Turns a slot's eight pairs by (c, s).  HALVES: pair i is (x_i, y_i); ADJ: x holds
// pairs 0..3 as (2i, 2i + 1), y pairs 4..7.
template <bool ADJ>
__device__ __forceinline__ void turn8(const float (&x)[8], const float (&y)[8], const float (&c)[8],
                                      const float (&s)[8], float (&u)[8], float (&v)[8]) {
  if (ADJ) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u[2 * i] = x[2 * i] * c[i] - x[2 * i + 1] * s[i];
      u[2 * i + 1] = x[2 * i + 1] * c[i] + x[2 * i] * s[i];
      v[2 * i] = y[2 * i] * c[4 + i] - y[2 * i + 1] * s[4 + i];
      v[2 * i + 1] = y[2 * i + 1] * c[4 + i] + y[2 * i] * s[4 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u[i] = x[i] * c[i] - y[i] * s[i];
      v[i] = y[i] * c[i] + x[i] * s[i];
    }
  }
}

}  // namespace rope
}  // namespace vc
