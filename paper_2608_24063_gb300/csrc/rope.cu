// Rotary positions with several axes (viscache_mrope).
//
// Frequency i of `half` turns the value pair (a_i, b_i) of every head by the
// angle w_i = pos[axis(i)] * theta^(-i / half):
//     a' = a cos w - b sin w,   b' = b cos w + a sin w
// (inverse: the sign of w flipped, which is also the gradient).
//
// Two loads, two stores and no reuse but of the angles: bound by memory.  The
// angles depend on the row alone, so a block takes a few rows and computes
// each (row, frequency)'s cosine and sine once, into shared memory; a thread
// then keeps the eight pairs of its (row, slot) in registers and walks over
// the heads, 16 values (two or four 16-byte loads) at a time.  32768 rows of 72
// heads of 128 in bf16 (1.21 GB): 198 us, 6.1 TB/s, 90% of a plain copy's rate.  16
// rows of 32 heads: 2.3 us, a launch.
//
// The phase is an integer: F_i = theta^(-i/half) / 2pi in units of 2^-64 turn,
// so pos * F_i modulo 2^64 is the reduced angle without any range reduction,
// for every 32-bit position, negative ones too.  Its top 32 bits become the
// argument of sincospif (error about 2^-26 turn; F_i itself is good to 45 bits:
// one fp64 power and up to 63 products, so the phase of position 2^20 is off by
// 2^-27 turn at most, and that of 2^31 - 1 by 2^-16).
#include <math.h>

#include "kernels.h"
#include "profile.h"
#include "vc_common.cuh"

namespace vc {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeHeadLanes = 8;     // heads a block works on at once
constexpr int kRopeBatch = 2;         // heads a thread has in flight

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

// Block: rows [blockIdx.x * RT, ...) with RT = 32 / SLOTS, heads of share
// blockIdx.y of gridDim.y.  Thread: slot t % SLOTS (16 values of a head), head
// lane (t / SLOTS) % 8, row t / (8 SLOTS).  Slots past the rotated part of a
// head copy their values.
template <typename T, int D, bool ADJ>
__global__ void __launch_bounds__(kRopeThreads) mrope_kernel(const __grid_constant__ RopeArgs a,
                                                             const T* q, T* q_out, const T* k,
                                                             T* k_out) {
  constexpr int SLOTS = D / 16;
  constexpr int RT = kRopeThreads / (kRopeHeadLanes * SLOTS);
  constexpr int HALF = D / 2;                       // table row; a.half <= HALF are used
  static_assert(RT * HALF == kRopeThreads, "one angle a thread");
  __shared__ float2 cs[RT][HALF];
  const int t = threadIdx.x;
  const int64_t r0 = (int64_t)blockIdx.x * RT;
  const int slot = t % SLOTS, hl = t / SLOTS % kRopeHeadLanes, lr = t / (SLOTS * kRopeHeadLanes);
  const int64_t row = r0 + lr;
  const bool turns = slot < a.half / 8;
  // element offsets of the slot's two 8-value runs within a head
  const int o0 = turns && !ADJ ? slot * 8 : slot * 16;
  const int o1 = turns && !ADJ ? a.half + slot * 8 : slot * 16 + 8;
  const int H = row < a.n_rows ? a.Hq + a.Hkv : 0, step = gridDim.y * kRopeHeadLanes;
  Raw8<T> x[kRopeBatch], y[kRopeBatch];
  auto load = [&](int h0) {
#pragma unroll
    for (int n = 0; n < kRopeBatch; ++n) {
      const int h = h0 + n * step;
      if (h < H) {
        const T* src = (h < a.Hq ? q + row * a.q_stride + (int64_t)h * D
                                 : k + row * a.k_stride + (int64_t)(h - a.Hq) * D);
        x[n].load(src + o0);
        y[n].load(src + o1);
      }
    }
  };
  int h0 = blockIdx.y * kRopeHeadLanes + hl;
  load(h0);                                         // in flight while the angles are computed
  {
    const int i = t % HALF;
    const int64_t ar = r0 + t / HALF;
    if (i < a.half && ar < a.n_rows) {
      const int32_t pos = __ldg(a.positions + (int64_t)a.axis[i] * a.n_rows + ar);
      const uint64_t phase = (uint64_t)(int64_t)pos * a.freq[i];
      const float turn = (float)(int32_t)(phase >> 32) * 0x1p-31f;    // half turns in [-1, 1)
      float s, c;
      sincospif(turn, &s, &c);
      cs[t / HALF][i] = make_float2(c, a.inverse ? -s : s);
    }
  }
  __syncthreads();
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 v = turns ? cs[lr][slot * 8 + i] : make_float2(1.f, 0.f);
    c[i] = v.x;
    s[i] = v.y;
  }
  // kBatch heads at a time, all loads before the first store: the output may
  // be the input, so the compiler would not move a load over a store by itself
  for (; h0 < H; h0 += kRopeBatch * step) {
    if (h0 != (int)(blockIdx.y * kRopeHeadLanes) + hl) load(h0);
#pragma unroll
    for (int n = 0; n < kRopeBatch; ++n) {
      const int h = h0 + n * step;
      if (h >= H) break;
      T* dst = h < a.Hq ? q_out + row * a.q_out_stride + (int64_t)h * D
                        : k_out + row * a.k_out_stride + (int64_t)(h - a.Hq) * D;
      float xa[8], ya[8], u[8], v[8];
      x[n].get(xa);
      y[n].get(ya);
      if (!turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[i] = xa[i];
          v[i] = ya[i];
        }
      } else if (ADJ) {
        // pairs (2i, 2i + 1): x holds pairs 0..3 of the slot, y pairs 4..7
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[2 * i] = xa[2 * i] * c[i] - xa[2 * i + 1] * s[i];
          u[2 * i + 1] = xa[2 * i + 1] * c[i] + xa[2 * i] * s[i];
          v[2 * i] = ya[2 * i] * c[4 + i] - ya[2 * i + 1] * s[4 + i];
          v[2 * i + 1] = ya[2 * i + 1] * c[4 + i] + ya[2 * i] * s[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[i] = xa[i] * c[i] - ya[i] * s[i];
          v[i] = ya[i] * c[i] + xa[i] * s[i];
        }
      }
      store8(dst + o0, u);
      store8(dst + o1, v);
    }
  }
}

template <typename T, int D, bool ADJ>
cudaError_t launch_t(const RopeArgs& a, const void* q, void* q_out, const void* k, void* k_out, cudaStream_t st) {
  constexpr int RT = kRopeThreads / (kRopeHeadLanes * (D / 16));
  const int64_t rb = (a.n_rows + RT - 1) / RT;
  // few rows: the heads are shared out over blocks as well, while every block
  // has an SM of its own (each recomputes its rows' angles).  40 heads of 128,
  // us with one share / with shares / with shares for four blocks an SM: 16 rows
  // 3.7 / 2.6 / 2.6, 256 rows 4.0 / 3.2 / 4.0, 512 rows 4.1 / 4.2 / 5.9
  const int64_t hmax = (a.Hq + a.Hkv + kRopeHeadLanes - 1) / kRopeHeadLanes;
  const int64_t want = kv8_sm_count() / rb;
  const unsigned hs = (unsigned)(want < 1 ? 1 : want > hmax ? hmax : want);
  ProfileScope ps("mrope", st);
  mrope_kernel<T, D, ADJ><<<dim3((unsigned)rb, hs), kRopeThreads, 0, st>>>(
      a, static_cast<const T*>(q), static_cast<T*>(q_out), static_cast<const T*>(k), static_cast<T*>(k_out));
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_d(const RopeArgs& a, int d, bool adj, const void* q, void* q_out, const void* k, void* k_out,
                     cudaStream_t st) {
  if (d == 128)
    return adj ? launch_t<T, 128, true>(a, q, q_out, k, k_out, st)
               : launch_t<T, 128, false>(a, q, q_out, k, k_out, st);
  return adj ? launch_t<T, 64, true>(a, q, q_out, k, k_out, st)
             : launch_t<T, 64, false>(a, q, q_out, k, k_out, st);
}

}  // namespace

cudaError_t launch_mrope(const RopeArgs& a, int dtype, int d, bool adjacent, const void* q, void* q_out,
                         const void* k, void* k_out, cudaStream_t st) {
  return dtype == VC_BF16 ? launch_d<__nv_bfloat16>(a, d, adjacent, q, q_out, k, k_out, st)
                          : launch_d<float>(a, d, adjacent, q, q_out, k, k_out, st);
}

}  // namespace vc
