// Query and key heads normed and rotated in one pass (viscache_norm_mrope), and the
// gradient (viscache_norm_mrope_grad).
//
// A head's values x (d of them, weights w, angles R of the row):
//     r = 1 / sqrt(sum x^2 / d + eps),  n = x r,  y = R (n w).
// Backward, g = R^T dy and h = g w:
//     dx = r (h - n sum(h n) / d),   dw = sum over rows and heads of g n.
//
// Both are bound by memory: a row is read once and written once (forward), rows and
// their output's gradients read once and one written (backward).  A thread holds 16
// values of a head (its slot: the eight pairs that eight frequencies turn), so the
// sums over a head are three or two shuffles and the rest stays in registers, as in
// rope.cu.
//
// 32768 rows of 72 heads of 128 in bf16 (1.21 GB): 209 us, 5.8 TB/s, 87% of a plain copy's rate (the
// rotation alone: 198 us).  Gradient of 12544 rows of 32 heads (308 MB): 82 us, 3.8 TB/s, 57%: 16
// warps an SM at 116 registers keep too little in flight; two rows ahead of each thread are no
// faster, smaller blocks slower (cold 89 and 103 against 89).  In fp32, cold: 394 us (6.1 TB/s, 92%) and
// 118 us (5.2 TB/s, 79%).  16 rows of 32 heads: a launch.
//
// Sums of squares that pass fp32's range are taken again of values times 2^-70: the
// branch costs nothing where it is not taken.
#include "kernels.h"
#include "norm_grid.h"
#include "profile.h"
#include "rope.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace rope;

constexpr int kThreads = 256;
constexpr int kHeadLanes = 8;         // heads a forward block works on at once

// Sum over the SLOTS neighbouring lanes of a head; every lane gets it.
template <int SLOTS>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
  for (int o = 1; o < SLOTS; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

__device__ __forceinline__ float squares(const float (&x)[8], const float (&y)[8], float scale) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = x[i] * scale, b = y[i] * scale;
    s = fmaf(a, a, s);
    s = fmaf(b, b, s);
  }
  return s;
}

// 1 / sqrt(mean + eps) in two factors (the second 1 but where the squares pass
// fp32's range); all lanes of the warp call it.
template <int D>
__device__ __forceinline__ float2 inverse_norm(const float (&x)[8], const float (&y)[8], float eps) {
  constexpr int SLOTS = D / 16;
  constexpr float kSmall = 0x1p-70f;
  float ss = head_sum<SLOTS>(squares(x, y, 1.f));
  const bool over = !(ss <= 3.402823466e38f);
  if (!__any_sync(0xffffffffu, over)) return make_float2(rsqrtf(ss * (1.f / D) + eps), 1.f);
  const float small = head_sum<SLOTS>(squares(x, y, kSmall));
  return over ? make_float2(rsqrtf(small * (1.f / D)), kSmall) : make_float2(rsqrtf(ss * (1.f / D) + eps), 1.f);
}

struct Slot {
  int o0, o1;          // the slot's two 8-value runs within a head
  bool turns;
  template <bool ADJ>
  static __device__ __forceinline__ Slot of(int slot, int half) {
    Slot s;
    s.turns = slot < half / 8;
    s.o0 = s.turns && !ADJ ? slot * 8 : slot * 16;
    s.o1 = s.turns && !ADJ ? half + slot * 8 : slot * 16 + 8;
    return s;
  }
};

// Block: rows [blockIdx.x * RT, ...) with RT = 32 / SLOTS, heads of share blockIdx.y
// of gridDim.y.  Thread: slot t % SLOTS, head lane (t / SLOTS) % 8, row t / (8 SLOTS).
// Slots past the rotated part of a head are normed alone.
template <typename T, int D, bool ADJ>
__global__ void __launch_bounds__(kThreads) norm_mrope_kernel(const __grid_constant__ RopeArgs a,
                                                              const __grid_constant__ NormRope p) {
  constexpr int SLOTS = D / 16;
  constexpr int RT = kThreads / (kHeadLanes * SLOTS);
  constexpr int HALF = D / 2;
  static_assert(RT * HALF == kThreads, "one angle a thread");
  __shared__ float2 cs[RT][HALF];
  const int t = threadIdx.x;
  const int64_t r0 = (int64_t)blockIdx.x * RT;
  const int slot = t % SLOTS, hl = t / SLOTS % kHeadLanes, lr = t / (SLOTS * kHeadLanes);
  const int64_t row = r0 + lr;
  const Slot sl = Slot::of<ADJ>(slot, a.half);
  const bool live = row < a.n_rows;
  const int H = a.Hq + a.Hkv, step = gridDim.y * kHeadLanes;
  const int base = blockIdx.y * kHeadLanes;     // (the same for the block: shuffles need whole warps)
  const T* const q = static_cast<const T*>(p.q) + row * a.q_stride;
  const T* const k = static_cast<const T*>(p.k) + row * a.k_stride;
  T* const qo = static_cast<T*>(p.q_out) + row * a.q_out_stride;
  T* const ko = static_cast<T*>(p.k_out) + row * a.k_out_stride;
  Raw8<T> x, y, nx, ny;
  auto load = [&](int h, Raw8<T>& u, Raw8<T>& v) {
    if (live && h < H) {
      const T* src = h < a.Hq ? q + (int64_t)h * D : k + (int64_t)(h - a.Hq) * D;
      u.load(src + sl.o0);
      v.load(src + sl.o1);
    }
  };
  load(base + hl, nx, ny);                      // in flight while the angles are computed
  {
    const int i = t % HALF;
    const int64_t ar = r0 + t / HALF;
    if (i < a.half && ar < a.n_rows) cs[t / HALF][i] = angle(a, i, ar);
  }
  __syncthreads();
  float c[8], s[8], wx[8], wy[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 v = sl.turns ? cs[lr][slot * 8 + i] : make_float2(1.f, 0.f);
    c[i] = v.x;
    s[i] = v.y;
  }
  int weights = -1;                             // whose weights wx, wy are
  for (int h0 = base; h0 < H; h0 += step) {
    const int h = h0 + hl;
    x = nx;
    y = ny;
    load(h + step, nx, ny);
    const int kind = h < a.Hq ? 0 : 1;
    if (kind != weights && h < H) {
      weights = kind;
      const T* w = static_cast<const T*>(kind ? p.k_weight : p.q_weight);
      Raw8<T> u, v;
      u.load(w + sl.o0);
      v.load(w + sl.o1);
      u.get(wx);
      v.get(wy);
    }
    float xa[8], ya[8], u[8], v[8];
    x.get(xa);
    y.get(ya);
    const bool on = live && h < H;
    if (!on) {
#pragma unroll
      for (int i = 0; i < 8; ++i) xa[i] = ya[i] = 0.f;
    }
    const float2 r = inverse_norm<D>(xa, ya, p.eps);
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      xa[i] = xa[i] * r.y * r.x * wx[i];
      ya[i] = ya[i] * r.y * r.x * wy[i];
    }
    T* dst = h < a.Hq ? qo + (int64_t)h * D : ko + (int64_t)(h - a.Hq) * D;
    if (sl.turns) {
      turn8<ADJ>(xa, ya, c, s, u, v);
      store8(dst + sl.o0, u);
      store8(dst + sl.o1, v);
    } else {
      store8(dst + sl.o0, xa);
      store8(dst + sl.o1, ya);
    }
  }
}

// Backward.  Blocks [0, nq) take the query heads, the others the key heads, so a
// thread sums one weight's gradient (16 channels of its slot) in registers; a block
// walks over groups of RB rows, whose angles it computes once.  The block's sums go
// to the workspace, one row of D a block.
template <typename T, int D, bool ADJ>
__global__ void __launch_bounds__(kThreads) norm_mrope_grad_kernel(const __grid_constant__ RopeArgs a,
                                                                   const __grid_constant__ NormRopeGrad p) {
  constexpr int SLOTS = D / 16, GROUPS = kThreads / SLOTS, HALF = D / 2, RB = kGradRows;
  __shared__ float2 cs[RB][HALF];                // frequency 8 slot + i at i * SLOTS + slot: no two slots on a bank
  __shared__ float sums[kThreads / 32][D];
  const int t = threadIdx.x, slot = t % SLOTS, grp = t / SLOTS;
  const bool isk = (int)blockIdx.x >= p.nq;
  const int H = isk ? a.Hkv : a.Hq;
  const int64_t xs = isk ? a.k_stride : a.q_stride, gs = isk ? p.k_dy_stride : p.q_dy_stride;
  const int64_t os = isk ? a.k_out_stride : a.q_out_stride;
  const T* const X = static_cast<const T*>(isk ? p.k : p.q);
  const T* const G = static_cast<const T*>(isk ? p.k_dy : p.q_dy);
  T* const O = static_cast<T*>(isk ? p.k_out : p.q_out);
  const Slot sl = Slot::of<ADJ>(slot, a.half);
  float wx[8], wy[8], dx[8], dy[8];
  {
    const T* w = static_cast<const T*>(isk ? p.k_weight : p.q_weight);
    Raw8<T> u, v;
    u.load(w + sl.o0);
    v.load(w + sl.o1);
    u.get(wx);
    v.get(wy);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) dx[i] = dy[i] = 0.f;
  const int first = isk ? (int)blockIdx.x - p.nq : (int)blockIdx.x;
  const int blocks = isk ? (int)gridDim.x - p.nq : p.nq;
  // items of a group of rows: (row, head), GROUPS of them at once; the next one's values are in flight
  const int dl = GROUPS / H, dh = GROUPS - dl * H, lr0 = grp / H, h0 = grp - lr0 * H;
  Raw8<T> x, y, g, k;
  auto load = [&](int64_t r0, int rows, int lr, int h) {
    if (lr >= rows) return;
    const T* xp = X + (r0 + lr) * xs + (int64_t)h * D;
    const T* gp = G + (r0 + lr) * gs + (int64_t)h * D;
    x.load(xp + sl.o0);
    y.load(xp + sl.o1);
    g.load(gp + sl.o0);
    k.load(gp + sl.o1);
  };
  for (int64_t r0 = (int64_t)first * RB; r0 < a.n_rows; r0 += (int64_t)blocks * RB) {
    const int rows = (int)(a.n_rows - r0 < RB ? a.n_rows - r0 : RB);
    load(r0, rows, lr0, h0);
    __syncthreads();                            // the angles before are read
    for (int i = t; i < RB * HALF; i += kThreads)
      if (i % HALF < a.half && r0 + i / HALF < a.n_rows)
        cs[i / HALF][i % 8 * SLOTS + i % HALF / 8] = angle(a, i % HALF, r0 + i / HALF);
    __syncthreads();
    int lr = lr0, h = h0;
    for (int left = rows * H; left > 0; left -= GROUPS) {     // (the same for the block: shuffles need whole warps)
      const bool on = lr < rows;
      const int row_of = on ? lr : 0;
      T* dst = O + (r0 + lr) * os + (int64_t)h * D;
      float xa[8], ya[8], ga[8], gb[8];
      if (on) {
        x.get(xa);
        y.get(ya);
        g.get(ga);
        k.get(gb);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) xa[i] = ya[i] = ga[i] = gb[i] = 0.f;
      }
      lr += dl;
      h += dh;
      if (h >= H) {
        h -= H;
        ++lr;
      }
      load(r0, rows, lr, h);
      if (sl.turns) {
        float c[8], s[8], u[8], v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 w = cs[row_of][i * SLOTS + slot];
          c[i] = w.x;
          s[i] = w.y;                           // (the table holds -sin: R^T)
        }
        turn8<ADJ>(ga, gb, c, s, u, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          ga[i] = u[i];
          gb[i] = v[i];
        }
      }
      const float2 r = inverse_norm<D>(xa, ya, p.eps);
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xa[i] = xa[i] * r.y * r.x;              // n
        ya[i] = ya[i] * r.y * r.x;
        dx[i] = fmaf(ga[i], xa[i], dx[i]);
        dy[i] = fmaf(gb[i], ya[i], dy[i]);
        ga[i] *= wx[i];                         // h
        gb[i] *= wy[i];
        m = fmaf(ga[i], xa[i], m);
        m = fmaf(gb[i], ya[i], m);
      }
      m = head_sum<SLOTS>(m) * (1.f / D);
      if (on) {
        const float rr = r.x * r.y;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          xa[i] = rr * (ga[i] - xa[i] * m);
          ya[i] = rr * (gb[i] - ya[i] * m);
        }
        store8(dst + sl.o0, xa);
        store8(dst + sl.o1, ya);
      }
    }
  }
  // the block's sums: lanes of a slot, then warps
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int o = SLOTS; o < 32; o <<= 1) {
      dx[i] += __shfl_xor_sync(0xffffffffu, dx[i], o);
      dy[i] += __shfl_xor_sync(0xffffffffu, dy[i], o);
    }
  if ((t & 31) < SLOTS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sums[t >> 5][sl.o0 + i] = dx[i];
      sums[t >> 5][sl.o1 + i] = dy[i];
    }
  }
  __syncthreads();
  if (t < D) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) v += sums[w][t];
    p.partial[(int64_t)blockIdx.x * D + t] = v;
  }
}

// Weight gradients: the blocks' sums added up, 32 channels of one weight a block.
__global__ void __launch_bounds__(256) norm_weight_grad_kernel(const float* __restrict__ partial, int d, int nq, int nk,
                                                               float* __restrict__ dwq, float* __restrict__ dwk) {
  dep_wait();
  __shared__ float part[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool isk = blockIdx.y != 0;
  const int first = isk ? nq : 0, n = isk ? nk : nq, col = blockIdx.x * 32 + lane;
  float v = 0.f;
  for (int b = warp; b < n; b += 8) v += partial[(int64_t)(first + b) * d + col];
  part[warp][lane] = v;
  __syncthreads();
  float* out = isk ? dwk : dwq;
  if (warp == 0 && out) {
    v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += part[w][lane];
    out[col] = v;
  }
}

template <typename T, int D, bool ADJ>
cudaError_t forward_t(const RopeArgs& a, const NormRope& p, cudaStream_t st) {
  constexpr int RT = kThreads / (kHeadLanes * (D / 16));
  const int64_t rb = (a.n_rows + RT - 1) / RT;
  const int64_t hmax = (a.Hq + a.Hkv + kHeadLanes - 1) / kHeadLanes;
  const int64_t want = kv8_sm_count() / rb;       // as in rope.cu: few rows share their heads out over blocks
  const unsigned hs = (unsigned)(want < 1 ? 1 : want > hmax ? hmax : want);
  ProfileScope ps("norm_mrope", st);
  norm_mrope_kernel<T, D, ADJ><<<dim3((unsigned)rb, hs), kThreads, 0, st>>>(a, p);
  return cudaGetLastError();
}

template <typename T, int D, bool ADJ>
cudaError_t grad_t(const RopeArgs& a, NormRopeGrad& p, float* dwq, float* dwk, cudaStream_t st) {
  const NormGradGrid g = norm_grad_grid(a.n_rows, a.Hq, a.Hkv);
  p.nq = g.nq;
  ProfileScope ps("norm_mrope_grad", st);
  norm_mrope_grad_kernel<T, D, ADJ><<<(unsigned)(g.nq + g.nk), kThreads, 0, st>>>(a, p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_dep(norm_weight_grad_kernel, dim3(D / 32, 2), dim3(256), 0, st, (const float*)p.partial, D, g.nq, g.nk,
                    dwq, dwk);
}

}  // namespace

#define VC_DISPATCH(F, ...)                                                                       \
  (dtype == VC_BF16 ? (d == 128 ? (adjacent ? F<__nv_bfloat16, 128, true>(__VA_ARGS__)            \
                                            : F<__nv_bfloat16, 128, false>(__VA_ARGS__))          \
                                : (adjacent ? F<__nv_bfloat16, 64, true>(__VA_ARGS__)             \
                                            : F<__nv_bfloat16, 64, false>(__VA_ARGS__)))          \
                    : (d == 128 ? (adjacent ? F<float, 128, true>(__VA_ARGS__)                    \
                                            : F<float, 128, false>(__VA_ARGS__))                  \
                                : (adjacent ? F<float, 64, true>(__VA_ARGS__)                     \
                                            : F<float, 64, false>(__VA_ARGS__))))

cudaError_t launch_norm_mrope(const RopeArgs& a, const NormRope& p, int dtype, int d, bool adjacent, cudaStream_t st) {
  return VC_DISPATCH(forward_t, a, p, st);
}

cudaError_t launch_norm_mrope_grad(const RopeArgs& a, NormRopeGrad& p, int dtype, int d, bool adjacent, float* dwq,
                                   float* dwk, cudaStream_t st) {
  return VC_DISPATCH(grad_t, a, p, dwq, dwk, st);
}

}  // namespace vc
