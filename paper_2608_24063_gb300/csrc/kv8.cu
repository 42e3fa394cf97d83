// The 8-bit paged cache written (viscache_kv8_append) and read back
// (viscache_kv8_read).
//
// Both are one pass over the step's rows: 2 or 4 bytes a value on one side, one
// on the other, bound by memory.  A unit is one (page touched by the step, KV
// head, K or V): the page's rows of that head are one contiguous block of
// codes with one scale.  A block looks its page up once and takes a share of
// the page's units in turn, the next unit's values in flight while it works on
// the current one: it reduces the largest magnitude of the rows it has to write
// (held in registers, 16 values a vector) and writes the codes.  Where the page
// held tokens of the request before, their codes are re-encoded by the same
// block if the scale grew, so no block waits for another and nothing is
// written twice.  At 128 dimensions in bf16: append of 32768 rows of 8 heads (201
// MB) 35 us, 5.7 TB/s; read of 16 caches of up to 12544 tokens, 4 heads (389 MB) 70
// us, 5.5 TB/s (84% of a plain copy's rate: what is left is the start and the last
// blocks of 70 us, and a look-up before each block's first load); append of 64
// requests' next tokens 4.0 us, three memory round trips after the launch.
#include "kernels.h"
#include "kv8.cuh"
#include "profile.h"

namespace vc {
namespace {

using namespace kv8;

// The u-th page touched by the step's rows, requests in order.
struct Touch {
  int r, j;              // request, page within the request
  int row0, first;       // packed row of token `first`, the request's first written token
  int len;               // tokens of the request
};

// Called by one whole warp; false where the step touches fewer pages.  Each
// lane counts the pages of four consecutive requests at a time, so the loads
// of 128 requests are in flight together.
template <int PAGE>
__device__ __forceinline__ bool find_touch(const vc_kv8_step& s, int u, int32_t* status, Touch& out) {
  const int lane = threadIdx.x & 31;
  int base = 0;
  for (int r0 = 0; r0 < s.n_req; r0 += 128) {
    Req8 q[4];
    int cnt[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + 4 * lane + i;
      q[i] = r < s.n_req ? load_req(s, PAGE, r, status) : Req8{0, 0, 0};
      const int lo = max(q[i].len - q[i].m, 0);
      cnt[i] = q[i].len > lo ? (q[i].len - 1) / PAGE - lo / PAGE + 1 : 0;
      sum += cnt[i];
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += x;
    }
    const int total = __shfl_sync(0xffffffffu, incl, 31);
    if (u < base + total) {
      const int src = __ffs(__ballot_sync(0xffffffffu, u < base + incl)) - 1;
      Touch t = {};
      int at = base + incl - sum;                       // pages before this lane's requests
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (u >= at && u < at + cnt[i]) {
          const int old = q[i].len - q[i].m, lo = max(old, 0);
          t.r = r0 + 4 * lane + i;
          t.j = lo / PAGE + (u - at);
          t.first = lo;
          t.row0 = q[i].row0 + (lo - old);
          t.len = q[i].len;
        }
        at += cnt[i];
      }
      out.r = __shfl_sync(0xffffffffu, t.r, src);
      out.j = __shfl_sync(0xffffffffu, t.j, src);
      out.row0 = __shfl_sync(0xffffffffu, t.row0, src);
      out.first = __shfl_sync(0xffffffffu, t.first, src);
      out.len = __shfl_sync(0xffffffffu, t.len, src);
      return true;
    }
    base += total;
  }
  return false;
}

template <int D, int PAGE>
struct UnitCfg {
  static constexpr int VECS = PAGE * D / 16;            // 16-value vectors of a unit
  static constexpr int THREADS = VECS / 2 < 64 ? 64 : VECS / 2 > 256 ? 256 : VECS / 2;
  static constexpr int NV = VECS / THREADS;             // vectors of a thread
  static constexpr int VPR = D / 16;                    // vectors of a row
  // 1280 threads an SM where two vectors a thread fit their registers (16-bit
  // rows: append 41.2 -> 39.0 us, read 75 -> 72 us on the long cases against
  // 1024 threads; 1536 and 2048 spill)
  static constexpr int blocks(int value_bytes) { return NV <= 2 && value_bytes == 2 ? 1280 / THREADS : 1; }
  static_assert(NV * THREADS == VECS, "whole vectors");
};

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// Sixteen values as they lie in memory.
template <typename T>
struct Raw16 {
  uint4 w[sizeof(T)];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void get(float (&v)[16]) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[8 * i + 2 * k] = __uint_as_float(x[k] << 16);
          v[8 * i + 2 * k + 1] = __uint_as_float(x[k] & 0xffff0000u);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[4 * i] = __uint_as_float(w[i].x); v[4 * i + 1] = __uint_as_float(w[i].y);
        v[4 * i + 2] = __uint_as_float(w[i].z); v[4 * i + 3] = __uint_as_float(w[i].w);
      }
    }
  }
  // the largest magnitude as the bits of an fp32 number; at least infinity's
  // where a value is infinite or NaN
  __device__ __forceinline__ uint32_t largest() const {
    if constexpr (sizeof(T) == 2) {
      __nv_bfloat162 m = __float2bfloat162_rn(0.f);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) m = __hmax2_nan(m, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&x[k])));
      }
      const uint32_t b = *reinterpret_cast<const uint32_t*>(&m);
      return max(b << 16, b & 0xffff0000u);
    } else {
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        m = max(m, max(w[i].x & 0x7fffffffu, w[i].y & 0x7fffffffu));
        m = max(m, max(w[i].z & 0x7fffffffu, w[i].w & 0x7fffffffu));
      }
      return m;
    }
  }
  // the same over the finite values alone
  __device__ __forceinline__ uint32_t largest_finite() const {
    float v[16], m = 0.f;
    get(v);
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (finite(v[k])) m = fmaxf(m, fabsf(v[k]));
    return __float_as_uint(m);
  }
};
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&v)[16]) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  *reinterpret_cast<uint4*>(p + 8) = make_uint4(w[4], w[5], w[6], w[7]);
}
__device__ __forceinline__ void store16(float* p, const float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<float4*>(p + 4 * i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}

// Sixteen values times `inv` as codes; with CHECK what is not finite becomes NaN and
// products stop at `top`.
template <bool CHECK>
__device__ __forceinline__ uint4 encode16(const float (&v)[16], float inv, float top) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float y = v[4 * i + k];
      if constexpr (CHECK) x[k] = finite(y) ? fminf(fmaxf(y * inv, -top), top) : __uint_as_float(0x7fffffffu);
      else x[k] = y * inv;
    }
    w[i] = f32x2_to_e4m3x2(x[0], x[1]) | f32x2_to_e4m3x2(x[2], x[3]) << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void decode16(const uint4& c, float (&v)[16]) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t h = e4m3x2_to_f16x2(w[i >> 1] >> (16 * (i & 1)));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

// Block 0 checks every request and every page that the step touches, and stores
// the call's status; the other blocks skip what is wrong silently.  A thread
// takes a request; those that touch more than two pages are then looked at by
// the whole warp.
template <int PAGE>
__device__ __forceinline__ void check_step(const vc_kv8& c, const vc_kv8_step& s, int32_t* status) {
  __shared__ int32_t err;
  if (threadIdx.x == 0) err = VC_OK;
  __syncthreads();
  const int lane = threadIdx.x & 31;
  for (int r0 = (int)threadIdx.x - lane; r0 < s.n_req; r0 += blockDim.x) {
    const int r = r0 + lane;
    int j0 = 0, cnt = 0;
    if (r < s.n_req) {
      const Req8 q = load_req(s, PAGE, r, &err);
      const int lo = max(q.len - q.m, 0);
      j0 = lo / PAGE;
      cnt = q.len > lo ? (q.len - 1) / PAGE - j0 + 1 : 0;
      for (int k = 0; k < min(cnt, 2); ++k) load_page(s, c.n_pages, r, j0 + k, &err);
    }
    for (uint32_t many = __ballot_sync(0xffffffffu, cnt > 2); many; many &= many - 1) {
      const int src = __ffs(many) - 1;
      const int first = __shfl_sync(0xffffffffu, j0, src), n = __shfl_sync(0xffffffffu, cnt, src);
      for (int k = 2 + lane; k < n; k += 32) load_page(s, c.n_pages, r0 + src, first + k, &err);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) *status = err;
}

// A block's page: the touch, the page and the slots [a, b) of the step's tokens;
// false where there is nothing to do.  All threads of the block call it.
struct PageJob {
  int64_t row;           // packed row of slot 0 (it may lie before the first)
  int p, a, b;
};
template <int PAGE>
__device__ __forceinline__ bool find_job(const vc_kv8& c, const vc_kv8_step& s, int32_t* status, PageJob& job) {
  if (blockIdx.x == 0) {
    if (blockIdx.y == 0) check_step<PAGE>(c, s, status);
    return false;
  }
  __shared__ PageJob sj;
  if (threadIdx.x < 32) {
    Touch x = {};
    const bool ok = find_touch<PAGE>(s, (int)blockIdx.x - 1, nullptr, x);
    if (threadIdx.x == 0) {
      sj.p = ok ? load_page(s, c.n_pages, x.r, x.j, nullptr) : -1;
      sj.a = max(x.first - x.j * PAGE, 0);
      sj.b = min(x.len - x.j * PAGE, PAGE);
      sj.row = (int64_t)x.row0 + (x.j * PAGE - x.first);
    }
  }
  __syncthreads();
  job = sj;
  return job.p >= 0;
}

// Unit u of a page: KV head u % Hkv of K (u < Hkv) or of V.
template <typename T, int D, int PAGE>
__global__ void __launch_bounds__(UnitCfg<D, PAGE>::THREADS, UnitCfg<D, PAGE>::blocks(sizeof(T))) kv8_append_kernel(
    const __grid_constant__ vc_kv8 c, const __grid_constant__ vc_kv8_step s, const __grid_constant__ Kv8Rows rows,
    int32_t* status) {
  using C = UnitCfg<D, PAGE>;
  __shared__ uint32_t red[2][C::THREADS / 32];
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  PageJob job;
  if (!find_job<PAGE>(c, s, status, job)) return;
  const int a = job.a, b = job.b;                       // slots [0, a) hold older tokens
  Raw16<T> next[C::NV];
  auto load = [&](int u) {
    const bool isv = u >= c.Hkv;
    const int g = isv ? u - c.Hkv : u;
    const int64_t rstep = isv ? rows.v_row : rows.k_row;
    const T* src = static_cast<const T*>(isv ? rows.V : rows.K) + (int64_t)g * (isv ? rows.v_head : rows.k_head) +
                   job.row * rstep;
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int vec = t + i * C::THREADS, slot = vec / C::VPR, part = vec % C::VPR;
      if (slot >= a && slot < b) next[i].load(src + (int64_t)slot * rstep + part * 16);
    }
  };
  int u = blockIdx.y, turn = 0;
  load(u);
  for (; u < 2 * c.Hkv; u += gridDim.y) {
    const bool isv = u >= c.Hkv;
    const int g = isv ? u - c.Hkv : u;
    float* scale = (isv ? c.V_scale : c.K_scale) + (int64_t)job.p * c.Hkv + g;
    uint8_t* codes = static_cast<uint8_t*>(isv ? c.V_codes : c.K_codes) + ((int64_t)job.p * c.Hkv + g) * (PAGE * D);
    const float old = a > 0 ? *scale : 0.f;
    Raw16<T> cur[C::NV];
#pragma unroll
    for (int i = 0; i < C::NV; ++i) cur[i] = next[i];
    if (u + (int)gridDim.y < 2 * c.Hkv) load(u + gridDim.y);
    // the block's largest magnitude; with a value that is not finite among them,
    // once more over the finite ones
    auto block_max = [&](uint32_t m) {
      m = __reduce_max_sync(0xffffffffu, m);
      if (lane == 0) red[turn][warp] = m;
      turn ^= 1;
      __syncthreads();                          // (the other row is read before the next barrier)
#pragma unroll
      for (int k = 0; k < C::THREADS / 32; ++k) m = max(m, red[turn ^ 1][k]);
      return m;
    };
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int slot = (t + i * C::THREADS) / C::VPR;
      if (slot >= a && slot < b) m = max(m, cur[i].largest());
    }
    m = block_max(m);
    const bool all_finite = m < 0x7f800000u;
    if (!all_finite) {
      m = 0u;
#pragma unroll
      for (int i = 0; i < C::NV; ++i) {
        const int slot = (t + i * C::THREADS) / C::VPR;
        if (slot >= a && slot < b) m = max(m, cur[i].largest_finite());
      }
      m = block_max(m);
    }
    const float amax = __uint_as_float(m);
    const float now = fmaxf(old, pow2_scale(amax));
    const float inv = pow2_inverse(now);
    // at the largest scale, 2^120, a code of 256 would stand for 2^128: no number
    const bool largest = now >= 0x1p120f;
    const float top = largest ? 240.f : 448.f;
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int vec = t + i * C::THREADS, slot = vec / C::VPR;
      if (slot >= a && slot < b) {
        float v[16];
        cur[i].get(v);
        *reinterpret_cast<uint4*>(codes + (size_t)vec * 16) =
            all_finite && !largest ? encode16<false>(v, inv, top) : encode16<true>(v, inv, top);
      }
    }
    if (now > old) {
      // older codes under the larger scale: value * old is exact (e4m3 has four
      // bits above 2^-135), the division by a power of two as well
      for (int vec = t; vec < a * C::VPR; vec += C::THREADS) {
        uint4* w = reinterpret_cast<uint4*>(codes + (size_t)vec * 16);
        float y[16];
        decode16(*w, y);
#pragma unroll
        for (int k = 0; k < 16; ++k) y[k] *= old;
        *w = encode16<true>(y, inv, top);
      }
    }
    if (t == 0) *scale = now;
  }
}

template <typename T, int D, int PAGE>
__global__ void __launch_bounds__(UnitCfg<D, PAGE>::THREADS, UnitCfg<D, PAGE>::blocks(sizeof(T))) kv8_read_kernel(
    const __grid_constant__ vc_kv8 c, const __grid_constant__ vc_kv8_step s, const __grid_constant__ Kv8Rows rows,
    int32_t* status) {
  using C = UnitCfg<D, PAGE>;
  const int t = threadIdx.x;
  PageJob job;
  if (!find_job<PAGE>(c, s, status, job)) return;
  const int a = job.a, b = job.b;
  uint4 next[C::NV];
  float nscale = 0.f;
  auto load = [&](int u) {
    const bool isv = u >= c.Hkv;
    const int64_t unit = (int64_t)job.p * c.Hkv + (isv ? u - c.Hkv : u);
    nscale = __ldg((isv ? c.V_scale : c.K_scale) + unit);
    const uint8_t* codes = static_cast<const uint8_t*>(isv ? c.V_codes : c.K_codes) + unit * (PAGE * D);
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int vec = t + i * C::THREADS, slot = vec / C::VPR;
      if (slot >= a && slot < b) next[i] = __ldg(reinterpret_cast<const uint4*>(codes + (size_t)vec * 16));
    }
  };
  int u = blockIdx.y;
  load(u);
  for (; u < 2 * c.Hkv; u += gridDim.y) {
    const bool isv = u >= c.Hkv;
    const int g = isv ? u - c.Hkv : u;
    const int64_t rstep = isv ? rows.v_row : rows.k_row;
    T* dst = static_cast<T*>(isv ? rows.V : rows.K) + (int64_t)g * (isv ? rows.v_head : rows.k_head) +
             job.row * rstep;
    const float scale = nscale;
    uint4 cur[C::NV];
#pragma unroll
    for (int i = 0; i < C::NV; ++i) cur[i] = next[i];
    if (u + (int)gridDim.y < 2 * c.Hkv) load(u + gridDim.y);
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int vec = t + i * C::THREADS, slot = vec / C::VPR, part = vec % C::VPR;
      if (slot >= a && slot < b) {
        float v[16];
        decode16(cur[i], v);
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] *= scale;
        store16(dst + (int64_t)slot * rstep + part * 16, v);
      }
    }
  }
}

// Pages the step may touch: a request with m > 0 rows touches at most
// ceil(m / page) + 1.
template <int PAGE>
int64_t most_pages(const vc_kv8_step& s) {
  return s.n_rows / PAGE + 2 * (int64_t)(s.n_req < s.n_rows ? s.n_req : s.n_rows);
}

template <typename T, int D, int PAGE>
cudaError_t launch_t(bool append, const vc_kv8& c, const vc_kv8_step& s, const Kv8Rows& rows, int32_t* status,
                     cudaStream_t st) {
  ProfileScope ps(append ? "kv8_append" : "kv8_read", st);
  // blocks a page: as many as make the device full at 1280 threads an SM, since
  // a step of few rows is as long as one block's turn; three (two with
  // fp32 rows or four vectors a thread) where there are pages enough, so that
  // the last blocks to start are short.  Us with 152 * 8 blocks in all and no least number / so:
  //   64 requests' next tokens, 8 KV heads of 128, pages of 64: append 6.0 / 5.4, read 4.9 / 3.7
  //   32 of 4096 tokens, 8 of 128, pages of 64: append 121.8 / 120.4, read 141.6 / 134.5
  //   32 of 4096 tokens, 8 of 128, pages of 16: append 165.1 / 140.7, read 189.7 / 147.5
  //   32 of 4096 tokens, 4 of 64, pages of 16: append 92.4 / 61.9, read 101.7 / 63.3
  const int64_t pages = most_pages<PAGE>(s);
  constexpr int threads = UnitCfg<D, PAGE>::THREADS;
  int64_t split = ((int64_t)kv8_sm_count() * (1280 / threads) + pages - 1) / pages;
  constexpr int least = UnitCfg<D, PAGE>::blocks(sizeof(T)) > 1 ? 3 : 2;
  if (split < least) split = least;
  if (split > 2 * c.Hkv) split = 2 * c.Hkv;
  const dim3 grid((unsigned)pages + 1, (unsigned)split);
  if (append) kv8_append_kernel<T, D, PAGE><<<grid, UnitCfg<D, PAGE>::THREADS, 0, st>>>(c, s, rows, status);
  else kv8_read_kernel<T, D, PAGE><<<grid, UnitCfg<D, PAGE>::THREADS, 0, st>>>(c, s, rows, status);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_p(bool append, const vc_kv8& c, const vc_kv8_step& s, const Kv8Rows& rows, int32_t* status,
                     cudaStream_t st) {
  switch (c.page) {
    case 16: return launch_t<T, D, 16>(append, c, s, rows, status, st);
    case 32: return launch_t<T, D, 32>(append, c, s, rows, status, st);
    case 64: return launch_t<T, D, 64>(append, c, s, rows, status, st);
    default: return launch_t<T, D, 128>(append, c, s, rows, status, st);
  }
}

cudaError_t launch(bool append, const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8Rows& rows,
                   int32_t* status, cudaStream_t st) {
  if (s.n_rows == 0) return cudaMemsetAsync(status, 0, sizeof(int32_t), st);
  if (dtype == VC_BF16)
    return c.d == 128 ? launch_p<__nv_bfloat16, 128>(append, c, s, rows, status, st)
                      : launch_p<__nv_bfloat16, 64>(append, c, s, rows, status, st);
  return c.d == 128 ? launch_p<float, 128>(append, c, s, rows, status, st)
                    : launch_p<float, 64>(append, c, s, rows, status, st);
}

}  // namespace

cudaError_t launch_kv8_append(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8Rows& rows,
                              int32_t* status, cudaStream_t st) {
  return launch(true, c, s, dtype, rows, status, st);
}

cudaError_t launch_kv8_read(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8Rows& rows,
                            int32_t* status, cudaStream_t st) {
  return launch(false, c, s, dtype, rows, status, st);
}

}  // namespace vc
