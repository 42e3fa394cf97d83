// A cache held to a budget (viscache_kv8_evict): of each request and KV head the keep
// heaviest tokens stay and move together in place.
//
// Two kernels.  The first finds each (request, head)'s keep-th largest weight: keys that
// order like the weights (NaN lowest, protected tokens as +inf), three radix passes of
// 11, 11 and 10 bits over them with a histogram in shared memory, the keys themselves in
// shared memory where they fit; then one pass writes the tokens that stay, in order,
// ties by place.  Reads 4 bytes a token.
//
// The second moves codes, scales and weights of what stays behind the first gap: bound
// by memory, 2 d + 8 bytes a token each way for K and V.  A page's new scale needs all
// of its new tokens, and its old tokens may be read by pages before it, so a unit (K or V
// of a request and head) goes through its pages in waves: a wave's blocks (a cluster)
// load all of its tokens into registers, meet, and write.  A token only moves towards
// the front, so what a later wave reads lies in its own pages or behind them: the next
// wave's loads are issued before the current one's are waited for.  An e4m3 code under a
// power-of-two scale is re-encoded by a power of two, and only where that is not 1.
//
// 16 caches of up to 12544 tokens, 8 heads of 128, cut to 3136 (201 MB): 75 us from cold memory, the
// selection 19 of them, against 30 at a plain copy's rate: a wave is a chain of its loads, the
// largest value, the codes and the stores, 25 waves long.  A batch a page over its budget
// (16 requests of 1088 tokens, 4 heads): 15 us a call, two launches and their chains.
#include "kernels.h"
#include "kv8.cuh"
#include "kv8_sched.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace kv8;

// ---------------------------------------------------------------------------
// which tokens stay

constexpr int kSelThreads = 512;
constexpr int kBins = 2048;
constexpr int kMostCached = 24576;    // keys in shared memory: 96 KB, two blocks an SM

// Orders like the weight: NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w == w)) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
constexpr uint32_t kInfKey = 0xff800000u;
constexpr int kNoGap = 0x7fffffff;    // a request that is left as it is

// Exclusive sums of x and y over the block, and the totals; `scan`: a word a warp.
__device__ __forceinline__ int2 block_scan(int x, int* scan, int& total_x, int y, int* scan_y, int& total_y) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int ix = scan_warp(x), iy = scan_warp(y);
  if (lane == 31) {
    scan[warp] = ix;
    scan_y[warp] = iy;
  }
  __syncthreads();
  int bx = 0, by = 0;
  total_x = total_y = 0;
  for (int w = 0; w < kSelThreads / 32; ++w) {
    if (w < warp) {
      bx += scan[w];
      by += scan_y[w];
    }
    total_x += scan[w];
    total_y += scan_y[w];
  }
  return make_int2(bx + ix - x, by + iy - y);
}

__global__ void __launch_bounds__(kSelThreads) kv8_evict_select_kernel(const __grid_constant__ vc_kv8 c,
                                                                       const __grid_constant__ vc_kv8_step s,
                                                                       const __grid_constant__ Kv8EvictArgs a,
                                                                       int cached) {
  extern __shared__ uint32_t cache[];
  __shared__ int hist[kBins];
  __shared__ int scan[2][kSelThreads / 32];
  __shared__ int err, found_bin, found_need, found_all, gap;
  const int t = threadIdx.x, r = blockIdx.y, g = blockIdx.x, shift = __ffs(c.page) - 1;      // (pages are powers of two)
  if (t == 0) err = VC_OK;
  __syncthreads();
  const int cap = s.max_pages * c.page;
  int len = __ldg(s.seq_lens + r), keep = __ldg(a.keep + r);
  if (len < 0 || len > cap || keep < 0 || keep > a.max_keep) {
    if (t == 0) err = VC_ERR_DEVICE_INDEX;
    len = min(max(len, 0), cap);
    keep = min(max(keep, 0), a.max_keep);
  }
  const int pages = (len + c.page - 1) / c.page;
  bool bad = false;
  for (int j = t; j < pages; j += kSelThreads) bad = load_page(s, c.n_pages, r, j, nullptr) < 0 || bad;
  bad = __syncthreads_or(bad) != 0;
  const int64_t unit = (int64_t)r * c.Hkv + g;
  int32_t* kept = a.kept + unit * a.max_keep;
  if (bad || len <= keep) {
    if (!bad)
      for (int i = t; i < len; i += kSelThreads) kept[i] = i;
    if (t == 0) a.units[unit] = {kNoGap, len, bad ? VC_ERR_DEVICE_INDEX : err, 0};
    return;
  }
  if (keep == 0) {                              // nothing to choose
    if (t == 0) a.units[unit] = {0, 0, err, 0};
    return;
  }
  const int32_t* table = s.block_table + (int64_t)r * s.max_pages;
  auto fetch = [&](int i) {
    if (i < a.sink || i >= len - a.recent) return kInfKey;
    const int p = __ldg(table + (i >> shift));
    return weight_key(__ldg(a.weights + (((p * c.Hkv + g) << shift) + (i & (c.page - 1)))));
  };
  const bool held = len <= cached;
  if (held) {
    // eight tokens at a time: their pages, then their weights
    constexpr int kAtOnce = 8;
    for (int i0 = t; i0 < len; i0 += kAtOnce * kSelThreads) {
      int p[kAtOnce];
      float w[kAtOnce];
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const int i = i0 + n * kSelThreads;
        p[n] = i < len ? __ldg(table + (i >> shift)) : 0;
      }
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const int i = i0 + n * kSelThreads;
        w[n] = i < len ? __ldg(a.weights + (((p[n] * c.Hkv + g) << shift) + (i & (c.page - 1)))) : 0.f;
      }
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const int i = i0 + n * kSelThreads;
        if (i < len) cache[i] = i < a.sink || i >= len - a.recent ? kInfKey : weight_key(w[n]);
      }
    }
  }
  auto key = [&](int i) { return held ? cache[i] : fetch(i); };      // (of other threads' too: past a barrier)
  // the keep-th largest key: digit by digit from the top
  uint32_t prefix = 0u, mask = 0u;
  int need = keep;                              // how many of the keys under the prefix stay
  bool all = false;
  for (int pass = 0; pass < 3 && !all; ++pass) {
    const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = t; i < kBins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int i = t; i < len; i += kSelThreads) {
      const uint32_t k = key(i);
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> low) & ((1u << bits) - 1u)], 1);
    }
    __syncthreads();
    // threads from the top bin down
    constexpr int per = kBins / kSelThreads;
    int mine = 0;
#pragma unroll
    for (int i = 0; i < per; ++i) mine += hist[kBins - 1 - (t * per + i)];
    int total, unused;
    int above = block_scan(mine, scan[0], total, 0, scan[1], unused).x;
    if (above < need && need <= above + mine) {
      for (int i = 0; i < per; ++i) {
        const int b = kBins - 1 - (t * per + i), n = hist[b];
        if (need <= above + n) {
          found_bin = b;
          found_need = need - above;
          found_all = need == above + n;
          break;
        }
        above += n;
      }
    }
    __syncthreads();
    prefix |= (uint32_t)found_bin << low;
    mask |= ((1u << bits) - 1u) << low;
    need = found_need;
    all = found_all != 0;                       // every key under the prefix stays
    __syncthreads();
  }
  // tokens in order: those above the prefix, and of those under it the first `need`
  if (t == 0) gap = len;
  const int per = ((len + kSelThreads - 1) / kSelThreads) | 1;    // (odd: no two lanes on a bank)
  const int i0 = min(t * per, len), i1 = min(i0 + per, len);
  auto stays_over = [&](uint32_t k) { return all ? k >= prefix : k > prefix; };
  int over = 0, ties = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key(i);
    over += stays_over(k) ? 1 : 0;
    ties += k == prefix && !all ? 1 : 0;
  }
  int total, unused;
  const int2 before = block_scan(over, scan[0], total, ties, scan[1], unused);
  int tie = before.y, at = before.x + min(tie, need), first_gap = len;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key(i);
    bool stays = stays_over(k);
    if (k == prefix && !all) stays = tie++ < need;
    if (stays) kept[at++] = i;
    else first_gap = min(first_gap, i);
  }
  if (first_gap < len) atomicMin(&gap, first_gap);
  __syncthreads();
  if (t == 0) a.units[unit] = {gap, keep, err, 0};
}

// ---------------------------------------------------------------------------
// what stays moves together

// 16 caches of up to 12544 tokens cut to 3136, 8 heads of 128, us of both kernels (cold): 256 threads 90,
// 512 75, 1024 75; 32 KB of codes a step and 512 threads 87.
constexpr int kMoveThreads = 512, kMoveBytes = 16384;   // codes of a block's step
constexpr int kNV = kMoveBytes / 16 / kMoveThreads;     // 16-code vectors of a thread

// The largest magnitude of sixteen codes, NaN left out.
__device__ __forceinline__ float largest_code(const uint4& w) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  __half2 m = __float2half2_rn(0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t b = e4m3x2_to_f16x2(x[i] >> (16 * h));
      m = __hmax2(m, __habs2(*reinterpret_cast<const __half2*>(&b)));
    }
  }
  return fmaxf(__low2float(m), __high2float(m));
}

// Sixteen codes times f = 2^k, 2^-24 <= f <= 2^15, to nearest even.  In fp16: a product that is not exact there
// is below 2^-20, which e4m3 rounds to 0 like anything below 2^-10.
__device__ __forceinline__ uint4 scale_codes(const uint4& w, float f) {
  const __half2 f2 = __float2half2_rn(f);
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t r[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t b = e4m3x2_to_f16x2(x[i] >> (16 * h));
      const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&b), f2);
      unsigned short o;
      asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(o) : "r"(*reinterpret_cast<const uint32_t*>(&z)));
      r[h] = o;
    }
    y[i] = r[0] | r[1] << 16;
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}

// Grid: clusters of C blocks, one for each unit: (request, head) x {K, V}.
template <int D>
__global__ void __launch_bounds__(kMoveThreads, 2) kv8_evict_move_kernel(const __grid_constant__ vc_kv8 c,
                                                                      const __grid_constant__ vc_kv8_step s,
                                                                      const __grid_constant__ Kv8EvictArgs a, int C) {
  constexpr int VPR = D / 16, TS = kMoveBytes / D;      // vectors of a token, tokens of a step
  __shared__ uint32_t amax[2][TS / 16];                 // by wave & 1 and page of the step
  dep_wait();
  const int t = threadIdx.x;
  const int rank = (int)blockIdx.x % C, u = (int)blockIdx.x / C;
  const bool isv = (u & 1) != 0;
  const int unit = u >> 1, r = unit / c.Hkv, g = unit - r * c.Hkv;
  if (blockIdx.x == 0) {
    // the call's status, and the lengths (seq_lens itself may be where they go)
    int32_t e = VC_OK;
    for (int i = t; i < s.n_req; i += kMoveThreads) {
      const Kv8Unit x = a.units[(int64_t)i * c.Hkv];
      a.new_lens[i] = x.len;
      if (x.err != VC_OK) e = x.err;
    }
    e = __syncthreads_or(e != VC_OK) ? VC_ERR_DEVICE_INDEX : VC_OK;
    if (t == 0) *a.status = e;
  }
  const Kv8Unit un = a.units[unit];
  const int shift = __ffs(c.page) - 1;
  const int first = un.gap & ~(c.page - 1);             // token from which pages are written
  if (first >= un.len) return;                          // (the whole cluster)
  const int steps = (un.len - first + TS - 1) / TS, waves = (steps + C - 1) / C;
  const int32_t* table = s.block_table + (int64_t)r * s.max_pages;
  const int32_t* kept = a.kept + (int64_t)unit * a.max_keep;
  uint8_t* codes = static_cast<uint8_t*>(isv ? c.V_codes : c.K_codes);
  float* scales = isv ? c.V_scale : c.K_scale;
  for (int i = t; i < 2 * (TS / 16); i += kMoveThreads) amax[i / (TS / 16)][i % (TS / 16)] = 0u;

  // (page, head) slot of a token of this head: slot / page is the scale's index
  auto slot_of = [&](int token) {
    const int p = __ldg(table + (token >> shift));
    return ((p * c.Hkv + g) << shift) + (token & (c.page - 1));      // (all slots of a pool: below 2^31)
  };
  // A wave's loads hang on one another: kept tokens, their pages, codes.  Each is sent for a wave before the
  // next one needs it.
  struct Wave {
    uint4 w[kNV];
    float scale[kNV], weight;
  };
  struct Places {
    int of[kNV], weight;                        // kept tokens, then their slots; of the token whose weight the thread moves
  };
  Wave cur, nxt;
  Places tokens, slots;
  const int part = t % VPR;
  auto token = [&](int wave, int i) { return first + (wave * C + rank) * TS + (t + i * kMoveThreads) / VPR; };
  auto weight_token = [&](int wave) { return first + (wave * C + rank) * TS + t; };
  auto moves_weight = [&](int wave) { return !isv && t < TS && weight_token(wave) < un.len; };
  auto load_tokens = [&](int wave) {
#pragma unroll
    for (int i = 0; i < kNV; ++i)
      if (token(wave, i) < un.len) tokens.of[i] = __ldg(kept + token(wave, i));
    if (moves_weight(wave)) tokens.weight = __ldg(kept + weight_token(wave));
  };
  auto load_slots = [&](int wave) {
#pragma unroll
    for (int i = 0; i < kNV; ++i)
      if (token(wave, i) < un.len) slots.of[i] = slot_of(tokens.of[i]);
    if (moves_weight(wave)) slots.weight = slot_of(tokens.weight);
  };
  auto load = [&](int wave, Wave& x) {
#pragma unroll
    for (int i = 0; i < kNV; ++i)
      if (token(wave, i) < un.len) {
        x.w[i] = __ldcg(reinterpret_cast<const uint4*>(codes + (int64_t)slots.of[i] * D) + part);
        x.scale[i] = __ldcg(scales + (slots.of[i] >> shift));
      }
    if (moves_weight(wave)) x.weight = __ldcg(a.weights + slots.weight);
  };
  load_tokens(0);
  load_slots(0);
  load_tokens(1);
  load(0, cur);
  load_slots(1);
  load_tokens(2);
  __syncthreads();                                      // amax is cleared
  for (int wave = 0; wave < waves; ++wave) {
    load(wave + 1, nxt);
    load_slots(wave + 2);
    load_tokens(wave + 3);
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const bool on = token(wave, i) < un.len;
      const float m = on ? largest_code(cur.w[i]) * cur.scale[i] : 0.f;
      const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
      // (a warp's tokens lie on one page)
      if ((t & 31) == 0) atomicMax(&amax[wave & 1][(t + i * kMoveThreads) / VPR >> shift], top);
    }
    __syncwarp();
    if (C > 1) tc::cluster_sync();
    else __syncthreads();
    // all of the wave's tokens are in registers: its pages may be written
#pragma unroll
    for (int i = 0; i < kNV; ++i) {
      const int to = token(wave, i);
      if (to < un.len) {
        const int slot = (t + i * kMoveThreads) / VPR;
        const float now = pow2_scale(__uint_as_float(amax[wave & 1][slot >> shift]));
        // a token of zeros may have any scale: a factor past e4m3's range is not needed
        const float f = fminf(cur.scale[i] * pow2_inverse(now), 0x1p20f);
        uint4 y = cur.w[i];
        if (f != 1.f) y = f <= 0x1p15f ? scale_codes(y, fmaxf(f, 0x1p-24f)) : scale_codes(scale_codes(y, 0x1p8f), f * 0x1p-8f);
        const int dst = slot_of(to);
        reinterpret_cast<uint4*>(codes + (int64_t)dst * D)[part] = y;
        if (part == 0 && (to & (c.page - 1)) == 0) scales[dst >> shift] = now;
      }
    }
    if (moves_weight(wave)) a.weights[slot_of(weight_token(wave))] = cur.weight;
    __syncthreads();
    if (t < TS / 16) amax[wave & 1][t] = 0u;            // (used again two barriers on)
    cur = nxt;
  }
}

template <int D>
cudaError_t launch_move(const vc_kv8& c, const vc_kv8_step& s, const Kv8EvictArgs& a, cudaStream_t st) {
  const int64_t units = (int64_t)s.n_req * c.Hkv * 2;
  const int64_t most = (int64_t)s.max_pages * c.page < a.max_keep ? (int64_t)s.max_pages * c.page : a.max_keep;
  const int64_t steps = (most * D + kMoveBytes - 1) / kMoveBytes;
  // blocks of a unit: while there are SMs without one (two an SM: 93 us instead of 75 in the case above, whose
  // 240 units fill the device; a wave's end is felt)
  int C = 1;
  while (C < 8 && units * C < kv8_sm_count() && C < steps) C *= 2;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * C));
  cfg.blockDim = dim3(kMoveThreads);
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = g_dependent_launch.load(std::memory_order_relaxed) ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kv8_evict_move_kernel<D>, c, s, a, C);
}

}  // namespace

cudaError_t launch_kv8_evict(const vc_kv8& c, const vc_kv8_step& s, const Kv8EvictArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = kv8_allow_smem(reinterpret_cast<const void*>(kv8_evict_select_kernel), kMostCached * 4, allowed);
  if (e != cudaSuccess) return e;
  const int64_t cap = (int64_t)s.max_pages * c.page;
  const int cached = (int)(cap < kMostCached ? cap : kMostCached);
  ProfileScope ps("kv8_evict", st);
  kv8_evict_select_kernel<<<dim3((unsigned)c.Hkv, (unsigned)s.n_req), kSelThreads, sizeof(uint32_t) * cached, st>>>(
      c, s, a, cached);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return c.d == 128 ? launch_move<128>(c, s, a, st) : launch_move<64>(c, s, a, st);
}

}  // namespace vc
