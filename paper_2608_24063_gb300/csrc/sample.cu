// The next token of each row of logits (viscache_sample): temperature, top-k, top-p,
// min-p and a given random number.
//
// w_i = 2^-z_i, z_i = (M - x_i) log2(e) / T.  What the filters keep is a prefix of the order by
// (logit descending, index), so each filter is a cut: a logit, and how many of the tokens
// that tie with it, lowest index first.  The token is where the kept weights, in order of
// index, first pass u times their sum.
//
// Reads the logits once: a cluster of C blocks holds a row in shared memory, and
// everything after works there.  Passes: (1) load, maximum; (2) weights summed, with
// top-k or top-p into a histogram of buckets of 1/16 in z; (3) for a cut that falls
// inside a bucket, histograms of ever finer ranges of keys until one logit is left;
// (4) sums of the kept weights of each thread's run of tokens, a scan, and the one warp
// that holds the token looks through its run.
//
// A token is a whole number: an answer off by one border is wrong, and rows have up to
// 262144 borders, so weights are computed to about 40 bits (pairs of fp32 numbers, a table
// of 2^(-i/64) and a polynomial of degree 4) and added as 64-bit whole numbers: exact in
// any order, so atomics and the split over blocks do not change a result.
#include "kernels.h"
#include "kv8_sched.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using kv8::scan_warp;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBuckets = 1024;
constexpr float kPerZ = 16.f;                   // buckets of 1 in z: z < 64
constexpr int kTableBits = 47;

// 2^(47 - i / 64), rounded
__constant__ uint64_t kPowers[64] = {
    0x800000000000ull, 0x7e9f06067a43ull, 0x7d41d96db915ull, 0x7be86fb98569ull, 0x7a92be8a9243ull, 0x7940bb9e2d00ull,
    0x77f25ccdee6dull, 0x76a7980f6ccaull, 0x75606373ee92ull, 0x741cb5281e26ull, 0x72dc8373be42ull, 0x719fc4b95f45ull,
    0x70666f76154aull, 0x6f307a412f07ull, 0x6dfddbcbed79ull, 0x6cce8ae13c58ull, 0x6ba27e656b4full, 0x6a79ad55e7f7ull,
    0x69540ec8f895ull, 0x683199ed7796ull, 0x6712460a8fc2ull, 0x65f60a7f7939ull, 0x64dcdec33718ull, 0x63c6ba6455ddull,
    0x62b39508aa83ull, 0x61a3666d124cull, 0x609626653338ull, 0x5f8bccdb3d3aull, 0x5e8451cfac06ull, 0x5d7fad59099full,
    0x5c7dd7a3b17eull, 0x5b7ec8f19469ull, 0x5a827999fcefull, 0x5988e2095489ull, 0x5891fac0e956ull, 0x579dbc56b485ull,
    0x56ac1f752151ull, 0x55bd1cdad49full, 0x54d0ad5a753eull, 0x53e6c9da74b3ull, 0x52ff6b54d8a9ull, 0x521a8ad704f3ull,
    0x513821818625ull, 0x50582887dcb9ull, 0x4f7a993048d1ull, 0x4e9f6cd39680ull, 0x4dc69cdceaa7ull, 0x4cf022c9905cull,
    0x4c1bf828c6dcull, 0x4b4a169b900cull, 0x4a7a77d47f7cull, 0x49ad159789f3ull, 0x48e1e9b9d589ull, 0x4818ee218a33ull,
    0x47521cc5a2e7ull, 0x468d6fadbf2eull, 0x45cae0f1f546ull, 0x450a6abaa4b7ull, 0x444c0740496dull, 0x438fb0cb4f47ull,
    0x42d561b3e624ull, 0x421d1461d66full, 0x4166c34c5616ull, 0x40b268f9de02ull
};

// Weights of a row's logits.
struct Weights {
  float M, ch, cl;                              // the maximum times `small`; log2(e) / (T small) = ch + cl
  float small;                                  // 1; 2^-90 where T is past 2^90: then M - x stays in range
  int q;                                        // a weight of 1 is 2^q
  const uint64_t* table;

  __device__ __forceinline__ uint64_t one() const { return (uint64_t)1 << q; }
  // z to fp32, never decreasing as x falls; infinite (or NaN, of an infinite T) for -inf
  __device__ __forceinline__ float z_of(float x) const {
    x *= small;
    return x == M ? 0.f : (M - x) * ch;
  }
  __device__ __forceinline__ int bucket(float x) const { return (int)fminf(z_of(x) * kPerZ, (float)(kBuckets - 1)); }
  __device__ __forceinline__ uint64_t of(float x) const {
    x *= small;
    if (x == M) return one();
    const float d = M - x;
    const float zh = d * ch;
    if (!(zh < 63.f)) return 0;
    // d's rounding, and z in two parts
    const float b = d - M, de = (M - (d - b)) + (-x - b);
    const float zl = fmaf(de, ch, fmaf(d, cl, fmaf(d, ch, -zh)));
    const float jf = rintf(zh * 64.f);
    const float g = fmaf(jf, -1.f / 64.f, zh);  // exact, |g| <= 1/128
    const int j = (int)jf;
    const uint64_t ti = table[j & 63];
    const float th = (float)(uint32_t)(ti >> 24) * 0x1p-23f, tl = (float)(uint32_t)(ti & 0xffffffu) * 0x1p-47f;
    // 2^-(g + zl) = e^-y, y = yh + yl
    constexpr float kLn2 = 0.693147182f, kLn2Lo = -1.904654323e-9f;
    const float yh = g * kLn2;
    const float yl = fmaf(zl, kLn2, fmaf(g, kLn2Lo, fmaf(g, kLn2, -yh)));
    const float sq = yh * yh * fmaf(yh, fmaf(yh, 1.f / 24.f, -1.f / 6.f), 0.5f);
    // T (1 - yh + (sq - yl)) - T, in two parts
    const float p = th * yh;
    const float e = sq - yl, r = fmaf(th, e, fmaf(tl, e, fmaf(-tl, yh, -fmaf(th, yh, -p))));
    const int64_t v = (int64_t)ti - __float2ll_rn(p * 0x1p47f) + __float2ll_rn(r * 0x1p47f);
    const int sh = (j >> 6) + kTableBits - q;
    return sh > 60 ? 0 : sh == 0 ? (uint64_t)v : ((uint64_t)v + ((uint64_t)1 << (sh - 1))) >> sh;
  }
};

// Orders like the logit.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}

// What a row's blocks share.
struct Shared {
  uint64_t table[64];
  uint64_t mass[2][kBuckets], mass_all[kBuckets];       // the block's, by turn; the cluster's
  uint32_t count[2][kBuckets], count_all[kBuckets];
  uint64_t warp_mass[kWarps];
  uint32_t warp_count[kWarps];
  uint64_t mine[8][2];                                  // what the block tells the others, by turn
  uint64_t found[4];
};

static_assert(sizeof(Shared) % 16 == 0, "the slice behind it is read in vectors");

struct Row {
  int C, rank, turn, told;
  Shared* sm;

  __device__ __forceinline__ void sync() const {
    __syncwarp();
    if (C > 1) tc::cluster_sync();
    else __syncthreads();
  }
  template <typename V>
  __device__ __forceinline__ V read(const V* p, int rank_of) const {
    const uint32_t at = tc::map_to_rank(tc::smem_u32(p), (uint32_t)rank_of);
    if constexpr (sizeof(V) == 8) {
      uint64_t v;
      asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
      return (V)v;
    } else {
      uint32_t v;
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
      return (V)v;
    }
  }
};

// A cut of the order: logits with keys above `key` are before it, and of those equal to
// it the first `ties`.
struct Cut {
  uint32_t key, ties;
};

template <typename T>
__device__ __forceinline__ float element(const uint8_t* data, int i);
template <>
__device__ __forceinline__ float element<float>(const uint8_t* data, int i) {
  return reinterpret_cast<const float*>(data)[i];
}
template <>
__device__ __forceinline__ float element<__nv_bfloat16>(const uint8_t* data, int i) {
  return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(data)[i] << 16);
}

// Calls f(x) for every element of vectors t, t + kThreads, ... of the slice.
template <typename T, typename F>
__device__ __forceinline__ void each(const uint8_t* data, int vecs, F f) {
  constexpr int E = 16 / sizeof(T);
  for (int v = threadIdx.x; v < vecs; v += kThreads) {
    const uint4 w = reinterpret_cast<const uint4*>(data)[v];
    const uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if constexpr (sizeof(T) == 4) f(__uint_as_float(b[i]));
      else f(__uint_as_float(i & 1 ? b[i >> 1] & 0xffff0000u : b[i >> 1] << 16));
    }
  }
}

__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Sum of x over the cluster; with `before` also of the threads in front of this one
// (blocks by rank, then threads).  All threads call it.
__device__ __forceinline__ uint64_t cluster_sum(Row& row, uint64_t x, uint64_t* before) {
  Shared& sm = *row.sm;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint64_t incl = scan_warp(x);
  __syncthreads();                              // (what was in the words is read)
  if (lane == 31) sm.warp_mass[warp] = incl;
  __syncthreads();
  uint64_t b = 0, sum = 0;
  for (int w = 0; w < kWarps; ++w) {
    const uint64_t v = sm.warp_mass[w];
    if (w < warp) b += v;
    sum += v;
  }
  b += incl - x;
  if (row.C > 1) {
    uint64_t* word = &sm.mine[row.told & 7][0];
    ++row.told;
    if (threadIdx.x == 0) *word = sum;
    row.sync();
    uint64_t all = 0;
    for (int c = 0; c < row.C; ++c) {
      const uint64_t v = row.read(word, c);
      if (c < row.rank) b += v;
      all += v;
    }
    sum = all;
  }
  if (before) *before = b;
  return sum;
}

__device__ __forceinline__ uint64_t cluster_max(Row& row, uint64_t x) {
  Shared& sm = *row.sm;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const uint64_t y = __shfl_xor_sync(0xffffffffu, x, o);
    if (y > x) x = y;
  }
  __syncthreads();
  if (lane == 0) sm.warp_mass[warp] = x;
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) {
    const uint64_t y = sm.warp_mass[w];
    if (y > x) x = y;
  }
  if (row.C > 1) {
    uint64_t* word = &sm.mine[row.told & 7][0];
    ++row.told;
    if (threadIdx.x == 0) *word = x;
    row.sync();
    for (int c = 0; c < row.C; ++c) {
      const uint64_t y = row.read(word, c);
      if (y > x) x = y;
    }
  }
  return x;
}

// The cluster's histogram from its blocks', into count_all and mass_all.  Blocks fill
// the turn's histogram, then all call it.
__device__ __forceinline__ void clear_histogram(Row& row) {
  Shared& sm = *row.sm;
  row.turn ^= 1;
  for (int i = threadIdx.x; i < kBuckets; i += kThreads) {
    sm.mass[row.turn][i] = 0;
    sm.count[row.turn][i] = 0;
  }
  __syncthreads();
}
__device__ __forceinline__ void join_histogram(Row& row) {
  Shared& sm = *row.sm;
  row.sync();
  for (int i = threadIdx.x; i < kBuckets; i += kThreads) {
    uint64_t m = 0;
    uint32_t n = 0;
    for (int c = 0; c < row.C; ++c) {
      if (row.C > 1) {
        m += row.read(&sm.mass[row.turn][i], c);
        n += row.read(&sm.count[row.turn][i], c);
      } else {
        m = sm.mass[row.turn][i];
        n = sm.count[row.turn][i];
      }
    }
    sm.mass_all[i] = m;
    sm.count_all[i] = n;
  }
  __syncthreads();
}
// The first bucket at whose end the running count (or mass) reaches `need` (>= 1): its
// index, and the count and mass before it; false if all together do not.
struct Place {
  int bucket;
  uint64_t count, mass;                         // before it
};
__device__ __forceinline__ bool find_place(Row& row, bool by_mass, uint64_t need, Place& at) {
  Shared& sm = *row.sm;
  constexpr int per = kBuckets / kThreads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t m[per], ms = 0;
  uint32_t n[per], ns = 0;
#pragma unroll
  for (int i = 0; i < per; ++i) {
    m[i] = sm.mass_all[threadIdx.x * per + i];
    n[i] = sm.count_all[threadIdx.x * per + i];
    ms += m[i];
    ns += n[i];
  }
  const uint64_t im = scan_warp(ms);
  const uint32_t in = scan_warp(ns);
  if (lane == 31) {
    sm.warp_mass[warp] = im;
    sm.warp_count[warp] = in;
  }
  if (threadIdx.x == 0) sm.found[0] = kBuckets;
  __syncthreads();
  uint64_t bm = im - ms, bn = in - ns;
  for (int w = 0; w < warp; ++w) {
    bm += sm.warp_mass[w];
    bn += sm.warp_count[w];
  }
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const uint64_t from = by_mass ? bm : bn, to = from + (by_mass ? m[i] : n[i]);
    if (from < need && need <= to) {
      sm.found[0] = threadIdx.x * per + i;
      sm.found[1] = bn;
      sm.found[2] = bm;
    }
    bm += m[i];
    bn += n[i];
  }
  __syncthreads();
  at.bucket = (int)sm.found[0];
  at.count = sm.found[1];
  at.mass = sm.found[2];
  __syncthreads();
  return at.bucket < kBuckets;
}

// Where in bucket `at` the count (or mass) reaches `need`: the cut, and the mass up to it.
template <typename T>
__device__ __forceinline__ Cut find_cut(Row& row, const Weights& wt, const uint8_t* data, int vecs, bool by_mass,
                                        uint64_t need, Place at, uint64_t& mass) {
  // the keys of the bucket
  uint64_t lo = 0, hi = 0;                      // as largest of ~key and of key
  each<T>(data, vecs, [&](float x) {
    if (x != -INFINITY && wt.bucket(x) == at.bucket) {
      const uint32_t k = key_of(x);
      hi = max(hi, (uint64_t)k);
      lo = max(lo, (uint64_t)(~k));
    }
  });
  uint32_t top = (uint32_t)cluster_max(row, hi), low = ~(uint32_t)cluster_max(row, lo);
  mass = at.mass;
  uint64_t count = at.count;
  Shared& sm = *row.sm;
  for (;;) {
    const int bits = 32 - __clz((int)(top - low) | 1);
    const int shift = bits > 10 ? bits - 10 : 0;
    clear_histogram(row);
    each<T>(data, vecs, [&](float x) {
      const uint32_t k = key_of(x);
      if (k >= low && k <= top) {
        const uint32_t b = (top - k) >> shift;
        atomicAdd(&sm.count[row.turn][b], 1u);
        atomicAdd(reinterpret_cast<unsigned long long*>(&sm.mass[row.turn][b]), (unsigned long long)wt.of(x));
      }
    });
    join_histogram(row);
    Place p;
    find_place(row, by_mass, need - (by_mass ? mass : count), p);
    mass += p.mass;
    count += p.count;
    top -= (uint32_t)p.bucket << shift;
    if (shift == 0) {
      Cut cut;
      cut.key = top;
      const uint64_t w = wt.of(logit_of(top));
      cut.ties = (uint32_t)(by_mass ? (need - mass + w - 1) / w : need - count);
      mass += cut.ties * w;
      return cut;
    }
    const uint32_t width = (1u << shift) - 1u;
    low = top - low > width ? top - width : low;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sm = *reinterpret_cast<Shared*>(smem);
  uint8_t* data = smem + sizeof(Shared);
  constexpr int E = 16 / sizeof(T);
  const int t = threadIdx.x, lane = t & 31;
  Row row;
  row.C = a.C;
  row.rank = (int)blockIdx.x % a.C;
  row.turn = 0;
  row.told = 0;
  row.sm = &sm;
  const int r = (int)blockIdx.x / a.C;
  if (t < 64) sm.table[t] = kPowers[t];

  // (1) the slice: vectors of 16 bytes from the row's first byte rounded down; what is not
  // the row's, and NaN, as -inf
  const T* x0 = static_cast<const T*>(a.logits) + (int64_t)r * a.stride;
  const int a0 = (int)((reinterpret_cast<uintptr_t>(x0) & 15u) / sizeof(T));
  const int all_vecs = (a0 + (int)a.vocab + E - 1) / E;
  const int first = row.rank * a.vecs, vecs = max(0, min(a.vecs, all_vecs - first));
  float M = -INFINITY;
  for (int v = t; v < vecs; v += kThreads) {
    const int e0 = (first + v) * E - a0;        // element of the vector's start
    uint4 w;
    uint32_t* b = reinterpret_cast<uint32_t*>(&w);
    if (e0 >= 0 && e0 + E <= a.vocab) {
      w = __ldg(reinterpret_cast<const uint4*>(x0 + e0));
    } else {
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          b[i] = e0 + i >= 0 && e0 + i < a.vocab ? __float_as_uint((float)x0[e0 + i]) : 0xff800000u;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t h[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int e = e0 + 2 * i + k;
            h[k] = e >= 0 && e < a.vocab ? (uint32_t)reinterpret_cast<const uint16_t*>(x0)[e] : 0xff80u;
          }
          b[i] = h[0] | h[1] << 16;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        if ((b[i] & 0x7fffffffu) > 0x7f800000u) b[i] = 0xff800000u;
        M = fmaxf(M, __uint_as_float(b[i]));
      } else {
        if ((b[i] & 0x7fffu) > 0x7f80u) b[i] = (b[i] & 0xffff0000u) | 0xff80u;
        if ((b[i] & 0x7fff0000u) > 0x7f800000u) b[i] = (b[i] & 0xffffu) | 0xff800000u;
        M = fmaxf(M, fmaxf(__uint_as_float(b[i] << 16), __uint_as_float(b[i] & 0xffff0000u)));
      }
    }
    reinterpret_cast<uint4*>(data)[v] = w;
  }
  M = logit_of((uint32_t)cluster_max(row, key_of(M)));
  const float temp = __ldg(a.temperature + r);
  const bool greedy = !(temp > 0.f);
  Weights wt;
  wt.small = temp > 0x1p90f ? 0x1p-90f : 1.f;
  wt.M = M * wt.small;
  wt.q = a.q;
  wt.table = sm.table;
  {
    const double c = greedy ? 0.0 : 1.4426950408889634074 / ((double)temp * (double)wt.small);
    wt.ch = (float)c;
    wt.cl = isinf(wt.ch) ? 0.f : (float)(c - (double)wt.ch);
  }
  const int32_t k = a.top_k ? __ldg(a.top_k + r) : 0;
  const float p = a.top_p ? __ldg(a.top_p + r) : 1.f;
  const float mp = a.min_p ? __ldg(a.min_p + r) : 0.f;
  float u = __ldg(a.u + r);
  u = u > 0.f ? u : 0.f;

  // (2), (3) the cuts
  Cut cut_k = {0u, 0xffffffffu}, cut_p = {0u, 0xffffffffu};
  uint64_t least = 1;                           // weights below it are not kept
  if (mp > 0.f) least = max((uint64_t)1, (uint64_t)__double2ull_rn((double)fminf(mp, 1.f) * (double)wt.one()));
  const bool by_k = !greedy && k > 0 && k < a.vocab, by_p = !greedy && p < 1.f;
  if (M == -INFINITY) {
    if (row.rank == 0 && t == 0) {
      a.token[r] = -1;
      if (a.logprob) a.logprob[r] = __uint_as_float(0x7fffffffu);
    }
  } else {
    if (by_k || by_p) {
      clear_histogram(row);
      each<T>(data, vecs, [&](float x) {
        const uint64_t w = wt.of(x);
        if (w != 0) {
          const int b = wt.bucket(x);
          atomicAdd(&sm.count[row.turn][b], 1u);
          atomicAdd(reinterpret_cast<unsigned long long*>(&sm.mass[row.turn][b]), (unsigned long long)w);
        }
      });
      join_histogram(row);
      uint64_t mass = 0, part = 0;
      // (the total: need it before the histogram is overwritten)
      for (int i = t; i < kBuckets; i += kThreads) part += sm.mass_all[i];
      part = warp_sum(part);
      __syncthreads();
      if (lane == 0) sm.warp_mass[t >> 5] = part;
      __syncthreads();
      for (int w = 0; w < kWarps; ++w) mass += sm.warp_mass[w];
      __syncthreads();
      Place pk, pp;
      const bool cut_by_k = by_k && find_place(row, false, (uint64_t)k, pk);
      // top-p alone: its place on the same histogram
      auto need_of = [&](uint64_t total) {
        const double x = ceil((double)fmaxf(p, 0.f) * (double)total);
        return min(total, max((uint64_t)1, (uint64_t)x));
      };
      if (cut_by_k) {
        // (top-p's bucket lies at top-k's or before it: the histogram is kept in registers' stead by a second look)
        cut_k = find_cut<T>(row, wt, data, vecs, false, (uint64_t)k, pk, mass);
        if (by_p) {
          clear_histogram(row);
          each<T>(data, vecs, [&](float x) {
            if (key_of(x) >= cut_k.key) {
              const uint64_t w = wt.of(x);
              const int b = wt.bucket(x);
              atomicAdd(&sm.count[row.turn][b], 1u);
              atomicAdd(reinterpret_cast<unsigned long long*>(&sm.mass[row.turn][b]), (unsigned long long)w);
            }
          });
          join_histogram(row);
        }
      }
      if (by_p) {
        const uint64_t need = need_of(mass);
        uint64_t unused;
        if (find_place(row, true, need, pp)) cut_p = find_cut<T>(row, wt, data, vecs, true, need, pp, unused);
      }
    }
    // (4) runs of tokens: thread t has vectors [t * run, t * run + run) of the slice
    const int run = ((a.vecs + kThreads - 1) / kThreads) | 1;     // (odd: lanes on different banks)
    const int v0 = min(t * run, vecs), v1 = min(v0 + run, vecs);
    const uint32_t ck = max(cut_k.key, cut_p.key);
    // tokens equal to the cut's logit that stay: of the two cuts the one that keeps fewer
    uint32_t ties = 0xffffffffu;
    if (cut_k.key == ck) ties = min(ties, cut_k.ties);
    if (cut_p.key == ck) ties = min(ties, cut_p.ties);
    uint64_t tie0 = 0;                          // such tokens in front of the run
    if (greedy) {
      // the first of the largest
      uint64_t best = 0;
      for (int e = v0 * E; e < v1 * E && best == 0; ++e)
        if (element<T>(data, e) == M) best = 0xffffffffull - (uint32_t)(first * E - a0 + e);
      best = cluster_max(row, best);
      if (row.rank == 0 && t == 0) {
        a.token[r] = (int32_t)(0xffffffffull - best);
        if (a.logprob) a.logprob[r] = 0.f;
      }
    } else {
      if (ties != 0xffffffffu) {
        uint32_t n = 0;
        for (int e = v0 * E; e < v1 * E; ++e) n += key_of(element<T>(data, e)) == ck ? 1u : 0u;
        cluster_sum(row, n, &tie0);
      }
      auto weight = [&](int e, uint64_t& tie) -> uint64_t {
        const float x = element<T>(data, e);
        const uint32_t key = key_of(x);
        if (key < ck) return 0;
        if (key == ck && tie++ >= ties) return 0;
        const uint64_t w = wt.of(x);
        return w >= least ? w : 0;
      };
      uint64_t sum = 0, tie = tie0;
      for (int e = v0 * E; e < v1 * E; ++e) sum += weight(e, tie);
      uint64_t before;
      const uint64_t total = cluster_sum(row, sum, &before);
      // running sum > u * total, in whole numbers
      uint64_t target = (uint64_t)((double)u * (double)total);
      if (u >= 1.f || target >= total) target = total - 1;
      const bool mine = before <= target && target < before + sum;
      const uint32_t who = __ballot_sync(0xffffffffu, mine);
      if (who) {
        // the warp looks through that lane's run, 32 tokens at a time
        const int src = __ffs(who) - 1;
        const int b0 = __shfl_sync(0xffffffffu, v0, src) * E, b1 = __shfl_sync(0xffffffffu, v1, src) * E;
        uint64_t at = __shfl_sync(0xffffffffu, before, src), seen = __shfl_sync(0xffffffffu, tie0, src);
        for (int e0 = b0; e0 < b1; e0 += 32) {
          const int e = e0 + lane;
          const bool tied = e < b1 && key_of(element<T>(data, e)) == ck;
          const uint32_t tied_all = __ballot_sync(0xffffffffu, tied);
          uint64_t rank = seen + __popc(tied_all & ((1u << lane) - 1u));
          const uint64_t w = e < b1 ? weight(e, rank) : 0;
          const uint64_t upto = at + scan_warp(w);
          const uint32_t hit = __ballot_sync(0xffffffffu, upto > target);
          if (hit) {
            if (lane == __ffs(hit) - 1) {
              a.token[r] = first * E - a0 + e;
              if (a.logprob) {
                const float x = element<T>(data, e);
                const float total_f = (float)total, rest = (float)(total - w) / total_f;
                float lp;
                if (rest < 0.5f) lp = log1pf(-rest);
                else if (w >= (1u << 26)) lp = logf((float)w / total_f);
                else lp = (float)(-((double)M - (double)x) / (double)temp) - logf(total_f * exp2f(-(float)wt.q));
                a.logprob[r] = lp;
              }
            }
            break;
          }
          at = __shfl_sync(0xffffffffu, upto, 31);
          seen += __popc(tied_all);
        }
      }
    }
  }
  // (no block leaves while another may read its words)
  row.sync();
}

template <typename T>
cudaError_t launch_t(SampleArgs a, int64_t n_rows, cudaStream_t st) {
  constexpr int E = 16 / sizeof(T);
  const int64_t vecs = (a.vocab + E - 1) / E + 1;       // (a row that starts inside a vector has one more)
  // blocks of a row: so many that a slice leaves room for a second block on the SM, and
  // that few rows use the device
  int C = 1;
  while (C < 8 && ((vecs + C - 1) / C * 16 > 64 * 1024 || (n_rows * C < kv8_sm_count() && vecs / C > 2 * kThreads))) C *= 2;
  a.C = C;
  a.vecs = (int)((vecs + C - 1) / C);
  const size_t smem = sizeof(Shared) + (size_t)a.vecs * 16;
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = kv8_allow_smem(reinterpret_cast<const void*>(sample_kernel<T>), 200 * 1024, allowed);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n_rows * C));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  ProfileScope ps("sample", st);
  return cudaLaunchKernelEx(&cfg, sample_kernel<T>, a);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, int dtype, int64_t n_rows, cudaStream_t st) {
  return dtype == VC_BF16 ? launch_t<__nv_bfloat16>(a, n_rows, st) : launch_t<float>(a, n_rows, st);
}

}  // namespace vc
