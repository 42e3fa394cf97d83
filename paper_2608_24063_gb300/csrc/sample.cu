// The next token of each row of logits (viscache_sample): temperature, top-k, top-p,
// min-p and a given random number.
//
// w_i = 2^-z_i, z_i = (M - x_i) log2(e) / T.  What the filters keep is a prefix of the order by
// (logit descending, index), so each filter is a cut: a logit, and how many of the tokens
// that tie with it, lowest index first.  The token is where the kept weights, in order of
// index, first pass u times their sum.
//
// Reads the logits once: a cluster of C blocks holds a row in shared memory, and
// everything after works there.  A token is a whole number: an answer off by one border is
// wrong, and rows have up to 262144 borders, so weights are computed to about 38 bits
// (pairs of fp32 numbers, a table of 2^(-i/64) and a polynomial of degree 4) and added as
// 64-bit whole numbers: exact in any order, so neither atomics nor the split over blocks
// change a result.  Such a weight costs some sixty instructions, and what bounds large
// batches is that arithmetic, so it is done as rarely as the cuts allow, and for bf16 logits
// once for each value where there are many of them:
//   - without filters once for each token;
//   - with filters, the tokens are counted by buckets of 1/16 in z first (no weight).  What
//     top-k keeps, and where top-p's cut can lie (a bucket's weights differ by 4.4%), follows
//     from the counts.  If that is kMostListed tokens or fewer, they are listed, one block puts
//     them in order and does the rest on the list; for top-p alone the sum of all
//     weights is taken once;
//   - a larger nucleus: the sums of all weights and of those in buckets before the cut's
//     are taken in one pass, by runs of tokens, and the cut is narrowed by counts of ever finer
//     ranges of keys; weights are taken again of the tokens in the cut's buckets alone;
//   - a larger top-k goes through histograms of counts and weights.
// Then the kept weights of each thread's run of tokens are summed (and the tokens that tie with the cut counted, in the
// same pass: in one of their own 3 us of 66 more) and scanned, and the one warp that
// holds the token looks through its run.
//
// 256 rows of 131072 in bf16, a fifth each greedy, all filters, none, and two of top-p alone with nuclei of
// thousands (67 MB): 135 us, bound by the passes' instructions and the clusters' meetings, a plain read
// 10 us.  64 rows of 50001 without filters 18 us, one row of 32000 with all of them 13 us, a chain of
// eight steps between blocks.  In place of the cuts from counts, histograms of weights by 64-bit
// atomics: 441, 31 and 52 us.  Two blocks an SM leave a thread 64 registers: the fp32 kernel spills 32
// bytes (352 of loads), the bf16 one none.
#include <cstddef>

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
constexpr int kTableBits = 48;
constexpr int kCopies = 8;                      // of the table (one: 3 to 6% slower, lanes wait for one another's banks)
// Vectors of a slice from which the weights of bf16 logits are taken from a table.  Without filters, with it and
// without, us: 500 vectors (a row of 32000) 14.4 and 14.4, 1000 (64 rows of 32000) 16.7 and 18.8, 4096 (64 of
// 131072) 27.3 and 39.3; with top_p the last 61 and 74.
constexpr int kTableFrom = 512;
constexpr int kMostListed = 1024;
// Lists up to here are put in order by counting, longer ones by a sort.  A row of 32000, us: 10 tokens 14.5 and 16.5,
// 100 16.7 and 18.8, 200 18.5 and 20.8, 256 20.9 and 21.0, 400 28.7 and 22.2.
constexpr uint32_t kFew = 192;
constexpr int kMostBlocks = 8;                  // of a row

// 2^(48 - i / 64), rounded
__constant__ uint64_t kPowers[64] = {
    0x1000000000000ull, 0xfd3e0c0cf487ull, 0xfa83b2db722aull, 0xf7d0df730ad1ull, 0xf5257d152487ull, 0xf281773c5a00ull,
    0xefe4b99bdcdbull, 0xed4f301ed994ull, 0xeac0c6e7dd24ull, 0xe8396a503c4cull, 0xe5b906e77c83ull, 0xe33f8972be8aull,
    0xe0ccdeec2a95ull, 0xde60f4825e0full, 0xdbfbb797daf2ull, 0xd99d15c278b0ull, 0xd744fccad69dull, 0xd4f35aabcfeeull,
    0xd2a81d91f12bull, 0xd06333daef2bull, 0xce248c151f85ull, 0xcbec14fef272ull, 0xc9b9bd866e2full, 0xc78d74c8abbaull,
    0xc5672a115507ull, 0xc346ccda2497ull, 0xc12c4cca6671ull, 0xbf1799b67a73ull, 0xbd08a39f580cull, 0xbaff5ab2133eull,
    0xb8fbaf4762fcull, 0xb6fd91e328d1ull, 0xb504f333f9deull, 0xb311c412a911ull, 0xb123f581d2acull, 0xaf3b78ad690aull,
    0xad583eea42a1ull, 0xab7a39b5a93full, 0xa9a15ab4ea7cull, 0xa7cd93b4e965ull, 0xa5fed6a9b151ull, 0xa43515ae09e7ull,
    0xa27043030c49ull, 0xa0b0510fb971ull, 0x9ef5326091a1ull, 0x9d3ed9a72d00ull, 0x9b8d39b9d54eull, 0x99e0459320b8ull,
    0x9837f0518db9ull, 0x96942d372018ull, 0x94f4efa8fef7ull, 0x935a2b2f13e7ull, 0x91c3d373ab12ull, 0x9031dc431467ull,
    0x8ea4398b45cdull, 0x8d1adf5b7e5cull, 0x8b95c1e3ea8cull, 0x8a14d575496full, 0x88980e8092dbull, 0x871f61969e8dull,
    0x85aac367cc48ull, 0x843a28c3acdeull, 0x82cd8698ac2cull, 0x8164d1f3bc03ull
};

// A power as the larger 24 bits and the rest of 1 = 2^0, and as a whole number (minus what the magic numbers
// below bring in).
struct alignas(16) Power {
  float hi, lo;
  int64_t whole;
};
// 1.5 * 2^23: the low bits of a sum with it are the rounded number
constexpr float kMagic = 12582912.f;
constexpr int kMagicBits = 0x4b400000;

// Weights of a row's logits.
struct Weights {
  float M, ch, cl;                              // the maximum times `small`; log2(e) / (T small) = ch + cl
  float small;                                  // 1; 2^-90 where T is past 2^90: then M - x stays in range
  int q;                                        // a weight of 1 is 2^q
  const Power* table;                           // the lane's copy

  __device__ __forceinline__ uint64_t one() const { return (uint64_t)1 << q; }
  // z to fp32, never decreasing as x falls; infinite (or NaN, of an infinite T) for -inf
  __device__ __forceinline__ float z_of(float x) const { return (M - x * small) * ch; }
  __device__ __forceinline__ int bucket(float x) const { return (int)fminf(z_of(x) * kPerZ, (float)(kBuckets - 1)); }
  __device__ __forceinline__ uint64_t of(float x) const {
    x *= small;
    const float d = M - x, zh = fminf(d * ch, 64.f);
    // d's rounding, and z in two parts
    const float b = d - M, de = (M - (d - b)) + (-x - b);
    const float zl = fmaf(de, ch, fmaf(d, cl, fmaf(d, ch, -zh)));
    const float t = fmaf(zh, 64.f, kMagic);
    const float g = fmaf(t - kMagic, -1.f / 64.f, zh);          // exact, |g| <= 1/128
    const int j = __float_as_int(t) - kMagicBits;
    const Power power = table[(j & 63) * kCopies];
    // 2^-(g + zl) = e^-y, y = yh + yl
    constexpr float kLn2 = 0.693147182f, kLn2Lo = -1.904654323e-9f;
    const float yh = g * kLn2;
    const float yl = fmaf(zl, kLn2, fmaf(g, kLn2Lo, fmaf(g, kLn2, -yh)));
    const float e = fmaf(yh * yh, fmaf(yh, fmaf(yh, 1.f / 24.f, -1.f / 6.f), 0.5f), -yl);
    // T (1 - yh + e) - T = r - p: whole numbers of 2^-29, and of 2^-37 of what they leave
    const float p = power.hi * yh;
    const float r = fmaf(power.hi, e, fmaf(power.lo, e, fmaf(-power.lo, yh, -fmaf(power.hi, yh, -p))));
    const float t1 = fmaf(p, 0x1p29f, kMagic);
    const float rest = r - fmaf(t1 - kMagic, -0x1p-29f, p);
    const float t2 = fmaf(rest, 0x1p37f, kMagic);
    const int64_t v = power.whole - (int64_t)__float_as_int(t1) * (1 << 19) + (int64_t)__float_as_int(t2) * (1 << 11);
    // half a unit of what is left is added (q is below kTableBits); nothing is left of z above 63
    const int sh = (j >> 6) + kTableBits - 1 - q;
    return zh < 63.f && sh < 60 ? (((uint64_t)v >> sh) + 1) >> 1 : 0;
  }
};

// Orders like the logit: 32 bits, or 16 of a bf16 number.
template <typename T>
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f), k = b >> 31 ? ~b : b | 0x80000000u;
  return sizeof(T) == 4 ? k : k >> 16;
}
template <typename T>
__device__ __forceinline__ float logit_of(uint32_t k) {
  if (sizeof(T) == 2) k = k << 16 | (k >> 15 ? 0u : 0xffffu);
  return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}

// What a row's blocks share.
struct alignas(16) Shared {
  Power table[64 * kCopies];
  uint64_t mass[2][kBuckets], mass_all[kBuckets];       // the block's, by turn; the cluster's
  uint32_t count[2][kBuckets], count_all[kBuckets];
  uint64_t warp_mass[kWarps];
  uint32_t warp_count[kWarps];
  uint64_t words[kWarps][3];
  uint64_t mine[8][4];                                  // what the block tells the others, by turn
  uint64_t found[4];
  uint32_t listed;                                      // the block's tokens on the list (in mass[1])
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

// Calls f(x, e) for elements e of the slice: of vectors v0, v0 + step, .. below v1.
template <typename T, typename F>
__device__ __forceinline__ void walk(const uint8_t* data, int v0, int v1, int step, F f) {
  constexpr int E = 16 / sizeof(T);
  for (int v = v0; v < v1; v += step) {
    const uint4 w = reinterpret_cast<const uint4*>(data)[v];
    const uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if constexpr (sizeof(T) == 4) f(__uint_as_float(b[i]), v * E + i);
      else f(__uint_as_float(i & 1 ? b[i >> 1] & 0xffff0000u : b[i >> 1] << 16), v * E + i);
    }
  }
}
template <typename T, typename F>
__device__ __forceinline__ void each(const uint8_t* data, int vecs, F f) {
  walk<T>(data, threadIdx.x, vecs, kThreads, f);
}

__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Sum of x over the block.
__device__ __forceinline__ uint64_t block_sum(Shared& sm, uint64_t x) {
  x = warp_sum(x);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sm.warp_mass[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0;
  for (int w = 0; w < kWarps; ++w) x += sm.warp_mass[w];
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
    // (a lane a block: one latency)
    const uint64_t v = lane < row.C ? row.read(word, lane) : 0;
    sum = warp_sum(v);
    b += warp_sum(lane < row.rank ? v : 0);
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
    x = lane < row.C ? row.read(word, lane) : 0;
#pragma unroll
    for (int o = kMostBlocks / 2; o > 0; o >>= 1) {
      const uint64_t y = __shfl_xor_sync(0xffffffffu, x, o);
      if (y > x) x = y;
    }
    x = __shfl_sync(0xffffffffu, x, 0);
  }
  return x;
}

// Sums of a and b over the cluster, and of c; or of c's halves the largest each.
__device__ __forceinline__ void cluster_words(Row& row, uint64_t& a, uint64_t& b, uint64_t& c, bool halves) {
  Shared& sm = *row.sm;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto join = [&](uint64_t x, uint64_t y) {
    if (!halves) return x + y;
    const uint32_t hi = max((uint32_t)(x >> 32), (uint32_t)(y >> 32)), lo = max((uint32_t)x, (uint32_t)y);
    return (uint64_t)hi << 32 | lo;
  };
  a = warp_sum(a);
  b = warp_sum(b);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) c = join(c, __shfl_xor_sync(0xffffffffu, c, o));
  uint64_t(*words)[3] = sm.words;
  __syncthreads();
  if (lane == 0) {
    words[warp][0] = a;
    words[warp][1] = b;
    words[warp][2] = c;
  }
  __syncthreads();
  a = b = c = 0;
  for (int w = 0; w < kWarps; ++w) {
    a += words[w][0];
    b += words[w][1];
    c = join(c, words[w][2]);
  }
  if (row.C == 1) return;
  uint64_t* word = sm.mine[row.told & 7];
  ++row.told;
  if (threadIdx.x == 0) {
    word[0] = a;
    word[1] = b;
    word[2] = c;
  }
  row.sync();
  const bool on = lane < row.C;
  a = warp_sum(on ? row.read(word, lane) : 0);
  b = warp_sum(on ? row.read(word + 1, lane) : 0);
  c = on ? row.read(word + 2, lane) : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) c = join(c, __shfl_xor_sync(0xffffffffu, c, o));
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
// The same of histograms of counts alone.
__device__ __forceinline__ void clear_counts(Row& row) {
  row.turn ^= 1;
  for (int i = threadIdx.x; i < kBuckets; i += kThreads) row.sm->count[row.turn][i] = 0;
  __syncthreads();
}
__device__ __forceinline__ void join_counts(Row& row) {
  Shared& sm = *row.sm;
  row.sync();
  for (int i = threadIdx.x; i < kBuckets; i += kThreads) {
    uint32_t v[kMostBlocks], n = 0;             // (all blocks' at once)
#pragma unroll
    for (int c = 0; c < kMostBlocks; ++c) v[c] = c < row.C ? row.read(&sm.count[row.turn][i], c) : 0u;
#pragma unroll
    for (int c = 0; c < kMostBlocks; ++c) n += v[c];
    sm.count_all[i] = n;
    sm.mass_all[i] = 0;
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
  each<T>(data, vecs, [&](float x, int) {
    if (x != -INFINITY && wt.bucket(x) == at.bucket) {
      const uint32_t k = key_of<T>(x);
      hi = max(hi, (uint64_t)k);
      lo = max(lo, (uint64_t)(~k));
    }
  });
  uint32_t top = (uint32_t)cluster_max(row, hi), low = ~(uint32_t)cluster_max(row, lo);
  mass = at.mass;
  uint64_t count = at.count;
  Shared& sm = *row.sm;
  for (int turn = 0; turn < 40; ++turn) {       // (each at least halves the range of 32-bit keys)
    const int bits = 32 - __clz((int)(top - low) | 1);
    const int shift = bits > 10 ? bits - 10 : 0;
    clear_histogram(row);
    each<T>(data, vecs, [&](float x, int) {
      const uint32_t k = key_of<T>(x);
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
      const uint64_t w = wt.of(logit_of<T>(top));
      cut.ties = (uint32_t)(by_mass ? (need - mass + w - 1) / w : need - count);
      mass += cut.ties * w;
      return cut;
    }
    const uint32_t width = (1u << shift) - 1u;
    low = top - low > width ? top - width : low;
  }
  return Cut{low, 0xffffffffu};
}

// The row's answer: token `at` of weight w among kept weights `total`.
__device__ __forceinline__ void write_token(const Weights& wt, uint32_t at, uint64_t w, uint64_t total, float z,
                                            int32_t* token, float* logprob) {
  *token = (int32_t)at;
  if (!logprob) return;
  const float total_f = (float)total, rest = (float)(total - w) / total_f;
  if (rest < 0.5f) *logprob = log1pf(-rest);
  else if (w >= (1u << 26)) *logprob = logf((float)w / total_f);
  else *logprob = -z - logf(total_f * exp2f(-(float)wt.q));
}

// Buckets that can hold the end of the first tokens whose weights reach the share p of all,
// from the counts of the buckets: a bucket's weights lie between 2^-(b + 1) / 16 and 2^-b / 16.
// The share reached at a bucket's end is largest where its tokens and those before weigh
// most and the others least.
__device__ __forceinline__ int2 share_buckets(Row& row, float p) {
  Shared& sm = *row.sm;
  constexpr int per = kBuckets / kThreads;
  constexpr float kRoom = 1e-4f;                // (more than z's and the sums' rounding)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float lo[per], hi[per], ls = 0.f, hs = 0.f;
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const int b = threadIdx.x * per + i;
    const float n = (float)sm.count_all[b];
    lo[i] = n * tc::ex2(-(float)(b + 1) / kPerZ);
    hi[i] = n * tc::ex2(-(float)b / kPerZ);
    ls += lo[i];
    hs += hi[i];
  }
  const float il = scan_warp(ls), ih = scan_warp(hs);
  float2* word = reinterpret_cast<float2*>(sm.warp_mass);
  __syncthreads();
  if (lane == 31) word[warp] = make_float2(il, ih);
  if (threadIdx.x == 0) sm.warp_count[0] = sm.warp_count[1] = kBuckets - 2;      // (the last that counts anything)
  __syncthreads();
  float bl = il - ls, bh = ih - hs, tl = 0.f, th = 0.f;
  for (int w = 0; w < kWarps; ++w) {
    const float2 v = word[w];
    if (w < warp) {
      bl += v.x;
      bh += v.y;
    }
    tl += v.x;
    th += v.y;
  }
#pragma unroll
  for (int i = 0; i < per; ++i) {
    bl += lo[i];
    bh += hi[i];
    if (bh >= (p - kRoom) * (bh + fmaxf(tl - bl, 0.f))) atomicMin(&sm.warp_count[0], (uint32_t)(threadIdx.x * per + i));
    if (bl >= (p + kRoom) * (bl + fmaxf(th - bh, 0.f))) atomicMin(&sm.warp_count[1], (uint32_t)(threadIdx.x * per + i));
  }
  __syncthreads();
  const int2 b = make_int2((int)sm.warp_count[0], (int)sm.warp_count[1]);
  __syncthreads();
  return b;
}

// floor(x * total) of an fp32 x in [0, 1) and a total below 2^62, exactly (fp64 is slow here); `rest`: whether
// something was cut off.
__device__ __forceinline__ uint64_t times(float x, uint64_t total, bool& rest) {
  const uint32_t b = __float_as_uint(x);
  const int s = 150 - (int)(b >> 23);           // x = m 2^-s
  const uint64_t m = (b & 0x7fffffu) | 0x800000u, lo = total * m, hi = __umul64hi(total, m);
  rest = x > 0.f;
  if (!(x > 0.f) || s >= 128 || s > 149) return 0;      // (below 2^-126 times 2^62)
  if (s >= 64) {
    rest = lo != 0 || (s > 64 && (hi & (((uint64_t)1 << (s - 64)) - 1)) != 0);
    return hi >> (s - 64);
  }
  rest = (lo & (((uint64_t)1 << s) - 1)) != 0;
  return hi << (64 - s) | lo >> s;
}
// Where a token is drawn: running sum > u * total.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t total) {
  bool rest;
  return u >= 1.f ? total - 1 : min(total - 1, times(u, total, rest));
}
// top_p of the weights `total`, in whole numbers, at least 1.
__device__ __forceinline__ uint64_t share_of(float p, uint64_t total) {
  bool rest = false;
  const uint64_t x = times(fmaxf(p, 0.f), total, rest);
  return min(total, max((uint64_t)1, x + (rest ? 1 : 0)));
}

// The cut where the weights of the keys in [low, top], the largest first, reach `need`.
template <typename T>
__device__ __forceinline__ Cut narrow(Row& row, const Weights& wt, const uint8_t* data, int vecs, uint32_t top,
                                      uint32_t low, uint64_t need) {
  Shared& sm = *row.sm;
  for (int turn = 0; turn < 40; ++turn) {       // (each at least halves the range of 32-bit keys)
    const int bits = 32 - __clz((int)(top - low) | 1);
    const int shift = bits > 10 ? bits - 10 : 0;
    const uint32_t width = (1u << shift) - 1u;
    clear_counts(row);
    each<T>(data, vecs, [&](float x, int) {
      const uint32_t k = key_of<T>(x);
      if (k >= low && k <= top) atomicAdd(&sm.count[row.turn][(top - k) >> shift], 1u);
    });
    join_counts(row);
    // bounds of the bins' weights (single keys: the weights themselves); find_place ends with a barrier
    auto fill = [&](bool upper) {
      for (int b = threadIdx.x; b < kBuckets; b += kThreads) {
        const uint64_t n = sm.count_all[b];
        if (n == 0) continue;
        const uint32_t first = top - ((uint32_t)b << shift), last = first - low > width ? first - width : low;
        const uint64_t w = wt.of(logit_of<T>(upper ? first : last)), room = shift > 0 ? (w >> 30) + 1 : 0;
        sm.mass_all[b] = n * (upper ? w + room : w - min(w, room));
      }
      __syncthreads();
    };
    Place p, q;
    fill(true);
    if (!find_place(row, true, need, p)) return Cut{low, 0xffffffffu};  // (all of them: not by the bounds)
    if (shift == 0) {
      Cut cut;
      cut.key = top - (uint32_t)p.bucket;
      const uint64_t w = wt.of(logit_of<T>(cut.key));
      cut.ties = (uint32_t)((need - p.mass + w - 1) / w);
      return cut;
    }
    // the cut lies in bins p .. q; where that is more than one, it is looked for by the weights themselves:
    // in bin p, in the bins up to the middle, or in the rest, so every turn at least halves the range
    fill(false);
    const int end = find_place(row, true, need, q) ? max(q.bucket, p.bucket) : kBuckets - 1, mid = (p.bucket + end) >> 1;
    auto last_of = [&](int b) {
      const uint32_t at = top - ((uint32_t)b << shift);
      return (uint32_t)b << shift > top - low || at - low < width ? low : at - width;
    };
    const uint32_t p_first = top - ((uint32_t)p.bucket << shift), p_last = last_of(p.bucket), m_last = last_of(mid),
                   e_last = last_of(end);
    uint64_t m0 = 0, m1 = 0, m2 = 0;
    each<T>(data, vecs, [&](float x, int) {
      const uint32_t k = key_of<T>(x);
      if (k > top || k < m_last) return;
      const uint64_t w = wt.of(x);
      if (k > p_first) m0 += w;
      else if (k >= p_last) m1 += w;
      else m2 += w;
    });
    cluster_words(row, m0, m1, m2, false);
    need = need > m0 ? need - m0 : 1;
    top = p_first;
    uint32_t to = p_last;
    if (end > p.bucket && need > m1) {
      need -= m1;
      to = m_last;
      if (mid > p.bucket && need <= m2) {
        top = p_last - 1;
      } else {
        need = need > m2 ? need - m2 : 1;
        if (m_last == low) return Cut{low, 0xffffffffu};              // (nothing is left: all of them)
        top = m_last - 1;
        to = e_last;
      }
    }
    low = max(low, to);
  }
  return Cut{low, 0xffffffffu};
}

// What the filters keep of the tokens in buckets up to `upto`, on a list of rank 0, and the
// token; `total`: the weights of which top_p is a share where there is no top_k.
template <typename T>
__device__ __forceinline__ void from_list(Row& row, const Weights& wt, const uint8_t* data, int vecs, int index0,
                                          int upto, uint32_t k, bool by_p, float p, uint64_t total, uint64_t least,
                                          float u, int32_t* token, float* logprob) {
  Shared& sm = *row.sm;
  const int t = threadIdx.x;
  // words of key and ~index: the block's, then all in order
  uint64_t *list = sm.mass[1], *order = sm.mass[0];
  if (t == 0) sm.listed = 0;
  __syncthreads();
  each<T>(data, vecs, [&](float x, int e) {
    if (wt.z_of(x) * kPerZ < (float)(upto + 1)) {
      list[atomicAdd(&sm.listed, 1u)] = (uint64_t)key_of<T>(x) << 32 | (uint32_t)~(index0 + e);
    }
  });
  row.sync();
  if (row.rank != 0) return;
  // the others' lists behind this block's, a warp a block
  const int lane = t & 31, from = t >> 5;
  const uint32_t count = lane < row.C ? row.read(&sm.listed, lane) : 0u, ends = scan_warp(count);
  const uint32_t n = __shfl_sync(0xffffffffu, ends, 31);
  static_assert(kMostBlocks <= kWarps, "a warp for each block");
  if (from > 0 && from < row.C) {
    const uint32_t m = __shfl_sync(0xffffffffu, count, from), at = __shfl_sync(0xffffffffu, ends, from) - m;
    for (uint32_t i = lane; i < m; i += 32) order[at + i] = row.read(&list[i], from);
  }
  const uint32_t own = __shfl_sync(0xffffffffu, count, 0);
  constexpr int per = kMostListed / kThreads;
  static_assert(kMostListed <= kBuckets && per == 2, "the histograms' words hold the list, a thread a pair of it");
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const uint32_t e = t + i * kThreads;
    if (e < own) order[e] = list[e];
    else if (e >= n) order[e] = 0;
  }
  __syncthreads();
  uint64_t* upto_sum = sm.mass[1];
  const bool few = n <= kFew;
  if (few) {
    // (a token's place is the number of those before it)
    const uint64_t me = order[t];
    uint32_t place = 0;
    if (t < (int)n)
      for (uint32_t j = 0; j < n; ++j) place += order[j] > me ? 1u : 0u;
    __syncthreads();
    if (t < (int)n) order[place] = me;
    __syncthreads();
  } else {
    // a bitonic sort, whose steps of 32 and less stay inside a warp's 64 words
    const uint32_t most = 2u << (31 - __clz((int)(n - 1)));
    for (uint32_t size = 2; size <= most; size *= 2) {
      for (uint32_t d = size / 2; d > 0; d /= 2) {
        if ((uint32_t)t < most / 2) {
          const uint32_t e = 2 * t - (t & (d - 1));
          const uint64_t x = order[e], y = order[e + d];
          if ((x < y) == ((e & size) == 0)) {
            order[e] = y;
            order[e + d] = x;
          }
        }
        if (d > 32 || (d == 1 && size >= 64)) __syncthreads();
        else __syncwarp();
      }
    }
  }
  const uint32_t nk = min(n, k);
  uint64_t mine[per], sum = 0;
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const uint32_t r = t * per + i;
    mine[i] = r < nk ? wt.of(logit_of<T>((uint32_t)(order[r] >> 32))) : 0;
    sum += mine[i];
  }
  const uint64_t incl = scan_warp(sum);
  if ((t & 31) == 31) sm.warp_mass[t >> 5] = incl;
  if (t == 0) sm.found[0] = sm.found[1] = nk;
  for (int i = t; i < kBuckets; i += kThreads) sm.mass_all[i] = 0;
  __syncthreads();
  uint64_t before = incl - sum, all = 0;
  for (int w = 0; w < kWarps; ++w) {
    if (w < (t >> 5)) before += sm.warp_mass[w];
    all += sm.warp_mass[w];
  }
  const uint64_t need = by_p ? share_of(p, total != 0 ? total : all) : 0;
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const uint32_t r = t * per + i;
    const uint64_t from = before;
    before += mine[i];
    if (r < nk) {
      upto_sum[r] = before;
      // the first to reach top_p's share, and the first below min_p (at least one stays)
      if (by_p && from < need && need <= before) sm.found[0] = r + 1;
      if (r > 0 && mine[i] < least) atomicMin(reinterpret_cast<unsigned long long*>(&sm.found[1]), (unsigned long long)r);
    }
  }
  __syncthreads();
  const uint32_t kept = (uint32_t)min(sm.found[0], sm.found[1]);
  const uint64_t sum_kept = upto_sum[kept - 1];
  const uint64_t target = target_of(u, sum_kept);
  uint32_t at[per];
#pragma unroll
  for (int i = 0; i < per; ++i) {
    const uint32_t r = t * per + i;
    at[i] = r < kept ? ~(uint32_t)order[r] : 0xffffffffu;
  }
  auto write = [&](int i) {
    write_token(wt, at[i], mine[i], sum_kept, wt.z_of(logit_of<T>((uint32_t)(order[t * per + i] >> 32))) * 0.693147182f,
                token, logprob);
  };
  if (few) {
#pragma unroll
    for (int i = 0; i < per; ++i) sm.mass_all[t * per + i] = mine[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < per; ++i) {
      if (at[i] == 0xffffffffu) break;
      uint64_t cum = 0;
      for (uint32_t j = 0; j < kept; ++j) cum += ~(uint32_t)order[j] <= at[i] ? sm.mass_all[j] : 0;
      if (target < cum && target >= cum - mine[i]) write(i);
    }
    return;
  }
  // first the 256 indexes that hold it, then it
  static_assert(kSampleMaxVocab <= 256 * kBuckets, "a bucket for each 256 indexes");
#pragma unroll
  for (int i = 0; i < per; ++i)
    if (at[i] != 0xffffffffu)
      atomicAdd(reinterpret_cast<unsigned long long*>(&sm.mass_all[at[i] >> 8]), (unsigned long long)mine[i]);
  __syncthreads();
  Place block, one;
  find_place(row, true, target + 1, block);
  for (int i = t; i < kBuckets; i += kThreads) sm.mass_all[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < per; ++i)
    if (at[i] != 0xffffffffu && (int)(at[i] >> 8) == block.bucket) sm.mass_all[at[i] & 255] = mine[i];
  __syncthreads();
  find_place(row, true, target + 1 - block.mass, one);
#pragma unroll
  for (int i = 0; i < per; ++i)
    if (at[i] == (uint32_t)(block.bucket << 8 | one.bucket)) write(i);
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
  {
    // a copy for each lane of a quarter warp, which is what loads 16 bytes at a time: on banks of its own
    static_assert(kThreads == 64 * kCopies, "a thread for each");
    const uint64_t x = kPowers[t / kCopies];
    sm.table[t] = {(float)(uint32_t)(x >> 25) * 0x1p-23f, (float)(uint32_t)(x & 0x1ffffffu) * 0x1p-48f,
                   (int64_t)x + ((int64_t)kMagicBits << 19) - ((int64_t)kMagicBits << 11)};
  }

  // weights of bf16 logits by their bits, in the histograms' words while these are not in use: of each sign the
  // kSigned magnitudes up to the largest that counts
  constexpr int kSigned = 3 * kBuckets / 2, kNoTable = 1 << 24;
  static_assert(offsetof(Shared, mass_all) == offsetof(Shared, mass) + sizeof(Shared::mass), "one table");
  uint64_t* const by_bits = reinterpret_cast<uint64_t*>(smem + offsetof(Shared, mass));
  int top_bits = kNoTable;

  // (1) the slice: vectors of 16 bytes from the row's first byte rounded down; what is not
  // the row's, and NaN, as -inf
  const T* x0 = static_cast<const T*>(a.logits) + (int64_t)r * a.stride;
  const int a0 = (int)((reinterpret_cast<uintptr_t>(x0) & 15u) / sizeof(T));
  const int all_vecs = (a0 + (int)a.vocab + E - 1) / E;
  const int first = row.rank * a.vecs, vecs = max(0, min(a.vecs, all_vecs - first));
  float M = -INFINITY;
  auto edge = [&](int e0) {                     // a vector that is not all the row's
    uint4 w;
    uint32_t* b = reinterpret_cast<uint32_t*>(&w);
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
    return w;
  };
  constexpr int kLoads = 4;                     // vectors of a thread in flight
  for (int vb = t; vb < vecs; vb += kLoads * kThreads) {
    uint4 w[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int v = vb + n * kThreads, e0 = (first + v) * E - a0;     // element of the vector's start
      if (v < vecs && e0 >= 0 && e0 + E <= a.vocab) w[n] = __ldg(reinterpret_cast<const uint4*>(x0 + e0));
    }
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int v = vb + n * kThreads, e0 = (first + v) * E - a0;
      if (v >= vecs) break;
      if (!(e0 >= 0 && e0 + E <= a.vocab)) w[n] = edge(e0);
      uint32_t b[4] = {w[n].x, w[n].y, w[n].z, w[n].w};
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
      reinterpret_cast<uint4*>(data)[v] = make_uint4(b[0], b[1], b[2], b[3]);
    }
  }
  const float temp = __ldg(a.temperature + r);
  const bool greedy = !(temp > 0.f);
  Weights wt;
  wt.small = temp > 0x1p90f ? 0x1p-90f : 1.f;
  {
    // log2(e) / T in two parts, in fp32 alone (fp64 is slow here); T no less than 2^-127, so that it is an fp32 number
    constexpr float kHi = 1.44269502f, kLo = 1.92596303e-8f;
    const float T1 = fmaxf(temp, 0x1p-127f) * wt.small;
    wt.ch = greedy || T1 == INFINITY ? 0.f : __fdiv_rn(kHi, T1);
    wt.cl = wt.ch == 0.f ? 0.f : __fdiv_rn(fmaf(-wt.ch, T1, kHi) + kLo, T1);
  }
  M = logit_of<T>((uint32_t)cluster_max(row, key_of<T>(M)));
  if (M == INFINITY) {
    // these share everything: 0 for them, nothing for the others
    for (int v = t; v < vecs; v += kThreads) {
      uint4 w = reinterpret_cast<uint4*>(data)[v];
      uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) b[i] = b[i] == 0x7f800000u ? 0u : 0xff800000u;
        else b[i] = ((b[i] & 0xffffu) == 0x7f80u ? 0u : 0xff80u) | (b[i] >> 16 == 0x7f80u ? 0u : 0xff800000u);
      }
      reinterpret_cast<uint4*>(data)[v] = make_uint4(b[0], b[1], b[2], b[3]);
    }
    M = 0.f;
    __syncthreads();
  }
  wt.M = M * wt.small;
  wt.q = a.q;
  wt.table = sm.table + (t & (kCopies - 1));
  const int32_t k = a.top_k ? __ldg(a.top_k + r) : 0;
  const float p = a.top_p ? __ldg(a.top_p + r) : 1.f;
  const float mp = a.min_p ? __ldg(a.min_p + r) : 0.f;
  float u = __ldg(a.u + r);
  u = u > 0.f ? u : 0.f;

  auto fill_table = [&]() {
    if constexpr (sizeof(T) == 2) {
      if (a.vecs < kTableFrom) return;
      // (a logit 64 in z below the maximum has no weight, and one past the largest magnitude here is further below)
      const float largest = wt.ch > 0.f && wt.small == 1.f ? fmaxf(fabsf(M), fabsf(M - __fdiv_rn(64.f, wt.ch))) : INFINITY;
      top_bits = min((int)(__float_as_uint(largest) >> 16) + 1, 0x7f80);
      for (int i = t; i < 2 * kSigned; i += kThreads) {
        const int bits = top_bits - (i < kSigned ? i : i - kSigned);
        const float x = __uint_as_float((uint32_t)max(bits, 0) << 16 | (i < kSigned ? 0u : 0x80000000u));
        by_bits[i] = x <= M ? wt.of(x) : 0;
      }
      __syncthreads();
    }
  };
  auto weight_of = [&](float x) -> uint64_t {
    if constexpr (sizeof(T) == 2) {
      const uint32_t b = __float_as_uint(x);
      const int i = top_bits - (int)(b >> 16 & 0x7fffu);
      if (i < kSigned) return i < 0 ? 0 : by_bits[i + (b >> 31 ? kSigned : 0)];
    }
    return wt.of(x);
  };

  // the cuts
  uint64_t least = 1;                           // weights below it are not kept
  if (mp > 0.f) least = max((uint64_t)1, (uint64_t)__float2ull_rn(fminf(mp, 1.f) * (float)wt.one()));
  const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.f;
  // runs of tokens: thread t has vectors [t * run, t * run + run) of the slice
  const int run = ((a.vecs + kThreads - 1) / kThreads) | 1;       // (odd: lanes on different banks)
  const int v0 = min(t * run, vecs), v1 = min(v0 + run, vecs), index0 = first * E - a0;
  int32_t* const token = a.token + r;
  float* const logprob = a.logprob ? a.logprob + r : nullptr;
  if (M == -INFINITY) {
    if (row.rank == 0 && t == 0) {
      *token = -1;
      if (logprob) *logprob = __uint_as_float(0x7fffffffu);
    }
  } else if (greedy) {
    // the first of the largest
    uint64_t best = 0;
    walk<T>(data, v0, v1, 1, [&](float x, int e) {
      if (x == M) best = max(best, (uint64_t)(0xffffffffull - (uint32_t)(index0 + e)));
    });
    best = cluster_max(row, best);
    if (row.rank == 0 && t == 0) {
      *token = (int32_t)(0xffffffffull - best);
      if (logprob) *logprob = 0.f;
    }
  } else {
    Cut cut_k = {0u, 0xffffffffu}, cut_p = {0u, 0xffffffffu};
    bool done = false, have_sum = false;
    uint64_t sum = 0;                           // kept weights of the run
    uint32_t top = 0;                           // with have_sum: those of keys above it
    if (by_k || by_p) {
      clear_counts(row);
      each<T>(data, vecs, [&](float x, int) {
        const float z = wt.z_of(x) * kPerZ;
        if (z < (float)(kBuckets - 1)) atomicAdd(&sm.count[row.turn][(int)z], 1u);      // (beyond: no weight)
      });
      join_counts(row);
      Place pk;
      const bool cut_by_k = by_k && find_place(row, false, (uint64_t)k, pk);
      if (cut_by_k) {
        if (pk.count + sm.count_all[pk.bucket] <= kMostListed) {
          from_list<T>(row, wt, data, vecs, index0, pk.bucket, (uint32_t)k, by_p, p, 0, least, u, token, logprob);
          done = true;
        } else {
          uint64_t mass = 0;
          pk.mass = 0;
          cut_k = find_cut<T>(row, wt, data, vecs, false, (uint64_t)k, pk, mass);
          if (by_p) {
            uint64_t kept = 0, unused, tie0;    // all that top-k keeps
            uint32_t ties = 0;
            walk<T>(data, v0, v1, 1, [&](float x, int) { ties += key_of<T>(x) == cut_k.key ? 1u : 0u; });
            cluster_sum(row, ties, &tie0);
            walk<T>(data, v0, v1, 1, [&](float x, int) {
              const uint32_t key = key_of<T>(x);
              if (key > cut_k.key || (key == cut_k.key && tie0++ < cut_k.ties)) kept += wt.of(x);
            });
            kept = cluster_sum(row, kept, nullptr);
            clear_histogram(row);
            each<T>(data, vecs, [&](float x, int) {
              if (key_of<T>(x) >= cut_k.key) {
                const uint64_t w = wt.of(x);
                const int b = wt.bucket(x);
                atomicAdd(&sm.count[row.turn][b], 1u);
                atomicAdd(reinterpret_cast<unsigned long long*>(&sm.mass[row.turn][b]), (unsigned long long)w);
              }
            });
            join_histogram(row);
            const uint64_t need = share_of(p, kept);
            Place pp;
            if (find_place(row, true, need, pp)) cut_p = find_cut<T>(row, wt, data, vecs, true, need, pp, unused);
          }
        }
      } else if (by_p) {
        const int2 b = share_buckets(row, p);
        uint64_t n = 0, total = 0, above = 0;
        uint32_t hi = 0, lo = 0;                // the largest key and ~key
        for (int i = t; i <= b.y; i += kThreads) n += sm.count_all[i];
        n = block_sum(sm, n);
        const bool few = n <= kMostListed;
        // all weights, those before the cut's buckets, and the keys of those buckets
        const float z0 = few ? -1.f : (float)b.x, z1 = few ? -1.f : (float)(b.y + 1);
        const bool all = least == 1;
        fill_table();
        walk<T>(data, v0, v1, 1, [&](float x, int) {
          const uint64_t w = weight_of(x);
          const float z = wt.z_of(x) * kPerZ;
          total += w;
          if (z < z0) {
            above += w;
            if (!all && w >= least) sum += w;
          } else if (z < z1) {
            hi = max(hi, key_of<T>(x));
            lo = max(lo, ~key_of<T>(x));
          }
        });
        if (all) sum = above;
        uint64_t keys = (uint64_t)hi << 32 | lo;
        cluster_words(row, total, above, keys, true);
        if (few) {
          from_list<T>(row, wt, data, vecs, index0, b.y, 0xffffffffu, true, p, total, least, u, token, logprob);
          done = true;
        } else {
          const uint64_t need = share_of(p, total);
          top = (uint32_t)(keys >> 32);
          cut_p = narrow<T>(row, wt, data, vecs, top, ~(uint32_t)keys, need > above ? need - above : 1);
          have_sum = true;
        }
      }
    }
    if (!done) {
      const uint32_t ck = max(cut_k.key, cut_p.key);
      // tokens equal to the cut's logit that stay: of the two cuts the one that keeps fewer
      uint32_t ties = 0xffffffffu;
      if (cut_k.key == ck) ties = min(ties, cut_k.ties);
      if (cut_p.key == ck) ties = min(ties, cut_p.ties);
      auto counts = [&](uint64_t w) { return w >= least ? w : 0; };
      auto weight = [&](float x, uint64_t& tie) -> uint64_t {
        const uint32_t key = key_of<T>(x);
        if (key < ck) return 0;
        if (key == ck && tie++ >= ties) return 0;
        return counts(wt.of(x));
      };
      uint64_t tie0 = 0, before;                // tokens that tie with the cut in front of the run
      uint32_t tied = 0;                        // and in it
      if (have_sum && top - ck < (uint32_t)kBuckets) {
        // few different logits (of bf16 rows always): their weights from a table
        for (uint32_t i = t; i <= top - ck; i += kThreads) sm.mass_all[i] = counts(wt.of(logit_of<T>(top - i)));
        __syncthreads();
        walk<T>(data, v0, v1, 1, [&](float x, int) {
          const uint32_t key = key_of<T>(x);
          if (key <= top && key > ck) sum += sm.mass_all[top - key];
          tied += key == ck ? 1u : 0u;
        });
      } else if (ck == 0) {
        fill_table();
        walk<T>(data, v0, v1, 1, [&](float x, int) { sum += counts(weight_of(x)); });
      } else {
        const uint32_t last = have_sum ? top : 0xffffffffu;
        walk<T>(data, v0, v1, 1, [&](float x, int) {
          const uint32_t key = key_of<T>(x);
          if (key <= last && key > ck) sum += counts(wt.of(x));
          tied += key == ck ? 1u : 0u;
        });
      }
      if (ck != 0) {
        if (ties != 0xffffffffu) cluster_sum(row, tied, &tie0);
        const uint32_t stay = tie0 < ties ? min(tied, ties - (uint32_t)tie0) : 0u;
        sum += stay * counts(wt.of(logit_of<T>(ck)));
      }
      const uint64_t total = cluster_sum(row, sum, &before);
      // running sum > u * total, in whole numbers
      const uint64_t target = target_of(u, total);
      const bool mine = before <= target && target < before + sum;
      const uint32_t who = __ballot_sync(0xffffffffu, mine);
      if (who) {
        // the warp looks through that lane's run, 32 tokens at a time
        const int src = __ffs(who) - 1;
        const int b0 = __shfl_sync(0xffffffffu, v0, src) * E, b1 = __shfl_sync(0xffffffffu, v1, src) * E;
        uint64_t at = __shfl_sync(0xffffffffu, before, src), seen = __shfl_sync(0xffffffffu, tie0, src);
        for (int e0 = b0; e0 < b1; e0 += 32) {
          const int e = e0 + lane;
          const float x = e < b1 ? element<T>(data, e) : -INFINITY;
          const uint32_t equal = __ballot_sync(0xffffffffu, e < b1 && key_of<T>(x) == ck);
          uint64_t rank = seen + __popc(equal & ((1u << lane) - 1u));
          const uint64_t w = e < b1 ? weight(x, rank) : 0;
          const uint64_t upto = at + scan_warp(w);
          const uint32_t hit = __ballot_sync(0xffffffffu, upto > target);
          if (hit) {
            if (lane == __ffs(hit) - 1)
              write_token(wt, (uint32_t)(index0 + e), w, total, wt.z_of(x) * 0.693147182f, token, logprob);
            break;
          }
          at = __shfl_sync(0xffffffffu, upto, 31);
          seen += __popc(equal);
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
  while (C < kMostBlocks && ((vecs + C - 1) / C * 16 > 66 * 1024 || (n_rows * C < kv8_sm_count() && vecs / C > 2 * kThreads))) C *= 2;
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
