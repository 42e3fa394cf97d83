// The attention that cached tokens get, added up, many query rows a request
// (viscache_kv8_weigh on tcgen05).
//
// A token's sum runs over rows, so tokens are the M of the product: K tiles of 128
// tokens lie in shared memory for as long as a unit lasts and blocks of kN query
// rows stream past them; a thread of the epilogue owns a token (a lane of tensor
// memory) and adds up the exponentials of its columns in registers.  Nothing but the
// sums leaves the SM.
//
// A unit is (request, group of kTiles K tiles, KV head); its steps are the blocks of
// query rows that see it.  Persistent blocks, one per SM, share the line of steps
// equally (kv8_sched.cuh); a split unit's pieces are added up by whoever comes last,
// and the first piece holds the old weights, so that two who both come last write the
// same numbers.
//
// bf16 rows: K codes expanded to bf16 (exact) once a unit, query rows as they are, so
// the products are exact and only their fp32 sums round.  fp32 rows: two fp16 numbers
// of a row brought to [2^14, 2^15) (22 bits), K as fp16; the smaller parts are
// multiplied first.
//
// Warps (672 threads):
//   0-15   a unit's K tiles (codes expanded), then the epilogue: warp w reads lanes
//          32 (w % 4) .., columns of quarter w / 4
//   16-19  loaders: query rows of the next step, their lse
//   20     MMA issuer
// Tensor memory: two buffers of kN columns, one product's epilogue under the next one's
// MMAs.
//
// Numbers: the exponent is one fused multiply-add, product * (scale log2(e)) - lse log2(e),
// with factors that agree: the first is off by its rounding (2^-24 at most) and by what the
// tensor cores cut off a sum (kWeighCut, kv8_api.cu, by type and head size), so lse's
// factor, in two parts, is off by the same: a term that counts has a score near its lse,
// and the two cancel.  What is left of the cut on average, at scores of 15: 2 to 5e-7 either
// way by the data (-15e-7 to 5e-7 with one constant for all); flat rows, whose scores lie far
// below their lse, are off by the first factor's rounding times that distance (4e-7 at 7).
// Other roundings go either way and average out over a token's rows.
// A tile's terms are added in eight partial sums, tiles with a compensated sum, so 16384
// rows cost no more bits than 16.
//
// 2048 rows over 32768 tokens, 64 / 8 heads of 128 (1.07 TFLOP, 4.3 G exponentials): 0.93 ms, 1.16
// PFLOP/s, 61% of the cuBLAS rate.  Bound by the epilogue, of which the exponentials are the
// smaller part: at 1.00 ms it took 0.90 without them, 0.99 without MMAs, 0.66 with a quarter of
// the epilogue (loads from tensor memory, of lse, multiply-adds, sums, exponentials).  A product's
// MMAs take 1024 clocks, its exponentials 1190 (alone), all of it about 1600 at the 1.5 GHz that
// the card holds under it; the tensor pipe, the special functions and the issue of instructions
// are half busy each.  Eight epilogue warps 1.05; two groups of eight that take products in turn
// 1.14, four with buffers of 128 columns 1.10; all of a warp's columns loaded at once 1.06 ms.
// fp32 rows, the same chunk: 3.55 ms, two products a part and rows brought by four warps.
// Few steps a unit: 64 requests of 128 rows over up to 4096 tokens 261 us, 7 us a unit, a chain of its
// codes, products, sums and old weights (K expanded by the four loaders 353 us).  One fp32 step
// holds 128 rows in two parts.
#include "kernels.h"
#include "kv8.cuh"
#include "kv8_sched.cuh"
#include "kv8_tc.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace kv8;
using namespace tc;

constexpr int kParts = 4;                       // parts of a product's columns
constexpr int kEpiWarps = 4 * kParts, kLoadWarp0 = kEpiWarps, kLoadWarps = 4, kIssueWarp = kLoadWarp0 + kLoadWarps;
constexpr int kTcThreads = 32 * (kIssueWarp + 1);
constexpr int kKT = 128, kTiles = 3;            // tokens of a K tile, K tiles of a unit
constexpr int kGroup = kTiles * kKT;          // (the workspace holds 1024 sums or more a piece: 16 rows of d)
constexpr int kLoadThreads = 32 * kLoadWarps;

template <typename T, int D>
struct Cfg {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int N = F32 ? 128 : 256;     // query rows of a step
  static constexpr int COLS = N / kParts;       // columns of an epilogue warp
  static constexpr int NP = F32 ? 2 : 1;        // parts of a query value
  static constexpr uint32_t QPART = (uint32_t)N * D * 2, QSTAGE = NP * QPART;
  static constexpr uint32_t KTILE = (uint32_t)kKT * D * 2;
};

template <typename T, int D>
struct alignas(1024) SmemW {
  using C = Cfg<T, D>;
  uint8_t q[2][C::QSTAGE];                      // [stage][part][64-column block][row][128 bytes], swizzled
  uint8_t k[kTiles][C::KTILE];                  // [tile][64-column block][token][128 bytes], swizzled
  float neg_lse[2][C::N];                       // -lse log2(e) of the stage's rows; -inf for rows that add nothing
  float row_scale[2][C::F32 ? C::N : 1];        // power of two of an fp32 row
  uint64_t q_full[2], q_empty[2], l_full[2], l_empty[2], k_full, d_full[2], d_empty[2], done;
  int64_t scan[kTcThreads / 32];
  Share share;
  uint32_t tmem_base;
  int abort, all;
  int32_t err;
};

// 3-D tile load: box at (x = element, y = head, z = row) -> smem, completes on bar.
__device__ __forceinline__ void tma_load_3d(void* smem_dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(smem_dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

__device__ __forceinline__ uint64_t pack_f2(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 unpack_f2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul_f2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Byte offset of 16-byte piece c (8 columns) of row r in a tile of ROWS rows.
template <int ROWS>
__device__ __forceinline__ uint32_t piece16(int r, int c) {
  return (uint32_t)((c >> 3) * (ROWS * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

// Two codes as bf16 numbers (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_bf16x2(uint32_t pair) {
  const uint32_t h = e4m3x2_to_f16x2(pair);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&b);
}

// Adds a product's exponentials to the sum of the thread's token: columns of `taddr` on,
// -lse and powers of two of their rows; with EDGE only those in [from, to) see it.
// (All in log2 units.)
template <typename C, bool EDGE>
__device__ __forceinline__ void add_product(uint32_t taddr, const float* nl, const float* rs, float f, int from, int to,
                                            uint64_t* empty, float& acc, float& low) {
  const uint64_t f2 = pack_f2(f, f);
  uint64_t sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = 0ull;
  uint32_t x[2][16];
  tmem_ld16(taddr, x[0]);
#pragma unroll
  for (int ch = 0; ch < C::COLS / 16; ++ch) {
    uint32_t(&y)[16] = x[ch & 1];
    tmem_wait(y);
    if (ch + 1 < C::COLS / 16) {
      tmem_ld16(taddr + (ch + 1) * 16, x[(ch + 1) & 1]);
    } else {
      tc_fence_before();
      __syncwarp();
      if ((threadIdx.x & 31) == 0) mbar_arrive(empty);
    }
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      const float4 l4 = *reinterpret_cast<const float4*>(nl + ch * 16 + e);
      uint64_t g2[2] = {f2, f2};
      if constexpr (C::F32) {
        const float4 s4 = *reinterpret_cast<const float4*>(rs + ch * 16 + e);
        g2[0] = mul_f2(f2, pack_f2(s4.x, s4.y));
        g2[1] = mul_f2(f2, pack_f2(s4.z, s4.w));
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint64_t z = pack_f2(__uint_as_float(y[e + 2 * h]), __uint_as_float(y[e + 2 * h + 1]));
        const uint64_t l2 = h ? pack_f2(l4.z, l4.w) : pack_f2(l4.x, l4.y);
        const float2 v = unpack_f2(fma_f2(z, g2[h], l2));
        float p0 = ex2(v.x), p1 = ex2(v.y);
        if constexpr (EDGE) {
          const int col = ch * 16 + e + 2 * h;
          if (col < from || col >= to) p0 = 0.f;
          if (col + 1 < from || col + 1 >= to) p1 = 0.f;
        }
        sum[(e >> 1 | h) & 3] = add_f2(sum[(e >> 1 | h) & 3], pack_f2(p0, p1));
      }
    }
  }
  const float2 v = unpack_f2(add_f2(add_f2(sum[0], sum[1]), add_f2(sum[2], sum[3])));
  const float term = (v.x + v.y) - low, now = acc + term;
  low = (now - acc) - term;
  acc = now;
}

template <typename T, int D>
__global__ void __launch_bounds__(kTcThreads, 1) kv8_weigh_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                                                                      const __grid_constant__ vc_kv8 c,
                                                                      const __grid_constant__ vc_kv8_step s,
                                                                      const __grid_constant__ Kv8WeighArgs a) {
  using C = Cfg<T, D>;
  constexpr bool F32 = C::F32;
  constexpr int N = C::N;
  extern __shared__ __align__(1024) uint8_t smem_weigh[];
  SmemW<T, D>& sm = *reinterpret_cast<SmemW<T, D>*>(smem_weigh);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int G = a.Hq / c.Hkv, RB = N / G;       // (the host sends G <= N)
  const Steps<N, kGroup> line{c.Hkv, RB, c.page, a.causal};
  auto report = [&](int32_t err) {
    a.block_status[blockIdx.x] = err;
    if (blockIdx.x == 0) {
      a.status[0] = kStatusPerBlock;
      a.status[1] = (int32_t)gridDim.x;
    }
  };
  if ((smem_u32(smem_weigh) & 1023u) != 0) {            // (the swizzled tiles need it)
    if (threadIdx.x == 0) report(VC_ERR_UNSUPPORTED);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.q_full[i], F32 ? kLoadWarps : 1);   // (bf16: the copies' bytes)
      mbar_init(&sm.q_empty[i], 1);
      mbar_init(&sm.l_full[i], kLoadWarps);
      mbar_init(&sm.l_empty[i], kEpiWarps);             // (apart from the rows: their copy does not wait for the epilogue)
      mbar_init(&sm.d_full[i], 1);
      mbar_init(&sm.d_empty[i], kEpiWarps);
    }
    mbar_init(&sm.k_full, kEpiWarps);
    mbar_init(&sm.done, 1);
    sm.abort = 0;
    sm.err = VC_OK;
    fence_mbar_init();
  }
  __syncthreads();
  int32_t* const err = &sm.err;
  find_share<kTcThreads>(line, s, err, sm.share, sm.scan);       // ends with a barrier
  const Share& sh = sm.share;
  if (sh.begin >= sh.end) {
    if (threadIdx.x == 0) report(sm.err);
    return;
  }
  if (warp == kIssueWarp) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  // rows past a step's RB * G are never written: zeros
  if (!F32 && RB * G < N) {
    for (int v = threadIdx.x; v < (int)sizeof(sm.q) / 16; v += kTcThreads)
      reinterpret_cast<uint4*>(sm.q)[v] = make_uint4(0, 0, 0, 0);
    fence_proxy_async();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = sm.tmem_base;
  volatile int* abort = &sm.abort;
  Walk w;
  w.start(sh);
  int seg = 0;                                  // segments so far
  int step = 0;                                 // steps so far
  int prod = 0;                                 // products (K tile x step) so far
  bool ok = true;
  auto tiles_of = [&]() { return (w.u.kend + kKT - 1) / kKT; };

  if (warp == kIssueWarp) {
    constexpr uint32_t idesc = F32 ? idesc_f16(128, N) : idesc_bf16_f32(128, N);
    const uint64_t qd = desc_sw128(smem_u32(sm.q)), kd = desc_sw128(smem_u32(sm.k));
    do {
      ok = warp_wait(&sm.k_full, seg & 1, abort);
      const int nt = tiles_of();
      for (int j = w.t0; ok && j < w.t1; ++j, ++step) {
        const int st = step & 1;
        ok = warp_wait(&sm.q_full[st], (step >> 1) & 1, abort);
        for (int kt = 0; ok && kt < nt; ++kt, ++prod) {
          const int b = prod & 1;
          ok = warp_wait(&sm.d_empty[b], ((prod >> 1) & 1) ^ 1, abort);
          if (!ok) break;
          tc_fence_after();
          __syncwarp();
          const uint32_t d = tbase + b * 256;
          const uint64_t ad = kd + (uint32_t)kt * (C::KTILE / 16), bd = qd + (uint32_t)st * (C::QSTAGE / 16);
#pragma unroll
          for (int part = C::NP - 1; part >= 0; --part)
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              mma_f16_ss(d, ad + (kk >> 2) * (kKT * 128 / 16) + (kk & 3) * 2,
                         bd + part * (C::QPART / 16) + (kk >> 2) * (N * 128 / 16) + (kk & 3) * 2, idesc,
                         (part < C::NP - 1 || kk) ? 1u : 0u);
          mma_commit_elected(&sm.d_full[b]);
        }
        if (ok) mma_commit_elected(&sm.q_empty[st]);
      }
      ++seg;
    } while (ok && w.next(line, s, err));
    // every MMA is done before the block frees its tensor memory
    __syncwarp();
    mma_commit_elected(&sm.done);
    drain_wait(&sm.done, 0);
  } else if (warp >= kLoadWarp0) {
    // ---- loaders
    const int t = threadIdx.x - 32 * kLoadWarp0;
    if (!F32) prefetch_tmap(&tmQ);
    // -lse of the columns t, t + 128 of a step: row and head do not change from step to step
    constexpr int NL = N / kLoadThreads;
    int li[NL];
    const float* lp[NL];
    float lv[NL];
    int issued = 0;                             // steps whose copies were sent
    auto send_rows = [&](int row, int st) {     // bf16: a step's rows, by one thread
      issued = step + 1;
      if (t == 0) {
        mbar_arrive_expect_tx(&sm.q_full[st], (uint32_t)(RB * G * D * 2));
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
          tma_load_3d(sm.q[st] + x * N * 128, &tmQ, x * 64, w.u.g * G, row, &sm.q_full[st]);
      }
      __syncwarp();
    };
    do {
      const Req8 q = w.u.q;
      const int b0 = line.first_block(q, w.u.rt * kGroup);
      const int dead = max(0, q.m - q.len);     // the surplus first rows are no tokens
      auto fetch_lse = [&](int b) {
#pragma unroll
        for (int k = 0; k < NL; ++k) {
          const int i = (b0 + b) * RB + li[k];
          lv[k] = -INFINITY;
          if (li[k] < RB && i >= dead && i < q.m) {
            // (an infinite lse, which adds nothing, stays out of the product: its second factor may be negative or 0)
            const float l = __ldg(lp[k] + (int64_t)(b0 + b) * RB * a.Hq);
            if (fabsf(l) != INFINITY) lv[k] = -fmaf(l, a.lse_log2, l * a.lse_log2_lo);
          }
        }
      };
#pragma unroll
      for (int k = 0; k < NL; ++k) {
        const int x = t + k * kLoadThreads;
        li[k] = x / G;
        lp[k] = a.lse + (int64_t)(q.row0 + li[k]) * a.Hq + w.u.g * G + (x - li[k] * G);
      }
      fetch_lse(w.t0);
      for (int b = w.t0; ok && b < w.t1; ++b, ++step) {
        const int st = step & 1, i0 = (b0 + b) * RB;
        // (only who fills the stage waits: another could find the barrier two phases on)
        if (F32 || warp == kLoadWarp0) ok = warp_wait(&sm.q_empty[st], ((step >> 1) & 1) ^ 1, abort);
        if (!ok) break;
        uint8_t* dst = sm.q[st];
        if constexpr (!F32) {
          send_rows(q.row0 + i0, st);
        }
        ok = warp_wait(&sm.l_empty[st], ((step >> 1) & 1) ^ 1, abort);
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < NL; ++k) sm.neg_lse[st][t + k * kLoadThreads] = lv[k];
        if (b + 1 < w.t1) fetch_lse(b + 1);
        if constexpr (F32) {
          const T* q0 = static_cast<const T*>(a.q) + (int64_t)q.row0 * a.q_stride + (int64_t)w.u.g * G * D;
          // eight threads a row (four at D = 64): 16 values each
          constexpr int TPR = D / 16;
          const int part = t % TPR;
#pragma unroll 2
          for (int x = t / TPR; x < N; x += kLoadThreads / TPR) {
            const int i = i0 + x / G;
            float v[16];
            float amax = 0.f;
            if (x < RB * G && i >= dead && i < q.m) {
              const float4* src =
                  reinterpret_cast<const float4*>(q0 + (int64_t)i * a.q_stride + (int64_t)(x % G) * D + part * 16);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float4 f = __ldg(src + e);
                v[4 * e] = f.x; v[4 * e + 1] = f.y; v[4 * e + 2] = f.z; v[4 * e + 3] = f.w;
              }
            } else {
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(v[e]));
#pragma unroll
            for (int o = 1; o < TPR; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            const uint32_t ex = __float_as_uint(amax) & 0x7f800000u;
            // 2^-126 at least, so that it and its inverse are normal; a row that is not finite as it is
            const float p2 = ex == 0x7f800000u ? 1.f : __uint_as_float(max(ex, 15u << 23) - (14u << 23));
            const float inv = pow2_inverse(p2);
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float y0 = v[2 * e] * inv, y1 = v[2 * e + 1] * inv;
              hi[e] = half2_bits(y0, y1);
              lo[e] = half2_rest(y0, y1, hi[e]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              *reinterpret_cast<uint4*>(dst + piece16<N>(x, 2 * part + h)) =
                  make_uint4(hi[4 * h], hi[4 * h + 1], hi[4 * h + 2], hi[4 * h + 3]);
              *reinterpret_cast<uint4*>(dst + C::QPART + piece16<N>(x, 2 * part + h)) =
                  make_uint4(lo[4 * h], lo[4 * h + 1], lo[4 * h + 2], lo[4 * h + 3]);
            }
            if (part == 0) sm.row_scale[st][x] = p2;
          }
        }
        if constexpr (F32) {
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.q_full[st]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.l_full[st]);
      }
      ++seg;
    } while (ok && w.next(line, s, err));
    // copies that nobody will wait for have landed before the block ends
    if (!F32 && !ok && t == 0)
      for (int i = max(0, issued - 2); i < issued; ++i) drain_wait(&sm.q_full[i & 1], (i >> 1) & 1);
  } else {
    // ---- epilogue
    const int quarter = warp >> 2, col0 = quarter * C::COLS,    // columns of a warp: COLS from col0 on
              tok = (warp & 3) * 32 + lane;
    const uint32_t lane_base = tbase + ((uint32_t)(warp & 3) << 21) + col0;
    do {
      const int nt = tiles_of(), tok0 = w.u.rt * kGroup;
      const int b0 = line.first_block(w.u.q, tok0);
      {
        // K tiles: the unit before is done with them once all of these warps are here.  16 codes of a token a
        // thread at a time, kB of them in flight
        constexpr int VPR = D / 16, kB = kGroup * VPR / (32 * kEpiWarps);
        static_assert(kB * 32 * kEpiWarps == kGroup * VPR, "whole turns");
        const int t = threadIdx.x;
        int pid[kB];
        uint4 codes[kB];
#pragma unroll
        for (int i = 0; i < kB; ++i) {
          const int x = (t + i * 32 * kEpiWarps) / VPR;
          pid[i] = x < w.u.kend ? load_page(s, c.n_pages, w.u.r, (tok0 + x) / c.page, err) : -1;
        }
#pragma unroll
        for (int i = 0; i < kB; ++i) {
          const int v = t + i * 32 * kEpiWarps, x = tok0 + v / VPR;
          codes[i] = make_uint4(0, 0, 0, 0);
          if (pid[i] >= 0)
            codes[i] = __ldg(reinterpret_cast<const uint4*>(
                                 static_cast<const uint8_t*>(c.K_codes) +
                                 (((int64_t)pid[i] * c.Hkv + w.u.g) * c.page + x % c.page) * D) + v % VPR);
        }
        named_sync(1, 32 * kEpiWarps);
#pragma unroll
        for (int i = 0; i < kB; ++i) {
          const int v = t + i * 32 * kEpiWarps, x = v / VPR, part = v % VPR;
          const uint32_t b[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
          uint32_t y[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            y[2 * k] = F32 ? e4m3x2_to_f16x2(b[k]) : e4m3x2_to_bf16x2(b[k]);
            y[2 * k + 1] = F32 ? e4m3x2_to_f16x2(b[k] >> 16) : e4m3x2_to_bf16x2(b[k] >> 16);
          }
          uint8_t* tile = sm.k[x / kKT];
          *reinterpret_cast<uint4*>(tile + piece16<kKT>(x % kKT, 2 * part)) = make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4*>(tile + piece16<kKT>(x % kKT, 2 * part + 1)) = make_uint4(y[4], y[5], y[6], y[7]);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.k_full);
      }
      float fac[kTiles], acc[kTiles], low[kTiles], old[kTiles];
      int64_t slot[kTiles];                     // of the thread's token, -1 if it has none
#pragma unroll
      for (int kt = 0; kt < kTiles; ++kt) {
        const int x = kt * kKT + tok;
        slot[kt] = -1;
        fac[kt] = acc[kt] = low[kt] = old[kt] = 0.f;
        if (x < w.u.kend) {
          const int p = load_page(s, c.n_pages, w.u.r, (tok0 + x) / c.page, err);
          if (p >= 0) {
            slot[kt] = ((int64_t)p * c.Hkv + w.u.g) * c.page + (tok0 + x) % c.page;
            fac[kt] = __ldg(c.K_scale + (int64_t)p * c.Hkv + w.u.g) * a.scale_log2;
            // what the token had, unless it is one of the step's own: in the unit's first piece
            if (quarter == 0 && w.t0 == 0 && tok0 + x < w.u.q.len - w.u.q.m) old[kt] = a.weights[slot[kt]];
          }
        }
      }
      for (int j = w.t0; ok && j < w.t1; ++j, ++step) {
        const int st = step & 1;
        const float* nl = sm.neg_lse[st] + col0;
        const float* rs = sm.row_scale[st] + (F32 ? col0 : 0);
        const int i0 = (b0 + j) * RB;           // the step's first row
        const int dead = max(0, w.u.q.m - w.u.q.len);
        ok = warp_wait(&sm.l_full[st], (step >> 1) & 1, abort);
#pragma unroll
        for (int kt = 0; kt < kTiles; ++kt) {
          if (!ok || kt >= nt) break;
          const int b = prod & 1;
          ok = warp_wait(&sm.d_full[b], (prod >> 1) & 1, abort);
          if (!ok) break;
          ++prod;
          tc_fence_after();
          // rows i see token t where t <= len - m + i; what the copies brought of other requests' rows is masked too
          const int tk = tok0 + kt * kKT, seen = w.u.q.len - w.u.q.m + 1;
          const bool edge = (a.causal && tk + kKT - 1 >= seen + i0) || i0 < dead || i0 + RB > w.u.q.m;
          const int least = a.causal ? max(dead, tk + tok - seen + 1) : dead;
          const int from = min(max(0, least - i0), RB) * G - col0, to = min(w.u.q.m - i0, RB) * G - col0;
          if (edge) add_product<C, true>(lane_base + b * 256, nl, rs, fac[kt], from, to, &sm.d_empty[b], acc[kt], low[kt]);
          else add_product<C, false>(lane_base + b * 256, nl, rs, fac[kt], 0, 0, &sm.d_empty[b], acc[kt], low[kt]);
        }
        // the step's lse is read
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.l_empty[st]);
      }
      // the quarters' sums meet where K was: all of the unit's products are done
      float* part = reinterpret_cast<float*>(sm.k[0]);
      if (quarter != 0 && ok) {
#pragma unroll
        for (int kt = 0; kt < kTiles; ++kt) part[(quarter * kTiles + kt) * kKT + tok] = acc[kt] - low[kt];
      }
      __syncwarp();
      if (named_sync_any(1, 32 * kEpiWarps, !ok)) break;        // (all of them, or none)
      if (quarter == 0) {
        const bool whole = w.whole();
        const int first = w.first_block(sh), final = w.last_block(sh);
#pragma unroll
        for (int kt = 0; kt < kTiles; ++kt) {
          float v = acc[kt] - low[kt];
#pragma unroll
          for (int x = 1; x < kParts; ++x) v += part[(x * kTiles + kt) * kKT + tok];
          v += old[kt];
          if (whole) {
            if (slot[kt] >= 0) a.weights[slot[kt]] = v;
          } else {
            __stcg(a.part + (2 * (int64_t)blockIdx.x + ((int)blockIdx.x == first ? 1 : 0)) * kGroup + kt * kKT + tok, v);
          }
        }
        if (!whole) {
          named_sync(2, 128);
          if (warp == 0) {
            const bool all = piece_done(a.flags, 1, a.token, first, final);
            if (lane == 0) sm.all = all;
          }
          named_sync(2, 128);
          if (sm.all) {
#pragma unroll
            for (int kt = 0; kt < kTiles; ++kt) {
              float v = 0.f;
              for (int b = first; b <= final; ++b)
                v += __ldcg(a.part + (2 * (int64_t)b + (b == first ? 1 : 0)) * kGroup + kt * kKT + tok);
              if (slot[kt] >= 0) a.weights[slot[kt]] = v;
            }
          }
          named_sync(2, 128);                   // (sm.all is read before the next segment's is written)
        }
      }
      __syncwarp();
      ++seg;
    } while (w.next(line, s, err));
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    tc_fence_after();
    tmem_dealloc(tbase, 512);
  }
  if (threadIdx.x == 0) report(sm.abort ? VC_ERR_DEVICE_TIMEOUT : sm.err);
}

template <typename T, int D>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8WeighArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> allowed{0};
  constexpr size_t smem = sizeof(SmemW<T, D>);
  static_assert(smem <= 227 * 1024, "shared memory of an SM");
  const cudaError_t e = kv8_allow_smem(reinterpret_cast<const void*>(kv8_weigh_tc_kernel<T, D>), smem, allowed);
  if (e != cudaSuccess) return e;
  CUtensorMap mq = {};
  const int G = a.Hq / c.Hkv;
  if (!Cfg<T, D>::F32 && !kv8_rows_map(&mq, a.q, s.n_rows, a.Hq, D, a.q_stride, G, Cfg<T, D>::N / G))
    return cudaErrorInvalidValue;
  ProfileScope ps("kv8_weigh_tc", st);
  kv8_weigh_tc_kernel<T, D><<<(unsigned)kv8_sm_count(), kTcThreads, smem, st>>>(mq, c, s, a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_weigh_tc(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8WeighArgs& a,
                                cudaStream_t st) {
  if (dtype == VC_BF16) return c.d == 128 ? launch_t<__nv_bfloat16, 128>(c, s, a, st) : launch_t<__nv_bfloat16, 64>(c, s, a, st);
  return c.d == 128 ? launch_t<float, 128>(c, s, a, st) : launch_t<float, 64>(c, s, a, st);
}

}  // namespace vc
