// Attention over the 8-bit paged cache, few query rows a request
// (viscache_kv8_attention):
//     out[rho] = sum_t p_t V[t] / sum_t p_t,  p_t = 2^(c q[rho] . K[t] - m),
// c = scale * log2(e), over the pages of one request and KV head.
//
// Reads d bytes of K and of V a token for 8 or 16 query rows: bound by the
// codes' bytes as long as expanding them stays cheap.  One persistent block
// per SM takes an equal share of the line of key tiles (kv8_sched.cuh); a
// producer warp brings 128-token tiles into a shared-memory ring by TMA (one
// box a page: the page's rows of one head are contiguous); the other warps
// take the tiles' 16-token chunks in turn, each with its own running maximum,
// sum and output, added up at a segment's end.
//
// Products are m16n8k16 with 16 tokens (QK) or 16 output dimensions (PV) as M
// and 8 query rows as N, fp16 operands and fp32 sums: an e4m3 code is exactly an
// fp16 number, so codes are expanded to fp16 in registers (two a conversion) and
// never written anywhere.  The order of the contracted index is free, so a
// thread's 16-byte read of a K row serves four k-steps of QK: thread column tig
// holds dimensions tig * D/4 ... of its row.  For PV the order of the output
// dimensions is free: a thread reads 16 bytes of the rows of its four tokens,
// pairs them with byte permutations and converts.  QK leaves probabilities as
// (token, query); movmatrix turns them into PV's (query, token).
//
// Numbers: a query row is multiplied by the power of two that brings its largest
// magnitude to [2^14, 2^15), so that fp16 holds bf16 values exactly down to 2^-31 of
// it; fp32 calls use a second fp16 part of the row (22 bits down to 2^-17 of the
// largest, 2^-39 of it below) and of the probabilities.  Scores are scaled by the page's K scale in
// fp32.  Probabilities enter as p * 2^(13 - r) * V scale, r + m following the
// row's largest score + log2 of its V scale: a row's fixed point is set by its
// largest contribution, not by values that it does not see or that have no
// weight.  At most 2^15 in fp16, the largest above 2^12, so they keep 11 bits down
// to 2^-26 of the largest.  The row sum adds p before it is rounded.  The tensor
// core's fp32 sums cut off, so fp32 calls take a chunk's product from 0 and add it to
// the output to nearest: over 20000 tokens, 12 rows of 128, the error falls from 5.9e-6
// of the output to 3e-7, and 64 requests of 8192 tokens, 8 KV heads, take 213 us instead
// of 197 (8 rows), 337 instead of 308 (16 rows).  Both
// references follow with a slack of 2 (log2 units), which saves most rescales of
// the accumulators; r is a whole number and m a score, so that the probability 1
// of a dominant token is not rounded.
//
// 32 requests of up to 32768 tokens, 8 KV heads of 128, 8 query heads each (1.35
// GB): 221 us, 6.1 TB/s, 90% of a plain copy's rate.  One request of 777 tokens, 4
// KV heads: 10 us, a chain of launch, lengths, page numbers, codes, products and
// the join of its pieces.
#include <cudaTypedefs.h>

#include <mutex>

#include "kernels.h"
#include "kv8.cuh"
#include "kv8_mma.cuh"
#include "kv8_sched.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace kv8;

constexpr int kKT = 128;                        // tokens of a tile
constexpr int kChunks = kKT / 16;
constexpr float kSlack = 2.f;
constexpr int kPExp = 13;
constexpr float kLeastRef = -110.f;             // (2^(kPExp - r) stays a normal number; scales below 2^-100 alone: fewer bits)

// T: query type, D: head dimension, NQ: groups of 8 query rows of a unit.
// Warps: registers are granted to four warps at a time, so the consumers and
// the producer fill 8, 12 or 16 warps of 255, 168 or 128 registers, chosen by
// what the accumulators and the query fragments take.  64 requests of 8192
// tokens, 8 KV heads, us with 7 / 11 / 15 consumers: d = 64, 8 rows 154 / 132 /
// 127; d = 128, 8 rows 188 / 174 / 175 (fp32 rows 233 / 213 / 231); d = 128, 16
// rows 249 / 279 / 385.
template <typename T, int D, int NQ>
struct Cfg {
  static constexpr int NP = sizeof(T) == 4 ? 2 : 1;         // fp16 parts of a query value
  static constexpr int MT = 8 * NQ;                         // query rows of a unit
  static constexpr int REGS = D / 4 * NQ * (1 + 0.5 * NP);  // accumulators and query fragments
  static constexpr int WARPS = REGS <= 32 ? 15 : REGS <= 64 ? 11 : 7;
  static constexpr int THREADS = 32 * (WARPS + 1);
  static constexpr int STAGE = kKT * D;                     // bytes of K, and of V
  static constexpr int NST = D == 128 ? 5 : 10;
  static constexpr int SLOTS = 32768 / (MT * D * 4);        // outputs that the merge buffer holds
};

template <typename T, int D, int NQ>
struct Smem {
  using C = Cfg<T, D, NQ>;
  uint8_t ring[C::NST][2][C::STAGE];                        // [K, V]
  float merge[C::SLOTS][C::MT][D];
  float scale[C::NST][2][kChunks];                          // [K, V][page of the tile]
  float wm[C::WARPS][C::MT], wl[C::WARPS][C::MT];           // a segment's warp states: maxima, sums
  float wf[C::WARPS][C::MT];                                // and their factors
  float2 ml[C::MT];                                         // the segment's maximum and sum of each row
  uint64_t full[C::NST], empty[C::NST];
  int64_t scan[C::WARPS + 1];
  Share share;
  int abort, last;
  int nan_token[2];                                         // first token whose V has a NaN in an edge chunk: [segment & 1]
  int32_t err;                                              // the block's status
};

// 8 x 8 transpose of 16-bit values: lane (gid, tig) gives row gid, columns 2 tig, + 1
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Byte offset of 16-byte piece c of row r in a tile as TMA wrote it (128-byte
// rows with the 128-byte swizzle, 64-byte rows with the 64-byte one).
template <int D>
__device__ __forceinline__ uint32_t piece(int r, int c) {
  return D == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4))
                  : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}

// over the eight lanes of a thread column (the tokens of a query)
__device__ __forceinline__ float max_column(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
__device__ __forceinline__ float sum_column(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 4);
  x += __shfl_xor_sync(0xffffffffu, x, 8);
  return x + __shfl_xor_sync(0xffffffffu, x, 16);
}

template <typename T, int D, int NQ>
__global__ void __launch_bounds__(Cfg<T, D, NQ>::THREADS, 1)
kv8_attn_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                const __grid_constant__ vc_kv8 c, const __grid_constant__ vc_kv8_step s,
                const __grid_constant__ Kv8AttnArgs a) {
  using C = Cfg<T, D, NQ>;
  constexpr int NP = C::NP, MT = C::MT, NW = C::WARPS;
  constexpr int KS = D / 16;                    // k-steps of QK
  constexpr int NM = D / 16;                    // dimension tiles of PV
  extern __shared__ uint8_t smem_raw[];
  Smem<T, D, NQ>& sm = *reinterpret_cast<Smem<T, D, NQ>*>(tc::align1024(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.Hq / c.Hkv;
  const Line<MT, kKT> line{c.Hkv, G, c.page, a.causal};
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NST; ++i) {
      tc::mbar_init(&sm.full[i], 2);            // the copies' bytes, and the scales
      tc::mbar_init(&sm.empty[i], NW);
    }
    sm.abort = 0;
    sm.nan_token[0] = sm.nan_token[1] = kNoNan;
    sm.err = VC_OK;
    tc::fence_mbar_init();
  }
  __syncthreads();
  int32_t* const err = &sm.err;
  find_share<C::THREADS>(line, s, err, sm.share, sm.scan);        // ends with a barrier
  const Share& sh = sm.share;
  if (sh.begin >= sh.end) {
    if (threadIdx.x == 0) store_status(a, sm.err);
    return;
  }
  volatile int* abort = &sm.abort;
  Walk wk;
  wk.start(sh);
  const Unit& u = wk.u;
  const int &t0 = wk.t0, &t1 = wk.t1;           // the segment's tiles of its unit
  int fill = 0;                                 // tiles so far (ring position)

  if (warp == NW) {
    // ---- producer: lane -> (tile, page) of a batch of 32 pages; page numbers
    // and scales of the next batch load while this one's boxes are issued
    const int ppt = kKT / c.page, tpb = 32 / ppt;
    const int bt = lane / ppt, bp = lane % ppt;
    const uint32_t page_bytes = (uint32_t)c.page * D;
    tc::prefetch_tmap(&tmK);
    tc::prefetch_tmap(&tmV);
    bool ok = true;
    do {
      auto look = [&](int first, int& pid, float& ks, float& vs, bool& live) {
        const int tile = first + bt, j = tile * ppt + bp;
        live = tile < t1 && j * c.page < u.kend;
        pid = live ? load_page(s, c.n_pages, u.r, j, err) : -1;
        const int64_t at = (int64_t)max(pid, 0) * c.Hkv + u.g;
        ks = pid >= 0 ? __ldg(c.K_scale + at) : 0.f;
        vs = pid >= 0 ? __ldg(c.V_scale + at) : 0.f;
      };
      int pid, npid = -1;
      float ks, vs, nks = 0.f, nvs = 0.f;
      bool live, nlive = false;
      look(t0, pid, ks, vs, live);
      for (int tb = t0; ok && tb < t1; tb += tpb) {
        if (tb + tpb < t1) look(tb + tpb, npid, nks, nvs, nlive);
        const int nt = min(tpb, t1 - tb);
        for (int i = 0; i < nt; ++i, ++fill) {
          const int st = fill % C::NST;
          if (!tc::warp_wait(&sm.empty[st], ((fill / C::NST) & 1) ^ 1, abort)) {
            ok = false;
            break;
          }
          const bool mine = bt == i;
          const int pages = __popc(__ballot_sync(0xffffffffu, mine && live));
          if (lane == 0) tc::mbar_arrive_expect_tx(&sm.full[st], (uint32_t)pages * 2 * page_bytes);
          __syncwarp();
          if (mine && live) {
            // a page that does not exist counts with scale 0; page 0 stands in
            const int row = (max(pid, 0) * c.Hkv + u.g) * c.page;
            tc::tma_load_2d(sm.ring[st][0] + bp * page_bytes, &tmK, 0, row, &sm.full[st]);
            tc::tma_load_2d(sm.ring[st][1] + bp * page_bytes, &tmV, 0, row, &sm.full[st]);
          }
          if (mine) {
            sm.scale[st][0][bp] = ks;
            sm.scale[st][1][bp] = vs;
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&sm.full[st]);
        }
        pid = npid;
        ks = nks;
        vs = nvs;
        live = nlive;
      }
    } while (ok && wk.next(line, s, err));
    // every copy has landed before the block may end
    __syncwarp();
    if (lane == 0)
      for (int i = max(0, fill - C::NST); i < fill; ++i) tc::drain_wait(&sm.full[i % C::NST], (i / C::NST) & 1);
  } else {
  // ---- consumers: chunk k of the share's tiles (16 tokens each) goes to warp k % NW.
  // Every warp waits for every tile and frees it, whether it has a chunk of it
  // or not: a warp that passed over a tile could find the tile's barrier a phase
  // behind or two ahead of the one it waits for, and parities do not tell.
  const int gid = lane >> 2, tig = lane & 3;
  int off = warp;                               // the warp's first chunk of the next tile (or past it)
  bool ok = true;
  int seg = 0;                                  // segments so far
  do {
    uint32_t qf[NP][NQ][KS][2];
    float cs[NQ][2];
    load_q<T, D, NQ, NP>(static_cast<const T*>(a.q), a.q_stride, u, G, qf, cs);
    // keys that rows 8 n + 2 tig, + 1 see, and the fewest that any row of the unit sees
    int lim[NQ][2], lim_min = u.kend;
    const int base = u.q.len - u.q.m + 1, r0 = u.rt * MT;
    if (a.causal) lim_min = base + r0 / G;
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        cs[n][h] *= a.scale_log2;
        lim[n][h] = a.causal ? min(u.kend, base + (r0 + 8 * n + 2 * tig + h) / G) : u.kend;
      }
    float o[NQ][NM][4];
    // references of rows 8 n + 2 tig, + 1: m of the scores x, r + m of x + log2 of the page's V
    // scale, and rs = 2^(kPExp - r)
    float m[NQ][2], r[NQ][2], rs[NQ][2], l[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
      for (int i = 0; i < NM; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
      m[n][0] = m[n][1] = r[n][0] = r[n][1] = -INFINITY;
      rs[n][0] = rs[n][1] = 1.f;
      l[n][0] = l[n][1] = 0.f;
    }
    for (int tile = t0; tile < t1; ++tile, ++fill) {
      const int st = fill % C::NST;
      ok = ok && tc::warp_wait(&sm.full[st], (fill / C::NST) & 1, abort);
      if (!ok) continue;
      int ck = off;
      for (; ck < kChunks; ck += NW) {
        const int key0 = tile * kKT + 16 * ck;
        if (key0 >= u.kend) continue;
        const uint8_t* kt = sm.ring[st][0];
        const uint8_t* vt = sm.ring[st][1];
        const int pg = 16 * ck / c.page;
        const float ksc = sm.scale[st][0][pg], vsc = sm.scale[st][1][pg];
        const float vlog = scale_log2(vsc);     // (the producer has no time to spare with pages of 16)
        // scores of tokens gid (x[.][0], [1]) and gid + 8, queries 2 tig and 2 tig + 1
        float x[NQ][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          const uint4 w0 = *reinterpret_cast<const uint4*>(kt + piece<D>(16 * ck + gid, tig * (D / 64) + h));
          const uint4 w1 = *reinterpret_cast<const uint4*>(kt + piece<D>(16 * ck + gid + 8, tig * (D / 64) + h));
          const uint32_t b0[4] = {w0.x, w0.y, w0.z, w0.w}, b1[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t ka[4] = {e4m3x2_to_f16x2(b0[k]), e4m3x2_to_f16x2(b1[k]), e4m3x2_to_f16x2(b0[k] >> 16),
                                    e4m3x2_to_f16x2(b1[k] >> 16)};
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
              for (int p = 0; p < NP; ++p) mma_f16(x[n], ka, qf[p][n][4 * h + k][0], qf[p][n][4 * h + k][1]);
          }
        }
        // the V rows of tokens 2 tig, + 1, 2 tig + 8, + 9 (their latency under the softmax)
        constexpr int WPT = D / 32;             // 4-byte words of a thread's row piece
        uint32_t w[4][WPT];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = 16 * ck + 2 * tig + (k & 1) + 8 * (k >> 1);
          if constexpr (D == 128) {
            const uint4 y = *reinterpret_cast<const uint4*>(vt + piece<D>(row, gid));
            w[k][0] = y.x; w[k][1] = y.y; w[k][2] = y.z; w[k][3] = y.w;
          } else {
            const uint2 y = *reinterpret_cast<const uint2*>(vt + piece<D>(row, gid >> 1) + 8 * (gid & 1));
            w[k][0] = y.x; w[k][1] = y.y;
          }
        }
        const bool edge = key0 + 16 > lim_min;
        if (edge) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
          {
            const int key = key0 + 2 * tig + (k & 1) + 8 * (k >> 1);
            uint32_t bad = 0;
#pragma unroll
            for (int e = 0; e < WPT; ++e) {
              const uint32_t n = key >= u.kend ? 0xffffffffu : nan_codes(w[k][e]);   // beyond the unit's keys: whatever is there
              w[k][e] &= ~n;
              bad |= n;
            }
            if (bad && key < u.kend) atomicMin(&sm.nan_token[seg & 1], key);
          }
        }
        float top[NQ][2];
        bool up = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float fac = cs[n][h] * ksc;
            x[n][h] *= fac;
            x[n][2 + h] *= fac;
            if (edge) {
              if (key0 + gid >= lim[n][h]) x[n][h] = -INFINITY;
              if (key0 + gid + 8 >= lim[n][h]) x[n][2 + h] = -INFINITY;
            }
            top[n][h] = max_column(fmaxf(x[n][h], x[n][2 + h]));
            up = up || top[n][h] - m[n][h] > fminf(kSlack, r[n][h] + kSlack - vlog);
          }
        if (__any_sync(0xffffffffu, up)) {
          // the references rise: what was summed is scaled down (0 stays 0)
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            float g[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float was = r[n][h];
              if (top[n][h] - m[n][h] > kSlack) {
                l[n][h] *= tc::ex2(m[n][h] - top[n][h]);
                was -= top[n][h] - m[n][h];
                m[n][h] = top[n][h];
              }
              const float y = top[n][h] - m[n][h] + vlog;
              const float to = fmaxf(y > was + kSlack ? ceilf(y) : floorf(was), kLeastRef);
              g[h] = tc::ex2(was - to);
              r[n][h] = to;
              rs[n][h] = pow2_bits(kPExp - (int)to);
            }
#pragma unroll
            for (int i = 0; i < NM; ++i) {
              o[n][i][0] *= g[0]; o[n][i][1] *= g[1]; o[n][i][2] *= g[0]; o[n][i][3] *= g[1];
            }
          }
        }
        __syncwarp();                           // (the products take whole warps)
        uint32_t pf[NP][NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          const float r0m = m[n][0] == -INFINITY ? 0.f : m[n][0], r1m = m[n][1] == -INFINITY ? 0.f : m[n][1];
          // (finite, also where a row sees nothing of a page far above its reference)
          const float c0 = fminf(vsc * rs[n][0], 0x1p127f), c1 = fminf(vsc * rs[n][1], 0x1p127f);
#pragma unroll
          for (int h = 0; h < 2; ++h) {         // token gid, gid + 8
            const float p0 = tc::ex2(x[n][2 * h] - r0m), p1 = tc::ex2(x[n][2 * h + 1] - r1m);
            l[n][0] += p0;
            l[n][1] += p1;
            const uint32_t hi = pack_f16(p0 * c0, p1 * c1);
            pf[0][n][h] = transpose8(hi);
            if (NP == 2) pf[NP - 1][n][h] = transpose8(pack_rest(p0 * c0, p1 * c1, hi));
          }
        }
        // PV: dimensions gid * D/8 + 4 e + 2 k (row gid of the tile) and + 1 (row gid + 8)
#pragma unroll
        for (int e = 0; e < WPT; ++e) {
          const uint32_t lo[2] = {__byte_perm(w[0][e], w[1][e], 0x5140), __byte_perm(w[0][e], w[1][e], 0x7362)};
          const uint32_t hi[2] = {__byte_perm(w[2][e], w[3][e], 0x5140), __byte_perm(w[2][e], w[3][e], 0x7362)};
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t va[4] = {e4m3x2_to_f16x2(lo[k]), e4m3x2_to_f16x2(lo[k] >> 16), e4m3x2_to_f16x2(hi[k]),
                                    e4m3x2_to_f16x2(hi[k] >> 16)};
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
              if constexpr (NP == 2) {
                // the tensor core cuts its sums off, the smaller part first; added up to nearest
                float y[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(y, va, pf[NP - 1][n][0], pf[NP - 1][n][1]);
                mma_f16(y, va, pf[0][n][0], pf[0][n][1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][2 * e + k][i] += y[i];
              } else {
                mma_f16(o[n][2 * e + k], va, pf[0][n][0], pf[0][n][1]);
              }
            }
          }
        }
      }
      off = ck - kChunks;
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&sm.empty[st]);
    }
    // ---- the segment's end: the warps' states are added up
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[n][h] = sum_column(l[n][h]);
        if (gid == 0) {
          sm.wm[warp][8 * n + 2 * tig + h] = m[n][h];
          sm.wl[warp][8 * n + 2 * tig + h] = l[n][h];
        }
      }
    __syncwarp();                               // (the named barriers take whole warps)
    if (tc::named_sync_any(1, 32 * NW, !ok)) break;         // some warp gave up: all stop
    const int nan_from = sm.nan_token[seg & 1];
    ++seg;
    if (threadIdx.x == 0) sm.nan_token[seg & 1] = kNoNan;   // (noted from the next segment on)
    // row r's states are put together by warp r (and r + NW): lane k has warp k's
    for (int row = warp; row < MT; row += NW) {
      const float x = lane < NW ? sm.wm[lane][row] : -INFINITY;
      const float y = lane < NW ? sm.wl[lane][row] : 0.f;
      float mx = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      mx = max_column(mx);
      // (a state without a maximum holds 0, or NaN)
      const float f = x == -INFINITY ? 1.f : tc::ex2(x - mx);
      float sum = y * f;
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      sum = sum_column(sum);
      if (lane < NW) sm.wf[lane][row] = f;
      if (lane == 0) sm.ml[row] = make_float2(mx, sum);
    }
    __syncwarp();
    tc::named_sync(1, 32 * NW);
    // outputs in true units of the row's maximum
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const float2 f = *reinterpret_cast<const float2*>(&sm.wf[warp][8 * n + 2 * tig]);
      const float g0 = f.x * pow2_inverse(rs[n][0]), g1 = f.y * pow2_inverse(rs[n][1]);
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        o[n][i][0] *= g0; o[n][i][1] *= g1; o[n][i][2] *= g0; o[n][i][3] *= g1;
      }
    }
    // A thread holds dimensions gid * D/8 ... of rows 8 n + 2 tig, + 1, as D/32
    // 16-byte pieces each; pieces are XOR-permuted by the row.
    auto spot = [](int row, int pc4) { return row * (D / 4) + (pc4 ^ ((row >> 1) & 3) * (D / 64)); };
    auto put = [&](bool add) {
      float4* slot = reinterpret_cast<float4*>(&sm.merge[warp % C::SLOTS][0][0]);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < D / 32; ++e) {
            float4* at = slot + spot(8 * n + 2 * tig + h, gid * (D / 32) + e);
            float (&y)[4] = o[n][2 * e], (&z)[4] = o[n][2 * e + 1];
            if (add) {
              const float4 v = *at;
              y[h] += v.x; y[2 + h] += v.y; z[h] += v.z; z[2 + h] += v.w;
            } else {
              *at = make_float4(y[h], y[2 + h], z[h], z[2 + h]);
            }
          }
    };
    // groups of SLOTS warps, the last first: each adds the group after it
    constexpr int GROUPS = (NW + C::SLOTS - 1) / C::SLOTS;
#pragma unroll
    for (int gi = GROUPS - 1; gi >= 0; --gi) {
      if (warp / C::SLOTS == gi) {
        if (gi < GROUPS - 1 && warp + C::SLOTS < NW) put(true);
        put(false);
      }
      tc::named_sync(1, 32 * NW);
    }
    // items of four dimensions of a row
    constexpr int ITEMS = MT * D / 4, IPT = (ITEMS + 32 * NW - 1) / (32 * NW);
    float M[IPT], L[IPT];
    float4 y[IPT];
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      const int it = threadIdx.x + k * 32 * NW;
      if (it >= ITEMS) break;
      const int row = it / (D / 4);
      M[k] = sm.ml[row].x;
      L[k] = sm.ml[row].y;
      y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int b = 0; b < (NW < C::SLOTS ? NW : C::SLOTS); ++b) {
        const float4 z = reinterpret_cast<const float4*>(&sm.merge[b][0][0])[spot(row, it % (D / 4))];
        y[k].x += z.x; y[k].y += z.y; y[k].z += z.z; y[k].w += z.w;
      }
      const int rho = r0 + row, nan_to = min(t1 * kKT, a.causal ? min(u.kend, base + rho / G) : u.kend);
      if (nan_from < nan_to && rho < u.q.m * G) {
        const uint32_t bad = nan_dims<4>(c, s, u.r, u.g, nan_from, nan_to, it % (D / 4) * 4);
        const float nan = __uint_as_float(0x7fffffffu);
        if (bad & 1u) y[k].x = nan;
        if (bad & 2u) y[k].y = nan;
        if (bad & 4u) y[k].z = nan;
        if (bad & 8u) y[k].w = nan;
      }
    }
    const bool whole = wk.whole();
    bool write = true;
    int first = 0, final = 0;
    if (!whole) {
      // a piece of a unit: to the workspace; the unit's last piece to arrive adds them up
      first = wk.first_block(sh);
      final = wk.last_block(sh);
      const int64_t mine = 2 * (int64_t)blockIdx.x + (t0 == 0 ? 1 : 0);
#pragma unroll
      for (int k = 0; k < IPT; ++k) {
        const int it = threadIdx.x + k * 32 * NW;
        if (it >= ITEMS) break;
        reinterpret_cast<float4*>(a.part_o + mine * MT * D)[it] = y[k];
        if (it % (D / 4) == 0) a.part_ml[mine * MT + it / (D / 4)] = make_float2(M[k], L[k]);
      }
      __syncwarp();
      tc::named_sync(1, 32 * NW);
      if (warp == 0) {
        const bool all = piece_done(a.flags, 1, a.token, first, final);
        if (lane == 0) sm.last = all;
        __syncwarp();
      }
    }
    tc::named_sync(1, 32 * NW);                 // states and merge buffer are read: the next segment may write
    if (!whole) write = sm.last;
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      const int it = threadIdx.x + k * 32 * NW;
      if (it >= ITEMS) break;
      const int row = it / (D / 4), rho = u.rt * MT + row;
      if (!write || rho >= u.q.m * G) continue;
      if (!whole) {
        auto slot = [&](int b) { return 2 * (int64_t)b + (b == first ? 1 : 0); };
        float mx = -INFINITY, lx = 0.f;
        float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
        // four pieces' loads at a time; what was summed is scaled to a new maximum
#pragma unroll 1
        for (int b0 = first; b0 <= final; b0 += 4) {
          float2 ml[4];
          float4 v[4];
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            ml[b] = make_float2(-INFINITY, 0.f);
            v[b] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (b0 + b <= final) {
              ml[b] = __ldcg(&a.part_ml[slot(b0 + b) * MT + row]);
              v[b] = __ldcg(reinterpret_cast<const float4*>(a.part_o + slot(b0 + b) * MT * D) + it);
            }
          }
          const float nm = fmaxf(mx, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)));
          const float g = mx == -INFINITY ? 1.f : tc::ex2(mx - nm);
          mx = nm;
          lx *= g;
          z.x *= g; z.y *= g; z.z *= g; z.w *= g;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const float wt = ml[b].x == -INFINITY ? 1.f : tc::ex2(ml[b].x - nm);
            lx = fmaf(ml[b].y, wt, lx);
            z.x = fmaf(v[b].x, wt, z.x);
            z.y = fmaf(v[b].y, wt, z.y);
            z.z = fmaf(v[b].z, wt, z.z);
            z.w = fmaf(v[b].w, wt, z.w);
          }
        }
        M[k] = mx;
        L[k] = lx;
        y[k] = z;
      }
      const float inv = L[k] > 0.f ? 1.f / L[k] : (L[k] == L[k] ? 0.f : L[k]);    // no token: zeros; NaN stays
      const int i = rho / G, j = rho - i * G;
      const int64_t at = (int64_t)(u.q.row0 + i) * a.Hq + u.g * G + j;
      T* dst = static_cast<T*>(a.out) + at * D + it % (D / 4) * 4;
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(dst) = make_float4(y[k].x * inv, y[k].y * inv, y[k].z * inv, y[k].w * inv);
      } else {
        const __nv_bfloat162 b0 = __floats2bfloat162_rn(y[k].x * inv, y[k].y * inv);
        const __nv_bfloat162 b1 = __floats2bfloat162_rn(y[k].z * inv, y[k].w * inv);
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
      }
      if (a.lse && it % (D / 4) == 0) a.lse[at] = L[k] == 0.f ? -INFINITY : fmaf(M[k], 0.6931471805599453f, logf(L[k]));
    }
  } while (wk.next(line, s, err));
  if (!ok && lane == 0) set_status(err, VC_ERR_DEVICE_TIMEOUT);
  }
  __syncthreads();
  if (threadIdx.x == 0) store_status(a, sm.err);
}

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

}  // namespace

// The pool as rows of d codes; a box is a page's rows of one head.
bool kv8_pool_map(CUtensorMap* m, const void* base, const vc_kv8& c) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
  if (!enc) return false;
  cuuint64_t dims[2] = {(cuuint64_t)c.d, (cuuint64_t)c.n_pages * c.Hkv * c.page};
  cuuint64_t strides[1] = {(cuuint64_t)c.d};
  cuuint32_t box[2] = {(cuuint32_t)c.d, (cuuint32_t)c.page};
  cuuint32_t es[2] = {1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, c.d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool kv8_rows_map(CUtensorMap* m, const void* q, int64_t n_rows, int Hq, int d, int64_t stride, int heads, int rows) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = encode_fn();
  if (!enc) return false;
  cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)Hq, (cuuint64_t)n_rows};
  cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)stride * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)rows};
  cuuint32_t es[3] = {1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

template <typename T, int D, int NQ>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  using C = Cfg<T, D, NQ>;
  constexpr size_t smem = sizeof(Smem<T, D, NQ>) + 1024;
  static_assert(smem <= 232448, "shared memory of a block");
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = kv8_allow_smem(reinterpret_cast<const void*>(kv8_attn_kernel<T, D, NQ>), smem, allowed);
  if (e != cudaSuccess) return e;
  CUtensorMap mk, mv;
  if (!kv8_pool_map(&mk, c.K_codes, c) || !kv8_pool_map(&mv, c.V_codes, c)) return cudaErrorInvalidValue;
  // no more blocks than the line can have tiles
  const int64_t G = a.Hq / c.Hkv;
  const int64_t units = ((int64_t)s.n_rows * G / C::MT + (s.n_req < s.n_rows ? s.n_req : s.n_rows)) * c.Hkv;
  const int64_t tiles = units * (((int64_t)s.max_pages * c.page + kKT - 1) / kKT);
  const int64_t sms = kv8_sm_count();
  ProfileScope ps("kv8_attn", st);
  kv8_attn_kernel<T, D, NQ><<<(unsigned)(tiles < sms ? tiles : sms), C::THREADS, smem, st>>>(mk, mv, c, s, a);
  return cudaGetLastError();
}

// Units of 8 query rows where the requests have no more on average (a decode
// step of up to 8 query heads a KV head), else of 16.  Us with units of 8 / of
// 16, d = 128, 8 KV heads: 64 requests of 8192 tokens, 8 rows 173 / 240, 16 rows
// 327 / 248; one request, 8 rows 13.5 / 17.7, 16 rows 15.7 / 20.5 (twice the
// units keep more SMs busy there, which a length on the device does not tell).
template <typename T, int D>
cudaError_t launch_q(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  const int64_t rows = (int64_t)s.n_rows * (a.Hq / c.Hkv);
  return rows <= 8 * (int64_t)s.n_req ? launch_t<T, D, 1>(c, s, a, st) : launch_t<T, D, 2>(c, s, a, st);
}

}  // namespace

int kv8_sm_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 1;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 1;
  if (n > kKv8MaxCtas) n = kKv8MaxCtas;
  cached[dev].store(n, std::memory_order_relaxed);
  return n;
}

cudaError_t kv8_allow_smem(const void* kernel, size_t bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

int kv8_attn_rows_mma() { return 16; }

cudaError_t launch_kv8_attn_mma(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8AttnArgs& a,
                                cudaStream_t st) {
  if (dtype == VC_BF16)
    return c.d == 128 ? launch_q<__nv_bfloat16, 128>(c, s, a, st) : launch_q<__nv_bfloat16, 64>(c, s, a, st);
  return c.d == 128 ? launch_q<float, 128>(c, s, a, st) : launch_q<float, 64>(c, s, a, st);
}

}  // namespace vc
