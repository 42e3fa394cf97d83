// Attention over the 8-bit paged cache, few query rows a request
// (viscache_kv8_attention):
//     out[rho] = sum_t p_t V[t] / sum_t p_t,  p_t = 2^(c q[rho] . K[t] - m),
// c = scale * log2(e), over the pages of one request and KV head.
//
// Reads d bytes of K and of V a token for at most 16 query rows: bound by the
// codes' bytes as long as expanding them stays cheap.  One persistent block
// per SM takes an equal share of the line of key tiles (kv8_sched.cuh); a
// producer warp brings 128-token tiles into a shared-memory ring by TMA (one
// box a page: the page's rows of one head are contiguous), eight warps take
// 16 tokens of a tile each.
//
// Products are m16n8k16 with the query rows as M, fp16 operands and fp32 sums:
// an e4m3 code is exactly an fp16 number, so codes are expanded to fp16 in
// registers (two a conversion) and never written anywhere.  The order of the
// contracted index is free, so a thread's 16-byte read of a K row serves four
// k-steps of QK: thread column tig holds dimensions tig * D/4 ... of its row.
// For PV the columns (output dimensions) are permuted the same way: a thread
// reads 16 bytes of the rows of its four tokens, pairs them with byte
// permutations and converts.  Accumulators of QK are the A operand of PV.
//
// Numbers: a query row is divided by the power of two below its largest
// magnitude, which makes fp16 hold bf16 values exactly (down to 2^-14 of that
// magnitude, then to 2^-24 of it); fp32 calls use a second fp16 part of the
// row and of the probabilities.  Scores are scaled by the page's K scale in
// fp32.  Probabilities enter as p * 2^12 * (V scale / largest V scale so far
// of the warp): at most 2^14 in fp16, so they keep 11 bits down to 2^-26 of
// the largest.  The row sum adds them before they are rounded.  The maximum
// m follows the scores with a slack of 2 (log2 units), which saves most
// rescales of the accumulators.
#include <cudaTypedefs.h>

#include <mutex>

#include "kernels.h"
#include "kv8.cuh"
#include "kv8_sched.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace kv8;

constexpr int kWarps = 8;                       // consumer warps
constexpr int kThreads = 32 * (kWarps + 1);     // and the producer
constexpr int kKT = 128;                        // tokens of a tile, 16 a warp
constexpr int kMT = 16;                         // query rows of a unit
constexpr float kSlack = 2.f;
constexpr float kPScale = 4096.f;               // 2^12

template <int D>
struct Cfg {
  static constexpr int STAGE = kKT * D;                     // bytes of K, and of V
  static constexpr int NST = D == 128 ? 5 : 10;
};

template <int D>
struct Smem {
  uint8_t ring[Cfg<D>::NST][2][Cfg<D>::STAGE];              // [K, V]
  float merge[4][kMT][D];
  float scale[Cfg<D>::NST][2][kKT / 16];                    // [K, V][page of the tile]
  float wm[kWarps][kMT], wl[kWarps][kMT], wv[kWarps];       // a segment's warp states
  uint64_t full[Cfg<D>::NST], empty[Cfg<D>::NST];
  int64_t scan[kThreads / 32];
  Share share;
  int abort, last;
};

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

// Byte offset of 16-byte piece c of row r in a tile as TMA wrote it (128-byte
// rows with the 128-byte swizzle, 64-byte rows with the 64-byte one).
template <int D>
__device__ __forceinline__ uint32_t piece(int r, int c) {
  return D == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4))
                  : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}

__device__ __forceinline__ float max_quad(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float sum_quad(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

// The warp's query fragments (row gid and gid + 8 of the unit), normalised,
// and each row's power of two.
template <typename T, int D, int NP>
__device__ __forceinline__ void load_q(const T* q, int64_t q_stride, const Unit& u, int G, int Hq,
                                       uint32_t (&f)[NP][D / 16][4], float (&qs)[2]) {
  constexpr int DPT = D / 4;                    // dimensions of a thread
  const int gid = (threadIdx.x & 31) >> 2, tig = threadIdx.x & 3;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int rho = u.rt * kMT + gid + 8 * h;
    float x[DPT];
    float amax = 0.f;
    if (rho < u.q.m * G) {
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
    amax = max_quad(amax);
    const uint32_t ex = __float_as_uint(amax) & 0x7f800000u;
    // zero, tiny or not finite rows as they are; 2^126 at most, whose inverse is normal
    qs[h] = ex == 0u || ex == 0x7f800000u ? 1.f : __uint_as_float(min(ex, 253u << 23));
    const float inv = pow2_inverse(qs[h]);
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const float a0 = x[4 * s] * inv, a1 = x[4 * s + 1] * inv, a2 = x[4 * s + 2] * inv, a3 = x[4 * s + 3] * inv;
      f[0][s][h] = pack_f16(a0, a1);            // k = 2 tig, + 1
      f[0][s][2 + h] = pack_f16(a2, a3);        // k = 2 tig + 8, + 9
      if (NP == 2) {
        f[NP - 1][s][h] = pack_rest(a0, a1, f[0][s][h]);
        f[NP - 1][s][2 + h] = pack_rest(a2, a3, f[0][s][2 + h]);
      }
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) kv8_attn_kernel(const __grid_constant__ CUtensorMap tmK,
                                                               const __grid_constant__ CUtensorMap tmV,
                                                               const __grid_constant__ vc_kv8 c,
                                                               const __grid_constant__ vc_kv8_step s,
                                                               const __grid_constant__ Kv8AttnArgs a) {
  using C = Cfg<D>;
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;    // fp16 parts of a query value and of a probability
  constexpr int KS = D / 16;                    // k-steps of QK
  constexpr int NT = D / 8;                     // output column tiles of PV
  extern __shared__ uint8_t smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(tc::align1024(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.Hq / c.Hkv;
  const Line<kMT, kKT> line{c.Hkv, G, c.page, a.causal};
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NST; ++i) {
      tc::mbar_init(&sm.full[i], 1);
      tc::mbar_init(&sm.empty[i], kWarps);
    }
    sm.abort = 0;
    tc::fence_mbar_init();
  }
  find_share<kThreads>(line, s, a.status, sm.share, sm.scan);     // ends with a barrier
  const Share& sh = sm.share;
  if (sh.begin >= sh.end) return;
  volatile int* abort = &sm.abort;
  Walk wk;
  wk.start(sh);
  const Unit& u = wk.u;
  const int &t0 = wk.t0, &t1 = wk.t1;           // the segment's tiles of its unit
  int fill = 0;                                 // tiles so far (ring position)

  if (warp == kWarps) {
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
        pid = live ? load_page(s, c.n_pages, u.r, j, a.status) : -1;
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
          if (mine) {
            sm.scale[st][0][bp] = ks;
            sm.scale[st][1][bp] = vs;
          }
          const int pages = __popc(__ballot_sync(0xffffffffu, mine && live));
          __syncwarp();
          if (lane == 0) tc::mbar_arrive_expect_tx(&sm.full[st], (uint32_t)pages * 2 * page_bytes);
          __syncwarp();
          if (mine && live) {
            // a page that does not exist counts with scale 0; page 0 stands in
            const int row = (max(pid, 0) * c.Hkv + u.g) * c.page;
            tc::tma_load_2d(sm.ring[st][0] + bp * page_bytes, &tmK, 0, row, &sm.full[st]);
            tc::tma_load_2d(sm.ring[st][1] + bp * page_bytes, &tmV, 0, row, &sm.full[st]);
          }
        }
        pid = npid;
        ks = nks;
        vs = nvs;
        live = nlive;
      }
    } while (ok && wk.next(line, s, a.status));
    // every copy has landed before the block may end
    __syncwarp();
    if (lane == 0)
      for (int i = max(0, fill - C::NST); i < fill; ++i) tc::drain_wait(&sm.full[i % C::NST], (i / C::NST) & 1);
    return;
  }

  // ---- consumers: warp w has tokens 16 w .. 16 w + 15 of every tile
  const int gid = lane >> 2, tig = lane & 3;
  const int wpage = 16 * warp / c.page;         // the page of the tile they lie in
  bool ok = true;
  do {
    uint32_t qf[NP][KS][4];
    float qs[2];
    load_q<T, D, NP>(static_cast<const T*>(a.q), a.q_stride, u, G, a.Hq, qf, qs);
    const float cs0 = a.scale_log2 * qs[0], cs1 = a.scale_log2 * qs[1];
    // keys each row sees, and the fewest that any row of the unit sees
    int lim0 = u.q.len, lim1 = u.q.len, lim_min = u.kend;
    if (a.causal) {
      const int base = u.q.len - u.q.m + 1, r0 = u.rt * kMT;
      lim0 = base + (r0 + gid) / G;
      lim1 = base + (r0 + gid + 8) / G;
      lim_min = base + r0 / G;
    }
    lim0 = min(lim0, u.kend);
    lim1 = min(lim1, u.kend);
    float o[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f, vref = 0.f;
    for (int tile = t0; tile < t1; ++tile, ++fill) {
      const int st = fill % C::NST;
      ok = ok && tc::warp_wait(&sm.full[st], (fill / C::NST) & 1, abort);
      if (!ok) continue;
      const int key0 = tile * kKT + 16 * warp;
      if (key0 < u.kend) {
        const uint8_t* kt = sm.ring[st][0];
        const uint8_t* vt = sm.ring[st][1];
        const float ksc = sm.scale[st][0][wpage], vsc = sm.scale[st][1][wpage];
        // scores of keys key0 + gid (n = gid of tile 0) and + 8
        float x[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int row = 16 * warp + 8 * n + gid;
          x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
#pragma unroll
          for (int h = 0; h < D / 64; ++h) {
            const uint4 w = *reinterpret_cast<const uint4*>(kt + piece<D>(row, tig * (D / 64) + h));
            const uint32_t b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t b0 = e4m3x2_to_f16x2(b[k]), b1 = e4m3x2_to_f16x2(b[k] >> 16);
              mma_f16(x[n], qf[0][4 * h + k], b0, b1);
              if (NP == 2) mma_f16(x[n], qf[NP - 1][4 * h + k], b0, b1);
            }
          }
        }
        const float f0 = cs0 * ksc, f1 = cs1 * ksc;
        const bool edge = key0 + 16 > lim_min;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          x[n][0] *= f0; x[n][1] *= f0; x[n][2] *= f1; x[n][3] *= f1;
          if (edge) {
            const int key = key0 + 8 * n + 2 * tig;
            if (key >= lim0) x[n][0] = -INFINITY;
            if (key + 1 >= lim0) x[n][1] = -INFINITY;
            if (key >= lim1) x[n][2] = -INFINITY;
            if (key + 1 >= lim1) x[n][3] = -INFINITY;
          }
        }
        const float t0m = max_quad(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1])));
        const float t1m = max_quad(fmaxf(fmaxf(x[0][2], x[0][3]), fmaxf(x[1][2], x[1][3])));
        const bool up0 = t0m > m0 + kSlack, up1 = t1m > m1 + kSlack, upv = vsc > vref;
        if (__any_sync(0xffffffffu, up0 || up1) || upv) {
          // the references rise: what was summed is scaled down (0 stays 0)
          float g0 = up0 ? tc::ex2(m0 - t0m) : 1.f, g1 = up1 ? tc::ex2(m1 - t1m) : 1.f;
          if (up0) m0 = t0m;
          if (up1) m1 = t1m;
          l0 *= g0;
          l1 *= g1;
          if (upv) {
            const float gv = vref * pow2_inverse(vsc);
            vref = vsc;
            g0 *= gv;
            g1 *= gv;
          }
#pragma unroll
          for (int i = 0; i < NT; ++i) { o[i][0] *= g0; o[i][1] *= g0; o[i][2] *= g1; o[i][3] *= g1; }
        }
        const float r0 = m0 == -INFINITY ? 0.f : m0, r1 = m1 == -INFINITY ? 0.f : m1;
        const float pc = vsc * pow2_inverse(vref) * kPScale;
        uint32_t pf[NP][4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const float p0 = tc::ex2(x[n][0] - r0), p1 = tc::ex2(x[n][1] - r0);
          const float p2 = tc::ex2(x[n][2] - r1), p3 = tc::ex2(x[n][3] - r1);
          l0 += p0 + p1;
          l1 += p2 + p3;
          pf[0][2 * n] = pack_f16(p0 * pc, p1 * pc);
          pf[0][2 * n + 1] = pack_f16(p2 * pc, p3 * pc);
          if (NP == 2) {
            pf[NP - 1][2 * n] = pack_rest(p0 * pc, p1 * pc, pf[0][2 * n]);
            pf[NP - 1][2 * n + 1] = pack_rest(p2 * pc, p3 * pc, pf[0][2 * n + 1]);
          }
        }
        // PV: tokens 2 tig, + 1 (b0) and 2 tig + 8, + 9 (b1), dimensions gid * D/8 ...
        constexpr int WPT = D / 32;             // 4-byte words of a thread's row piece
        uint32_t w[4][WPT];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = 16 * warp + 2 * tig + (k & 1) + 8 * (k >> 1);
          if constexpr (D == 128) {
            const uint4 y = *reinterpret_cast<const uint4*>(vt + piece<D>(row, gid));
            w[k][0] = y.x; w[k][1] = y.y; w[k][2] = y.z; w[k][3] = y.w;
          } else {
            const uint2 y = *reinterpret_cast<const uint2*>(vt + piece<D>(row, gid >> 1) + 8 * (gid & 1));
            w[k][0] = y.x; w[k][1] = y.y;
          }
          if (edge && key0 - 16 * warp + row >= u.kend) {   // beyond the unit's keys: whatever is there
#pragma unroll
            for (int e = 0; e < WPT; ++e) w[k][e] = 0u;
          }
        }
#pragma unroll
        for (int e = 0; e < WPT; ++e) {
          const uint32_t lo0 = __byte_perm(w[0][e], w[1][e], 0x5140), hi0 = __byte_perm(w[0][e], w[1][e], 0x7362);
          const uint32_t lo1 = __byte_perm(w[2][e], w[3][e], 0x5140), hi1 = __byte_perm(w[2][e], w[3][e], 0x7362);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t b0 = e4m3x2_to_f16x2((k < 2 ? lo0 : hi0) >> (16 * (k & 1)));
            const uint32_t b1 = e4m3x2_to_f16x2((k < 2 ? lo1 : hi1) >> (16 * (k & 1)));
            mma_f16(o[4 * e + k], pf[0], b0, b1);
            if (NP == 2) mma_f16(o[4 * e + k], pf[NP - 1], b0, b1);
          }
        }
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&sm.empty[st]);
    }
    // ---- the segment's end: the warps' states are added up
    l0 = sum_quad(l0);
    l1 = sum_quad(l1);
    if (tig == 0) {
      sm.wm[warp][gid] = m0;
      sm.wm[warp][gid + 8] = m1;
      sm.wl[warp][gid] = l0;
      sm.wl[warp][gid + 8] = l1;
    }
    if (tc::named_sync_any(1, 32 * kWarps, !ok)) break;     // some warp gave up: all stop
    // as the last step has them: thread: row t / 16, dimensions (t % 16) * D/16 ...
    // (read here, before the next barrier: a fast warp may overwrite them in
    // the next segment).  A state without a maximum holds 0, or NaN.
    const int row = threadIdx.x >> 4, part = threadIdx.x & 15;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm.wm[w][row]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float x = sm.wm[w][row];
      L = fmaf(sm.wl[w][row], x == -INFINITY ? 1.f : tc::ex2(x - M), L);
    }
    float M0 = -INFINITY, M1 = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      M0 = fmaxf(M0, sm.wm[w][gid]);
      M1 = fmaxf(M1, sm.wm[w][gid + 8]);
    }
    {
      const float g0 = m0 == -INFINITY ? 0.f : tc::ex2(m0 - M0) * (vref / kPScale);
      const float g1 = m1 == -INFINITY ? 0.f : tc::ex2(m1 - M1) * (vref / kPScale);
#pragma unroll
      for (int i = 0; i < NT; ++i) { o[i][0] *= g0; o[i][1] *= g0; o[i][2] *= g1; o[i][3] *= g1; }
    }
    // a thread's columns: dimensions tig * D/4 + (0 .. NT-1) from the even
    // accumulator columns, + NT ... from the odd ones; 16-byte chunks XOR-permuted
    constexpr int CPT = D / 16;                 // chunks of a thread and row
    auto chunk = [](int row, int ch) { return ch ^ (ch / CPT * 2 + (row & 1)); };
    float4* slot = reinterpret_cast<float4*>(&sm.merge[warp & 3][0][0]);
    auto put = [&](bool add) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = gid + 8 * h;
#pragma unroll
        for (int e = 0; e < CPT; ++e) {
          const int odd = e >= CPT / 2, i = 4 * (e - (odd ? CPT / 2 : 0));
          float4* at = slot + row * (D / 4) + chunk(row, CPT * tig + e);
          const int k = 2 * h + odd;
          if (add) {
            const float4 y = *at;
            o[i][k] += y.x; o[i + 1][k] += y.y; o[i + 2][k] += y.z; o[i + 3][k] += y.w;
          } else {
            *at = make_float4(o[i][k], o[i + 1][k], o[i + 2][k], o[i + 3][k]);
          }
        }
      }
    };
    if (warp >= 4) put(false);
    tc::named_sync(1, 32 * kWarps);
    if (warp < 4) {
      put(true);
      put(false);
    }
    tc::named_sync(1, 32 * kWarps);
    const int rho = u.rt * kMT + row;
    const bool real = rho < u.q.m * G;
    constexpr int EPT = D / 16;
    float y[EPT];
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 z =
            reinterpret_cast<const float4*>(&sm.merge[k][0][0])[row * (D / 4) + chunk(row, (part * EPT + e) / 4)];
        v.x += z.x; v.y += z.y; v.z += z.z; v.w += z.w;
      }
      y[e] = v.x; y[e + 1] = v.y; y[e + 2] = v.z; y[e + 3] = v.w;
    }
    bool write = real;
    if (!wk.whole()) {
      // a piece of a unit: to the workspace; the unit's last piece to arrive adds them up
      const int first = wk.first_block(sh), final = wk.last_block(sh);
      const int64_t mine = 2 * (int64_t)blockIdx.x + (t0 == 0 ? 1 : 0);
      float* po = a.part_o + (mine * kMT + row) * D + part * EPT;
#pragma unroll
      for (int e = 0; e < EPT; e += 4)
        *reinterpret_cast<float4*>(po + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
      if (part == 0) a.part_ml[mine * kMT + row] = make_float2(M, L);
      __threadfence();
      tc::named_sync(1, 32 * kWarps);
      if (threadIdx.x == 0) {
        sm.last = atomicAdd(&a.arrivals[first], 1) == final - first;
        __threadfence();
      }
      tc::named_sync(1, 32 * kWarps);
      write = real && sm.last;
      if (write) {
        M = -INFINITY;
        for (int b = first; b <= final; ++b)
          M = fmaxf(M, __ldcg(&a.part_ml[(2 * (int64_t)b + (b == first ? 1 : 0)) * kMT + row]).x);
        L = 0.f;
#pragma unroll
        for (int e = 0; e < EPT; ++e) y[e] = 0.f;
#pragma unroll 4
        for (int b = first; b <= final; ++b) {
          const int64_t at = (2 * (int64_t)b + (b == first ? 1 : 0)) * kMT + row;
          const float2 ml = __ldcg(&a.part_ml[at]);
          const float w = ml.x == -INFINITY ? 1.f : tc::ex2(ml.x - M);
          L = fmaf(ml.y, w, L);
#pragma unroll
          for (int e = 0; e < EPT; e += 4) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(a.part_o + at * D + part * EPT + e));
            y[e] = fmaf(v.x, w, y[e]);
            y[e + 1] = fmaf(v.y, w, y[e + 1]);
            y[e + 2] = fmaf(v.z, w, y[e + 2]);
            y[e + 3] = fmaf(v.w, w, y[e + 3]);
          }
        }
      }
    }
    if (write) {
      const float inv = L > 0.f ? 1.f / L : (L == L ? 0.f : L);      // no token: zeros; NaN stays
      const int i = rho / G, j = rho - i * G;
      const int64_t at = (int64_t)(u.q.row0 + i) * a.Hq + u.g * G + j;
      T* dst = static_cast<T*>(a.out) + at * D + part * EPT;
#pragma unroll
      for (int e = 0; e < EPT; e += 4) {
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(dst + e) =
              make_float4(y[e] * inv, y[e + 1] * inv, y[e + 2] * inv, y[e + 3] * inv);
        } else {
          const __nv_bfloat162 b0 = __floats2bfloat162_rn(y[e] * inv, y[e + 1] * inv);
          const __nv_bfloat162 b1 = __floats2bfloat162_rn(y[e + 2] * inv, y[e + 3] * inv);
          *reinterpret_cast<uint2*>(dst + e) = make_uint2(*reinterpret_cast<const uint32_t*>(&b0),
                                                          *reinterpret_cast<const uint32_t*>(&b1));
        }
      }
      if (a.lse && part == 0) a.lse[at] = L == 0.f ? -INFINITY : fmaf(M, 0.6931471805599453f, logf(L));
    }
  } while (wk.next(line, s, a.status));
  if (!ok && lane == 0) set_status(a.status, VC_ERR_DEVICE_TIMEOUT);
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

namespace {

template <typename T, int D>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  constexpr size_t smem = sizeof(Smem<D>) + 1024;
  static std::atomic<bool> attr{false};
  if (!attr.load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(kv8_attn_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)smem);
    if (e != cudaSuccess) return e;
    attr.store(true, std::memory_order_relaxed);
  }
  CUtensorMap mk, mv;
  if (!kv8_pool_map(&mk, c.K_codes, c) || !kv8_pool_map(&mv, c.V_codes, c)) return cudaErrorInvalidValue;
  // no more blocks than the line can have tiles
  const int64_t G = a.Hq / c.Hkv;
  const int64_t units = ((int64_t)s.n_rows * G / kMT + (s.n_req < s.n_rows ? s.n_req : s.n_rows)) * c.Hkv;
  const int64_t tiles = units * (((int64_t)s.max_pages * c.page + kKT - 1) / kKT);
  const int64_t sms = kv8_sm_count();
  ProfileScope ps("kv8_attn", st);
  kv8_attn_kernel<T, D><<<(unsigned)(tiles < sms ? tiles : sms), kThreads, smem, st>>>(mk, mv, c, s, a);
  return cudaGetLastError();
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

int kv8_attn_rows_mma() { return kMT; }

cudaError_t launch_kv8_attn_mma(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8AttnArgs& a,
                                cudaStream_t st) {
  if (dtype == VC_BF16)
    return c.d == 128 ? launch_t<__nv_bfloat16, 128>(c, s, a, st) : launch_t<__nv_bfloat16, 64>(c, s, a, st);
  return c.d == 128 ? launch_t<float, 128>(c, s, a, st) : launch_t<float, 64>(c, s, a, st);
}

}  // namespace vc
