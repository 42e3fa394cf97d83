// Attention over the 8-bit paged cache, many query rows a request, bf16 rows
// (viscache_kv8_attention on tcgen05).
//
// A unit has 256 packed query rows (two tiles of 128 rows, one TMEM lane a row)
// over tiles of 128 tokens: 4 * 256 * 128 * d flops a tile, so it is bound by
// the tensor cores once the softmax and the expansion of the codes run beside
// them.  Persistent blocks, one per SM, share out the line of key tiles
// (kv8_sched.cuh).  Warps (512 threads, register shares set per warpgroup):
//   0-3, 4-7  softmax of row tile A, B: one thread a row
//   8-11      converters: a tile's codes from the staging buffer, e4m3 -> fp16,
//             into 128-byte-swizzled K and V tiles, two stages each; the unit's
//             query rows too
//   12        one thread issues the MMAs
//   13        loader: page numbers, scales, and a bulk copy per page into the
//             staging buffer (one tile of K and one of V)
// Tensor memory: S_A, S_B (128 columns each; P over the first 64 as fp16
// pairs), O_A, O_B (d columns each).  Order of issue per tile t:
//   PV_A(t) S_A(t+1) PV_B(t) S_B(t+1)
// so one row tile's softmax works while the other's products run.  MMAs of one
// thread execute in order, so S_A(t+1) may overwrite the P_A(t) that PV_A(t)
// reads, and s_full of tile t + 1 says that PV(t) is done too.
//
// Numbers: query rows are divided by the power of two below their largest
// magnitude, codes multiplied by their page's scale over the tile's largest
// one, so both are fp16 without rounding (but for pages 2^-14 of their tile).
// A row's maximum may be passed by 2^10 before O is rescaled; P = 2^(x - m + 4)
// times (V scale of the tile / the largest so far), at most 2^14, keeps 11
// bits down to 2^-18 of its reference.  Row sums are fp32, of unrounded terms.
#include "kernels.h"
#include "kv8.cuh"
#include "kv8_sched.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace kv8;
using namespace tc;

constexpr int kTcThreads = 512;
constexpr int kTcMT = 256, kTcKT = 128;
constexpr int kConvWarp0 = 8, kConvWarps = 4, kIssueWarp = 12, kLoadWarp = 13;
constexpr float kTcSlack = 10.f;                // log2 units
constexpr int kTcPExp = 4;
constexpr uint32_t kBlk = 128 * 128;            // 128 rows x 128 bytes (64 fp16 columns)
constexpr uint32_t kSCol = 0, kOCol = 256;
constexpr int kRefs = 8;                        // tiles whose scales are kept (the loader is at most 4 ahead)

template <int D>
struct TcSmem {
  uint8_t q[2][D / 64][kBlk];                   // query rows of the unit, [row tile][64-column block]
  uint8_t k[2][D / 64][kBlk];                   // [stage][block]
  uint8_t v[2][D / 64][kBlk];
  uint8_t code[2][kTcKT * D];                   // a tile's codes as they are in the cache, [K, V]
  float qs[kTcMT];                              // power of two of each query row
  float ref[kRefs][2];                          // largest page scales of tile t, at t % kRefs, [K, V]
  float part[kRefs][2][8];                      // each 16-token group's share of them
  uint64_t q_full, q_empty, k_full[2], k_empty[2], v_full[2], v_empty[2], ref_full[kRefs];
  uint64_t code_full[2], code_empty[2];
  uint64_t s_full[2], p_full[2], o_full[2], done;
  int64_t scan[kTcThreads / 32];
  Share share;
  uint32_t tmem_base;
  int abort, last[2];
};

// Instruction descriptor, kind::f16: A, B fp16, D fp32; B K-major, or MN-major.
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t M, uint32_t N, bool b_mn) {
  return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((N >> 3) << 17) | ((M >> 4) << 24);
}

// D[tmem] (+)= A[tmem] * B[smem], issued by one thread.
__device__ __forceinline__ void mma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t hmul2_bits(uint32_t a, __half2 f) {
  const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&a), f);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Sixteen codes times a power of two, as 32 bytes of row `row`, column chunk c
// (16 columns) of a tile: the two 16-byte pieces are written in an order that
// keeps the eight lanes of a row on different banks.
__device__ __forceinline__ void expand16(uint8_t* tile, int row, int c, const uint4& w, float factor) {
  const __half2 f = __float2half2_rn(factor);
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = hmul2_bits(e4m3x2_to_f16x2(x[i]), f);
    y[2 * i + 1] = hmul2_bits(e4m3x2_to_f16x2(x[i] >> 16), f);
  }
  uint8_t* base = tile + (c >> 2) * kBlk + row * 128;
  const int ch = 2 * (c & 3), r7 = row & 7;
  const uint4 lo = make_uint4(y[0], y[1], y[2], y[3]), hi = make_uint4(y[4], y[5], y[6], y[7]);
  const bool swap = (c & 4) != 0;
  *reinterpret_cast<uint4*>(base + (((ch + swap) ^ r7) << 4)) = swap ? hi : lo;
  *reinterpret_cast<uint4*>(base + (((ch + !swap) ^ r7) << 4)) = swap ? lo : hi;
}

template <int D>
__global__ void __launch_bounds__(kTcThreads, 1) kv8_attn_tc_kernel(const __grid_constant__ vc_kv8 c,
                                                                    const __grid_constant__ vc_kv8_step s,
                                                                    const __grid_constant__ Kv8AttnArgs a) {
  extern __shared__ uint8_t smem_raw[];
  TcSmem<D>& sm = *reinterpret_cast<TcSmem<D>*>(align1024(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.Hq / c.Hkv;
  const Line<kTcMT, kTcKT> line{c.Hkv, G, c.page, a.causal};
  if (threadIdx.x == 0) {
    mbar_init(&sm.q_full, kConvWarps);
    mbar_init(&sm.q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.k_full[i], kConvWarps);
      mbar_init(&sm.k_empty[i], 1);
      mbar_init(&sm.v_full[i], kConvWarps);
      mbar_init(&sm.v_empty[i], 1);
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.p_full[i], 4);
      mbar_init(&sm.o_full[i], 1);
    }
    for (int i = 0; i < kRefs; ++i) mbar_init(&sm.ref_full[i], 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.code_full[i], 1);
      mbar_init(&sm.code_empty[i], kConvWarps);
    }
    mbar_init(&sm.done, 1);
    sm.abort = 0;
    fence_mbar_init();
  }
  find_share<kTcThreads>(line, s, a.status, sm.share, sm.scan);   // ends with a barrier
  const Share& sh = sm.share;
  if (sh.begin >= sh.end) return;
  if (warp == kIssueWarp) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = sm.tmem_base;
  volatile int* abort = &sm.abort;
  Walk w;
  w.start(sh);
  int seg = 0;                                  // segments so far
  int t = 0;                                    // tiles so far
  auto rows_of = [&]() { return min(kTcMT, w.u.q.m * G - w.u.rt * kTcMT); };

  if (warp >= kConvWarp0 + kConvWarps) {
    // registers a thread: 128 at launch; 184 + 184 + 72 + 72 = 4 * 128
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == kIssueWarp && lane == 0) {
      // ---- MMA issuer
      constexpr uint32_t id_s = idesc_f16(128, kTcKT, false), id_o = idesc_f16(128, D, true);
      bool ok = true;
      int np[2] = {0, 0};                       // P tiles consumed per row tile
      // descriptors hold addresses in units of 16 bytes: offsets are added to them
      const uint64_t qd = desc_sw128(smem_u32(sm.q)), kd = desc_sw128(smem_u32(sm.k));
      const uint64_t vd = desc_sw128_mn(smem_u32(sm.v), kBlk);
      constexpr uint32_t kRows16 = sizeof(sm.q[0]) / 16;      // a row tile, a stage
      auto issue_s = [&](int x, int st) {
        const uint64_t ad = qd + (uint32_t)x * kRows16, bd = kd + (uint32_t)st * kRows16;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = ((kk >> 2) * kBlk + (kk & 3) * 32) / 16;
          mma_bf16(tbase + kSCol + x * kTcKT, ad + off, bd + off, id_s, kk ? 1u : 0u);
        }
        mma_commit(&sm.s_full[x]);
      };
      auto issue_pv = [&](int x, int st, bool first) -> bool {
        if (!mbar_wait(&sm.p_full[x], np[x] & 1, abort)) return false;
        ++np[x];
        tc_fence_after();
        const uint64_t bd = vd + (uint32_t)st * kRows16;
#pragma unroll
        for (int kk = 0; kk < kTcKT / 16; ++kk)
          mma_f16_ta(tbase + kOCol + x * D, tbase + kSCol + x * kTcKT + kk * 8, bd + kk * 2048 / 16, id_o,
                     (!first || kk) ? 1u : 0u);
        return true;
      };
      do {
        const bool two = rows_of() > 128;
        ok = mbar_wait(&sm.q_full, seg & 1, abort) && mbar_wait(&sm.k_full[t & 1], (t >> 1) & 1, abort);
        if (!ok) break;
        tc_fence_after();
        issue_s(0, t & 1);
        if (two) issue_s(1, t & 1);
        mma_commit(&sm.k_empty[t & 1]);
        for (int j = w.t0; ok && j < w.t1; ++j, ++t) {
          const int st = t & 1, sn = (t + 1) & 1;
          const bool more = j + 1 < w.t1;
          if (!mbar_wait(&sm.v_full[st], (t >> 1) & 1, abort) || !issue_pv(0, st, j == w.t0)) {
            ok = false;
            break;
          }
          if (!more) mma_commit(&sm.o_full[0]);
          if (more) {
            if (!mbar_wait(&sm.k_full[sn], ((t + 1) >> 1) & 1, abort)) {
              ok = false;
              break;
            }
            tc_fence_after();
            issue_s(0, sn);
          }
          if (two) {
            if (!issue_pv(1, st, j == w.t0)) {
              ok = false;
              break;
            }
            if (!more) mma_commit(&sm.o_full[1]);
          }
          mma_commit(&sm.v_empty[st]);
          if (more) {
            if (two) issue_s(1, sn);
            mma_commit(&sm.k_empty[sn]);
          }
        }
        if (ok) mma_commit(&sm.q_empty);
        ++seg;
      } while (ok && w.next(line, s, a.status));
      // every MMA is done before the block frees its tensor memory
      mma_commit(&sm.done);
      drain_wait(&sm.done, 0);
    }
    if (warp == kLoadWarp) {
      // ---- loader: lane -> (tile, page) of a batch of 32 pages; page numbers and
      // scales of the next batch load while this one's copies are issued
      const int ppt = kTcKT / c.page, tpb = 32 / ppt;
      const int bt = lane / ppt, bp = lane % ppt;
      const uint32_t page_bytes = (uint32_t)c.page * D;
      bool ok = true;
      int copied[2] = {0, 0};                   // tiles of K and of V under way or landed
      do {
        auto look = [&](int first, int& pid, float& ks, float& vs, bool& live) {
          const int tile = first + bt, j = tile * ppt + bp;
          live = tile < w.t1 && j * c.page < w.u.kend;
          pid = live ? load_page(s, c.n_pages, w.u.r, j, a.status) : -1;
          const int64_t at = (int64_t)max(pid, 0) * c.Hkv + w.u.g;
          ks = pid >= 0 ? __ldg(c.K_scale + at) : 0.f;
          vs = pid >= 0 ? __ldg(c.V_scale + at) : 0.f;
        };
        int pid, npid = -1;
        float ks, vs, nks = 0.f, nvs = 0.f;
        bool live, nlive = false;
        look(w.t0, pid, ks, vs, live);
        for (int tb = w.t0; ok && tb < w.t1; tb += tpb) {
          if (tb + tpb < w.t1) look(tb + tpb, npid, nks, nvs, nlive);
          // each tile's largest scales
          float kref = ks, vref = vs;
          for (int o = 1; o < ppt; o <<= 1) {
            kref = fmaxf(kref, __shfl_xor_sync(0xffffffffu, kref, o));
            vref = fmaxf(vref, __shfl_xor_sync(0xffffffffu, vref, o));
          }
          const float kf = ks * pow2_inverse(kref), vf = vs * pow2_inverse(vref);
          const int nt = min(tpb, w.t1 - tb);
          for (int i = 0; i < nt; ++i, ++t) {
            const bool mine = bt == i;
            const int rt = t % kRefs;
            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine && live)) * page_bytes;
            const int64_t at = ((int64_t)max(pid, 0) * c.Hkv + w.u.g) * (int64_t)page_bytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              if (!warp_wait(&sm.code_empty[h], (t & 1) ^ 1, abort)) {
                ok = false;
                break;
              }
              if (h == 0 && mine) {
                if (bp == 0) {
                  sm.ref[rt][0] = kref;
                  sm.ref[rt][1] = vref;
                }
                for (int e = 0; e < c.page / 16; ++e) {
                  sm.part[rt][0][bp * (c.page / 16) + e] = kf;
                  sm.part[rt][1][bp * (c.page / 16) + e] = vf;
                }
              }
              __syncwarp();
              if (lane == 0) {
                if (h == 0) mbar_arrive(&sm.ref_full[rt]);
                mbar_arrive_expect_tx(&sm.code_full[h], bytes);
              }
              ++copied[h];
              __syncwarp();
              // (a page that does not exist has scale 0: page 0 stands in)
              if (mine && live)
                bulk_load(sm.code[h] + bp * page_bytes, static_cast<const uint8_t*>(h ? c.V_codes : c.K_codes) + at,
                          page_bytes, &sm.code_full[h]);
            }
            if (!ok) break;
          }
          pid = npid;
          ks = nks;
          vs = nvs;
          live = nlive;
        }
      } while (ok && w.next(line, s, a.status));
      // every copy has landed before the block may end
      __syncwarp();
      if (lane == 0)
        for (int h = 0; h < 2; ++h)
          if (copied[h] > 0) drain_wait(&sm.code_full[h], (copied[h] - 1) & 1);
    }
  } else if (warp >= kConvWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    // ---- converters
    const int i = threadIdx.x - 32 * kConvWarp0;
    bool ok = true;
    do {
      // the unit's query rows, once the last S of the segment before is done
      if (!warp_wait(&sm.q_empty, (seg & 1) ^ 1, abort)) break;
      {
        const int rows = rows_of();
        constexpr int QL = D / 8;               // lanes of a query row
#pragma unroll 4
        for (int r = i / QL; r < kTcMT; r += 128 / QL) {
          const int qc = i % QL;
          uint4 y = make_uint4(0u, 0u, 0u, 0u);
          if (r < rows) {
            const int rho = w.u.rt * kTcMT + r, qi = rho / G, qj = rho - qi * G;
            y = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) +
                                                     (int64_t)(w.u.q.row0 + qi) * a.q_stride +
                                                     (int64_t)(w.u.g * G + qj) * D + qc * 8));
          }
          const uint32_t b[4] = {y.x, y.y, y.z, y.w};
          float x[8], amax = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(b[e] << 16);
            x[2 * e + 1] = __uint_as_float(b[e] & 0xffff0000u);
            amax = fmaxf(amax, fmaxf(fabsf(x[2 * e]), fabsf(x[2 * e + 1])));
          }
#pragma unroll
          for (int o = QL / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
          const uint32_t ex = __float_as_uint(amax) & 0x7f800000u;
          const float qs = ex == 0u || ex >= 0x7f000000u ? 1.f : __uint_as_float(ex);
          const float inv = pow2_inverse(qs);
          uint8_t* dst = sm.q[r >> 7][qc >> 3] + (r & 127) * 128 + (((qc & 7) ^ (r & 7)) << 4);
          *reinterpret_cast<uint4*>(dst) =
              make_uint4(half2_bits(x[0] * inv, x[1] * inv), half2_bits(x[2] * inv, x[3] * inv),
                         half2_bits(x[4] * inv, x[5] * inv), half2_bits(x[6] * inv, x[7] * inv));
          if (qc == 0) sm.qs[r] = qs;
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full);
      for (int j = w.t0; ok && j < w.t1; ++j, ++t) {
        const int st = t & 1;
        const int left = w.u.kend - j * kTcKT;  // tokens of the tile
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // K, then V: the codes have landed, the stage is free
          ok = warp_wait(&sm.code_full[h], t & 1, abort) &&
               warp_wait(h ? &sm.v_empty[st] : &sm.k_empty[st], ((t >> 1) & 1) ^ 1, abort);
          if (!ok) break;
          constexpr int LPR = D / 16, RP = 128 / LPR;   // lanes of a row (16 codes each), rows at once
          const int key0 = i / LPR, ch = i % LPR;
          uint8_t* tile = h ? sm.v[st][0] : sm.k[st][0];
          const float* part = sm.part[t % kRefs][h];
#pragma unroll
          for (int n = 0; n < 128 / RP; ++n) {
            const int key = key0 + RP * n;
            uint4 y = *reinterpret_cast<const uint4*>(sm.code[h] + key * D + ch * 16);
            if (key >= left) y = make_uint4(0u, 0u, 0u, 0u);    // not a token: whatever was there
            expand16(tile, key, ch, y, part[key >> 4]);
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&sm.code_empty[h]);
            mbar_arrive(h ? &sm.v_full[st] : &sm.k_full[st]);
          }
        }
      }
      ++seg;
    } while (ok && w.next(line, s, a.status));
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    // ---- softmax of row tile X, one row a thread
    const int X = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lane_off = (uint32_t)((warp & 3) << 5) << 16;
    const uint32_t s_col = tbase + lane_off + kSCol + X * kTcKT;
    const uint32_t o_col = tbase + lane_off + kOCol + X * D;
    bool ok = true;
    int ns = 0, no = 0;                         // S tiles and finished O of this row tile
    do {
      if (X == 1 && rows_of() <= 128) {         // no rows in this half
        t += w.t1 - w.t0;
        continue;
      }
      const int rho = w.u.rt * kTcMT + X * 128 + row;
      const bool real = rho < w.u.q.m * G;
      const int qi = rho / G, qj = rho - qi * G;
      int lim = w.u.kend;
      if (a.causal) lim = min(lim, w.u.q.len - w.u.q.m + 1 + qi);
      float m = -INFINITY, l = 0.f, cs = 0.f, vmax = 0.f;
      for (int j = w.t0; j < w.t1; ++j, ++t) {
        ok = ok && warp_wait(&sm.ref_full[t % kRefs], (t / kRefs) & 1, abort) && warp_wait(&sm.s_full[X], ns & 1, abort);
        if (!ok) continue;
        ++ns;
        tc_fence_after();
        if (j == w.t0) cs = a.scale_log2 * sm.qs[X * 128 + row];
        // (f > 0, so that a masked score stays -inf: scores below 1e-37 are 0)
        const float f = fmaxf(cs * sm.ref[t % kRefs][0], 1e-37f), vr = sm.ref[t % kRefs][1];
        float x[8][16];
        {
          uint32_t v[8][16];
#pragma unroll
          for (int p = 0; p < 8; ++p) tmem_ld16(s_col + p * 16, v[p]);
          tmem_wait_only();
#pragma unroll
          for (int p = 0; p < 8; ++p) {
            reg_fence(v[p]);
#pragma unroll
            for (int q = 0; q < 16; ++q) x[p][q] = __uint_as_float(v[p][q]);
          }
        }
        const int valid = lim - j * kTcKT;
        if (__any_sync(0xffffffffu, valid < kTcKT)) {
#pragma unroll
          for (int p = 0; p < 8; ++p)
#pragma unroll
            for (int q = 0; q < 16; ++q)
              if (p * 16 + q >= valid) x[p][q] = -INFINITY;
        }
        float b[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          b[p] = fmaxf(x[2 * p][0], x[2 * p + 1][0]);
#pragma unroll
          for (int q = 1; q < 16; ++q) b[p] = fmax3(b[p], x[2 * p][q], x[2 * p + 1][q]);
        }
        const float tm = fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])) * f;
        const bool raise = tm > m + kTcSlack, vraise = vr > vmax;
        float g = 1.f;
        if (raise) {
          g = ex2(m - tm);                      // 0 on the first
          l *= g;
          m = tm;
        }
        if (vraise) {
          // one step above, so that a tile with a page of the next size fits
          const float up = vr * 2.f;
          g *= vmax * pow2_inverse(up);
          vmax = up;
        }
        if (j > w.t0 && __any_sync(0xffffffffu, raise || vraise)) {
          // PV of the tile before is done (s_full) and the next waits for this P
#pragma unroll 1
          for (int p = 0; p < D / 16; ++p) {
            uint32_t v[16];
            tmem_ld16(o_col + p * 16, v);
            tmem_wait(v);
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = __float_as_uint(__uint_as_float(v[q]) * g);
            tmem_st16(o_col + p * 16, v);
          }
        }
        // exponent of P's factor: 2^4 times the tile's share of vmax, not below 2^-26
        const int lc = vr > 0.f ? max(-30, (int)(__float_as_uint(vr) >> 23) - (int)(__float_as_uint(vmax) >> 23)) : -30;
        const float mm = (m == -INFINITY ? 0.f : m) - (float)(lc + kTcPExp);
        const float2 sc = make_float2(f, f), nm = make_float2(-mm, -mm);
        float2 l0 = make_float2(0.f, 0.f), l1 = make_float2(0.f, 0.f);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t y16[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const int k = 32 * h + 2 * q;
            const float2 y = __ffma2_rn(make_float2(x[k >> 4][k & 15], x[k >> 4][(k & 15) + 1]), sc, nm);
            const float2 e = make_float2(ex2(y.x), ex2(y.y));
            if (q & 1) l1 = __fadd2_rn(l1, e);
            else l0 = __fadd2_rn(l0, e);
            y16[q] = half2_bits(e.x, e.y);
          }
          tmem_st16(s_col + h * 16, y16);
        }
        const float2 ls = __fadd2_rn(l0, l1);
        l += (ls.x + ls.y) * __uint_as_float((uint32_t)(127 - lc - kTcPExp) << 23);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[X]);
      }
      ok = ok && warp_wait(&sm.o_full[X], no & 1, abort);
      ++no;
      if (named_sync_any(1 + X, 128, !ok)) break;
      tc_fence_after();
      // O in units of vmax * 2^-4
      const float ou = vmax * __uint_as_float((uint32_t)(127 - kTcPExp) << 23);
      const bool whole = w.whole();
      const int64_t at = (int64_t)(w.u.q.row0 + qi) * a.Hq + w.u.g * G + qj;
      auto put_out = [&](int col, const float (&y)[16], float inv) {
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.out) + at * D + col;
        uint32_t b8[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const __nv_bfloat162 b2 = __floats2bfloat162_rn(y[2 * q] * inv, y[2 * q + 1] * inv);
          b8[q] = *reinterpret_cast<const uint32_t*>(&b2);
        }
        *reinterpret_cast<uint4*>(dst) = make_uint4(b8[0], b8[1], b8[2], b8[3]);
        *reinterpret_cast<uint4*>(dst + 8) = make_uint4(b8[4], b8[5], b8[6], b8[7]);
      };
      auto put_lse = [&](float M, float L) {
        if (a.lse) a.lse[at] = L == 0.f ? -INFINITY : fmaf(M, 0.6931471805599453f, logf(L));
      };
      auto inverse_of = [](float L) { return L > 0.f ? 1.f / L : (L == L ? 0.f : L); };
      const int64_t mine = 2 * (int64_t)blockIdx.x + (w.t0 == 0 ? 1 : 0);
      const float inv = whole ? inverse_of(l) * ou : ou;
#pragma unroll 1
      for (int p = 0; p < D / 16; ++p) {
        uint32_t v[16];
        tmem_ld16(o_col + p * 16, v);
        tmem_wait(v);
        float y[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) y[q] = __uint_as_float(v[q]);
        if (whole) {
          if (real) put_out(p * 16, y, inv);
        } else {
          float* po = a.part_o + ((mine * 2 + X) * 128 + row) * D + p * 16;
#pragma unroll
          for (int q = 0; q < 16; q += 4)
            *reinterpret_cast<float4*>(po + q) =
                make_float4(y[q] * inv, y[q + 1] * inv, y[q + 2] * inv, y[q + 3] * inv);
        }
      }
      tc_fence_before();
      if (whole) {
        if (real) put_lse(m, l);
      } else {
        a.part_ml[(mine * 2 + X) * 128 + row] = make_float2(m, l);
        const int first = w.first_block(sh), final = w.last_block(sh);
        __threadfence();
        named_sync(1 + X, 128);
        if (row == 0) {
          sm.last[X] = atomicAdd(&a.arrivals[2 * first + X], 1) == final - first;
          __threadfence();
        }
        named_sync(1 + X, 128);
        if (sm.last[X] && real) {
          auto slot = [&](int b) { return ((2 * (int64_t)b + (b == first ? 1 : 0)) * 2 + X) * 128 + row; };
          float M = -INFINITY, L = 0.f;
          for (int b = first; b <= final; ++b) M = fmaxf(M, __ldcg(&a.part_ml[slot(b)]).x);
          for (int b = first; b <= final; ++b) {
            const float2 ml = __ldcg(&a.part_ml[slot(b)]);
            L = fmaf(ml.y, ml.x == -INFINITY ? 1.f : ex2(ml.x - M), L);
          }
          const float il = inverse_of(L);
#pragma unroll 1
          for (int p = 0; p < D / 16; ++p) {
            float y[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) y[q] = 0.f;
            for (int b = first; b <= final; ++b) {
              const int64_t k = slot(b);
              const float mx = __ldcg(&a.part_ml[k]).x;
              const float wt = mx == -INFINITY ? 1.f : ex2(mx - M);
              const float4* src = reinterpret_cast<const float4*>(a.part_o + k * D + p * 16);
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const float4 z = __ldcg(src + q);
                y[4 * q] = fmaf(z.x, wt, y[4 * q]);
                y[4 * q + 1] = fmaf(z.y, wt, y[4 * q + 1]);
                y[4 * q + 2] = fmaf(z.z, wt, y[4 * q + 2]);
                y[4 * q + 3] = fmaf(z.w, wt, y[4 * q + 3]);
              }
            }
            put_out(p * 16, y, il);
          }
          put_lse(M, L);
        }
      }
    } while (w.next(line, s, a.status));
    if (!ok && lane == 0) set_status(a.status, VC_ERR_DEVICE_TIMEOUT);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    tc_fence_after();
    tmem_dealloc(tbase, 512);
  }
  if (threadIdx.x == 0 && sm.abort) set_status(a.status, VC_ERR_DEVICE_TIMEOUT);
}

template <int D>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  constexpr size_t smem = sizeof(TcSmem<D>) + 1024;
  static std::atomic<bool> attr{false};
  if (!attr.load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(kv8_attn_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)smem);
    if (e != cudaSuccess) return e;
    attr.store(true, std::memory_order_relaxed);
  }
  const int64_t G = a.Hq / c.Hkv;
  const int64_t units = ((int64_t)s.n_rows * G / kTcMT + (s.n_req < s.n_rows ? s.n_req : s.n_rows)) * c.Hkv;
  const int64_t tiles = units * (((int64_t)s.max_pages * c.page + kTcKT - 1) / kTcKT);
  const int64_t sms = kv8_sm_count();
  ProfileScope ps("kv8_attn_tc", st);
  kv8_attn_tc_kernel<D><<<(unsigned)(tiles < sms ? tiles : sms), kTcThreads, smem, st>>>(c, s, a);
  return cudaGetLastError();
}

}  // namespace

int kv8_attn_rows_tc() { return kTcMT; }

cudaError_t launch_kv8_attn_tc(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  return c.d == 128 ? launch_t<128>(c, s, a, st) : launch_t<64>(c, s, a, st);
}

}  // namespace vc
