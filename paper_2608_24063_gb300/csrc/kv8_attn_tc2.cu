// Attention over the 8-bit paged cache, long chunks of bf16 query rows
// (viscache_kv8_attention on tcgen05): 256 rows a unit.
//
// Where there is work for every SM, two row tiles share a tile's expansion and each
// other's waits: a chunk of 2048 rows over 32768 tokens (64 query heads, 8 KV heads
// of 128) takes 1479 us, 1.44 PFLOP/s, against 2039 us with one row tile; 512 packed rows
// tie.  Bound by a row tile's chain (scores, softmax, products) and the tensor cores
// about equally: before the pages' exponents, which cost 3%, it would have taken 1255 us
// without exponentials, maxima and expansion; the products alone take 1111.
//
// A unit has 256 packed query rows (two tiles of 128 rows, one TMEM lane a row)
// over tiles of 128 tokens: 4 * 256 * 128 * d flops a tile, so it is bound by
// the tensor cores once the softmax and the expansion of the codes run beside
// them.  Persistent blocks, one per SM, share out the line of key tiles
// (kv8_sched.cuh).
//
// S = Q K^T runs on the codes as they are (kind::f8f6f4): a query value is the
// sum of its rounding to e4m3 and the rest in e5m2 (split8, kv8_tc.cuh), exact
// down to 2^-13 of its row's largest, which lies in [128, 256), and within 2^-21 of
// it below.  Two products at twice the rate cost what one fp16 product does, and K
// needs no expansion: TMA writes its tiles.
// O = P V runs in fp16: P needs more than e4m3's range, so V is expanded,
// once for both row tiles.
//
// Warps (512 threads, register shares set per warpgroup):
//   0-3, 4-7  softmax of row tile A, B: one thread a row
//   8-11      converters: V codes from the staging buffer, e4m3 -> fp16, into
//             128-byte-swizzled tiles, two stages; the unit's query rows too
//   12        MMA issuer
//   13        loader: page numbers, scales, a TMA box per page of K, a bulk
//             copy per page of V
// Tensor memory: S_A, S_B (128 columns each; P over the first 64 as fp16
// pairs), O_A, O_B (d columns each).  Order of issue per tile t:
//   PV_A(t) S_A(t+1) PV_B(t) S_B(t+1)
// so one row tile's softmax works while the other's products run.  P arrives in
// two halves, and the first half's products run while the second's exponentials
// do (5% of a long chunk; four parts or a first quarter lost 3%).  MMAs of one
// thread execute in order, so S_A(t+1) may overwrite the P_A(t) that PV_A(t)
// reads, and s_full of tile t + 1 says that PV(t) is done too.
//
// Numbers: query rows are scaled by a power of two to a largest magnitude in
// [128, 256).  Scores are scaled by their page's K scale in fp32.  V codes are fp16
// numbers as they are; a page's V scale enters with P (RowRefs, kv8_tc.cuh), so that
// a row depends on no page that it does not see: P = 2^(x + log2 V scale - reference
// + 5).  A reference may be passed by 2^10 before O is rescaled, so P is at most 2^15
// and its largest above 2^4: it keeps 11 bits down to 2^-18 of the largest.  Row sums
// are fp32, of unrounded terms.
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

constexpr int kTcThreads = 512;
constexpr int kTcMT = 256, kTcKT = 128;
constexpr int kConvWarp0 = 8, kConvWarps = 4, kIssueWarp = 12, kLoadWarp = 13;
constexpr float kTcSlack = 10.f;                // log2 units
constexpr int kTcPExp = 5;
constexpr uint32_t kSCol = 0, kOCol = 256;
constexpr int kKStages = 3, kVStages = 2, kCodeStages = 2;
constexpr int kRefs = 8;                        // tiles whose scales are kept (the loader is at most 4 ahead)

template <int D>
struct TcSmem {
  uint8_t v[kVStages][D / 64][kBlk];            // V as fp16, [stage][64-column block]
  uint8_t q[2][2][128 * D];                     // query rows of the unit, [row tile][rounding, rest]
  uint8_t k[kKStages][kTcKT * D];               // K codes
  uint8_t code[kCodeStages][kTcKT * D];         // V codes as they are in the cache
  float qs[kTcMT];                              // power of two of each query row
  float kscale[kRefs][8];                       // K scale of each 16-token group of tile t, at t % kRefs
  float vlog[kRefs][8];                         // log2 of its V scale
  uint64_t q_full, q_empty, k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
  uint64_t code_full[kCodeStages], code_empty[kCodeStages], ref_full[kRefs];
  uint64_t s_full[2], p_full[2], p_half[2], o_full[2], done;
  int64_t scan[kTcThreads / 32];
  Share share;
  uint32_t tmem_base;
  int abort, last[2];
  int nan_token[2][2][4];                       // first token whose V has a NaN in a mixed tile: [row tile][its segment & 1][warp]
  int32_t err;                                  // the block's status
};

template <int D>
__global__ void __launch_bounds__(kTcThreads, 1) kv8_attn_tc2_kernel(const __grid_constant__ CUtensorMap tmK,
                                                                    const __grid_constant__ vc_kv8 c,
                                                                    const __grid_constant__ vc_kv8_step s,
                                                                    const __grid_constant__ Kv8AttnArgs a) {
  extern __shared__ uint8_t smem_raw[];
  TcSmem<D>& sm = *reinterpret_cast<TcSmem<D>*>(align1024(smem_raw));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // (warp: uniform)
  const int G = a.Hq / c.Hkv;
  const Line<kTcMT, kTcKT> line{c.Hkv, G, c.page, a.causal};
  if (threadIdx.x == 0) {
    mbar_init(&sm.q_full, kConvWarps);
    mbar_init(&sm.q_empty, 1);
    for (int i = 0; i < kKStages; ++i) {
      mbar_init(&sm.k_full[i], 1);
      mbar_init(&sm.k_empty[i], 1);
    }
    for (int i = 0; i < kVStages; ++i) {
      mbar_init(&sm.v_full[i], kConvWarps);
      mbar_init(&sm.v_empty[i], 1);
    }
    for (int i = 0; i < kCodeStages; ++i) {
      mbar_init(&sm.code_full[i], 1);
      mbar_init(&sm.code_empty[i], kConvWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.p_half[i], 4);
      mbar_init(&sm.p_full[i], 4);
      mbar_init(&sm.o_full[i], 1);
    }
    for (int i = 0; i < kRefs; ++i) mbar_init(&sm.ref_full[i], 1);
    mbar_init(&sm.done, 1);
    for (int i = 0; i < 16; ++i) sm.nan_token[i >> 3][i >> 2 & 1][i & 3] = kNoNan;
    sm.abort = 0;
    sm.err = VC_OK;
    fence_mbar_init();
  }
  __syncthreads();
  int32_t* const err = &sm.err;
  find_share<kTcThreads>(line, s, err, sm.share, sm.scan);        // ends with a barrier
  const Share& sh = sm.share;
  if (sh.begin >= sh.end) {
    if (threadIdx.x == 0) store_status(a, sm.err);
    return;
  }
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
    if (warp == kIssueWarp) {
      // ---- MMA issuer
      constexpr uint32_t id_s = idesc_e4m3(128, kTcKT), id_rest = idesc_e5m2_e4m3(128, kTcKT);
      constexpr uint32_t id_o = idesc_f16_bmn(128, D);
      bool ok = true;
      int np[2] = {0, 0};                       // P tiles consumed per row tile
      const uint64_t qd = desc_codes<D>(smem_u32(sm.q)), kd = desc_codes<D>(smem_u32(sm.k));
      const uint64_t vd = desc_sw128_mn(smem_u32(sm.v), kBlk);
      // descriptors hold addresses in units of 16 bytes
      constexpr uint32_t kV16 = sizeof(sm.v[0]) / 16, kK16 = sizeof(sm.k[0]) / 16;
      constexpr uint32_t kQ16 = sizeof(sm.q[0]) / 16, kQPart16 = sizeof(sm.q[0][0]) / 16;
      auto issue_s = [&](int x, int st) {
        const uint64_t ad = qd + (uint32_t)x * kQ16, bd = kd + (uint32_t)st * kK16;
        __syncwarp();
#pragma unroll
        for (int kk = 0; kk < 2 * (D / 32); ++kk)             // 32 columns: 2 x 16 bytes
          mma_f8_ss(tbase + kSCol + x * kTcKT, ad + (kk & 1) * kQPart16 + (kk >> 1) * 2, bd + (kk >> 1) * 2,
                    kk & 1 ? id_rest : id_s, kk ? 1u : 0u);
        mma_commit_elected(&sm.s_full[x]);
      };
      // P comes in two halves
      auto issue_pv = [&](int x, int st, bool first) -> bool {
        const uint64_t bd = vd + (uint32_t)st * kV16;
        if (!warp_wait(&sm.p_half[x], np[x] & 1, abort)) return false;
        tc_fence_after();
        __syncwarp();
#pragma unroll
        for (int kk = 0; kk < kTcKT / 32; ++kk)
          mma_f16_ts(tbase + kOCol + x * D, tbase + kSCol + x * kTcKT + kk * 8, bd + kk * 2048 / 16, id_o,
                     (!first || kk) ? 1u : 0u);
        if (!warp_wait(&sm.p_full[x], np[x] & 1, abort)) return false;
        ++np[x];
        tc_fence_after();
        __syncwarp();
#pragma unroll
        for (int kk = kTcKT / 32; kk < kTcKT / 16; ++kk)
          mma_f16_ts(tbase + kOCol + x * D, tbase + kSCol + x * kTcKT + kk * 8, bd + kk * 2048 / 16, id_o,
                     (!first || kk) ? 1u : 0u);
        return true;
      };
      do {
        const bool two = rows_of() > 128;
        int ks = t % kKStages;
        ok = warp_wait(&sm.q_full, seg & 1, abort) && warp_wait(&sm.k_full[ks], (t / kKStages) & 1, abort);
        if (!ok) break;
        tc_fence_after();
        issue_s(0, ks);
        if (two) issue_s(1, ks);
        mma_commit_elected(&sm.k_empty[ks]);
        for (int j = w.t0; ok && j < w.t1; ++j, ++t) {
          const int st = t % kVStages;
          const bool more = j + 1 < w.t1;
          ks = (t + 1) % kKStages;
          if (!warp_wait(&sm.v_full[st], (t / kVStages) & 1, abort) || !issue_pv(0, st, j == w.t0)) {
            ok = false;
            break;
          }
          if (!more) mma_commit_elected(&sm.o_full[0]);
          if (more) {
            if (!warp_wait(&sm.k_full[ks], ((t + 1) / kKStages) & 1, abort)) {
              ok = false;
              break;
            }
            tc_fence_after();
            issue_s(0, ks);
          }
          if (two) {
            if (!issue_pv(1, st, j == w.t0)) {
              ok = false;
              break;
            }
            if (!more) mma_commit_elected(&sm.o_full[1]);
          }
          mma_commit_elected(&sm.v_empty[st]);
          if (more) {
            if (two) issue_s(1, ks);
            mma_commit_elected(&sm.k_empty[ks]);
          }
        }
        if (ok) mma_commit_elected(&sm.q_empty);
        ++seg;
      } while (ok && w.next(line, s, err));
      // every MMA is done before the block frees its tensor memory
      __syncwarp();
      mma_commit_elected(&sm.done);
      drain_wait(&sm.done, 0);
    }
    if (warp == kLoadWarp) {
      // ---- loader: lane -> (tile, page) of a batch of 32 pages; page numbers and
      // scales of the next batch load while this one's copies are issued
      const int ppt = kTcKT / c.page, tpb = 32 / ppt;
      const int bt = lane / ppt, bp = lane % ppt;
      const uint32_t page_bytes = (uint32_t)c.page * D;
      bool ok = true;
      int nk = 0;                               // K tiles under way or landed (t counts V tiles)
      prefetch_tmap(&tmK);
      do {
        auto look = [&](int first, int& pid, float& ks, float& vs, bool& live) {
          const int tile = first + bt, j = tile * ppt + bp;
          live = tile < w.t1 && j * c.page < w.u.kend;
          pid = live ? load_page(s, c.n_pages, w.u.r, j, err) : -1;
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
          const float vlog = scale_log2(vs);
          const int nt = min(tpb, w.t1 - tb);
          // (a page that does not exist has scale 0: page 0 stands in)
          const int row = (max(pid, 0) * c.Hkv + w.u.g) * c.page;
          for (int i = 0; i < nt; ++i, ++t) {
            const bool mine = bt == i;
            const int rt = t % kRefs, kst = t % kKStages, cst = t % kCodeStages;
            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine && live)) * page_bytes;
            ok = warp_wait(&sm.k_empty[kst], ((t / kKStages) & 1) ^ 1, abort);
            if (!ok) break;
            if (mine) {
              for (int e = 0; e < c.page / 16; ++e) {
                sm.kscale[rt][bp * (c.page / 16) + e] = ks;
                sm.vlog[rt][bp * (c.page / 16) + e] = vlog;
              }
            }
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(&sm.ref_full[rt]);
              mbar_arrive_expect_tx(&sm.k_full[kst], bytes);
            }
            ++nk;
            __syncwarp();
            if (mine && live) tma_load_2d(sm.k[kst] + bp * page_bytes, &tmK, 0, row, &sm.k_full[kst]);
            ok = warp_wait(&sm.code_empty[cst], ((t / kCodeStages) & 1) ^ 1, abort);
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(&sm.code_full[cst], bytes);
            __syncwarp();
            if (mine && live)
              bulk_load(sm.code[cst] + bp * page_bytes, static_cast<const uint8_t*>(c.V_codes) + (int64_t)row * D,
                        page_bytes, &sm.code_full[cst]);
          }
          pid = npid;
          ks = nks;
          vs = nvs;
          live = nlive;
        }
      } while (ok && w.next(line, s, err));
      // every copy has landed before the block may end
      __syncwarp();
      if (lane == 0) {
        for (int i = max(0, nk - kKStages); i < nk; ++i) drain_wait(&sm.k_full[i % kKStages], (i / kKStages) & 1);
        for (int i = max(0, t - kCodeStages); i < t; ++i)
          drain_wait(&sm.code_full[i % kCodeStages], (i / kCodeStages) & 1);
      }
    }
  } else if (warp >= kConvWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    // ---- converters
    const int i = threadIdx.x - 32 * kConvWarp0;
    bool ok = true;
    int seg1 = 0;                               // segments in which row tile B had rows
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
          // largest magnitude to [128, 256), by 2^126 at most; rows that are not finite as they are
          const uint32_t ex = __float_as_uint(amax) & 0x7f800000u;
          const float qs = ex == 0x7f800000u ? 1.f : __uint_as_float(max(ex, 8u << 23) - (7u << 23));
          const float inv = pow2_inverse(qs);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] *= inv;
          uint2 top, rest;
          split8(x, top, rest);
          const uint32_t off = code_piece<D>(r & 127, qc);
          *reinterpret_cast<uint2*>(sm.q[r >> 7][0] + off) = top;
          *reinterpret_cast<uint2*>(sm.q[r >> 7][1] + off) = rest;
          if (qc == 0) sm.qs[r] = qs;
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full);
      // keys that every row of the unit sees; whether row tile B has rows
      const int lim_min = a.causal ? w.u.q.len - w.u.q.m + 1 + w.u.rt * kTcMT / G : w.u.kend;
      const bool two = rows_of() > 128;
      for (int j = w.t0; j < w.t1; ++j, ++t) {
        const int st = t % kVStages, cst = t % kCodeStages;
        const int left = w.u.kend - j * kTcKT;  // tokens of the tile
        // the codes have landed, the stage is free
        ok = warp_wait(&sm.code_full[cst], (t / kCodeStages) & 1, abort) &&
             warp_wait(&sm.v_empty[st], ((t / kVStages) & 1) ^ 1, abort);
        if (!ok) break;
        constexpr int LPR = D / 16, RP = 128 / LPR;     // lanes of a row (16 codes each), rows at once
        const int key0 = i / LPR, ch = i % LPR;
        const bool mixed = (j + 1) * kTcKT > lim_min;           // some rows do not see all of it
        if (mixed) {                            // (a pass of its own: 4% of a long chunk within the loop below)
#pragma unroll 1
          for (int key = key0; key < min(left, 128); key += RP) {
            uint4* at = reinterpret_cast<uint4*>(sm.code[cst] + key * D + ch * 16);
            uint4 y = *at;
            if (drop_nan(y)) {
              *at = y;
              for (int k = 0; k < 4; ++k) {
                atomicMin(&sm.nan_token[0][seg & 1][k], j * kTcKT + key);
                if (two) atomicMin(&sm.nan_token[1][seg1 & 1][k], j * kTcKT + key);
              }
            }
          }
        }
#pragma unroll
        for (int n = 0; n < 128 / RP; ++n) {
          const int key = key0 + RP * n;
          uint4 y = *reinterpret_cast<const uint4*>(sm.code[cst] + key * D + ch * 16);
          if (key >= left) y = make_uint4(0u, 0u, 0u, 0u);      // not a token: whatever was there
          expand16(sm.v[st][0], key, ch, y);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sm.code_empty[cst]);
          mbar_arrive(&sm.v_full[st]);
        }
      }
      ++seg;
      seg1 += two;
    } while (ok && w.next(line, s, err));
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
        ++seg;
        continue;
      }
      const int rho = w.u.rt * kTcMT + X * 128 + row;
      const bool real = rho < w.u.q.m * G;
      const int qi = rho / G, qj = rho - qi * G;
      int lim = w.u.kend;
      if (a.causal) lim = min(lim, w.u.q.len - w.u.q.m + 1 + qi);
      RowRefs ref;
      ref.clear();
      float cs = 0.f;
      for (int j = w.t0; j < w.t1; ++j, ++t) {
        // S first: then the scales' (and the query rows') barriers are at the phase
        // asked for, also where this row tile sat out the segments before
        ok = ok && warp_wait(&sm.s_full[X], ns & 1, abort) &&
             warp_wait(&sm.ref_full[t % kRefs], (t / kRefs) & 1, abort) &&
             (j > w.t0 || warp_wait(&sm.q_full, seg & 1, abort));
        if (!ok) continue;
        ++ns;
        tc_fence_after();
        if (j == w.t0) cs = a.scale_log2 * sm.qs[X * 128 + row];
        // factor of each 16 scores (above 0, so that a masked one stays -inf)
        float f[8];
        {
          const float4 k0 = *reinterpret_cast<const float4*>(&sm.kscale[t % kRefs][0]);
          const float4 k1 = *reinterpret_cast<const float4*>(&sm.kscale[t % kRefs][4]);
          f[0] = k0.x; f[1] = k0.y; f[2] = k0.z; f[3] = k0.w;
          f[4] = k1.x; f[5] = k1.y; f[6] = k1.z; f[7] = k1.w;
#pragma unroll
          for (int p = 0; p < 8; ++p) f[p] = fmaxf(cs * f[p], 1e-37f);
        }
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
        float b[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) {
          b[p] = fmaxf(x[p][0], x[p][1]);
#pragma unroll
          for (int q = 2; q < 16; q += 2) b[p] = fmax3(b[p], x[p][q], x[p][q + 1]);
          b[p] *= f[p];
        }
        const float* vlog = sm.vlog[t % kRefs];
        float g;
        const bool moved = ref.raise(b, vlog, kTcSlack, g);
        if (j > w.t0 && __any_sync(0xffffffffu, moved)) {
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
        __syncwarp();                           // (whole warps store P)
        const float mr = ref.base(), lift = kTcPExp - ref.value_base();
        float ev[8];                            // exponent of each 16-token group's page in P
        {
          const float4 v0 = *reinterpret_cast<const float4*>(vlog), v1 = *reinterpret_cast<const float4*>(vlog + 4);
          ev[0] = v0.x; ev[1] = v0.y; ev[2] = v0.z; ev[3] = v0.w; ev[4] = v1.x; ev[5] = v1.y; ev[6] = v1.z; ev[7] = v1.w;
#pragma unroll
          for (int p = 0; p < 8; ++p) ev[p] = fmaxf(ev[p] + lift, kLeastShare);
        }
        float2 ls = make_float2(0.f, 0.f);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t y16[16];
#pragma unroll
          for (int gr = 0; gr < 2; ++gr) {      // 16 tokens: one page's
            const int p = 2 * h + gr;
            const float e = ev[p], back = ex2(-e);      // (what P's sum takes for the row's)
            const float2 nm = make_float2(e - mr, e - mr);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float2 y = __ffma2_rn(make_float2(x[p][2 * q], x[p][2 * q + 1]), make_float2(f[p], f[p]), nm);
              const float2 ex = make_float2(ex2(y.x), ex2(y.y));
              sum = q ? __fadd2_rn(sum, ex) : ex;
              y16[8 * gr + q] = half2_bits(ex.x, ex.y);
            }
            ls = __ffma2_rn(sum, make_float2(back, back), ls);
          }
          tmem_st16(s_col + h * 16, y16);
          if (h == 1) {                         // the first half may be multiplied
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.p_half[X]);
          }
        }
        ref.l += ls.x + ls.y;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[X]);
      }
      ok = ok && warp_wait(&sm.o_full[X], no & 1, abort);
      ++no;
      ++seg;
      if (named_sync_any(1 + X, 128, !ok)) break;
      tc_fence_after();
      // O in units of 2^(r - kTcPExp)
      const float2 ou = pow2_factors((int)ref.value_base() - kTcPExp);
      const bool whole = w.whole();
      const int64_t at = (int64_t)(w.u.q.row0 + qi) * a.Hq + w.u.g * G + qj;
      auto put_out = [&](int64_t at, int col, const float (&y)[16], float inv) {
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
      auto put_lse = [&](int64_t at, float M, float L) {
        if (a.lse) a.lse[at] = L == 0.f ? -INFINITY : fmaf(M, 0.6931471805599453f, logf(L));
      };
      const int64_t mine = 2 * (int64_t)blockIdx.x + (w.t0 == 0 ? 1 : 0);
      int& nan_token = sm.nan_token[X][(no - 1) & 1][warp & 3];
      const int nan_from = nan_token, nan_to = min(lim, w.t1 * kTcKT);
      __syncwarp();
      if (lane == 0) nan_token = kNoNan;
      const float inv = whole ? inverse_of(ref.l) : 1.f;
#pragma unroll 1
      for (int p = 0; p < D / 16; ++p) {
        uint32_t v[16];
        __syncwarp();                           // (whole warps read tensor memory)
        tmem_ld16(o_col + p * 16, v);
        tmem_wait(v);
        float y[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) y[q] = __uint_as_float(v[q]) * ou.x * inv * ou.y;
        if (nan_from < nan_to && real) {
          const uint32_t bad = nan_dims<16>(c, s, w.u.r, w.u.g, nan_from, nan_to, p * 16);
#pragma unroll
          for (int q = 0; q < 16; ++q)
            if (bad >> q & 1u) y[q] = __uint_as_float(0x7fffffffu);
        }
        if (whole) {
          if (real) put_out(at, p * 16, y, 1.f);
        } else {
          // (four columns of the row tile's rows side by side)
          float4* po = reinterpret_cast<float4*>(a.part_o + (mine * 2 + X) * 128 * D) + p * 4 * 128 + row;
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (real) po[q * 128] = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
        }
      }
      tc_fence_before();
      if (whole) {
        if (real) put_lse(at, ref.m, ref.l);
      } else {
        if (real) a.part_ml[(mine * 2 + X) * 128 + row] = make_float2(ref.m, ref.l);
        const int first = w.first_block(sh), final = w.last_block(sh);
        __syncwarp();                           // (the named barriers take whole warps)
        named_sync(1 + X, 128);
        if ((warp & 3) == 0) {
          const bool all = piece_done(a.flags + X, 2, a.token, first, final);
          if (lane == 0) sm.last[X] = all;
          __syncwarp();
        }
        named_sync(1 + X, 128);
        if (sm.last[X]) {
          const int rows = min(128, w.u.q.m * G - w.u.rt * kTcMT - X * 128);
          join_pieces<D>(a, first, final, 2, X, rows, [&](int jr, int col, const float (&y)[16], float M, float L) {
            const int jrho = w.u.rt * kTcMT + X * 128 + jr, ji = jrho / G;
            const int64_t jat = (int64_t)(w.u.q.row0 + ji) * a.Hq + w.u.g * G + (jrho - ji * G);
            put_out(jat, col, y, inverse_of(L));
            if (col == 0) put_lse(jat, M, L);
          });
        }
      }
    } while (w.next(line, s, err));
    if (!ok && lane == 0) set_status(err, VC_ERR_DEVICE_TIMEOUT);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    tc_fence_after();
    tmem_dealloc(tbase, 512);
  }
  if (threadIdx.x == 0) store_status(a, sm.abort ? VC_ERR_DEVICE_TIMEOUT : sm.err);
}

template <int D>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  constexpr size_t smem = sizeof(TcSmem<D>) + 1024;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = kv8_allow_smem(reinterpret_cast<const void*>(kv8_attn_tc2_kernel<D>), smem, allowed);
  if (e != cudaSuccess) return e;
  CUtensorMap mk;
  if (!kv8_pool_map(&mk, c.K_codes, c)) return cudaErrorInvalidValue;
  const int64_t G = a.Hq / c.Hkv;
  const int64_t units = ((int64_t)s.n_rows * G / kTcMT + (s.n_req < s.n_rows ? s.n_req : s.n_rows)) * c.Hkv;
  const int64_t tiles = units * (((int64_t)s.max_pages * c.page + kTcKT - 1) / kTcKT);
  const int64_t sms = kv8_sm_count();
  ProfileScope ps("kv8_attn_tc2", st);
  kv8_attn_tc2_kernel<D><<<(unsigned)(tiles < sms ? tiles : sms), kTcThreads, smem, st>>>(mk, c, s, a);
  return cudaGetLastError();
}

}  // namespace

int kv8_attn_rows_tc2() { return kTcMT; }

cudaError_t launch_kv8_attn_tc2(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  return c.d == 128 ? launch_t<128>(c, s, a, st) : launch_t<64>(c, s, a, st);
}

}  // namespace vc
