// Attention over the 8-bit paged cache, many query rows a request
// (viscache_kv8_attention on tcgen05): 128 rows a unit, bf16 or fp32.
//
// A unit has 128 packed query rows (one TMEM lane a row) over tiles of 128 tokens.
// A tile's scores come from one of two S buffers, so its softmax runs while the
// next tile's products do.  Persistent blocks, one per SM, share out the line of
// key tiles (kv8_sched.cuh).
//
// bf16 rows.  S = Q K^T runs on the codes as they are (kind::f8f6f4): a query value is
// the sum of its rounding to e4m3 and the rest in e5m2 (split8, kv8_tc.cuh), exact down
// to 2^-13 of its row's largest, which lies in [128, 256), and within 2^-21 of it below.
// Two products at twice the rate cost what one fp16 product does, and K needs no
// expansion: TMA writes its tiles.  O = P V runs in fp16: P needs more than e4m3's
// range, so V is expanded.
// fp32 rows.  Rows and probabilities are sums of two fp16 numbers (22 bits), and K
// and V are both expanded to fp16 (exact), K a tile ahead of V.
//
// Warps (512 threads, register shares set per warpgroup):
//   0-3    softmax, one thread a row
//   4-11   converters: codes from the staging ring, e4m3 -> fp16, into
//          128-byte-swizzled tiles; the unit's query rows too
//   12     MMA issuer
//   13     loader: page numbers, scales, a TMA box (K, bf16 rows) or a bulk copy
//          per page
// Tensor memory: S_0, S_1 (128 columns each; P over them: fp16 pairs in the first
// 64 columns, of fp32 calls the rest of each in the others), O, and in fp32 calls
// the sum of earlier O.  Order of issue:
//   S(0) S(1) PV(0) S(2) PV(1) ...
// MMAs of one thread execute in order, so S(t+2) may overwrite the P(t) that PV(t)
// reads.  P arrives in two halves: the first half's products run while the second's
// exponentials do.
//
// Numbers: query rows are scaled by a power of two to a largest magnitude in
// [128, 256), of fp32 calls in [2^14, 2^15) (their parts keep 2^-39 of it).  Scores
// are scaled by their page's K scale in fp32.  V codes are fp16 numbers as they are;
// a page's V scale enters with P (RowRefs, kv8_tc.cuh), so that a row depends on no
// page that it does not see: P = 2^(x + log2 V scale - reference + 5) (fp32: + 13).
// A reference may be passed by 2^10 (fp32: 2^2) before O is rescaled, so P is at most
// 2^15 and its largest above 2^4 (2^12): it keeps 11 bits down to 2^-18 of the largest
// (fp32: 22 bits down to 2^-15, and 2^-37 of it below).  Row sums are fp32, of unrounded
// terms.  The tensor cores' fp32 sums
// cut off, so in fp32 calls the smaller parts are added first and O goes into a
// sum beside it every four tiles: the error over 29000 tokens falls from 2.5e-5
// of the output to 1.3e-6 and the time rises by a tenth, with the exponentials'
// factor taken out of their exponents (3e-7 of each) included.
//
// Bound by the softmax's chain: one tile takes about 2200 clocks (its products
// 1024).  64 requests of 128 rows over 4096 tokens, 8 KV heads of 128: 192 us, 2.8
// TB/s of codes; fp32 rows 381 us.  Long chunks: kv8_attn_tc2.cu.
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
constexpr int kTcMT = 128, kTcKT = 128;
constexpr int kConvWarp0 = 4, kConvWarps = 8, kIssueWarp = 12, kLoadWarp = 13;
constexpr uint32_t kSCol = 0, kOCol = 256, kSumCol = 384;
constexpr int kRefs = 8;                        // tiles whose scales are kept (the loader is at most 5 ahead)

template <typename T, int D>
struct Cfg {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr float SLACK = F32 ? 2.f : 10.f;          // log2 units
  static constexpr int PEXP = F32 ? 13 : 5;
  // Tiles whose products O takes before it is added to the sum beside it (fp32: the
  // tensor core's sums lose about 2^-26 of O a step, a context of 29000 tokens 2.5e-5).
  static constexpr int FOLD = F32 ? 4 : 1 << 30;
  static __device__ __forceinline__ bool fresh(int i) { return i % FOLD == 0; }     // tile i begins O anew
  static constexpr int QPART = F32 ? kTcMT * D * 2 : kTcMT * D, KTILE = F32 ? kTcKT * D * 2 : kTcKT * D;
  static constexpr int KS = F32 ? 2 : 3, VS = F32 ? 1 : 2, CS = F32 ? 4 : 3;
};

template <typename T, int D>
struct Tc1Smem {
  using C = Cfg<T, D>;
  uint8_t q[2][C::QPART];                       // query rows of the unit, [larger part, rest]: fp16, or e4m3 and e5m2
  uint8_t k[C::KS][C::KTILE];                   // K as fp16, or its codes
  uint8_t v[C::VS][D / 64][kBlk];               // V as fp16, [stage][64-column block]
  uint8_t code[C::CS][kTcKT * D];               // codes as they are in the cache: K, K, V, K, V, ..., or V
  float qs[kTcMT];                              // power of two of each query row
  float kscale[kRefs][8];                       // K scale of each 16-token group of tile t, at t % kRefs
  float vlog[kRefs][8];                         // log2 of its V scale
  uint64_t q_full, q_empty, k_full[C::KS], k_empty[C::KS], v_full[C::VS], v_empty[C::VS], pv_done;
  uint64_t code_full[C::CS], code_empty[C::CS], ref_full[kRefs];
  uint64_t s_full[2], p_half[2], p_full, done;
  int64_t scan[kTcThreads / 32];
  Share share;
  uint32_t tmem_base;
  int abort, last;
  int nan_token[2][4];                          // first token whose V has a NaN in a mixed tile: [segment & 1][warp]
  int32_t err;                                  // the block's status
};

// Eight values of a query row.
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 x0 = __ldg(reinterpret_cast<const float4*>(p)), x1 = __ldg(reinterpret_cast<const float4*>(p) + 1);
  x[0] = x0.x; x[1] = x0.y; x[2] = x0.z; x[3] = x0.w;
  x[4] = x1.x; x[5] = x1.y; x[6] = x1.z; x[7] = x1.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 y = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t b[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(b[e] << 16);
    x[2 * e + 1] = __uint_as_float(b[e] & 0xffff0000u);
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kTcThreads, 1) kv8_attn_tc1_kernel(const __grid_constant__ CUtensorMap tmK,
                                                                      const __grid_constant__ vc_kv8 c,
                                                                      const __grid_constant__ vc_kv8_step s,
                                                                      const __grid_constant__ Kv8AttnArgs a) {
  using C = Cfg<T, D>;
  constexpr bool F32 = C::F32;
  constexpr int kKStages = C::KS, kVStages = C::VS, kCodeStages = C::CS;
  constexpr float kTcSlack = C::SLACK;
  constexpr int kTcPExp = C::PEXP;
  extern __shared__ uint8_t smem_raw[];
  Tc1Smem<T, D>& sm = *reinterpret_cast<Tc1Smem<T, D>*>(align1024(smem_raw));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // (warp: uniform)
  const int G = a.Hq / c.Hkv;
  const Line<kTcMT, kTcKT> line{c.Hkv, G, c.page, a.causal};
  if (threadIdx.x == 0) {
    mbar_init(&sm.q_full, kConvWarps);
    mbar_init(&sm.q_empty, 1);
    for (int i = 0; i < kKStages; ++i) {
      mbar_init(&sm.k_full[i], F32 ? kConvWarps : 1);
      mbar_init(&sm.k_empty[i], 1);
    }
    for (int i = 0; i < kVStages; ++i) {
      mbar_init(&sm.v_full[i], kConvWarps);
      mbar_init(&sm.v_empty[i], 1);
    }
    mbar_init(&sm.pv_done, 1);
    for (int i = 0; i < kCodeStages; ++i) {
      mbar_init(&sm.code_full[i], 1);
      mbar_init(&sm.code_empty[i], kConvWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.p_half[i], 4);              // (sent before the tile before's is looked for)
    }
    mbar_init(&sm.p_full, 4);
    for (int i = 0; i < kRefs; ++i) mbar_init(&sm.ref_full[i], 1);
    mbar_init(&sm.done, 1);
    for (int i = 0; i < 8; ++i) sm.nan_token[i >> 2][i & 3] = kNoNan;
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

  if (warp >= kConvWarp0 + kConvWarps) {
    // registers a thread: 128 at launch; 216 + 104 + 104 + 88 = 4 * 128
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kIssueWarp) {
      // ---- MMA issuer
      constexpr uint32_t id_s = F32 ? idesc_f16(128, kTcKT) : idesc_e4m3(128, kTcKT), id_o = idesc_f16_bmn(128, D);
      constexpr uint32_t id_rest = idesc_e5m2_e4m3(128, kTcKT);
      bool ok = true;
      const uint64_t qd = F32 ? desc_sw128(smem_u32(sm.q)) : desc_codes<D>(smem_u32(sm.q));
      const uint64_t kd = F32 ? desc_sw128(smem_u32(sm.k)) : desc_codes<D>(smem_u32(sm.k));
      const uint64_t vd = desc_sw128_mn(smem_u32(sm.v), kBlk);
      // descriptors hold addresses in units of 16 bytes
      constexpr uint32_t kV16 = sizeof(sm.v[0]) / 16, kK16 = C::KTILE / 16, kQ16 = C::QPART / 16, kBlk16 = kBlk / 16;
      auto issue_pv = [&](uint32_t s_col, uint64_t bd, int kk0, bool first) {
        tc_fence_after();
        __syncwarp();
#pragma unroll
        for (int k = 0; k < kTcKT / 32; ++k) {
          const int kk = kk0 + k;
          if (F32) mma_f16_ts(tbase + kOCol, s_col + 64 + kk * 8, bd + kk * 2048 / 16, id_o, (!first || k) ? 1u : 0u);
          mma_f16_ts(tbase + kOCol, s_col + kk * 8, bd + kk * 2048 / 16, id_o, (F32 || !first || k) ? 1u : 0u);
        }
      };
      do {
        ok = warp_wait(&sm.q_full, seg & 1, abort);
        for (int j = w.t0; ok && j <= w.t1; ++j) {
          if (j < w.t1) {
            const int tk = t + j - w.t0, ks = tk % kKStages;
            ok = warp_wait(&sm.k_full[ks], (tk / kKStages) & 1, abort);
            if (!ok) break;
            tc_fence_after();
            __syncwarp();
            const uint32_t d = tbase + kSCol + (tk & 1) * kTcKT;
            const uint64_t bd = kd + (uint32_t)ks * kK16;
            if constexpr (F32) {
#pragma unroll
              for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                  const uint32_t at = (kk >> 2) * kBlk16 + (kk & 3) * 2;
                  // (the rest first: the sum is large only while the larger parts are added)
                  mma_f16_ss(d, qd + (1 - part) * kQ16 + at, bd + at, id_s, (part || kk) ? 1u : 0u);
                }
            } else {
#pragma unroll
              for (int kk = 0; kk < 2 * (D / 32); ++kk)
                mma_f8_ss(d, qd + (kk & 1) * kQ16 + (kk >> 1) * 2, bd + (kk >> 1) * 2, kk & 1 ? id_rest : id_s,
                          kk ? 1u : 0u);
            }
            mma_commit_elected(&sm.s_full[tk & 1]);
            mma_commit_elected(&sm.k_empty[ks]);
          }
          if (j > w.t0) {
            const int tv = t + j - 1 - w.t0;
            const uint32_t s_col = tbase + kSCol + (tv & 1) * kTcKT;
            const int vs = tv % kVStages;
            const uint64_t bd = vd + (uint32_t)vs * kV16;
            ok = warp_wait(&sm.v_full[vs], (tv / kVStages) & 1, abort) && warp_wait(&sm.p_half[tv & 1], (tv >> 1) & 1, abort);
            if (!ok) break;
            issue_pv(s_col, bd, 0, C::fresh(j - 1 - w.t0));
            ok = warp_wait(&sm.p_full, tv & 1, abort);
            if (!ok) break;
            issue_pv(s_col, bd, kTcKT / 32, false);
            mma_commit_elected(&sm.pv_done);
            mma_commit_elected(&sm.v_empty[vs]);
          }
        }
        // (after the last PV: the softmax has read the rows' powers of two)
        if (ok) mma_commit_elected(&sm.q_empty);
        t += w.t1 - w.t0;
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
      int item = 0, nk = 0;                     // code tiles (and K tiles) under way or landed
      if (!F32) prefetch_tmap(&tmK);
      // the code tile of the pages that the lanes with `mine` hold
      auto put = [&](const void* codes, bool mine, int pid) {
        const int st = item % kCodeStages;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, mine)) * page_bytes;
        ok = warp_wait(&sm.code_empty[st], ((item / kCodeStages) & 1) ^ 1, abort);
        if (!ok) return;
        if (lane == 0) mbar_arrive_expect_tx(&sm.code_full[st], bytes);
        __syncwarp();
        // (a page that does not exist has scale 0: page 0 stands in)
        if (mine)
          bulk_load(sm.code[st] + bp * page_bytes,
                    static_cast<const uint8_t*>(codes) + ((int64_t)max(pid, 0) * c.Hkv + w.u.g) * page_bytes,
                    page_bytes, &sm.code_full[st]);
        ++item;
      };
      do {
        auto look = [&](int first, int& pid, float& ks, float& vs, bool& live) {
          const int tile = first + bt, j = tile * ppt + bp;
          live = tile < w.t1 && j * c.page < w.u.kend;
          pid = live ? load_page(s, c.n_pages, w.u.r, j, err) : -1;
          const int64_t at = (int64_t)max(pid, 0) * c.Hkv + w.u.g;
          ks = pid >= 0 ? __ldg(c.K_scale + at) : 0.f;
          vs = pid >= 0 ? __ldg(c.V_scale + at) : 0.f;
        };
        int pid, npid = -1, ppid = -1;          // this batch's pages, the next one's, the one's before
        float ks, vs, nks = 0.f, nvs = 0.f;
        bool live, nlive = false, plive = false;
        look(w.t0, pid, ks, vs, live);
        for (int tb = w.t0; ok && tb < w.t1; tb += tpb) {
          if (tb + tpb < w.t1) look(tb + tpb, npid, nks, nvs, nlive);
          const float vlog = scale_log2(vs);
          const int nt = min(tpb, w.t1 - tb);
          for (int i = 0; i < nt; ++i, ++t) {
            const int rt = t % kRefs;
            // (what reads this place's scales is done: the codes of the tile 2 before are expanded
            // once the PV of the one 5 before is)
            ok = F32 ? warp_wait(&sm.code_empty[item % kCodeStages], ((item / kCodeStages) & 1) ^ 1, abort)
                     : warp_wait(&sm.k_empty[t % kKStages], ((t / kKStages) & 1) ^ 1, abort);
            if (!ok) break;
            if (bt == i) {
              for (int e = 0; e < c.page / 16; ++e) {
                sm.kscale[rt][bp * (c.page / 16) + e] = ks;
                sm.vlog[rt][bp * (c.page / 16) + e] = vlog;
              }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.ref_full[rt]);
            if constexpr (F32) {
              put(c.K_codes, bt == i && live, pid);
              if (ok && tb + i > w.t0) {
                if (i > 0) put(c.V_codes, bt == i - 1 && live, pid);
                else put(c.V_codes, bt == tpb - 1 && plive, ppid);
              }
            } else {
              const int kst = t % kKStages;
              const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, bt == i && live)) * page_bytes;
              if (lane == 0) mbar_arrive_expect_tx(&sm.k_full[kst], bytes);
              ++nk;
              __syncwarp();
              if (bt == i && live)
                tma_load_2d(sm.k[kst] + bp * page_bytes, &tmK, 0, (max(pid, 0) * c.Hkv + w.u.g) * c.page,
                            &sm.k_full[kst]);
              put(c.V_codes, bt == i && live, pid);
            }
            if (!ok) break;
          }
          if (F32 && ok && tb + nt == w.t1) put(c.V_codes, bt == nt - 1 && live, pid);
          ppid = pid;
          plive = live;
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
        for (int i = max(0, item - kCodeStages); i < item; ++i)
          drain_wait(&sm.code_full[i % kCodeStages], (i / kCodeStages) & 1);
      }
    }
  } else if (warp >= kConvWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    // ---- converters
    const int i = threadIdx.x - 32 * kConvWarp0;
    bool ok = true;
    int item = 0;
    constexpr int LPR = D / 16, RP = 32 * kConvWarps / LPR;       // lanes of a row (16 codes each), rows at once
    const int key0 = i / LPR, ch = i % LPR;
    do {
      // the unit's query rows, once the segment before is done
      if (!warp_wait(&sm.q_empty, (seg & 1) ^ 1, abort)) break;
      {
        const int rows = min(kTcMT, w.u.q.m * G - w.u.rt * kTcMT);
        constexpr int QL = D / 8;               // lanes of a query row
#pragma unroll 2
        for (int r = i / QL; r < kTcMT; r += 32 * kConvWarps / QL) {
          const int qc = i % QL;
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
          if (r < rows) {
            const int rho = w.u.rt * kTcMT + r, qi = rho / G, qj = rho - qi * G;
            load8(static_cast<const T*>(a.q) + (int64_t)(w.u.q.row0 + qi) * a.q_stride +
                      (int64_t)(w.u.g * G + qj) * D + qc * 8, x);
          }
          float amax = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
#pragma unroll
          for (int o = QL / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
          // largest magnitude to [2^14, 2^15) or [2^7, 2^8), by 2^126 at most; rows that are not
          // finite as they are
          constexpr uint32_t kUp = (F32 ? 14u : 7u) << 23;
          const uint32_t ex = __float_as_uint(amax) & 0x7f800000u;
          const float qs = ex == 0x7f800000u ? 1.f : __uint_as_float(max(ex, kUp + (1u << 23)) - kUp);
          const float inv = pow2_inverse(qs);
          if constexpr (F32) {
            uint32_t top[4], rest[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float z0 = x[2 * e] * inv, z1 = x[2 * e + 1] * inv;
              top[e] = half2_bits(z0, z1);
              rest[e] = half2_rest(z0, z1, top[e]);
            }
            const uint32_t off = (uint32_t)((qc >> 3) * kBlk + r * 128 + (((qc & 7) ^ (r & 7)) << 4));
            *reinterpret_cast<uint4*>(sm.q[0] + off) = make_uint4(top[0], top[1], top[2], top[3]);
            *reinterpret_cast<uint4*>(sm.q[1] + off) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
          } else {
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = x[e] * inv;
            uint2 top, rest;
            split8(z, top, rest);
            const uint32_t off = code_piece<D>(r, qc);
            *reinterpret_cast<uint2*>(sm.q[0] + off) = top;
            *reinterpret_cast<uint2*>(sm.q[1] + off) = rest;
          }
          if (qc == 0) sm.qs[r] = qs;
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.q_full);
      // keys that every row of the unit sees
      const int lim_min = a.causal ? w.u.q.len - w.u.q.m + 1 + w.u.rt * kTcMT / G : w.u.kend;
      for (int j = w.t0; ok && j <= w.t1; ++j) {
        if (F32 && j < w.t1) {                  // K of tile j
          const int tk = t + j - w.t0, ks = tk % kKStages, st = item % kCodeStages;
          ok = warp_wait(&sm.code_full[st], (item / kCodeStages) & 1, abort) &&
               warp_wait(&sm.k_empty[ks], ((tk / kKStages) & 1) ^ 1, abort);
          if (!ok) break;
#pragma unroll
          for (int n = 0; n < 128 / RP; ++n) {
            const int key = key0 + RP * n;
            expand16(sm.k[ks], key, ch, *reinterpret_cast<const uint4*>(sm.code[st] + key * D + ch * 16));
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&sm.code_empty[st]);
            mbar_arrive(&sm.k_full[ks]);
          }
          ++item;
        }
        if (j > w.t0) {                         // V of tile j - 1
          const int tv = t + j - 1 - w.t0, vs = tv % kVStages, st = item % kCodeStages;
          const int left = w.u.kend - (j - 1) * kTcKT;            // tokens of the tile
          ok = warp_wait(&sm.code_full[st], (item / kCodeStages) & 1, abort) &&
               warp_wait(&sm.v_empty[vs], ((tv / kVStages) & 1) ^ 1, abort);
          if (!ok) break;
          const bool mixed = j * kTcKT > lim_min;               // some rows do not see all of it
          if (mixed) {                          // (a pass of its own: within the loop below it costs every tile)
#pragma unroll 1
            for (int key = key0; key < min(left, 128); key += RP) {
              uint4* at = reinterpret_cast<uint4*>(sm.code[st] + key * D + ch * 16);
              uint4 y = *at;
              if (drop_nan(y)) {
                *at = y;
                for (int k = 0; k < 4; ++k) atomicMin(&sm.nan_token[seg & 1][k], (j - 1) * kTcKT + key);
              }
            }
          }
#pragma unroll
          for (int n = 0; n < 128 / RP; ++n) {
            const int key = key0 + RP * n;
            uint4 y = *reinterpret_cast<const uint4*>(sm.code[st] + key * D + ch * 16);
            if (key >= left) y = make_uint4(0u, 0u, 0u, 0u);      // not a token: whatever was there
            expand16(sm.v[vs][0], key, ch, y);
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&sm.code_empty[st]);
            mbar_arrive(&sm.v_full[vs]);
          }
          ++item;
        }
      }
      t += w.t1 - w.t0;
      ++seg;
    } while (ok && w.next(line, s, err));
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ---- softmax, one row a thread
    const int row = threadIdx.x;
    const uint32_t lane_off = (uint32_t)(warp << 5) << 16;
    const uint32_t o_col = tbase + lane_off + kOCol, sum_col = tbase + lane_off + kSumCol;
    bool ok = true;
    do {
      const int rho = w.u.rt * kTcMT + row;
      const bool real = rho < w.u.q.m * G;
      const int qi = rho / G, qj = rho - qi * G;
      int lim = w.u.kend;
      if (a.causal) lim = min(lim, w.u.q.len - w.u.q.m + 1 + qi);
      RowRefs ref;
      ref.clear();
      float cs = 0.f;
      for (int j = w.t0; j < w.t1; ++j, ++t) {
        ok = ok && warp_wait(&sm.s_full[t & 1], (t >> 1) & 1, abort) &&
             warp_wait(&sm.ref_full[t % kRefs], (t / kRefs) & 1, abort) &&
             (j > w.t0 || warp_wait(&sm.q_full, seg & 1, abort));
        if (!ok) continue;
        tc_fence_after();
        const uint32_t s_col = tbase + lane_off + kSCol + (t & 1) * kTcKT;
        if (j == w.t0) cs = a.scale_log2 * sm.qs[row];
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
        const bool fold = j > w.t0 && C::fresh(j - w.t0);
        if (j > w.t0 && (fold || __any_sync(0xffffffffu, moved))) {
          // the PV of the tile before is done, the next waits for this P
          ok = warp_wait(&sm.pv_done, (t & 1) ^ 1, abort);
          if (!ok) continue;
          tc_fence_after();
          const bool sums = j - w.t0 > C::FOLD;             // O was added to the sum before
#pragma unroll 1
          for (int p = 0; p < D / 16; ++p) {
            uint32_t v[16], u[16];
            tmem_ld16(o_col + p * 16, v);
            if (F32 && sums) tmem_ld16(sum_col + p * 16, u);
            tmem_wait_only();
            reg_fence(v);
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = __float_as_uint(__uint_as_float(v[q]) * g);
            if (!fold) tmem_st16(o_col + p * 16, v);
            if (F32 && sums) {
              reg_fence(u);
#pragma unroll
              for (int q = 0; q < 16; ++q)
                v[q] = __float_as_uint(fmaf(__uint_as_float(u[q]), g, fold ? __uint_as_float(v[q]) : 0.f));
            }
            if (F32 && (fold || sums)) tmem_st16(sum_col + p * 16, v);
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
          uint32_t top[16], rest[16];
#pragma unroll
          for (int gr = 0; gr < 2; ++gr) {      // 16 tokens: one page's
            const int p = 2 * h + gr;
            const float e = ev[p];
            // (fp32: the factor after the exponential, so that the largest terms' exponents are small numbers)
            const float2 nm = F32 ? make_float2(-mr, -mr) : make_float2(e - mr, e - mr);
            const float pf = pow2_bits((int)fminf(e, 127.f));
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float2 y = __ffma2_rn(make_float2(x[p][2 * q], x[p][2 * q + 1]), make_float2(f[p], f[p]), nm);
              const float2 ex = make_float2(ex2(y.x), ex2(y.y));
              sum = q ? __fadd2_rn(sum, ex) : ex;
              if constexpr (F32) {
                const float2 pe = __fmul2_rn(ex, make_float2(pf, pf));
                top[8 * gr + q] = half2_bits(pe.x, pe.y);
                rest[8 * gr + q] = half2_rest(pe.x, pe.y, top[8 * gr + q]);
              } else {
                top[8 * gr + q] = half2_bits(ex.x, ex.y);
              }
            }
            if constexpr (F32) {
              ls = __fadd2_rn(ls, sum);
            } else {
              const float back = ex2(-e);       // (what P's sum takes for the row's)
              ls = __ffma2_rn(sum, make_float2(back, back), ls);
            }
          }
          tmem_st16(s_col + h * 16, top);
          if (F32) tmem_st16(s_col + 64 + h * 16, rest);
          if (h == 1) {                         // the first half may be multiplied
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.p_half[t & 1]);
          }
        }
        ref.l += ls.x + ls.y;
        // the PV of the tile before in turn, so that no wait for one is two phases behind
        ok = warp_wait(&sm.pv_done, (t & 1) ^ 1, abort);
        if (!ok) continue;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full);
      }
      ok = ok && warp_wait(&sm.pv_done, (t & 1) ^ 1, abort);
      ++seg;
      if (named_sync_any(1, 128, !ok)) break;
      tc_fence_after();
      // O in units of 2^(r - kTcPExp)
      const float2 ou = pow2_factors((int)ref.value_base() - kTcPExp);
      const bool whole = w.whole();
      const int64_t at = (int64_t)(w.u.q.row0 + qi) * a.Hq + w.u.g * G + qj;
      auto put_out = [&](int64_t at, int col, const float (&y)[16], float inv) {
        T* dst = static_cast<T*>(a.out) + at * D + col;
        if constexpr (F32) {
#pragma unroll
          for (int q = 0; q < 16; q += 4)
            *reinterpret_cast<float4*>(dst + q) =
                make_float4(y[q] * inv, y[q + 1] * inv, y[q + 2] * inv, y[q + 3] * inv);
        } else {
          uint32_t b8[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const __nv_bfloat162 b2 = __floats2bfloat162_rn(y[2 * q] * inv, y[2 * q + 1] * inv);
            b8[q] = *reinterpret_cast<const uint32_t*>(&b2);
          }
          *reinterpret_cast<uint4*>(dst) = make_uint4(b8[0], b8[1], b8[2], b8[3]);
          *reinterpret_cast<uint4*>(dst + 8) = make_uint4(b8[4], b8[5], b8[6], b8[7]);
        }
      };
      auto put_lse = [&](int64_t at, float M, float L) {
        if (a.lse) a.lse[at] = L == 0.f ? -INFINITY : fmaf(M, 0.6931471805599453f, logf(L));
      };
      const int64_t mine = 2 * (int64_t)blockIdx.x + (w.t0 == 0 ? 1 : 0);
      const int nan_from = sm.nan_token[(seg - 1) & 1][warp], nan_to = min(lim, w.t1 * kTcKT);
      __syncwarp();
      if (lane == 0) sm.nan_token[(seg - 1) & 1][warp] = kNoNan;
      const float inv = whole ? inverse_of(ref.l) : 1.f;
#pragma unroll 1
      for (int p = 0; p < D / 16; ++p) {
        uint32_t v[16];
        __syncwarp();                           // (whole warps read tensor memory)
        tmem_ld16(o_col + p * 16, v);
        tmem_wait(v);
        float y[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) y[q] = __uint_as_float(v[q]);
        if constexpr (F32) {
          if (w.t1 - w.t0 > C::FOLD) {
            tmem_ld16(sum_col + p * 16, v);
            tmem_wait(v);
#pragma unroll
            for (int q = 0; q < 16; ++q) y[q] += __uint_as_float(v[q]);
          }
        }
#pragma unroll
        for (int q = 0; q < 16; ++q) y[q] = y[q] * ou.x * inv * ou.y;
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
          float4* po = reinterpret_cast<float4*>(a.part_o + mine * 128 * D) + p * 4 * 128 + row;
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (real) po[q * 128] = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
        }
      }
      tc_fence_before();
      if (whole) {
        if (real) put_lse(at, ref.m, ref.l);
      } else {
        if (real) a.part_ml[mine * 128 + row] = make_float2(ref.m, ref.l);
        const int first = w.first_block(sh), final = w.last_block(sh);
        __syncwarp();                           // (the named barriers take whole warps)
        named_sync(1, 128);
        if (warp == 0) {
          const bool all = piece_done(a.flags, 1, a.token, first, final);
          if (lane == 0) sm.last = all;
          __syncwarp();
        }
        named_sync(1, 128);
        if (sm.last) {
          const int rows = min(kTcMT, w.u.q.m * G - w.u.rt * kTcMT);
          join_pieces<D>(a, first, final, 1, 0, rows, [&](int jr, int col, const float (&y)[16], float M, float L) {
            const int jrho = w.u.rt * kTcMT + jr, ji = jrho / G;
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

template <typename T, int D>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8AttnArgs& a, cudaStream_t st) {
  constexpr size_t smem = sizeof(Tc1Smem<T, D>) + 1024;
  static_assert(smem <= 232448, "shared memory of a block");
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = kv8_allow_smem(reinterpret_cast<const void*>(kv8_attn_tc1_kernel<T, D>), smem, allowed);
  if (e != cudaSuccess) return e;
  CUtensorMap mk = {};
  if (!Cfg<T, D>::F32 && !kv8_pool_map(&mk, c.K_codes, c)) return cudaErrorInvalidValue;
  const int64_t G = a.Hq / c.Hkv;
  const int64_t units = ((int64_t)s.n_rows * G / kTcMT + (s.n_req < s.n_rows ? s.n_req : s.n_rows)) * c.Hkv;
  const int64_t tiles = units * (((int64_t)s.max_pages * c.page + kTcKT - 1) / kTcKT);
  const int64_t sms = kv8_sm_count();
  ProfileScope ps("kv8_attn_tc1", st);
  kv8_attn_tc1_kernel<T, D><<<(unsigned)(tiles < sms ? tiles : sms), kTcThreads, smem, st>>>(mk, c, s, a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_attn_tc1(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8AttnArgs& a,
                                cudaStream_t st) {
  if (dtype == VC_BF16)
    return c.d == 128 ? launch_t<__nv_bfloat16, 128>(c, s, a, st) : launch_t<__nv_bfloat16, 64>(c, s, a, st);
  return c.d == 128 ? launch_t<float, 128>(c, s, a, st) : launch_t<float, 64>(c, s, a, st);
}

}  // namespace vc
