// The attention that cached tokens get, added up (viscache_kv8_weigh), few query rows
// a request:
//     A[t] = sum over rows rho that see t of exp(scale q[rho] . K[t] - lse[rho]),
// rho the packed rows of a request and KV head, weights[t] <- A[t] + (old or 0).
//
// Reads d bytes of K a token for 8 or 16 query rows, four bytes of weight either way:
// bound by the codes' bytes.  A token's sum needs no other token, so there is nothing
// to join: every warp takes an equal share of the line of 16- or 32-token chunks (requests,
// KV heads, chunks) and brings its chunks, which are contiguous in a page, into a ring of
// its own in shared memory by bulk copies, kStages - 1 ahead; no warp waits for another.
// The product is m16n8k16 with tokens as M and query rows as N (kv8_attn.cu says how
// codes become fragments); the queries' fragments stay in registers while the head lasts.
//
// Numbers: query rows as in kv8_attn.cu (powers of two, one fp16 part of bf16 rows,
// two of fp32 rows, 22 bits); the exponent is (product * scale - lse) * log2(e): product
// times the powers of two is exact, the subtraction is one fused multiply-add, so a large
// lse costs no bits.  The tensor cores cut a product's fp32 sums off; the scale is larger
// by what that is on average (kWeighCut, kv8_api.cu: fp32 rows of 128, whose weights at
// scores of 15 were short by 4.0e-6, are off by 1e-7 to 7e-7 on average).
//
// 32 requests of up to 32768 tokens, 64 / 8 heads of 128 (718 MB): 117 us, 6.1 TB/s, 92% of a plain
// copy's rate (138 us from cold memory).  6 x 5 fp32 rows over 3136 tokens: 8 us, a launch, the
// lengths, a page, a chunk.
//
// Requests of more rows than the fragments hold run over their rows 16 at a time for
// each chunk, which a warp's share does not count: one request of 256 rows among 63 of
// one, 4096 tokens each, takes 6.3 ms, all of one row 70 us.  Many rows belong to
// kv8_weigh_tc.cu.
#include "kernels.h"
#include "kv8.cuh"
#include "kv8_mma.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace kv8;

// Warps of a block, one block an SM, and stages of their rings, as shared memory and the
// registers of the fragments allow.  32 requests of up to 32768 tokens, 64 / 8 heads of 128, us: 8
// warps of 6 stages 147, 12 of 4 138, 16 of 3 147; in chunks of 16 tokens 16 warps of 4
// stages 151 (the work around a chunk counts), 24 warps 319 (registers).  6 x 5 fp32 rows
// over 3136 tokens: 12 warps 12.5, 16 warps 11.3.
template <typename T, int NQ>
constexpr int kWarps = sizeof(T) == 2 && NQ == 1 ? 12 : 16;

// A chunk of CT tokens in shared memory: its codes and the weights of its tokens.
template <int D, int CT>
struct alignas(16) Chunk {
  uint8_t k[CT][D];
  float weight[CT];
};
template <int D, int CT, int NW>
struct RingSmem {
  static constexpr int NST = CT == 16 || NW == 12 ? 4 : 3;      // stages of a warp's ring
  Chunk<D, CT> ring[NW][NST];
  uint64_t full[NW][NST];
  int scale_at[NW][NST];                    // (page, KV head) of the stage's chunk, -1 if there is no such page
  int abort;
  int32_t err;
};

template <typename T, int D, int NQ, int CT>
__global__ void __launch_bounds__(32 * kWarps<T, NQ>, 1)
kv8_weigh_kernel(const __grid_constant__ vc_kv8 c, const __grid_constant__ vc_kv8_step s,
                 const __grid_constant__ Kv8WeighArgs a) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1, KS = D / 16, MT = 8 * NQ, NS = CT / 16, NW = kWarps<T, NQ>;
  constexpr int kStages = RingSmem<D, CT, NW>::NST;
  extern __shared__ __align__(16) uint8_t smem_ring[];
  RingSmem<D, CT, NW>& sm = *reinterpret_cast<RingSmem<D, CT, NW>*>(smem_ring);
  int32_t& err = sm.err;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
  const int G = a.Hq / c.Hkv, shift = __ffs(c.page) - 1;      // (pages are powers of two)
  if (threadIdx.x == 0) {
    err = VC_OK;
    sm.abort = 0;
  }
  if (lane < kStages) tc::mbar_init(&sm.full[warp][lane], 1);
  tc::fence_mbar_init();
  __syncthreads();

  // the warp's share [at, end) of the line; requests without rows have no place on it
  auto chunks_of = [&](const Req8& q) { return q.m > 0 ? (int64_t)c.Hkv * ((q.len + CT - 1) / CT) : (int64_t)0; };
  int64_t total = 0;
  for (int r0 = 0; r0 < s.n_req; r0 += 32) {
    const Req8 q = r0 + lane < s.n_req ? load_req(s, c.page, r0 + lane, &err) : Req8{0, 0, 0};
    total += __shfl_sync(0xffffffffu, scan_warp(chunks_of(q)), 31);
  }
  const int64_t workers = (int64_t)gridDim.x * NW, me = (int64_t)warp * gridDim.x + blockIdx.x;
  const int64_t per = divide(total, workers), more = total - per * workers;
  int64_t at = me * per + (me < more ? me : more);
  const int64_t end = at + per + (me < more ? 1 : 0);
  if (at < end) {
    // the request that holds `at`
    Unit u;
    int64_t first = 0;                          // its first chunk
    u.r = -1;
    u.rt = 0;
    for (int r0 = 0; u.r < 0; r0 += 32) {
      const Req8 q = r0 + lane < s.n_req ? load_req(s, c.page, r0 + lane, &err) : Req8{0, 0, 0};
      const int64_t w = chunks_of(q), upto = first + scan_warp(w);
      const uint32_t has = __ballot_sync(0xffffffffu, at < upto);
      if (has) {
        const int src = __ffs(has) - 1;
        u.r = r0 + src;
        u.q.row0 = __shfl_sync(0xffffffffu, q.row0, src);
        u.q.m = __shfl_sync(0xffffffffu, q.m, src);
        u.q.len = __shfl_sync(0xffffffffu, q.len, src);
        first = __shfl_sync(0xffffffffu, upto - w, src);
      } else {
        first = __shfl_sync(0xffffffffu, upto, 31);
      }
    }
    // a place on the line: request, head, chunk of n
    struct Place {
      int r, g, ck, n;
    };
    auto next = [&](Place& p) {                 // (called while there is one); whether the request is another
      if (++p.ck < p.n) return false;
      p.ck = 0;
      if (++p.g < c.Hkv) return false;
      p.g = 0;
      for (;;) {
        const Req8 q = load_req(s, c.page, ++p.r, &err);
        if (q.m == 0 || q.len == 0) continue;
        p.n = (q.len + CT - 1) / CT;
        return true;
      }
    };
    Place cur;
    cur.r = u.r;
    cur.n = (u.q.len + CT - 1) / CT;
    cur.g = (int)divide(at - first, cur.n);
    cur.ck = (int)(at - first - (int64_t)cur.g * cur.n);
    Req8 q = u.q;                               // cur's request
    // the page's number as it is in the table: looked at an iteration later, when it has come
    auto fetch_page = [&](const Place& p) {
      return __ldg(s.block_table + (int64_t)p.r * s.max_pages + (p.ck * CT >> shift));
    };
    auto checked = [&](int pid) {
      if (pid >= 0 && pid < c.n_pages) return pid;
      set_status(&err, VC_ERR_DEVICE_INDEX);
      return -1;
    };
    // slot of token CT ck + i from the chunk's (page, head)
    auto slot0 = [&](int at_scale, int ck) { return ((int64_t)at_scale << shift) + (ck * CT & (c.page - 1)); };
    const int mine = gid + 8 * tig;             // the token that the lane writes (of 16: lanes with tig < 2)
    auto load = [&](const Place& p, int pid, int st) {
      if (lane != 0) return;
      uint64_t* bar = &sm.full[warp][st];
      auto& x = sm.ring[warp][st];
      const int sc = pid < 0 ? -1 : pid * c.Hkv + p.g;
      sm.scale_at[warp][st] = sc;
      if (pid < 0) {
        tc::mbar_arrive(bar);
        return;
      }
      const int64_t t0 = slot0(sc, p.ck);
      tc::mbar_arrive_expect_tx(bar, sizeof(Chunk<D, CT>));
      tc::bulk_load(x.k, static_cast<const uint8_t*>(c.K_codes) + t0 * D, CT * D, bar);
      tc::bulk_load(x.weight, a.weights + t0, 4 * CT, bar);
    };
    uint32_t qf[NP][NQ][KS][2];
    float qs[NQ][2], lse[NQ][2];
    int lim[NQ][2], lim_min = 0;
    auto rows = [&](int rt) {
      u.q = q;
      u.g = cur.g;
      u.rt = rt;
      // (rows that are no tokens count as 0: theirs may hold anything, and not causal nothing masks them)
      load_q<T, D, NQ, NP, true>(static_cast<const T*>(a.q), a.q_stride, u, G, qf, qs);
      const int base = q.len - q.m + 1, r0 = rt * MT;
      lim_min = a.causal ? base + r0 / G : 0x7fffffff;
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int rho = r0 + 8 * n + 2 * tig + h, i = rho / G;
          lim[n][h] = a.causal ? base + i : 0x7fffffff;
          // rows that are none, see nothing or are no tokens add exp(-inf)
          float l = INFINITY;
          if (i < q.m && base + i > 0) {
            l = __ldg(a.lse + (int64_t)(q.row0 + i) * a.Hq + cur.g * G + (rho - i * G));
            if (l == -INFINITY) l = INFINITY;
          }
          lse[n][h] = l;
        }
    };
    // the head of the ring: kStages - 1 chunks in front of cur
    Place head = cur;
    int64_t left = end - at;                    // chunks not yet sent for
    int raw = fetch_page(head);
    auto send = [&](int st) {
      if (left <= 0) return;
      load(head, checked(raw), st);
      if (--left > 0) {
        next(head);
        raw = fetch_page(head);
      }
    };
#pragma unroll 1
    for (int st = 0; st < kStages - 1; ++st) send(st);
    __syncwarp();
    float kscale = __ldg(c.K_scale + max(sm.scale_at[warp][0], 0)), nscale = 0.f;
    bool fresh = true, ok = true;               // fresh: the fragments are another head's
    uint32_t it = 0;
#pragma unroll 1
    for (; at < end; ++at, ++it) {
      const int st = it % kStages;
      __syncwarp();                             // (the stage before is read)
      send((st + kStages - 1) % kStages);
      __syncwarp();
      // the next chunk's scale
      if (at + 1 < end) nscale = __ldg(c.K_scale + max(sm.scale_at[warp][(st + 1) % kStages], 0));
      const int sc = sm.scale_at[warp][st];
      ok = tc::warp_wait(&sm.full[warp][st], (it / kStages) & 1, &sm.abort);
      if (!ok) break;
      const auto& ch = sm.ring[warp][st];
      const float old = cur.ck * CT + mine % CT < q.len - q.m ? ch.weight[mine % CT] : 0.f;
      const int tiles = (q.m * G + MT - 1) / MT;
      float sum[2 * NS];                        // of tokens gid + 8 i
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i) sum[i] = 0.f;
#pragma unroll 1
      for (int rt = 0; rt < tiles; ++rt) {
        if (tiles > 1 || fresh) rows(rt);
        fresh = false;
        const bool edge = cur.ck * CT + CT > lim_min;
#pragma unroll
        for (int sub = 0; sub < NS; ++sub) {
          // rows gid and gid + 8, the thread's D / 4 bytes of each; odd rows read their halves in the other order, so
          // that a quarter of a warp covers all banks
          uint4 x[2][D / 64];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint4* src = reinterpret_cast<const uint4*>(ch.k[16 * sub + 8 * i + gid]) + tig * (D / 64);
            if constexpr (D == 128) {
              const uint4 u0 = src[gid & 1], u1 = src[~gid & 1];
              x[i][0] = gid & 1 ? u1 : u0;
              x[i][1] = gid & 1 ? u0 : u1;
            } else {
              x[i][0] = src[0];
            }
          }
          float z[NQ][4];
#pragma unroll
          for (int n = 0; n < NQ; ++n) z[n][0] = z[n][1] = z[n][2] = z[n][3] = 0.f;
#pragma unroll
          for (int h = 0; h < D / 64; ++h) {
            const uint4 u0 = x[0][h], u1 = x[1][h];
            const uint32_t b0[4] = {u0.x, u0.y, u0.z, u0.w}, b1[4] = {u1.x, u1.y, u1.z, u1.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t ka[4] = {e4m3x2_to_f16x2(b0[k]), e4m3x2_to_f16x2(b1[k]), e4m3x2_to_f16x2(b0[k] >> 16),
                                      e4m3x2_to_f16x2(b1[k] >> 16)};
#pragma unroll
              for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int p = 0; p < NP; ++p) mma_f16(z[n], ka, qf[p][n][4 * h + k][0], qf[p][n][4 * h + k][1]);
            }
          }
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float f = qs[n][h] * kscale;
              float p0 = tc::ex2(fmaf(z[n][h] * f, a.scale, -lse[n][h]) * kLog2e);
              float p1 = tc::ex2(fmaf(z[n][2 + h] * f, a.scale, -lse[n][h]) * kLog2e);
              if (edge) {
                const int t = cur.ck * CT + 16 * sub + gid;
                if (t >= lim[n][h]) p0 = 0.f;
                if (t + 8 >= lim[n][h]) p1 = 0.f;
              }
              sum[2 * sub] += p0;
              sum[2 * sub + 1] += p1;
            }
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i) {
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
      }
      const float lo = tig & 1 ? sum[1] : sum[0], hi = tig & 1 ? sum[2 * NS - 1] : sum[2 * NS - 2];
      if (sc >= 0 && mine < CT && cur.ck * CT + mine < q.len)
        a.weights[slot0(sc, cur.ck) + mine] = old + (tig < 2 ? lo : hi);
      kscale = nscale;
      if (at + 1 < end) {
        if (next(cur)) q = load_req(s, c.page, cur.r, &err);
        fresh = cur.ck == 0;
      }
    }
    if (!ok) {
      // copies that nobody waited for have landed before the block ends
      if (lane == 0) set_status(&err, VC_ERR_DEVICE_TIMEOUT);
      for (int64_t k = 0; k < kStages && at + k < end - left; ++k, ++it)
        tc::drain_wait(&sm.full[warp][it % kStages], (it / kStages) & 1);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    a.block_status[blockIdx.x] = err;
    if (blockIdx.x == 0) {
      a.status[0] = kStatusPerBlock;
      a.status[1] = (int32_t)gridDim.x;
    }
  }
}

template <typename T, int D, int NQ, int CT>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8WeighArgs& a, cudaStream_t st) {
  using Smem = RingSmem<D, CT, kWarps<T, NQ>>;
  static_assert(sizeof(Smem) <= 227 * 1024, "shared memory of an SM");
  static std::atomic<uint64_t> allowed{0};
  const auto kernel = kv8_weigh_kernel<T, D, NQ, CT>;
  const cudaError_t e = kv8_allow_smem(reinterpret_cast<const void*>(kernel), sizeof(Smem), allowed);
  if (e != cudaSuccess) return e;
  ProfileScope ps("kv8_weigh", st);
  kernel<<<(unsigned)kv8_sm_count(), 32 * kWarps<T, NQ>, sizeof(Smem), st>>>(c, s, a);
  return cudaGetLastError();
}

template <typename T, int D, int NQ>
cudaError_t launch_c(const vc_kv8& c, const vc_kv8_step& s, const Kv8WeighArgs& a, cudaStream_t st) {
  return c.page >= 32 ? launch_t<T, D, NQ, 32>(c, s, a, st) : launch_t<T, D, NQ, 16>(c, s, a, st);
}

template <typename T, int D>
cudaError_t launch_q(const vc_kv8& c, const vc_kv8_step& s, const Kv8WeighArgs& a, cudaStream_t st) {
  // Fragments of 8 query rows where the requests have no more on average, of bf16 calls; else of 16.  Us with 8 / with
  // 16, cold: 64 requests of up to 4096 tokens, 16 rows 94 / 50, 24 rows 127 / 113, 128 rows 529 / 384; 8 rows of fp32 52 / 80;
  // fp32 24 rows 160 / 180, 48 rows 267 / 286 (the larger ones spill)
  const int64_t rows = (int64_t)s.n_rows * (a.Hq / c.Hkv);
  return rows <= 8 * (int64_t)s.n_req ? launch_c<T, D, 1>(c, s, a, st) : launch_c<T, D, 2>(c, s, a, st);
}

}  // namespace

cudaError_t launch_kv8_weigh(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8WeighArgs& a,
                             cudaStream_t st) {
  if (dtype == VC_BF16)
    return c.d == 128 ? launch_q<__nv_bfloat16, 128>(c, s, a, st) : launch_q<__nv_bfloat16, 64>(c, s, a, st);
  return c.d == 128 ? launch_q<float, 128>(c, s, a, st) : launch_q<float, 64>(c, s, a, st);
}

}  // namespace vc
