// The attention that cached tokens get, added up (viscache_kv8_weigh), few query rows
// a request:
//     A[t] = sum over rows rho that see t of exp(scale q[rho] . K[t] - lse[rho]),
// rho the packed rows of a request and KV head, weights[t] <- A[t] + (old or 0).
//
// Reads d bytes of K a token for 8 or 16 query rows, four bytes of weight either way:
// bound by the codes' bytes.  A token's sum needs no other token, so there is nothing
// to join: every warp takes an equal share of the line of 16-token chunks (requests,
// KV heads, chunks), a chunk's codes go from memory into registers as they are
// multiplied, and the next chunk's are in flight meanwhile.  The product is
// m16n8k16 with tokens as M and query rows as N (kv8_attn.cu says how codes become
// fragments); the queries' fragments stay in registers while the head lasts.
//
// Numbers: query rows as in kv8_attn.cu (powers of two, one fp16 part of bf16 rows,
// two of fp32 rows); the exponent is (product * scale - lse) * log2(e): product times
// the powers of two is exact, the subtraction is one fused multiply-add, so a large
// lse costs no bits.
//
// Requests of more rows than the fragments hold run over their rows 16 at a time for
// each chunk; many rows belong to kv8_weigh_tc.cu.
#include "kernels.h"
#include "kv8.cuh"
#include "kv8_mma.cuh"
#include "profile.h"
#include "tc_common.cuh"
#include "vc_common.cuh"

namespace vc {
namespace {

using namespace kv8;

constexpr int kWarps = 8;
constexpr int kWThreads = 32 * kWarps;

// A chunk on its way: codes of tokens gid and gid + 8 (this thread's D / 4 bytes of each),
// the page's scale, and the old weight of the token that the lane will write.
template <int D>
struct Chunk {
  uint4 k[2][D / 64];
  float scale, old;
};

template <typename T, int D, int NQ>
__global__ void __launch_bounds__(kWThreads, sizeof(T) == 4 || NQ == 2 ? 2 : 3)
kv8_weigh_kernel(const __grid_constant__ vc_kv8 c, const __grid_constant__ vc_kv8_step s,
                 const __grid_constant__ Kv8WeighArgs a) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1, KS = D / 16, MT = 8 * NQ;
  __shared__ int32_t err;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
  const int G = a.Hq / c.Hkv;
  if (threadIdx.x == 0) err = VC_OK;
  __syncthreads();

  // the warp's share [at, end) of the line; requests without rows have no place on it
  auto chunks_of = [&](const Req8& q) { return q.m > 0 ? (int64_t)c.Hkv * ((q.len + 15) / 16) : (int64_t)0; };
  int64_t total = 0;
  for (int r0 = 0; r0 < s.n_req; r0 += 32) {
    const Req8 q = r0 + lane < s.n_req ? load_req(s, c.page, r0 + lane, &err) : Req8{0, 0, 0};
    total += __shfl_sync(0xffffffffu, scan_warp(chunks_of(q)), 31);
  }
  const int64_t workers = (int64_t)gridDim.x * kWarps, me = (int64_t)warp * gridDim.x + blockIdx.x;
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
    // a place on the line: request, head, chunk
    struct Place {
      int r, g, ck, n;                          // n: chunks of the head
      Req8 q;
    };
    auto next = [&](Place& p) {                 // (called while there is one)
      if (++p.ck < p.n) return;
      p.ck = 0;
      if (++p.g < c.Hkv) return;
      p.g = 0;
      do {
        ++p.r;
        p.q = load_req(s, c.page, p.r, &err);
      } while (chunks_of(p.q) == 0);
      p.n = (p.q.len + 15) / 16;
    };
    Place cur;
    cur.r = u.r;
    cur.q = u.q;
    cur.n = (u.q.len + 15) / 16;
    cur.g = (int)divide(at - first, cur.n);
    cur.ck = (int)(at - first - (int64_t)cur.g * cur.n);
    auto page_of = [&](const Place& p) { return load_page(s, c.n_pages, p.r, p.ck * 16 / c.page, &err); };
    // slot of token 16 ck + i: ((page * Hkv + g) * page size) + slot in it
    auto slot0 = [&](const Place& p, int pid) {
      return ((int64_t)max(pid, 0) * c.Hkv + p.g) * c.page + p.ck * 16 % c.page;
    };
    const int mine = gid + 8 * tig;             // the token that lanes with tig < 2 write
    auto load = [&](const Place& p, int pid, Chunk<D>& x) {
      const int64_t t0 = slot0(p, pid);
      const uint8_t* codes = static_cast<const uint8_t*>(c.K_codes) + (t0 + gid) * D + tig * (D / 4);
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {
        x.k[0][h] = __ldg(reinterpret_cast<const uint4*>(codes) + h);
        x.k[1][h] = __ldg(reinterpret_cast<const uint4*>(codes + 8 * D) + h);
      }
      x.scale = __ldg(c.K_scale + (int64_t)max(pid, 0) * c.Hkv + p.g);
      const int t = p.ck * 16 + mine;
      x.old = tig < 2 && t < p.q.len - p.q.m ? a.weights[t0 + mine] : 0.f;
    };
    uint32_t qf[NP][NQ][KS][2];
    float qs[NQ][2], lse[NQ][2];
    int lim[NQ][2], lim_min = 0;
    auto rows = [&](const Place& p, int rt) {
      u.r = p.r;
      u.q = p.q;
      u.g = p.g;
      u.rt = rt;
      load_q<T, D, NQ, NP>(static_cast<const T*>(a.q), a.q_stride, u, G, qf, qs);
      const int base = p.q.len - p.q.m + 1, r0 = rt * MT;
      lim_min = a.causal ? base + r0 / G : 0x7fffffff;
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int rho = r0 + 8 * n + 2 * tig + h, i = rho / G;
          lim[n][h] = a.causal ? base + i : 0x7fffffff;
          // rows that are none, see nothing or are no tokens add exp(-inf)
          float l = INFINITY;
          if (i < p.q.m && base + i > 0) {
            l = __ldg(a.lse + (int64_t)(p.q.row0 + i) * a.Hq + p.g * G + (rho - i * G));
            if (l == -INFINITY) l = INFINITY;
          }
          lse[n][h] = l;
        }
    };
    Place nxt = cur;
    int pid = page_of(cur), npid = -1;
    Chunk<D> x, y;
    load(cur, pid, x);
    if (at + 1 < end) {
      next(nxt);
      npid = page_of(nxt);
    }
    int have_r = -1, have_g = -1;               // whose fragments the registers hold
    for (; at < end; ++at) {
      const int tiles = (cur.q.m * G + MT - 1) / MT;
      if (tiles == 1 && (cur.r != have_r || cur.g != have_g)) {
        rows(cur, 0);
        have_r = cur.r;
        have_g = cur.g;
      }
      Place after = nxt;
      int apid = -1;
      if (at + 1 < end) {
        load(nxt, npid, y);
        if (at + 2 < end) {
          next(after);
          apid = page_of(after);
        }
      }
      float sum[2] = {0.f, 0.f};                // of tokens gid, gid + 8
      for (int rt = 0; rt < tiles; ++rt) {
        if (tiles > 1) {
          rows(cur, rt);
          have_r = -1;
        }
        float z[NQ][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n) z[n][0] = z[n][1] = z[n][2] = z[n][3] = 0.f;
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
          const uint32_t b0[4] = {x.k[0][h].x, x.k[0][h].y, x.k[0][h].z, x.k[0][h].w};
          const uint32_t b1[4] = {x.k[1][h].x, x.k[1][h].y, x.k[1][h].z, x.k[1][h].w};
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
        const bool edge = cur.ck * 16 + 16 > lim_min;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float f = qs[n][h] * x.scale;
            float p0 = tc::ex2(fmaf(z[n][h] * f, a.scale, -lse[n][h]) * kLog2e);
            float p1 = tc::ex2(fmaf(z[n][2 + h] * f, a.scale, -lse[n][h]) * kLog2e);
            if (edge) {
              const int t = cur.ck * 16 + gid;
              if (t >= lim[n][h]) p0 = 0.f;
              if (t + 8 >= lim[n][h]) p1 = 0.f;
            }
            sum[0] += p0;
            sum[1] += p1;
          }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
      }
      if (pid >= 0 && tig < 2 && cur.ck * 16 + mine < cur.q.len)
        a.weights[slot0(cur, pid) + mine] = x.old + (tig == 0 ? sum[0] : sum[1]);
      cur = nxt;
      nxt = after;
      pid = npid;
      npid = apid;
      x = y;
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

template <typename T, int D, int NQ>
cudaError_t launch_t(const vc_kv8& c, const vc_kv8_step& s, const Kv8WeighArgs& a, cudaStream_t st) {
  ProfileScope ps("kv8_weigh", st);
  kv8_weigh_kernel<T, D, NQ><<<(unsigned)kv8_sm_count(), kWThreads, 0, st>>>(c, s, a);
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_q(const vc_kv8& c, const vc_kv8_step& s, const Kv8WeighArgs& a, cudaStream_t st) {
  const int64_t rows = (int64_t)s.n_rows * (a.Hq / c.Hkv);
  return rows <= 8 * (int64_t)s.n_req ? launch_t<T, D, 1>(c, s, a, st) : launch_t<T, D, 2>(c, s, a, st);
}

}  // namespace

cudaError_t launch_kv8_weigh(const vc_kv8& c, const vc_kv8_step& s, int dtype, const Kv8WeighArgs& a,
                             cudaStream_t st) {
  if (dtype == VC_BF16)
    return c.d == 128 ? launch_q<__nv_bfloat16, 128>(c, s, a, st) : launch_q<__nv_bfloat16, 64>(c, s, a, st);
  return c.d == 128 ? launch_q<float, 128>(c, s, a, st) : launch_q<float, 64>(c, s, a, st);
}

}  // namespace vc
