// C entry points of the rotary positions and of the 8-bit paged cache
// (include/viscache.h) and of the step around it (include/viscache_step.h):
// argument checks, workspace layout, launches.
#include <math.h>

#include <atomic>
#include <chrono>

#include "api_util.h"
#include "kernels.h"
#include "norm_grid.h"
#include "viscache_step.h"

namespace vc {
namespace {

constexpr double kInv2Pi = 0.15915494309189533577;

bool valid_cache(const vc_kv8* c) {
  if (!c || !c->K_codes || !c->V_codes || !c->K_scale || !c->V_scale) return false;
  if (!aligned16(c->K_codes) || !aligned16(c->V_codes) || !aligned16(c->K_scale) || !aligned16(c->V_scale))
    return false;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return false;
  if ((c->d != 64 && c->d != 128) || c->Hkv < 1 || c->Hkv > 1024 || c->n_pages < 1) return false;
  return (int64_t)c->n_pages * c->Hkv * c->page < (int64_t)1 << 31;
}

bool valid_step(const vc_kv8* c, const vc_kv8_step* s) {
  if (!s || !s->block_table || !s->seq_lens || !s->row_start) return false;
  if (s->n_req < 1 || s->n_req > 1024 || s->max_pages < 1 || s->n_rows < 0 || s->n_rows > (1 << 24)) return false;
  return (int64_t)s->max_pages * c->page <= (int64_t)1 << 30;
}

bool valid_type(int dtype) { return dtype == VC_BF16 || dtype == VC_F32; }

// Row or head strides in elements: whole 16-byte pieces.
bool valid_stride(int64_t stride, int64_t least, int dtype) {
  return stride >= least && stride % (dtype == VC_BF16 ? 8 : 4) == 0 && stride < (int64_t)1 << 40;
}

bool valid_rope(const vc_rope* rope, int dtype, int64_t n_rows, int32_t Hq, int32_t Hkv, int32_t d) {
  if (!rope || !valid_type(dtype) || (d != 64 && d != 128)) return false;
  if (n_rows < 0 || n_rows > (1 << 24) || Hq < 0 || Hkv < 0 || Hq > 4096 || Hkv > 4096) return false;
  if (rope->n_axes < 1 || rope->n_axes > 4 || !(rope->theta >= 1.0) || !isfinite(rope->theta)) return false;
  if ((rope->order != VC_ROPE_SECTIONED && rope->order != VC_ROPE_INTERLEAVED) ||
      (rope->pairing != VC_ROPE_HALVES && rope->pairing != VC_ROPE_ADJACENT))
    return false;
  int64_t half = 0;
  for (int a = 0; a < rope->n_axes; ++a) {
    if (rope->sections[a] < 0 || rope->sections[a] > d / 2) return false;
    half += rope->sections[a];
  }
  return half >= 8 && half % 8 == 0 && half <= d / 2;
}

// Rows of `heads` heads (none: nothing to look at).
bool valid_rows(const void* p, int64_t stride, int32_t heads, int32_t d, int dtype) {
  return heads == 0 || (p && aligned16(p) && valid_stride(stride, (int64_t)heads * d, dtype));
}

// Frequencies and their axes, positions and counts; strides and direction are the caller's.
void set_rope(RopeArgs& a, const vc_rope& rope, const int32_t* positions, int64_t n_rows, int32_t Hq, int32_t Hkv) {
  int half = 0;
  for (int x = 0; x < rope.n_axes; ++x) half += rope.sections[x];
  for (int i = 0; i < half; ++i) {
    if (rope.order == VC_ROPE_INTERLEAVED) {
      const int x = i % rope.n_axes;
      a.axis[i] = (uint8_t)(i < rope.n_axes * rope.sections[x] ? x : 0);
    } else {
      int x = 0;
      for (int upto = rope.sections[0]; i >= upto; upto += rope.sections[x]) ++x;
      a.axis[i] = (uint8_t)x;
    }
  }
  // theta^(-i / half) by one power, off by an ulp, and up to 63 products: within 2^-45
  const double r = pow(rope.theta, -1.0 / (double)half);
  double f = kInv2Pi;
  for (int i = 0; i < half; ++i, f *= r) a.freq[i] = (uint64_t)(f * 18446744073709551616.0);
  a.positions = positions;
  a.n_rows = n_rows;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.half = half;
}

// Workspace: status word and block count (256 bytes), the blocks' status
// words, flags, (max, sum) and outputs of the attention's split units.
struct Kv8Ws {
  size_t o_blocks = 0, o_flags = 0, o_ml = 0, o_o = 0, total = 0;
};
Kv8Ws kv8_ws(bool tc, int d) {
  Arena a;
  Kv8Ws w;
  a.take(kAlign);
  const size_t rows = (size_t)2 * kKv8MaxCtas * (tc ? kv8_attn_rows_tc2() : kv8_attn_rows_mma());
  w.o_blocks = a.take(sizeof(int32_t) * kKv8MaxCtas);      // at byte 256: prunekv_get_status reads it there
  w.o_flags = a.take(sizeof(uint64_t) * 2 * kKv8MaxCtas * 2);
  w.o_ml = a.take(sizeof(float2) * rows);
  w.o_o = a.take(sizeof(float) * rows * d);
  w.total = a.off;
  return w;
}

// A number of its own for every call, spread over 64 bits so that what happens
// to be in a workspace is none of them: a counter from a point that differs
// between processes, through the SplitMix64 finaliser.
uint64_t next_token() {
  static std::atomic<uint64_t> count{(uint64_t)std::chrono::steady_clock::now().time_since_epoch().count() ^
                                     (uint64_t)std::chrono::system_clock::now().time_since_epoch().count() << 20};
  uint64_t z = count.fetch_add(0x9E3779B97F4A7C15ull, std::memory_order_relaxed);
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  z ^= z >> 31;
  return z ? z : 1;
}

// The kernel of a call.  On tcgen05 (tc1): more than kTcRows packed rows of a KV
// head per request on average, so at least two 16-row units of the mma.sync kernel
// (fp32, whose tiles take twice as long: three),
// and more of those units than SMs, or of their tiles than kTcShare an SM: below
// that every unit there gets blocks of its own.  With 256-row units (tc2): bf16, at
// least kTc2Rows such rows, kTc2Tiles tiles and more than kTc2Share tiles of those
// units an SM: its segments cost more at their ends.  Lengths are on the device, so
// the block table's width stands for them.
// d = 128, 8 KV heads, us on mma.sync / tc1:
//   64 requests of 4096 tokens, 16 rows 146 / 164, 20 rows 267 / 164, 128 rows 1012 / 192
//   8 of 600 tokens, 24 rows 14.4 / 16.7, 48 rows 31.8 / 17.6
//   one of 8192 tokens, 20 rows 22.3 / 20.7, 128 rows 45.6 / 35.6
//   fp32, twice the rows: 8 of 4096, 24 rows 53.8 / 55.2, 36 rows 83 / 58, 256 rows 350 / 103
// on tc1 / tc2:
//   one of 32768 tokens, 320 rows 75 / 98, 512 rows 98.6 / 98.1, 8192 rows 1049 / 778
//   one of 8192 tokens, 1024 rows 56.4 / 58.6, 2048 rows 89.5 / 82.7
//   one of 4096 tokens, 8192 rows 162 / 156; 64 of 1000, 1024 rows 537 / 628
constexpr int64_t kTcRows = 16, kTcShare = 8, kTc2Rows = 512, kTc2Tiles = 64, kTc2Share = 16;
enum class Kernel { kMma, kTc1, kTc2 };
bool may_have_many_rows(int64_t n_rows, int64_t n_req, int32_t Hq, int32_t Hkv) {
  return n_rows * (Hq / Hkv) > kTcRows * n_req;
}
Kernel kernel_of(const vc_kv8& c, const vc_kv8_step& s, int dtype, int32_t Hq) {
  const int64_t rows = (int64_t)s.n_rows * Hq, sms = kv8_sm_count();
  if (rows / c.Hkv <= (dtype == VC_F32 ? 2 : 1) * kTcRows * s.n_req) return Kernel::kMma;
  const int64_t tiles = ((int64_t)s.max_pages * c.page + 127) / 128;
  if (rows / 16 <= sms && rows / 16 * tiles <= kTcShare * sms) return Kernel::kMma;
  const bool two = dtype == VC_BF16 && rows / c.Hkv >= kTc2Rows * s.n_req && tiles >= kTc2Tiles &&
                   rows / 256 * tiles > kTc2Share * sms;
  return two ? Kernel::kTc2 : Kernel::kTc1;
}

// viscache_kv8_weigh on tcgen05: more packed rows of a KV head per request on average than
// this.  The mma.sync kernel reads a chunk's codes once and its rows 16 at a time; the
// other expands each K tile once however many rows there are.  The average, because rows are
// on the device: a long request among short ones takes the mma.sync kernel, whose shares count
// chunks and not rows (64 requests of 4096 tokens, one of 256 rows and 63 of one: 6.3 ms).
// d = 128, 8 KV heads, lengths drawn up to those given, us on mma.sync / tcgen05 (cold):
//   bf16, 64 requests of 4096 tokens, 24 rows 113 / 259, 48 rows 169 / 259, 128 rows 384 / 261
//   8 of 8192 tokens, 48 rows 58 / 72, 128 rows 118 / 73; one of 8192, 48 rows 20 / 30, 128 rows 34 / 30
//   fp32, 64 of 4096, 24 rows 160 / 228, 48 rows 267 / 231; 8 of 8192, 24 rows 51 / 63, 48 rows 81 / 63
//   one of 8192, 24 rows 20 / 28, 48 rows 28 / 28
constexpr int64_t kWeighTcRows = 64, kWeighTcRowsF32 = 32;

// What the tensor cores cut off a score, on average, in 2^-24 of it ([kernel: few rows, many][bf16, fp32][d = 64,
// 128]): a product's fp32 sum is cut, not rounded, at each of its steps of 16 dimensions, fp32 rows have twice as many,
// and bf16 rows have fewer bits to lose.  Measured at scores of 15 and 38 (sums of the weights against 64 bits, 8
// requests of 256 rows and 64 of 2, 1024 tokens; normal and uniform values, rows and pages of different size, outlier
// channels, rows along a key), by data: few rows .2-.6, .4-1.5 | 2.1-3.2, 3.7-5.4; many .15-.6, .4-1.2 | .9-1.3, 1.4-2.4.
// The factors are set off by the middle; what is left is of the size of fp32's rounding of a score.
constexpr double kWeighCut[2][2][2] = {{{0.35, 0.8}, {2.4, 4.3}}, {{0.35, 0.75}, {1.1, 1.8}}};

bool valid_heads(int32_t Hq, int32_t Hkv) { return Hkv >= 1 && Hq >= Hkv && Hq <= 4096 && Hq % Hkv == 0; }

// The attention's line of key tiles (units of 8 rows at least): a block's share is
// counted in 31 bits.
bool short_line(const vc_kv8& c, const vc_kv8_step& s, int32_t Hq) {
  const int64_t row_tiles = (int64_t)s.n_rows * (Hq / c.Hkv) / 8 + s.n_req;
  return row_tiles * c.Hkv <= ((int64_t)1 << 37) / (((int64_t)s.max_pages * c.page + 127) / 128);
}

int kv8_rows_call(bool append, const vc_kv8* cache, const vc_kv8_step* step, int dtype, const Kv8Rows& rows,
                  void* ws, size_t ws_bytes, void* stream) {
  if (!valid_cache(cache) || !valid_step(cache, step) || !valid_type(dtype)) return VC_ERR_INVALID_ARG;
  if (step->n_rows > 0 && (!rows.K || !rows.V || !aligned16(rows.K) || !aligned16(rows.V))) return VC_ERR_INVALID_ARG;
  if (!valid_stride(rows.k_row, cache->d, dtype) || !valid_stride(rows.v_row, cache->d, dtype) ||
      !valid_stride(rows.k_head, cache->d, dtype) || !valid_stride(rows.v_head, cache->d, dtype))
    return VC_ERR_INVALID_ARG;
  const int wc = check_ws(ws, ws_bytes, kAlign);
  if (wc != VC_OK) return wc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t* status = static_cast<int32_t*>(ws);
  return cuda_status(append ? launch_kv8_append(*cache, *step, dtype, rows, status, st)
                            : launch_kv8_read(*cache, *step, dtype, rows, status, st));
}

}  // namespace
}  // namespace vc

using namespace vc;

extern "C" {

int viscache_mrope(const vc_rope* rope, const int32_t* positions, int dtype, int64_t n_rows, int32_t Hq,
                   int32_t Hkv, int32_t d, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                   int inverse, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
                   void* stream) {
  RopeArgs a = {};
  if (!valid_rope(rope, dtype, n_rows, Hq, Hkv, d)) return VC_ERR_INVALID_ARG;
  if (n_rows > 0) {
    if (!positions) return VC_ERR_INVALID_ARG;
    if (!valid_rows(q, q_stride, Hq, d, dtype) || !valid_rows(q_out, q_out_stride, Hq, d, dtype) ||
        !valid_rows(k, k_stride, Hkv, d, dtype) || !valid_rows(k_out, k_out_stride, Hkv, d, dtype))
      return VC_ERR_INVALID_ARG;
  }
  if (n_rows == 0 || Hq + Hkv == 0) return VC_OK;
  set_rope(a, *rope, positions, n_rows, Hq, Hkv);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.inverse = inverse != 0;
  return cuda_status(launch_mrope(a, dtype, d, rope->pairing == VC_ROPE_ADJACENT, q, q_out, k, k_out,
                                  static_cast<cudaStream_t>(stream)));
}

static bool valid_eps(float eps) { return eps >= 1e-20f && eps <= 1.f; }

int viscache_norm_mrope(const vc_rope* rope, const int32_t* positions, int dtype, int64_t n_rows, int32_t Hq,
                        int32_t Hkv, int32_t d, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        const void* q_weight, const void* k_weight, float eps, void* q_out, int64_t q_out_stride,
                        void* k_out, int64_t k_out_stride, void* stream) {
  RopeArgs a = {};
  if (!valid_rope(rope, dtype, n_rows, Hq, Hkv, d) || !valid_eps(eps)) return VC_ERR_INVALID_ARG;
  if (n_rows > 0) {
    if (!positions) return VC_ERR_INVALID_ARG;
    if (!valid_rows(q, q_stride, Hq, d, dtype) || !valid_rows(q_out, q_out_stride, Hq, d, dtype) ||
        !valid_rows(k, k_stride, Hkv, d, dtype) || !valid_rows(k_out, k_out_stride, Hkv, d, dtype) ||
        !valid_rows(q_weight, d, Hq > 0, d, dtype) || !valid_rows(k_weight, d, Hkv > 0, d, dtype))
      return VC_ERR_INVALID_ARG;
  }
  if (n_rows == 0 || Hq + Hkv == 0) return VC_OK;
  set_rope(a, *rope, positions, n_rows, Hq, Hkv);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  const NormRope p = {q, k, q_weight, k_weight, q_out, k_out, eps};
  return cuda_status(launch_norm_mrope(a, p, dtype, d, rope->pairing == VC_ROPE_ADJACENT,
                                       static_cast<cudaStream_t>(stream)));
}

size_t viscache_norm_mrope_grad_workspace_size(int64_t n_rows, int32_t Hq, int32_t Hkv, int32_t d) {
  if (n_rows < 0 || n_rows > (1 << 24) || Hq < 0 || Hkv < 0 || Hq > 4096 || Hkv > 4096 || (d != 64 && d != 128))
    return 0;
  return align_up(sizeof(float) * kNormGradBlocks * d);
}

int viscache_norm_mrope_grad(const vc_rope* rope, const int32_t* positions, int dtype, int64_t n_rows, int32_t Hq,
                             int32_t Hkv, int32_t d, const void* q, int64_t q_stride, const void* k,
                             int64_t k_stride, const void* q_out_grad, int64_t q_out_grad_stride,
                             const void* k_out_grad, int64_t k_out_grad_stride, const void* q_weight,
                             const void* k_weight, float eps, void* q_grad, int64_t q_grad_stride, void* k_grad,
                             int64_t k_grad_stride, float* q_weight_grad, float* k_weight_grad, void* ws,
                             size_t ws_bytes, void* stream) {
  RopeArgs a = {};
  if (!valid_rope(rope, dtype, n_rows, Hq, Hkv, d) || !valid_eps(eps)) return VC_ERR_INVALID_ARG;
  if ((Hq > 0 && (!q_weight_grad || !aligned16(q_weight_grad))) ||
      (Hkv > 0 && (!k_weight_grad || !aligned16(k_weight_grad))))
    return VC_ERR_INVALID_ARG;
  if (n_rows > 0) {
    if (!positions) return VC_ERR_INVALID_ARG;
    if (!valid_rows(q, q_stride, Hq, d, dtype) || !valid_rows(q_out_grad, q_out_grad_stride, Hq, d, dtype) ||
        !valid_rows(q_grad, q_grad_stride, Hq, d, dtype) || !valid_rows(k, k_stride, Hkv, d, dtype) ||
        !valid_rows(k_out_grad, k_out_grad_stride, Hkv, d, dtype) ||
        !valid_rows(k_grad, k_grad_stride, Hkv, d, dtype) || !valid_rows(q_weight, d, Hq > 0, d, dtype) ||
        !valid_rows(k_weight, d, Hkv > 0, d, dtype))
      return VC_ERR_INVALID_ARG;
  }
  const int wc = check_ws(ws, ws_bytes, viscache_norm_mrope_grad_workspace_size(n_rows, Hq, Hkv, d));
  if (wc != VC_OK) return wc;
  if (Hq + Hkv == 0) return VC_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n_rows == 0) {
    cudaError_t e = Hq > 0 ? cudaMemsetAsync(q_weight_grad, 0, sizeof(float) * d, st) : cudaSuccess;
    if (e == cudaSuccess && Hkv > 0) e = cudaMemsetAsync(k_weight_grad, 0, sizeof(float) * d, st);
    return cuda_status(e);
  }
  set_rope(a, *rope, positions, n_rows, Hq, Hkv);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_grad_stride;
  a.k_out_stride = k_grad_stride;
  a.inverse = 1;
  NormRopeGrad p = {q, k, q_out_grad, k_out_grad, q_weight, k_weight, q_grad, k_grad, q_out_grad_stride,
                    k_out_grad_stride, static_cast<float*>(ws), eps, 0};
  return cuda_status(launch_norm_mrope_grad(a, p, dtype, d, rope->pairing == VC_ROPE_ADJACENT,
                                            Hq > 0 ? q_weight_grad : nullptr, Hkv > 0 ? k_weight_grad : nullptr, st));
}

size_t viscache_kv8_workspace_size(int32_t n_rows, int32_t Hq, int32_t Hkv, int32_t d) {
  if (n_rows < 0 || n_rows > (1 << 24) || !valid_heads(Hq, Hkv) || (d != 64 && d != 128)) return 0;
  return kv8_ws(may_have_many_rows(n_rows, 1, Hq, Hkv), d).total;
}

int viscache_kv8_append(const vc_kv8* cache, const vc_kv8_step* step, int dtype, const void* K,
                        int64_t k_row_stride, int64_t k_head_stride, const void* V, int64_t v_row_stride,
                        int64_t v_head_stride, void* ws, size_t ws_bytes, void* stream) {
  const Kv8Rows rows = {const_cast<void*>(K), const_cast<void*>(V), k_row_stride, k_head_stride, v_row_stride,
                        v_head_stride};
  return kv8_rows_call(true, cache, step, dtype, rows, ws, ws_bytes, stream);
}

int viscache_kv8_read(const vc_kv8* cache, const vc_kv8_step* step, int dtype, void* K_hat, void* V_hat,
                      void* ws, size_t ws_bytes, void* stream) {
  if (!cache) return VC_ERR_INVALID_ARG;
  const int64_t row = (int64_t)cache->Hkv * cache->d;
  const Kv8Rows rows = {K_hat, V_hat, row, cache->d, row, cache->d};
  return kv8_rows_call(false, cache, step, dtype, rows, ws, ws_bytes, stream);
}

int viscache_kv8_attention(const vc_kv8* cache, const vc_kv8_step* step, int dtype, int32_t Hq, const void* q,
                           int64_t q_stride, float scale, int causal, void* out, float* lse, void* ws,
                           size_t ws_bytes, void* stream) {
  if (!valid_cache(cache) || !valid_step(cache, step) || !valid_type(dtype)) return VC_ERR_INVALID_ARG;
  if (!valid_heads(Hq, cache->Hkv) || (int64_t)step->n_rows * Hq >= (int64_t)1 << 31) return VC_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !isfinite(scale)) return VC_ERR_INVALID_ARG;
  if (step->n_rows > 0 && (!q || !out || !aligned16(q) || !aligned16(out) ||
                           !valid_stride(q_stride, (int64_t)Hq * cache->d, dtype)))
    return VC_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return VC_ERR_INVALID_ARG;
  if (!short_line(*cache, *step, Hq)) return VC_ERR_UNSUPPORTED;
  const Kernel kernel = kernel_of(*cache, *step, dtype, Hq);
  const Kv8Ws w = kv8_ws(kernel != Kernel::kMma, cache->d);
  const int wc = check_ws(ws, ws_bytes, w.total);
  if (wc != VC_OK) return wc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* base = static_cast<uint8_t*>(ws);
  if (step->n_rows == 0) return cuda_status(cudaMemsetAsync(base, 0, sizeof(int32_t), st));
  Kv8AttnArgs a = {};
  a.q = q;
  a.q_stride = q_stride;
  a.out = out;
  a.lse = lse;
  a.Hq = Hq;
  a.causal = causal != 0;
  a.scale_log2 = (scale == 0.f ? 1.0f / sqrtf((float)cache->d) : scale) * kLog2e;
  a.status = reinterpret_cast<int32_t*>(base);
  a.block_status = reinterpret_cast<int32_t*>(base + w.o_blocks);
  a.token = next_token();
  a.flags = reinterpret_cast<uint64_t*>(base + w.o_flags);
  a.part_ml = reinterpret_cast<float2*>(base + w.o_ml);
  a.part_o = reinterpret_cast<float*>(base + w.o_o);
  return cuda_status(kernel == Kernel::kMma   ? launch_kv8_attn_mma(*cache, *step, dtype, a, st)
                     : kernel == Kernel::kTc1 ? launch_kv8_attn_tc1(*cache, *step, dtype, a, st)
                                              : launch_kv8_attn_tc2(*cache, *step, a, st));
}

int viscache_kv8_weigh(const vc_kv8* cache, const vc_kv8_step* step, int dtype, int32_t Hq, const void* q,
                       int64_t q_stride, const float* lse, float scale, int causal, float* weights, void* ws,
                       size_t ws_bytes, void* stream) {
  if (!valid_cache(cache) || !valid_step(cache, step) || !valid_type(dtype)) return VC_ERR_INVALID_ARG;
  if (!valid_heads(Hq, cache->Hkv) || (int64_t)step->n_rows * Hq >= (int64_t)1 << 31) return VC_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || !isfinite(scale) || !weights || !aligned16(weights)) return VC_ERR_INVALID_ARG;
  if (step->n_rows > 0 && (!q || !aligned16(q) || !valid_stride(q_stride, (int64_t)Hq * cache->d, dtype) || !lse ||
                           (reinterpret_cast<uintptr_t>(lse) & 3u) != 0))
    return VC_ERR_INVALID_ARG;
  if (!short_line(*cache, *step, Hq)) return VC_ERR_UNSUPPORTED;
  const Kv8Ws w = kv8_ws(false, cache->d);      // (the outputs' place, 16 rows of d a piece, holds the sums of 384 tokens)
  const int wc = check_ws(ws, ws_bytes, w.total);
  if (wc != VC_OK) return wc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* base = static_cast<uint8_t*>(ws);
  if (step->n_rows == 0) return cuda_status(cudaMemsetAsync(base, 0, sizeof(int32_t), st));
  Kv8WeighArgs a = {};
  a.q = q;
  a.q_stride = q_stride;
  a.lse = lse;
  a.weights = weights;
  a.Hq = Hq;
  a.causal = causal != 0;
  // (a step there holds all heads of a group: 128 fit in both types)
  const bool many = (int64_t)step->n_rows * (Hq / cache->Hkv) > (dtype == VC_F32 ? kWeighTcRowsF32 : kWeighTcRows) * step->n_req &&
                    Hq / cache->Hkv <= 128;
  const double exact = scale == 0.f ? 1.0 / sqrt((double)cache->d) : (double)scale;
  const double cut = kWeighCut[many][dtype == VC_F32][cache->d == 128] * 0x1p-24;
  a.scale = (float)fmin(exact * (1.0 + cut), 3.4028234663852886e38);
  constexpr double kLog2eExact = 1.4426950408889634074;
  a.scale_log2 = (float)(exact * kLog2eExact);
  const double factor = exact > 0.0 ? (double)a.scale_log2 / exact * (1.0 - cut) : kLog2eExact;
  a.lse_log2 = (float)factor;
  a.lse_log2_lo = (float)(factor - (double)a.lse_log2);
  a.status = reinterpret_cast<int32_t*>(base);
  a.block_status = reinterpret_cast<int32_t*>(base + w.o_blocks);
  a.token = next_token();
  a.flags = reinterpret_cast<uint64_t*>(base + w.o_flags);
  a.part = reinterpret_cast<float*>(base + w.o_o);
  return cuda_status(many ? launch_kv8_weigh_tc(*cache, *step, dtype, a, st)
                          : launch_kv8_weigh(*cache, *step, dtype, a, st));
}

size_t viscache_kv8_evict_workspace_size(int32_t n_req, int32_t Hkv) {
  if (n_req < 1 || n_req > 1024 || Hkv < 1 || Hkv > 1024) return 0;
  return kAlign + align_up(sizeof(Kv8Unit) * n_req * Hkv);
}

int viscache_kv8_evict(const vc_kv8* cache, const vc_kv8_step* step, float* weights, const int32_t* keep,
                       int32_t max_keep, int32_t sink, int32_t recent, int32_t* kept, int32_t* new_lens, void* ws,
                       size_t ws_bytes, void* stream) {
  if (!valid_cache(cache) || !valid_step(cache, step)) return VC_ERR_INVALID_ARG;
  if (!weights || !aligned16(weights) || !keep || !kept || !new_lens) return VC_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(keep) | reinterpret_cast<uintptr_t>(kept) |
        reinterpret_cast<uintptr_t>(new_lens)) & 3u) != 0)
    return VC_ERR_INVALID_ARG;
  if (max_keep < 1 || max_keep > (1 << 30) || sink < 0 || recent < 0) return VC_ERR_INVALID_ARG;
  const int wc = check_ws(ws, ws_bytes, viscache_kv8_evict_workspace_size(step->n_req, cache->Hkv));
  if (wc != VC_OK) return wc;
  uint8_t* base = static_cast<uint8_t*>(ws);
  const Kv8EvictArgs a = {weights, keep, max_keep, sink, recent, kept, new_lens, reinterpret_cast<int32_t*>(base),
                          reinterpret_cast<Kv8Unit*>(base + kAlign)};
  return cuda_status(launch_kv8_evict(*cache, *step, a, static_cast<cudaStream_t>(stream)));
}

int viscache_sample(int dtype, int64_t n_rows, int64_t vocab, const void* logits, int64_t stride, const float* u,
                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                    int32_t* token, float* logprob, void* stream) {
  if (!valid_type(dtype) || n_rows < 0 || n_rows > 65535 || vocab < 1 || vocab > kSampleMaxVocab)
    return VC_ERR_INVALID_ARG;
  if (stride < vocab || stride >= (int64_t)1 << 40) return VC_ERR_INVALID_ARG;
  if (n_rows == 0) return VC_OK;
  if (!logits || !u || !temperature || !token) return VC_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(logits) & (dtype == VC_BF16 ? 1u : 3u)) != 0) return VC_ERR_INVALID_ARG;
  const void* words[] = {u, temperature, top_k, top_p, min_p, token, logprob};
  for (const void* w : words)
    if ((reinterpret_cast<uintptr_t>(w) & 3u) != 0) return VC_ERR_INVALID_ARG;
  SampleArgs a = {logits, stride, vocab, u, temperature, top_p, min_p, top_k, token, logprob, 47, 1, 0};
  while ((uint64_t)vocab > ((uint64_t)1 << 62) >> a.q) --a.q;
  return cuda_status(launch_sample(a, dtype, n_rows, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
