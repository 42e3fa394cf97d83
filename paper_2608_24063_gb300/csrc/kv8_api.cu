// C entry points of the rotary positions and of the 8-bit paged cache
// (include/viscache.h): argument checks, workspace layout, launches.
#include <math.h>

#include <atomic>
#include <chrono>

#include "api_util.h"
#include "kernels.h"

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

bool valid_heads(int32_t Hq, int32_t Hkv) { return Hkv >= 1 && Hq >= Hkv && Hq <= 4096 && Hq % Hkv == 0; }

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
  if (!rope || !valid_type(dtype) || (d != 64 && d != 128)) return VC_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > (1 << 24) || Hq < 0 || Hkv < 0 || Hq > 4096 || Hkv > 4096) return VC_ERR_INVALID_ARG;
  if (rope->n_axes < 1 || rope->n_axes > 4 || !(rope->theta >= 1.0) || !isfinite(rope->theta))
    return VC_ERR_INVALID_ARG;
  if ((rope->order != VC_ROPE_SECTIONED && rope->order != VC_ROPE_INTERLEAVED) ||
      (rope->pairing != VC_ROPE_HALVES && rope->pairing != VC_ROPE_ADJACENT))
    return VC_ERR_INVALID_ARG;
  int64_t half = 0;
  for (int a = 0; a < rope->n_axes; ++a) {
    if (rope->sections[a] < 0 || rope->sections[a] > d / 2) return VC_ERR_INVALID_ARG;
    half += rope->sections[a];
  }
  if (half < 8 || half % 8 != 0 || half > d / 2) return VC_ERR_INVALID_ARG;
  RopeArgs a = {};
  for (int i = 0; i < (int)half; ++i) {
    if (rope->order == VC_ROPE_INTERLEAVED) {
      const int x = i % rope->n_axes;
      a.axis[i] = (uint8_t)(i < rope->n_axes * rope->sections[x] ? x : 0);
    } else {
      int x = 0;
      for (int upto = rope->sections[0]; i >= upto; upto += rope->sections[x]) ++x;
      a.axis[i] = (uint8_t)x;
    }
  }
  if (n_rows > 0) {
    if (!positions) return VC_ERR_INVALID_ARG;
    if (Hq > 0 && (!q || !q_out || !aligned16(q) || !aligned16(q_out) ||
                   !valid_stride(q_stride, (int64_t)Hq * d, dtype) ||
                   !valid_stride(q_out_stride, (int64_t)Hq * d, dtype)))
      return VC_ERR_INVALID_ARG;
    if (Hkv > 0 && (!k || !k_out || !aligned16(k) || !aligned16(k_out) ||
                    !valid_stride(k_stride, (int64_t)Hkv * d, dtype) ||
                    !valid_stride(k_out_stride, (int64_t)Hkv * d, dtype)))
      return VC_ERR_INVALID_ARG;
  }
  if (n_rows == 0 || Hq + Hkv == 0) return VC_OK;
  // theta^(-i / half) by one power, off by an ulp, and up to 63 products: within 2^-45
  const double r = pow(rope->theta, -1.0 / (double)half);
  double f = kInv2Pi;
  for (int i = 0; i < (int)half; ++i, f *= r) a.freq[i] = (uint64_t)(f * 18446744073709551616.0);
  a.positions = positions;
  a.n_rows = n_rows;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.half = (int32_t)half;
  a.inverse = inverse != 0;
  return cuda_status(launch_mrope(a, dtype, d, rope->pairing == VC_ROPE_ADJACENT, q, q_out, k, k_out,
                                  static_cast<cudaStream_t>(stream)));
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
  // the attention's line of key tiles (units of 8 rows at least): a block's
  // share is counted in 31 bits
  const int64_t row_tiles = (int64_t)step->n_rows * (Hq / cache->Hkv) / 8 + step->n_req;
  if (row_tiles * cache->Hkv > ((int64_t)1 << 37) / (((int64_t)step->max_pages * cache->page + 127) / 128))
    return VC_ERR_UNSUPPORTED;
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

}  // extern "C"
