// How the attention kernels over the 8-bit cache share out their work.
//
// A unit is (request, row tile, KV head): MT consecutive packed rows of a
// request's group of query heads (row rho = i * G + j is query head j of the
// group at the request's row i) over the tiles of KT keys that any of them
// sees, at least one tile.  The units' tiles, in order of request, row tile,
// KV head, form one line (kv8_line.cuh) of T tiles; block i of N takes tiles
// of it in turn, T / N of them and one more for the first T % N blocks.  So every
// block has the same number of tiles whatever the lengths are, a long unit is split over blocks, and a
// block's piece of a unit is a "segment".  A segment that is not a whole unit
// leaves its partial sums in the workspace (at most two a block: the end of
// the unit before, the start of the one after); the block that finishes a
// unit's last segment adds them up in order.  Lengths are read on the device.
//
// Where the units are no more than the blocks (few requests), no block takes two:
// every unit gets whole blocks, ceil(tiles / per) of them with the least `per` that
// the blocks allow, if that is no more than kEndTiles above an equal share, since a
// segment's end costs as much as several tiles.  Us on the line / in whole blocks,
// 152 blocks: 24 units of 6 to 25 tiles 17.5 / 12.8, 144 of 8 to 32 31.6 / 29.7,
// 128 of 16 to 64 43.6 / 47.8, 128 of 64 to 256 116 / 152.
#pragma once

#include <cuda.h>

#include "kernels.h"
#include "kv8.cuh"
#include "kv8_line.cuh"

namespace vc {

// Tensor map of a pool's codes: rows of d bytes, a box is a page's rows of one
// head, swizzled over whole rows (128 bytes at d = 128, 64 at d = 64).
bool kv8_pool_map(CUtensorMap* m, const void* base, const vc_kv8& c);
// Tensor map of bf16 query rows [n_rows][Hq][d], `stride` elements between rows: a box is 64
// dimensions of `heads` heads (at most 256) of `rows` rows, swizzled over 128 bytes.
bool kv8_rows_map(CUtensorMap* m, const void* q, int64_t n_rows, int Hq, int d, int64_t stride, int heads, int rows);

namespace kv8 {

// What a segment's end costs, in tiles: measured on the few-rows kernel (the figures
// above), taken for the others too, whose tiles and ends both take longer.
constexpr int kEndTiles = 16;

// A split unit's pieces meet in the workspace without counters that would have
// to be cleared: a block that has stored its piece sets the piece's flag to the
// call's token, and then looks at the flags of all of the unit's pieces.  With a
// sequentially consistent fence between the two, the last block to set one sees
// them all; a block that sees them all adds the pieces up (two may: they write
// the same values) and clears the flags, so that a replayed graph, whose token
// is the same, finds them clear.  One warp calls it, after a barrier behind the
// block's stores.
__device__ __forceinline__ bool piece_done(uint64_t* flags, int step, uint64_t token, int first, int final) {
  const int lane = threadIdx.x & 31, n = final - first + 1;
  // block b's piece is its second (the unit's first) for b == first, else its first
  auto flag = [&](int k) -> volatile uint64_t* { return flags + (2 * (first + k) + (k == 0 ? 1 : 0)) * step; };
  __threadfence();
  if (lane == 0) *flag((int)blockIdx.x - first) = token;
  __threadfence();
  __syncwarp();
  bool all = true;
  for (int k = lane; k < n; k += 32) all = all && *flag(k) == token;
  all = __all_sync(0xffffffffu, all);
  if (all)
    for (int k = lane; k < n; k += 32) *flag(k) = 0;
  __threadfence();
  return all;
}

// The block's status, and that the status is the blocks'.
__device__ __forceinline__ void store_status(const Kv8AttnArgs& a, int32_t err) {
  a.block_status[blockIdx.x] = err;
  if (blockIdx.x == 0) {
    a.status[0] = kStatusPerBlock;
    a.status[1] = (int32_t)gridDim.x;
  }
}

template <typename Int>
__device__ __forceinline__ Int scan_warp(Int x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Int y = __shfl_up_sync(0xffffffffu, x, o);
    if ((int)(threadIdx.x & 31) >= o) x += y;
  }
  return x;
}

// Computes the block's share with all of the block's NT threads; `sh` and
// `scan` (one word a warp) are in shared memory.  Up to 32 requests: one warp,
// a request a lane.  More: each thread counts the tiles of consecutive
// requests, and a scan over the block places them on the line.  The thread
// whose requests hold the first tile of the share looks it up.  Ends with a
// barrier.
template <int NT, typename L>
__device__ __forceinline__ void find_share(const L& line, const vc_kv8_step& s, int32_t* status,
                                           Share& sh, int64_t* scan) {
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  if (s.n_req <= 32) {
    if (warp == 0) {
      const Req8 q = lane < s.n_req ? load_req(s, line.page, lane, status) : Req8{0, 0, 0};
      const int N = gridDim.x, rts = line.row_tiles(q);
      // (at most 32 (N + 1) if none is over N: no overflow)
      const int units = __reduce_add_sync(0xffffffffu, min(rts, N + 1) * min(line.Hkv, N + 1));
      int per = 0, mine = 0, before = 0;
      bool pieces = units <= N;
      if (pieces) {
        // pieces of at most `per` tiles; a unit has at most 2^23 tiles, N units fewer than 2^31
        int w = 0;
        for (int rt = 0; rt < rts; ++rt) w += line.Hkv * line.tiles(line.keys(q, rt));
        const int share = (__reduce_add_sync(0xffffffffu, w) + N - 1) / N;
        for (per = share;;) {
          mine = 0;
          for (int rt = 0; rt < rts; ++rt) mine += line.Hkv * ((line.tiles(line.keys(q, rt)) + per - 1) / per);
          before = scan_warp(mine) - mine;
          if (__shfl_sync(0xffffffffu, before + mine, 31) <= N) break;
          per += per / 8 + 1;
        }
        pieces = per <= share + kEndTiles;
      }
      if (pieces) {
        const int i = blockIdx.x;
        if (lane == 31) {
          sh.begin = 0;
          sh.end = i < before + mine ? 1 : 0;   // whether there is anything to do
        }
        if (i >= before && i < before + mine) {
          Unit u;
          u.r = lane;
          u.rt = 0;
          u.q = q;
          int at = i - before, k;               // the place among the request's blocks
          for (;; ++u.rt) {
            line.set(u);
            k = (u.tiles + per - 1) / per;
            if (at < line.Hkv * k) break;
            if (u.rt + 1 >= rts) {              // (as in set_first)
              set_status(status, VC_ERR_DEVICE_INDEX);
              at = line.Hkv * k - 1;
              break;
            }
            at -= line.Hkv * k;
          }
          u.g = at / k;
          sh.u = u;
          sh.pieces = k;
          sh.piece = at - u.g * k;
        }
      } else {
        const int64_t w = line.Hkv * line.request_tiles(q);
        const int64_t upto = scan_warp(w);
        Share x;
        set_range(x, __shfl_sync(0xffffffffu, upto, 31));
        if (lane == 0) {
          sh.begin = x.begin;
          sh.end = x.end;
          sh.per = x.per;
          sh.more = x.more;
          sh.pieces = 0;
        }
        if (x.begin < x.end && x.begin >= upto - w && x.begin < upto) set_first(line, sh, x.begin, upto - w, lane, q, status);
      }
    }
    __syncthreads();
    return;
  }
  const int per = (s.n_req + NT - 1) / NT;
  const int ra = min(t * per, s.n_req), rb = min(ra + per, s.n_req);
  int64_t sum = 0;
  for (int r = ra; r < rb; ++r) sum += line.Hkv * line.request_tiles(load_req(s, line.page, r, status));
  const int64_t upto = scan_warp(sum);
  if (lane == 31) scan[warp] = upto;
  __syncthreads();
  int64_t T = 0, before = 0;
  for (int w = 0; w < NT / 32; ++w) {
    if (w < warp) before += scan[w];
    T += scan[w];
  }
  Share x;
  set_range(x, T);
  if (t == 0) {
    sh.begin = x.begin;
    sh.end = x.end;
    sh.per = x.per;
    sh.more = x.more;
    sh.pieces = 0;
  }
  int64_t at = before + upto - sum;
  if (x.begin < x.end && x.begin >= at && x.begin < at + sum) {
    for (int r = ra; r < rb; ++r) {
      const Req8 q = load_req(s, line.page, r, status);
      const int64_t w = line.Hkv * line.request_tiles(q);
      if (x.begin < at + w) {
        set_first(line, sh, x.begin, at, r, q, status);
        break;
      }
      at += w;
    }
  }
  __syncthreads();
}

}  // namespace kv8
}  // namespace vc
