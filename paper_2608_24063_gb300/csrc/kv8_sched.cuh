// How the attention kernels over the 8-bit cache share out their work.
//
// A unit is (request, row tile, KV head): MT consecutive packed rows of a
// request's group of query heads (row rho = i * G + j is query head j of the
// group at the request's row i) over the tiles of KT keys that any of them
// sees, at least one tile.  The units' tiles, in order of request, row tile,
// KV head, form one line of T tiles; block i of N takes tiles
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

namespace vc {

// Tensor map of a pool's codes: rows of d bytes, a box is a page's rows of one
// head, swizzled over whole rows (128 bytes at d = 128, 64 at d = 64).
bool kv8_pool_map(CUtensorMap* m, const void* base, const vc_kv8& c);

namespace kv8 {

// What a segment's end costs, in tiles: measured on the few-rows kernel (the figures
// above), taken for the others too, whose tiles and ends both take longer.
constexpr int kEndTiles = 16;

// Place in the line: a unit and the request's numbers.
struct Unit {
  int r, rt, g;          // request, row tile, KV head
  Req8 q;
  int tiles;             // key tiles of the unit
  int kend;              // keys its rows see (0 .. q.len)
};

template <int MT, int KT>
struct Line {
  int Hkv, G, page, causal;

  __device__ __forceinline__ int row_tiles(const Req8& q) const { return (q.m * G + MT - 1) / MT; }
  // keys that the rows of row tile rt see together
  __device__ __forceinline__ int keys(const Req8& q, int rt) const {
    if (!causal) return q.len;
    const int last = min(q.m - 1, ((rt + 1) * MT - 1) / G);
    return min(q.len, max(0, q.len - q.m + last + 1));
  }
  __device__ __forceinline__ int tiles(int kend) const { return max(1, (kend + KT - 1) / KT); }
  // tiles of a request's units for one KV head
  __device__ __forceinline__ int64_t request_tiles(const Req8& q) const {
    const int n = row_tiles(q);
    if (!causal) return (int64_t)n * tiles(q.len);
    int64_t sum = 0;
    for (int rt = 0; rt < n; ++rt) sum += tiles(keys(q, rt));
    return sum;
  }
  __device__ __forceinline__ void set(Unit& u) const {
    u.kend = keys(u.q, u.rt);
    u.tiles = tiles(u.kend);
  }
  // the next unit (there is one)
  __device__ __forceinline__ void next(const vc_kv8_step& s, Unit& u, int32_t* status) const {
    if (++u.g < Hkv) return;
    u.g = 0;
    if (++u.rt >= row_tiles(u.q)) {
      u.rt = 0;
      do {
        ++u.r;
        u.q = load_req(s, page, u.r, status);
      } while (u.q.m == 0 && u.r + 1 < s.n_req);
    }
    set(u);
  }
};

// a / b, in 32 bits where that holds it (the division of a few microseconds'
// call is felt)
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// A block's share of the line.
struct Share {
  int64_t begin, end;      // the block's range of the line
  int64_t per;             // tiles of a block, T / N
  int more;                // the first T % N blocks have one more
  int64_t tile0;           // the first unit's first tile on the line
  Unit u;                  // the first unit
  int pieces, piece;       // above 0: the block has this piece of that unit and no more

  // the block that holds tile x of the line
  __device__ __forceinline__ int block_of(int64_t x) const {
    const int64_t y = x - more * (per + 1);
    return y < 0 ? (int)divide(x, per + 1) : more + (int)divide(y, per);
  }
};

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

// A role's walk over the block's segments.  Positions are relative to the
// share's begin (a share is below 2^31 tiles: the host refuses longer lines).
struct Walk {
  Unit u;                // the segment's unit
  int t0, t1;            // its tiles of the unit
  int left;              // tiles of the share from t0 on
  int rel;               // the unit's first tile, from the share's begin

  __device__ __forceinline__ void start(const Share& sh) {
    u = sh.u;
    if (sh.pieces > 0) {
      rel = 0;
      t0 = u.tiles * sh.piece / sh.pieces;
      t1 = u.tiles * (sh.piece + 1) / sh.pieces;
      left = t1 - t0;
      return;
    }
    left = (int)(sh.end - sh.begin);
    rel = (int)(sh.tile0 - sh.begin);
    t0 = -rel;
    t1 = left < u.tiles - t0 ? t0 + left : u.tiles;
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == u.tiles; }
  // the next segment; false at the share's end
  template <typename L>
  __device__ __forceinline__ bool next(const L& line, const vc_kv8_step& s, int32_t* status) {
    left -= t1 - t0;
    if (left <= 0) return false;
    rel += u.tiles;
    line.next(s, u, status);
    t0 = 0;
    t1 = left < u.tiles ? left : u.tiles;
    return true;
  }
  // the blocks that hold the unit's first and last tile
  __device__ __forceinline__ int first_block(const Share& sh) const {
    return sh.pieces > 0 ? (int)blockIdx.x - sh.piece : sh.block_of(sh.begin + rel);
  }
  __device__ __forceinline__ int last_block(const Share& sh) const {
    return sh.pieces > 0 ? (int)blockIdx.x - sh.piece + sh.pieces - 1 : sh.block_of(sh.begin + rel + u.tiles - 1);
  }
};

template <typename Int>
__device__ __forceinline__ Int scan_warp(Int x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Int y = __shfl_up_sync(0xffffffffu, x, o);
    if ((int)(threadIdx.x & 31) >= o) x += y;
  }
  return x;
}

// The block's range of a line of T tiles.
__device__ __forceinline__ void set_range(Share& sh, int64_t T) {
  const int N = (int)(T < (int64_t)gridDim.x ? T : (int64_t)gridDim.x);
  const int i = blockIdx.x;
  sh.per = N > 0 ? divide(T, N) : 0;
  sh.more = (int)(T - sh.per * N);
  sh.begin = i < N ? i * sh.per + min(i, sh.more) : 0;
  sh.end = i < N ? sh.begin + sh.per + (i < sh.more ? 1 : 0) : 0;
}

// Finds the tile `begin` within request r, whose first tile is `at`.
template <int MT, int KT>
__device__ __forceinline__ void set_first(const Line<MT, KT>& line, Share& sh, int64_t begin, int64_t at, int r,
                                          const Req8& q) {
  Unit u;
  u.r = r;
  u.rt = 0;
  u.q = q;
  for (;; ++u.rt) {
    line.set(u);
    const int64_t row = (int64_t)line.Hkv * u.tiles;
    if (begin < at + row) break;
    at += row;
  }
  u.g = (int)divide(begin - at, u.tiles);
  sh.tile0 = at + (int64_t)u.g * u.tiles;
  sh.u = u;
}

// Computes the block's share with all of the block's NT threads; `sh` and
// `scan` (one word a warp) are in shared memory.  Up to 32 requests: one warp,
// a request a lane.  More: each thread counts the tiles of consecutive
// requests, and a scan over the block places them on the line.  The thread
// whose requests hold the first tile of the share looks it up.  Ends with a
// barrier.
template <int NT, int MT, int KT>
__device__ __forceinline__ void find_share(const Line<MT, KT>& line, const vc_kv8_step& s, int32_t* status,
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
        if (x.begin < x.end && x.begin >= upto - w && x.begin < upto) set_first(line, sh, x.begin, upto - w, lane, q);
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
        set_first(line, sh, x.begin, at, r, q);
        break;
      }
      at += w;
    }
  }
  __syncthreads();
}

}  // namespace kv8
}  // namespace vc
