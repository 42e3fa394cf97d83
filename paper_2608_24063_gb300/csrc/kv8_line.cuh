// The lines that the kernels over the 8-bit cache share out (kv8_sched.cuh), and a
// block's walk over its share: whole numbers alone.  `S` is a step's device arrays with a
// load_req that reads them.  tests/test_kv8_line.py compiles this file for the host.
#pragma once

namespace vc {
namespace kv8 {

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
  // the next unit: there is one (request_tiles adds up what set gives)
  template <typename S>
  __device__ __forceinline__ bool next(const S& s, Unit& u, int32_t* status) const {
    if (++u.g < Hkv) return true;
    u.g = 0;
    if (++u.rt >= row_tiles(u.q)) {
      u.rt = 0;
      do {
        ++u.r;
        u.q = load_req(s, page, u.r, status);
      } while (u.q.m == 0 && u.r + 1 < s.n_req);
    }
    set(u);
    return true;
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

// The block's range of a line of T tiles.
__device__ __forceinline__ void set_range(Share& sh, int64_t T) {
  const int N = (int)(T < (int64_t)gridDim.x ? T : (int64_t)gridDim.x);
  const int i = blockIdx.x;
  sh.per = N > 0 ? divide(T, N) : 0;
  sh.more = (int)(T - sh.per * N);
  sh.begin = i < N ? i * sh.per + min(i, sh.more) : 0;
  sh.end = i < N ? sh.begin + sh.per + (i < sh.more ? 1 : 0) : 0;
}

// Finds the tile `begin` within request r, whose first tile is `at`.  Ends at the last
// row tile: a tile past it (a line longer than its units) would be an error, with status,
// looked at behind the loop (inside it the many-rows weighing kernel's registers come out
// otherwise: 2048 rows over 32768 tokens 934 us against 926).
template <typename L>
__device__ __forceinline__ void set_first(const L& line, Share& sh, int64_t begin, int64_t at, int r, const Req8& q,
                                          int32_t* status) {
  Unit u;
  u.r = r;
  u.rt = 0;
  u.q = q;
  const int rts = line.row_tiles(q);
  int64_t row;
  for (;; ++u.rt) {
    line.set(u);
    row = (int64_t)line.Hkv * u.tiles;
    if (begin < at + row || u.rt + 1 >= rts) break;
    at += row;
  }
  if (begin >= at + row) {
    set_status(status, VC_ERR_DEVICE_INDEX);
    at = begin - (row - 1);                     // (its last tile)
  }
  u.g = (int)divide(begin - at, u.tiles);
  sh.tile0 = at + (int64_t)u.g * u.tiles;
  sh.u = u;
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
  template <typename L, typename S>
  __device__ __forceinline__ bool next(const L& line, const S& s, int32_t* status) {
    left -= t1 - t0;
    if (left <= 0) return false;
    rel += u.tiles;
    if (!line.next(s, u, status)) return false;
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

// The line of steps: a unit's "row tile" is its group of K tiles, its "tiles" are the
// steps, RB = N / G request rows of all G heads of a group, that see any of it.
template <int N, int GROUP>
struct Steps {
  int Hkv, RB, page, causal;

  __device__ __forceinline__ int row_tiles(const Req8& q) const { return q.m > 0 ? (q.len + GROUP - 1) / GROUP : 0; }
  __device__ __forceinline__ int blocks(const Req8& q) const { return (q.m + RB - 1) / RB; }
  // the first step with a row that sees token t
  __device__ __forceinline__ int first_block(const Req8& q, int t) const {
    return causal ? max(0, t - (q.len - q.m)) / RB : 0;
  }
  __device__ __forceinline__ int keys(const Req8& q, int rt) const { return blocks(q) - first_block(q, rt * GROUP); }
  __device__ __forceinline__ int tiles(int steps) const { return steps; }
  __device__ __forceinline__ int64_t request_tiles(const Req8& q) const {
    const int n = row_tiles(q);
    // groups that start no later than the step's own tokens are seen by every row (where rows are more than
    // tokens the first ones see none)
    const int full = !causal ? n : q.len < q.m ? 0 : min(n, (q.len - q.m) / GROUP + 1);
    int64_t sum = (int64_t)full * blocks(q);
    for (int rt = full; rt < n; ++rt) sum += keys(q, rt);
    return sum;
  }
  __device__ __forceinline__ void set(Unit& u) const {
    u.kend = min(u.q.len - u.rt * GROUP, GROUP);      // tokens of the group
    u.tiles = keys(u.q, u.rt);
  }
  // the next unit; false where there is none, which no share asks for
  template <typename S>
  __device__ __forceinline__ bool next(const S& s, Unit& u, int32_t* status) const {
    if (++u.g < Hkv) return true;
    u.g = 0;
    if (++u.rt >= row_tiles(u.q)) {
      u.rt = 0;
      do {
        if (u.r + 1 >= s.n_req) {
          set_status(status, VC_ERR_DEVICE_INDEX);
          return false;
        }
        ++u.r;
        u.q = load_req(s, page, u.r, status);
      } while (row_tiles(u.q) == 0);
    }
    set(u);
    return true;
  }
};

}  // namespace kv8
}  // namespace vc
