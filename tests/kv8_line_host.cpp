// Host check of the sharing of work over the 8-bit cache (csrc/kv8_line.cuh): each tile of
// each unit is walked over exactly once, in range, for any lengths, rows and grids.
//
// Reads batches from standard input, one a line:
//   kind Hkv G causal page grid n_req  len m  len m ...
// (kind 0 .. 3: the lines below), prints "ok" or what is wrong for each.
#include <stdint.h>

#include <algorithm>
#include <iostream>
#include <map>
#include <sstream>
#include <string>
#include <tuple>
#include <vector>

#include "viscache.h"

#define __device__
#define __forceinline__ inline
static struct {
  int x;
} blockIdx, gridDim;
using std::max;
using std::min;

namespace vc {
namespace kv8 {
struct Req8 {
  int row0, m, len;
};
struct Batch {
  int n_req;
  std::vector<Req8> req;
};
inline void set_status(int32_t* status, int32_t code) {
  if (*status == VC_OK) *status = code;
}
struct Outside {};
inline Req8 load_req(const Batch& s, int, int r, int32_t*) {
  if (r < 0 || r >= s.n_req) throw Outside{};
  return s.req[r];
}
}  // namespace kv8
}  // namespace vc

#include "kv8_line.cuh"

using namespace vc::kv8;

template <typename L>
static std::string run(const L& line, const Batch& s, int grid) {
  std::ostringstream bad;
  std::map<std::tuple<int, int, int, int>, int> seen;
  std::vector<int64_t> upto{0};
  int64_t want = 0;
  for (int r = 0; r < s.n_req; ++r) {
    const int64_t n = line.request_tiles(s.req[r]);
    int64_t sum = 0;
    for (int rt = 0; rt < line.row_tiles(s.req[r]); ++rt) {
      const int tiles = line.tiles(line.keys(s.req[r], rt));
      if (tiles < 1) return "a unit without tiles";
      sum += tiles;
    }
    if (sum != n) {
      bad << "request " << r << ": " << n << " tiles on the line, " << sum << " in its units";
      return bad.str();
    }
    upto.push_back(upto.back() + line.Hkv * n);
    want += line.Hkv * sum;
  }
  gridDim.x = grid;
  for (int b = 0; b < grid; ++b) {
    blockIdx.x = b;
    Share sh = {};
    set_range(sh, upto.back());
    if (sh.begin >= sh.end) continue;
    int r = 0;
    while (!(sh.begin >= upto[r] && sh.begin < upto[r + 1])) ++r;
    int32_t status = VC_OK;
    set_first(line, sh, sh.begin, upto[r], r, s.req[r], &status);
    Walk w;
    w.start(sh);
    int64_t tiles = 0;
    do {
      const Req8& q = s.req[w.u.r];
      if (w.u.q.len != q.len || w.u.q.m != q.m || w.u.rt < 0 || w.u.rt >= line.row_tiles(q) || w.u.g < 0 ||
          w.u.g >= line.Hkv || w.t0 < 0 || w.t1 <= w.t0 || w.t1 > w.u.tiles ||
          w.u.tiles != line.tiles(line.keys(q, w.u.rt)))
        return "a place that is none";
      const int first = w.first_block(sh), last = w.last_block(sh);
      if (first < 0 || last >= grid || b < first || b > last || w.whole() != (first == last)) return "a piece of another block's";
      for (int t = w.t0; t < w.t1; ++t) ++seen[{w.u.r, w.u.rt, w.u.g, t}];
      tiles += w.t1 - w.t0;
      if (tiles > sh.end - sh.begin) return "more tiles than the share has";
    } while (w.next(line, s, &status));
    if (status != VC_OK) return "a status";
    if (tiles != sh.end - sh.begin) return "fewer tiles than the share has";
  }
  if ((int64_t)seen.size() != want) return "a tile that nobody takes";
  for (const auto& x : seen)
    if (x.second != 1) return "a tile taken twice";
  return "ok";
}

int main() {
  std::string text;
  while (std::getline(std::cin, text)) {
    std::istringstream in(text);
    int kind, Hkv, G, causal, page, grid, row0 = 0;
    Batch s;
    in >> kind >> Hkv >> G >> causal >> page >> grid >> s.n_req;
    for (int r = 0; r < s.n_req; ++r) {
      Req8 q;
      in >> q.len >> q.m;
      q.row0 = row0;
      row0 += q.m;
      s.req.push_back(q);
    }
    std::string out;
    try {
      switch (kind) {
        case 0: out = run(Line<16, 64>{Hkv, G, page, causal}, s, grid); break;
        case 1: out = run(Line<256, 128>{Hkv, G, page, causal}, s, grid); break;
        case 2: out = run(Steps<256, 384>{Hkv, 256 / G, page, causal}, s, grid); break;
        default: out = run(Steps<128, 384>{Hkv, 128 / G, page, causal}, s, grid); break;
      }
    } catch (const Outside&) {
      out = "a request past the last is read";
    }
    std::cout << out << std::endl;
  }
}
