// The steps of a batch's tiles, dealt out evenly: used by the latent attention
// kernels, absorbed and expanded.
//
// A tile is some consecutive query rows of one sequence, a step 64 keys of a
// tile.  The steps of all tiles, sequence after sequence, are numbered through,
// and share c of them is c * per .. (c + 1) * per - 1, whatever lengths the
// sequences have, so a batch of ragged contexts ends everywhere at once, and a
// prompt's early tiles count as the few steps they are.  Lengths are on the
// device: every wave forms the numbering of its share itself.
#pragma once

#include "msa_common.h"

namespace {

using namespace msa;

namespace steps {

constexpr int kKeys = 64;                // keys per step

struct TileGeom {
  int q_begin, q_rows, kv_len;
};
__device__ __forceinline__ TileGeom tile_geom(const msa_seqs& sq, int s) {
  const SeqGeom g = seq_geom(sq, s);
  TileGeom t;
  t.q_begin = g.q_begin;
  t.q_rows = static_cast<int>(max<int64_t>(0, min<int64_t>(min(g.q_rows, sq.max_q_rows), sq.total_q_rows - g.q_begin)));
  t.kv_len = min(g.kv_len, sq.max_kv_len);
  return t;
}
// Steps that tile x of a sequence is numbered with: those of its last row, at
// least one.  `ahead` keys lie before the sequence's first row.
struct TileSteps {
  int64_t ahead;
  int last_steps, tiles, rows;
  __device__ __forceinline__ TileSteps(const TileGeom& g, int rows_per_tile) {
    ahead = max(g.kv_len - g.q_rows, 0);
    last_steps = max(1, (g.kv_len + kKeys - 1) / kKeys);
    tiles = (g.q_rows + rows_per_tile - 1) / rows_per_tile;
    rows = rows_per_tile;
  }
  __device__ __forceinline__ int64_t one(int64_t x) const {        // of a tile that is not the last
    return (ahead + (x + 1) * rows + kKeys - 1) >> 6;
  }
  __device__ __forceinline__ int64_t of(int x) const { return x < tiles - 1 ? one(x) : last_steps; }
  // of tiles 0 .. x - 1, x < tiles: the sum of floor((a + y rows) / 64), y < x
  __device__ __forceinline__ int64_t before(int64_t x) const {
    const int64_t a = ahead + rows + kKeys - 1;
    if ((rows & (kKeys - 1)) == 0) return x * (a >> 6) + (rows >> 6) * (x * (x - 1) / 2);
    if ((rows & (rows - 1)) == 0) {      // floor((a + y rows) / 64) = floor((floor(a / rows) + y) / m), m = 64 / rows
      const int lg = 31 - __clz(rows), lm = 6 - lg;
      auto below = [&](int64_t n) {      // the sum of floor(i / m), i < n
        const int64_t q = n >> lm;
        return ((q * (q - 1) / 2) << lm) + q * (n & ((1 << lm) - 1));
      };
      return below((a >> lg) + x) - below(a >> lg);
    }
    // one(y + 64) = one(y) + rows
    const int64_t q = x >> 6;
    const int r = static_cast<int>(x & 63);
    int64_t part = 0, all = 0;
    for (int y = 0; y < (q > 0 ? 64 : r); ++y) {
      const int64_t c = one(y);
      all += c;
      if (y < r) part += c;
    }
    return q * all + 64 * rows * (q * (q - 1) / 2) + part + static_cast<int64_t>(r) * rows * q;
  }
  __device__ __forceinline__ int64_t total() const { return tiles < 1 ? 0 : before(tiles - 1) + last_steps; }
};

__device__ __forceinline__ int64_t scan_incl(int64_t v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const int64_t x = __shfl_up(static_cast<long long>(v), d);
    if (lane_id() >= d) v += x;
  }
  return v;
}

__device__ __forceinline__ int64_t last_lane(int64_t v) {
  return static_cast<int64_t>(readlane_u64(static_cast<uint64_t>(v), kWave - 1));
}

// A share's steps, tile by tile (the same in every lane):
//   for (Share sh(...); sh.more(); sh.next()): steps begin() .. end() - 1 of tile x of sequence s.
struct Share {
  const msa_seqs& sq;
  int rows, range;                       // query rows per tile; which share
  int64_t per, u, u_end;                 // steps per share; this share's that are left
  int s = 0, x = 0;
  TileGeom g{};
  TileSteps ts;
  int64_t tile_first = 0;                // first step of the tile

  __device__ __forceinline__ Share(const msa_seqs& seqs, int rows_per_tile, int ranges, int min_steps, int which)
      : sq(seqs), rows(rows_per_tile), range(which), ts(TileGeom{}, 1) {
    struct Chunk {
      int64_t incl;                      // steps up to and of sequence 64 c + lane
    };
    auto chunk = [&](int c) {
      const int i = 64 * c + lane_id();
      return Chunk{scan_incl(i < sq.num_seqs ? TileSteps(tile_geom(sq, i), rows).total() : 0)};
    };
    const int chunks = (sq.num_seqs + 63) >> 6;
    Chunk ch = chunk(0);
    int64_t total = last_lane(ch.incl);
    for (int c = 1; c < chunks; ++c) total += last_lane(chunk(c).incl);
    per = max<int64_t>(min_steps, (total + ranges - 1) / ranges);
    u = range * per;
    u_end = min(u + per, total);
    if (u >= u_end) return;
    int64_t base = 0;
    for (int c = 0;; ++c) {
      if (c > 0) ch = chunk(c);
      const int64_t all = last_lane(ch.incl);
      if (u < base + all) {
        const int j = __popcll(__ballot(u >= base + ch.incl));   // sequences that end before u
        s = 64 * c + j;
        tile_first = base + (j > 0 ? static_cast<int64_t>(readlane_u64(static_cast<uint64_t>(ch.incl), j - 1)) : 0);
        break;
      }
      base += all;
    }
    g = tile_geom(sq, s);
    ts = TileSteps(g, rows);
    if (ts.tiles > 1) {
      int lo = 0, hi = ts.tiles - 1;
      const bool closed = (rows & (rows - 1)) == 0 || (rows & (kKeys - 1)) == 0;
      // else as TileSteps::before, the sums within a period of 64 tiles one per lane
      const int64_t incl = closed ? 0 : scan_incl(ts.one(lane_id()));
      const int64_t all = last_lane(incl);
      auto before = [&](int y) {
        if (closed) return ts.before(y);
        const int64_t k = y >> 6;
        const int r = y & 63;
        const int64_t part = r > 0 ? static_cast<int64_t>(readlane_u64(static_cast<uint64_t>(incl), r - 1)) : 0;
        return k * all + 64 * rows * (k * (k - 1) / 2) + part + static_cast<int64_t>(r) * rows * k;
      };
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tile_first + before(mid) <= u) lo = mid; else hi = mid - 1;
      }
      x = lo;
      tile_first += before(x);
    }
  }
  __device__ __forceinline__ bool more() const { return u < u_end; }
  __device__ __forceinline__ int64_t begin() const { return u - tile_first; }
  __device__ __forceinline__ int64_t end() const { return min(ts.of(x), begin() + (u_end - u)); }
  // shares that have steps of this tile, from this one (which has its first) to that of its `visits`-th
  __device__ __forceinline__ int parts(int visits) const {
    return static_cast<int>((tile_first + visits - 1) / per) - range + 1;
  }
  __device__ __forceinline__ void next() {
    u += end() - begin();
    if (u >= u_end) return;
    tile_first += ts.of(x);
    if (++x == ts.tiles) {
      x = 0;
      do {
        g = tile_geom(sq, ++s);
      } while (g.q_rows < 1);            // steps are left, so a sequence with rows follows
      ts = TileSteps(g, rows);
    }
  }
};

}  // namespace steps
}  // namespace
