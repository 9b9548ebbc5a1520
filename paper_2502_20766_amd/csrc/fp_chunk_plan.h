// How chunk_attn divides the keys of a batch among workgroups: whole-number arithmetic on lengths, for the
// kernels and, as it is, for programs on the host.
#pragma once

#include <algorithm>

#include "fp_internal.h"

#define FP_BOTH __host__ __device__ __forceinline__

namespace fp {
namespace {

constexpr int kMaxList = FP_MAX_CACHE_LIST;

// A workgroup: `WAVES` waves of 32 rows, key tiles of `TILE` keys.
template <int WAVES, int TILE>
struct Geo {
  static constexpr int THREADS = 64 * WAVES, ROWS = 32 * WAVES, KEYS = TILE;
  static_assert(THREADS >= kMaxList, "the plan has one thread per sequence");
};

// Key tiles that a segment takes of the line beside its own: the cost of starting and ending a piece.
constexpr int kSegCost = 2;
// Fewest key tiles of a part: less than a segment's, so that every short one gets a part of its own.
constexpr int kPartTiles = 3;
// Key tiles from a segment's start or end within which a cut moves there.
constexpr int kSnapTiles = 4;

// A segment: sequence, KV head, its number there, its places in the line.
struct Segment {
  int seq, head, seg;
  int64_t start, end;
};

// a / b for 0 <= a < 2^62 and b > 0 where the result is below 2^45: an estimate, off by one at most, by a
// reciprocal in float64.  (The division itself is a call's worth of instructions, and the plan has six.)
FP_BOTH int64_t divide(int64_t a, int64_t b) {
  const double y = (double)b;
#ifdef __HIP_DEVICE_COMPILE__
  double r = __builtin_amdgcn_rcp(y);
#else
  double r = 1.f / (float)b;
#endif
  r = fma(fma(-y, r, 1.0), r, r);
  r = fma(fma(-y, r, 1.0), r, r);
  int64_t q = (int64_t)((double)a * r);
  const int64_t rest = a - q * b;
  if (rest < 0) --q;
  else if (rest >= b) ++q;
  return q;
}

// A line of `total` places in `parts` equal parts, the first total % parts of them one place longer.
struct Cut {
  int64_t per, rem;
  FP_BOTH Cut(int64_t total, int parts) : per(divide(total, parts)) { rem = total - per * parts; }
  FP_BOTH int64_t begin(int p) const { return per * p + std::min((int64_t)p, rem); }
  FP_BOTH int owner(int64_t x) const {
    const int64_t longer = rem * (per + 1);
    return (int)(x < longer ? divide(x, per + 1) : rem + divide(x - longer, per));
  }
};

// A sequence's segments of one KV head: segment i takes fixed + (i + 1) * step places, the last one fixed +
// its rows.
template <class G>
struct Series {
  int64_t fixed;
  int step, n, rows;
  FP_BOTH Series(const ChunkArgs &a, int width, int m, int len) {
    const int span = width * G::ROWS;
    rows = m * a.G;
    n = (int)((uint32_t)(rows + span - 1) / (uint32_t)span);
    fixed = a.G * (int64_t)(G::KEYS * kSegCost + (len > 0 ? G::KEYS + std::max(len - m, 0) : 0));
    step = len > 0 ? span : 0;
    if (len == 0) rows = 0;
  }
  FP_BOTH int64_t begin(int i) const { return i * fixed + (int64_t)step * ((int64_t)i * (i + 1) / 2); }
  FP_BOTH int64_t end(int i) const { return i + 1 < n ? begin(i + 1) : begin(i) + fixed + rows; }
  FP_BOTH int64_t whole() const { return n > 0 ? end(n - 1) : 0; }
};

// Parts that a line of `total` places is cut into: one for each cluster of workgroups, fewer of short lines.
template <class G>
FP_BOTH int parts_of(const ChunkArgs &a, int64_t total) {
  const int64_t want = divide(total, kPartTiles * G::KEYS * (int64_t)a.G);
  return (int)std::min(std::max(want, (int64_t)1), (int64_t)(a.wgs / a.width));
}

struct Part {
  int p, tile;          // number of the part, row tile of its segments
  int width;            // row tiles of a segment
  int64_t lo, hi;       // places; lo >= hi: none
};

// The part of workgroup `block` and its row tile of the part's segments.  Every number below wgs / width has
// one workgroup of row tile 0, also where no part has it: that one writes the record of the number, and the
// join looks at all of them.
//
// Workgroups of one XCD (every eighth) take neighbouring parts; where there is not work for all, the
// clusters are dealt out over the XCDs, `room` to each.  What an XCD then has left over, fewer than `width`,
// takes the numbers from 8 * room on, which no part has.
FP_BOTH Part place_of(const ChunkArgs &a, int block, int parts) {
  const int x = block & 7, y = block >> 3, room = a.wgs / 8 / a.width;
  Part r = {a.wgs / a.width, 0, a.width, 0, 0};
  if (block >= a.wgs) return r;
  if (8 * parts * a.width > 7 * a.wgs || parts > 8 * room) {
    const int wg = x * (a.wgs / 8) + y;
    r.p = wg / a.width;
    r.tile = wg - r.p * a.width;
  } else {
    const int c = y / a.width;
    r.p = c * 8 + x;
    r.tile = y - c * a.width;
  }
  return r;
}

// A cut of the line in segment [start, end) of it: at `x`, or where that is near an end there, which
// leaves short segments whole and long ones no short pieces.
template <class G>
FP_BOTH int64_t snap(const ChunkArgs &a, int64_t x, int64_t start, int64_t end) {
  const int64_t near = (int64_t)kSnapTiles * G::KEYS * a.G;
  return x - start <= near ? start : end - x <= near ? end : x;
}

// The segment of sequence `seq`, whose places begin at `start`, in which place `at` lies.
template <class G>
FP_BOTH Segment segment_at(const Series<G> &series, int64_t whole, int seq, int64_t start, int64_t at) {
  const int64_t in = at - start, head = divide(in, whole), z = in - head * whole;
  int lo = 0, hi = series.n;                         // begin(lo) <= z < begin(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (series.begin(mid) <= z) lo = mid;
    else hi = mid;
  }
  return {seq, (int)head, lo, at - z + series.begin(lo), at - z + series.end(lo)};
}

// Where a piece's keys lie, as Loader needs it.
struct Source {
  int row;              // cache slot whose pages are read
  int head;             // KV head
  int key0, limit;      // keys: first, and the sequence's tokens
  int once;             // no other workgroup reads these keys
};

// A run of key tiles of one row tile in one workgroup; every field is wave-uniform.
struct Piece {
  Source src;
  int t0, t1;           // tiles [t0, t1) of its keys that this row tile sees
  int row0, rows;       // rows of the sequence and KV head: first, and how many (0: none)
  int vis;              // keys that the sequence's first query sees (may be negative)
  int here;             // the part has any of the segment's tiles, or its start if it has none
  int begins, ends;     // the part has the segment's first tile, its last
  int64_t last;         // last place of the segment's last tile
  Segment s;
};

// The piece of a segment, of a sequence of `len` tokens, in the workgroup's part.
template <class G>
FP_BOTH Piece piece_of(const ChunkArgs &a, const Segment &s, int len, const Part &part) {
  Piece r;
  r.s = s;
  const int m = a.cu[s.seq + 1] - a.cu[s.seq];
  const int rows = m * a.G, span = part.width * G::ROWS;
  r.src.row = a.slot[s.seq];
  r.src.head = s.head;
  r.src.key0 = 0;
  r.src.limit = len;
  r.src.once = rows <= G::ROWS;
  r.vis = len - m + 1;
  // tiles that the segment's last row sees, and those in this part
  const int tile = G::KEYS * a.G;
  auto tiles_of = [&](int end) {
    const int keys = len > 0 ? std::max(r.vis + (end - 1) / a.G, 0) : 0;
    return (keys + G::KEYS - 1) / G::KEYS;
  };
  const int all = tiles_of(std::min((s.seg + 1) * span, rows));
  const int64_t first = s.start + kSegCost * (int64_t)tile;
  r.last = first + (int64_t)tile * all - 1;
  const int t0 = part.lo <= first ? 0 : (int)std::min(divide(part.lo - first, tile), (int64_t)all);
  const int t1 = part.hi >= s.end ? all
                 : part.hi <= first ? 0 : (int)std::min(divide(part.hi - first, tile), (int64_t)all);
  // (rows without a key belong to the part where they begin)
  const bool here = all > 0 ? t0 < t1 : part.lo <= s.start;
  r.row0 = s.seg * span + part.tile * G::ROWS;
  r.rows = here ? std::max(std::min(rows - r.row0, G::ROWS), 0) : 0;
  r.t0 = t0;
  r.t1 = r.rows > 0 ? std::max(std::min(t1, tiles_of(r.row0 + r.rows)), t0) : t0;
  r.here = here;
  r.begins = t0 == 0;
  r.ends = t1 == all;
  return r;
}

// Pieces of the segment of `p`, which begins in the part and goes on in later ones (0: it does not); `total`
// places in `parts` parts.
template <class G>
FP_BOTH int pieces_of(const ChunkArgs &a, int64_t total, int parts, const Part &part, const Piece &p) {
  if (!(p.here && p.begins && !p.ends)) return 0;
  // (a cut near the segment's end has moved there)
  const int64_t near = (int64_t)kSnapTiles * G::KEYS * a.G;
  const Cut cut(total, parts);
  return cut.owner(std::min(p.last, p.s.end - near - 1)) - part.p + 1;
}

// The record of a piece's segment, where there is one for every segment.
template <class G>
FP_BOTH int record_of(const ChunkArgs &a, const Piece &p) {
  const int n = Series<G>(a, a.width, a.cu[p.s.seq + 1] - a.cu[p.s.seq], 0).n;
  return a.base[p.s.seq] + p.s.head * n + p.s.seg;
}

}  // namespace
}  // namespace fp

#undef FP_BOTH
