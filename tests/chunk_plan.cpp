// How chunk_attn divides the keys of a batch, gone through on the host with the kernels' own arithmetic:
// every workgroup of a call in turn, what it reads of the keys and what it leaves for the join.
//
//   places            every workgroup count, width and number of parts: who has which part
//   batches SEED N    N drawn batches, among them many sequences without tokens
//   batch ROWS WGS WIDTH G HKV LEN:NEW ...   one batch (LEN -1: no slot)
//
// Prints a line of counts, or the first thing that is wrong, with status 1.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <string>
#include <vector>

#include "../paper_2502_20766_amd/csrc/fp_chunk_plan.h"

using namespace fp;

namespace {

std::string g_case;

[[noreturn]] void fail(const char *what, long a = 0, long b = 0, long c = 0) {
  printf("%s: %s (%ld, %ld, %ld)\n", g_case.c_str(), what, a, b, c);
  exit(1);
}

void places() {
  long n = 0;
  for (int wgs : {256, 512, 768})
    for (int width = 1; width <= 16; ++width)
      for (int parts = 1; parts <= wgs / width; ++parts) {
        ChunkArgs a;
        a.wgs = wgs;
        a.width = width;
        g_case = std::to_string(wgs) + " workgroups, width " + std::to_string(width) + ", " +
                 std::to_string(parts) + " parts";
        std::vector<int> keeps(wgs / width), works(parts * width);
        for (int block = 0; block < wgs + 70; ++block) {
          const Part r = place_of(a, block, parts);
          if (r.width != width || r.p < 0 || r.tile < 0 || r.tile >= width || r.lo < r.hi)
            fail("a workgroup's place", block, r.p, r.tile);
          if (r.tile == 0 && r.p < wgs / width) ++keeps[r.p];
          if (r.p < parts) ++works[r.p * width + r.tile];
        }
        for (int p = 0; p < wgs / width; ++p)
          if (keeps[p] != 1) fail("writers of a record", p, keeps[p]);
        for (int i = 0; i < parts * width; ++i)
          if (works[i] != 1) fail("workgroups of a part's row tile", i / width, i % width, works[i]);
        ++n;
      }
  printf("%ld\n", n);
}

struct Run {            // a piece of a row tile
  int p, t0, t1, begins, ends;
};

struct Counts {
  long cut = 0, joined = 0, dealt = 0, few = 0;
} g_counts;

struct Batch {
  int rows, wgs, width, G, hkv;
  std::vector<int> len, news;          // tokens (-1: no slot) and queries
};

template <class G>
void go(const Batch &b) {
  ChunkArgs a;
  memset(&a, 0, sizeof(a));
  a.G = b.G;
  a.hkv = b.hkv;
  a.batch = (int)b.len.size();
  a.wgs = b.wgs;
  a.width = b.width;
  a.rows = b.rows;
  const int most = a.wgs / a.width;
  int64_t records = 0;
  std::vector<int> len(a.batch);
  for (int i = 0; i < a.batch; ++i) {
    a.slot[i] = b.len[i] < 0 ? -1 : i;
    len[i] = std::max(b.len[i], 0);
    a.cu[i + 1] = a.cu[i] + b.news[i];
    const int64_t span = (int64_t)a.rows * a.width;
    a.base[i] = (int32_t)std::min<int64_t>(records, a.wgs);
    records += ((int64_t)b.news[i] * a.G + span - 1) / span * a.hkv;
  }
  if (a.cu[a.batch] == 0) return;
  a.by_segment = records <= most;
  a.records = a.by_segment ? (int)records : most;

  // the line: all segments in its order
  std::vector<Segment> line;
  std::vector<int64_t> start(a.batch + 1);
  for (int i = 0; i < a.batch; ++i) {
    const Series<G> series(a, a.width, b.news[i], len[i]);
    for (int h = 0; h < a.hkv; ++h)
      for (int s = 0; s < series.n; ++s) {
        const int64_t from = start[i] + h * series.whole();
        line.push_back({i, h, s, from + series.begin(s), from + series.end(s)});
      }
    start[i + 1] = start[i] + a.hkv * series.whole();
  }
  const int64_t total = start[a.batch];
  for (size_t i = 0; i < line.size(); ++i)
    if (line[i].start != (i ? line[i - 1].end : 0) || line[i].end <= line[i].start)
      fail("a segment's places", i);
  if (line.back().end != total || (int64_t)line.size() != records) fail("the line's end");
  auto number = [&](int64_t at) {      // of the segment that a place lies in
    return (int)(std::upper_bound(line.begin(), line.end(), at,
                                  [](int64_t x, const Segment &s) { return x < s.end; }) - line.begin());
  };

  const int parts = parts_of<G>(a, total);
  const Cut cut(total, parts);
  std::map<std::pair<int, int>, std::vector<Run>> runs;       // of segment and row tile
  std::vector<int> writers(a.wgs);
  std::vector<int4> record(a.wgs);
  auto write = [&](int at, int4 x) {
    if (at < 0 || at >= a.records) fail("a record out of range", at, a.records);
    ++writers[at];
    record[at] = x;
  };
  for (int block = 0; block < a.wgs + 9; ++block) {
    Part part = place_of(a, block, parts);
    if (part.p < parts)
      for (int i = 0; i < 2; ++i) {
        const int64_t at = cut.begin(part.p + i);
        int64_t x = total;
        if (at < total) {
          const Segment &s = line[number(at)];
          const Series<G> series(a, a.width, b.news[s.seq], len[s.seq]);
          const Segment f = segment_at(series, series.whole(), s.seq, start[s.seq], at);
          if (f.head != s.head || f.seg != s.seg || f.start != s.start || f.end != s.end)
            fail("the segment of a place", at);
          x = snap<G>(a, at, s.start, s.end);
        }
        (i ? part.hi : part.lo) = x;
      }
    const bool keeps = part.tile == 0;
    if (part.lo >= part.hi) {
      if (keeps && !a.by_segment && part.p < most) write(part.p, make_int4(0, 0, 0, 0));
      continue;
    }
    for (int i = number(part.lo);; ++i) {
      const Piece p = piece_of<G>(a, line[i], len[line[i].seq], part);
      if (p.rows > 0)
        runs[{i, part.tile}].push_back({part.p, p.t0, p.t1, p.begins, p.ends});
      const bool last = line[i].end >= part.hi;
      if (keeps) {
        const int4 rec = make_int4(pieces_of<G>(a, total, parts, part, p) | part.p << 16, line[i].seq,
                                   line[i].head, line[i].seg);
        if (a.by_segment) {
          if (p.here && p.begins) write(record_of<G>(a, p), rec);
        } else if (last) {
          write(part.p, rec);
        }
      }
      if (last) break;
    }
  }
  for (int i = 0; i < a.records; ++i)
    if (writers[i] != 1) fail("writers of a record", i, writers[i], a.records);

  // the join: the records of segments that it puts together
  std::map<int, int4> joins;
  for (int i = 0; i < a.records; ++i) {
    const int n = record[i].x & 0xFFFF;
    if (n == 0) continue;
    int at = 0;
    while (line[at].seq != record[i].y || line[at].head != record[i].z || line[at].seg != record[i].w)
      if (++at == (int)line.size()) fail("a record of no segment", i);
    if (n == 1 || !joins.emplace(at, record[i]).second) fail("pieces of a record", i, n);
  }
  for (int i = 0; i < (int)line.size(); ++i) {
    const Segment &s = line[i];
    const int m = b.news[s.seq], all_rows = m * a.G;
    for (int j = 0; j < a.width; ++j) {
      const int row0 = (s.seg * a.width + j) * a.rows, rows = std::min(all_rows - row0, a.rows);
      std::vector<Run> r = runs[{i, j}];
      if (rows <= 0) {
        if (!r.empty()) fail("a piece without rows", i, j);
        continue;
      }
      const int keys = len[s.seq] ? std::max(len[s.seq] - m + (row0 + rows - 1) / a.G + 1, 0) : 0;
      const int tiles = (keys + 63) / 64;
      std::sort(r.begin(), r.end(), [](const Run &x, const Run &y) { return x.p < y.p; });
      const auto join = joins.find(i);
      if (join == joins.end()) {
        if (r.size() != 1 || !r[0].begins || !r[0].ends || r[0].t0 != 0 || r[0].t1 != tiles)
          fail("a row tile that is not joined", i, j, (long)r.size());
        continue;
      }
      const int n = join->second.x & 0xFFFF, p0 = join->second.x >> 16;
      if ((int)r.size() != n) fail("pieces of a row tile", i, j, (long)r.size());
      int at = 0;
      for (int k = 0; k < n; ++k) {
        if (r[k].p != p0 + k || r[k].begins != (k == 0) || (r[k].begins && r[k].ends))
          fail("the part of a piece", i, j, k);
        if (r[k].t0 < r[k].t1) {
          if (r[k].t0 != at) fail("a gap or an overlap between pieces", i, j, k);
          at = r[k].t1;
        }
      }
      if (at != tiles) fail("keys that no piece has", i, j, at);
      ++g_counts.joined;
    }
  }
  ++g_counts.cut;
  const int room = a.wgs / 8 / a.width;
  if (parts <= 8 * room && 8 * parts * a.width <= 7 * a.wgs && most > 8 * room) {
    ++g_counts.dealt;
    if (!a.by_segment) ++g_counts.few;
  }
}

void run(const Batch &b) {
  g_case = "batch " + std::to_string(b.rows) + " " + std::to_string(b.wgs) + " " +
           std::to_string(b.width) + " " + std::to_string(b.G) + " " + std::to_string(b.hkv);
  for (size_t i = 0; i < b.len.size(); ++i)
    g_case += " " + std::to_string(b.len[i]) + ":" + std::to_string(b.news[i]);
  if (b.rows == 256) go<Geo<8, 64>>(b);
  else go<Geo<4, 64>>(b);
}

void batches(unsigned seed, int n) {
  std::mt19937 rng(seed);
  auto below = [&](int x) { return (int)(rng() % (unsigned)x); };
  auto size = [&](int most) {          // spread over its logarithm
    return (int)std::exp(std::log((double)most + 1) * ((rng() >> 8) * 0x1p-24));
  };
  for (int k = 0; k < n; ++k) {
    Batch b;
    const int heads[] = {1, 2, 4, 7, 16, 33}, kv[] = {1, 1, 2, 2, 3, 8};
    b.rows = below(2) ? 256 : 128;
    b.wgs = b.rows == 256 ? 256 : below(2) ? 768 : 512;
    b.width = 1 + below(16);
    b.G = heads[below(6)];
    b.hkv = kv[below(6)];
    const int batch = 1 + size(below(8) ? 9 : 255);
    // rows for about as many segments as there are parts, or for few
    const int many = (int)((int64_t)b.wgs * b.rows / b.G / b.hkv) * (1 + below(4)) / 2;
    for (int i = 0; i < batch; ++i) {
      const int idle = below(3), len = idle == 0 ? -1 : idle == 1 && below(2) ? 0 : size(below(4) ? 3000 : 90000);
      b.len.push_back(len);
      b.news.push_back(below(8) == 0 ? 0 : len <= 0 || below(8) == 0 ? 1 + (below(2) ? below(many / batch + 1) : size(many))
                                             : std::min(len + below(3), 1 + size(4000)));
    }
    run(b);
  }
}

}  // namespace

int main(int argc, char **argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "places") {
    places();
    return 0;
  }
  if (what == "batches" && argc == 4) {
    batches((unsigned)atoi(argv[2]), atoi(argv[3]));
  } else if (what == "batch" && argc > 7) {
    Batch b = {atoi(argv[2]), atoi(argv[3]), atoi(argv[4]), atoi(argv[5]), atoi(argv[6]), {}, {}};
    for (int i = 7; i < argc; ++i) {
      int len, news;
      if (sscanf(argv[i], "%d:%d", &len, &news) != 2) return 2;
      b.len.push_back(len);
      b.news.push_back(news);
    }
    run(b);
  } else {
    return 2;
  }
  printf("%ld %ld %ld %ld\n", g_counts.cut, g_counts.joined, g_counts.dealt, g_counts.few);
  return 0;
}
