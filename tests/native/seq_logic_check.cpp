// Host checks of the page lists and of the passes planned over them: random batches of forks,
// appends, compactions, truncations and closings against a plain model of every sequence's rows,
// with a page's contents written and read in the order the kernels may take; and for every plan,
// that each query meets every key of its context exactly once and no two results share a slot.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <vector>

#include "../../paper_2609_23286_amd/csrc/rv_ops.h"

namespace {
int g_fail = 0;
#define CHECK(c, ...)                                 \
  do {                                                \
    if (!(c) && ++g_fail < 20) {                      \
      std::fprintf(stderr, "%s:%d: ", __FILE__, __LINE__); \
      std::fprintf(stderr, __VA_ARGS__);              \
      std::fprintf(stderr, "\n");                     \
    }                                                 \
  } while (0)

using rv::PageBook;
std::mt19937 rng(12345);
int uniform(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }

struct World {
  PageBook book;
  int n_pages, max_seqs;
  int64_t max_rows;
  std::vector<std::vector<int>> page;         // contents
  std::map<int, std::vector<int>> rows;       // the model
  int next = 1;

  World(int pages, int seqs, int64_t max) : n_pages(pages), max_seqs(seqs), max_rows(max) {
    CHECK(book.init(pages, seqs, (int)((max + 63) / 64)), "init");
    page.assign(pages, std::vector<int>(64, 0));
  }
  std::vector<int> some(int most) {
    std::vector<int> all;
    for (auto& r : rows) all.push_back(r.first);
    std::shuffle(all.begin(), all.end(), rng);
    all.resize(std::min<size_t>(all.size(), uniform(0, most)));
    return all;
  }
  void verify() {
    std::vector<int> users(n_pages, 0);
    for (auto& r : rows) {
      CHECK(book.is_open(r.first) && book.len(r.first) == (int64_t)r.second.size(), "length of %d", r.first);
      for (int i = 0; i < book.pages(r.first); ++i) ++users[book.page(r.first, i)];
      for (size_t i = 0; i < r.second.size(); ++i)
        CHECK(page[book.page(r.first, i / 64)][i % 64] == r.second[i], "sequence %d row %zu", r.first, i);
    }
    int free = 0;
    for (int p = 0; p < n_pages; ++p) {
      CHECK(book.users(p) == users[p], "page %d has %d users, not %d", p, book.users(p), users[p]);
      free += users[p] == 0;
    }
    CHECK(free == book.free_pages(), "%d free pages, not %d", book.free_pages(), free);
    CHECK(book.can_open() == max_seqs - (int)rows.size(), "sequences to open");
  }
  // All reads of a batch see the pages as they were, or as the batch writes them, in any order: reads
  // are taken before and after the writes, and both must give the same.
  void append(const std::vector<int>& seqs) {
    std::vector<int> n;
    int64_t need = 0;
    for (int s : seqs) {
      int r = uniform(0, 3) ? uniform(0, 70) : uniform(0, 300);
      if (book.len(s) + r > max_rows) r = 0;
      n.push_back(r);
      need += book.append_pages(s, r);
    }
    if (need > book.free_pages()) return;
    struct Copy { int from, to, n; };
    std::vector<Copy> copies;
    std::vector<std::pair<std::pair<int, int>, int>> writes;
    for (size_t i = 0; i < seqs.size(); ++i) {
      if (n[i] == 0) continue;
      const int64_t start = book.len(seqs[i]);
      const int before = book.free_pages(), want = book.append_pages(seqs[i], n[i]);
      const int old = book.append(seqs[i], n[i]);
      CHECK(before - book.free_pages() == want, "pages taken");
      bool row = true;
      for (int k = 1; k < book.pages(seqs[i]); ++k) row = row && book.page(seqs[i], k) == book.page(seqs[i], k - 1) + 1;
      CHECK(book.in_a_row(seqs[i], 0) == row, "pages in a row");
      if (old >= 0) copies.push_back({old, book.page(seqs[i], start / 64), (int)(start % 64)});
      for (int k = 0; k < n[i]; ++k) {
        const int64_t r = start + k;
        writes.push_back({{book.page(seqs[i], r / 64), (int)(r % 64)}, next});
        rows[seqs[i]].push_back(next++);
      }
    }
    auto old_pages = page;
    std::set<std::pair<int, int>> written;
    for (auto& w : writes) {
      CHECK(written.insert(w.first).second, "a row written twice");
      page[w.first.first][w.first.second] = w.second;
    }
    for (auto& c : copies)
      for (int r = 0; r < c.n; ++r) {
        CHECK(page[c.from][r] == old_pages[c.from][r], "a copied row is written in the same batch");
        CHECK(written.insert({c.to, r}).second, "a copied row written twice");
      }
    for (auto& c : copies)
      for (int r = 0; r < c.n; ++r) page[c.to][r] = old_pages[c.from][r];
    book.release_dropped();
  }
  void compact(const std::vector<int>& seqs) {
    std::vector<int64_t> first, keep;
    int64_t need = 0;
    for (int s : seqs) {
      const int64_t len = book.len(s);
      first.push_back(uniform(0, (int)len));
      keep.push_back(len > first.back() ? uniform(1, (int)std::min<int64_t>(max_rows - first.back(), len)) : 0);
      if (keep.back() > 0) need += book.compact_pages(first.back(), first.back() + keep.back());
    }
    if (need > book.free_pages()) return;
    auto old_pages = page;
    std::set<int> fresh;
    for (size_t i = 0; i < seqs.size(); ++i) {
      const int s = seqs[i];
      if (keep[i] == 0) {
        book.truncate(s, first[i]);
        rows[s].resize(first[i]);
        continue;
      }
      auto was = rows[s];
      rows[s].resize(first[i]);
      for (int64_t k = 0; k < keep[i]; ++k) rows[s].push_back(was[uniform((int)first[i], (int)was.size() - 1)]);
      book.compact(s, first[i], first[i] + keep[i]);
      for (int k = (int)(first[i] / 64); k < book.pages(s); ++k) {
        CHECK(fresh.insert(book.page(s, k)).second, "a new page given twice");
        for (int r = 0; r < 64 && k * 64 + r < (int)rows[s].size(); ++r) page[book.page(s, k)][r] = rows[s][k * 64 + r];
      }
    }
    // no page that the batch wrote is one that some old list still reads
    for (int p : fresh) CHECK(book.users(p) == 1, "a new page with %d users", book.users(p));
    book.release_dropped();
  }

  void plan(bool frame, int n_heads, int group) {
    std::vector<int> all = some(40);
    std::sort(all.begin(), all.end());
    if (uniform(0, 1) && !all.empty()) all.push_back(all[0]);
    std::vector<rv::SeqSpan> span;
    for (int s : all) span.push_back({s, uniform(0, 3) ? uniform(1, 4) : uniform(1, 700)});
    int tok0 = uniform(0, 50);
    const int64_t max_slots = uniform(0, 3) ? 8192 : 300;
    for (size_t i = 0; i < span.size();) {
      rv::SeqArgs a{};
      a.n_queues = uniform(1, 9);
      const int done = rv::plan_seqs(book, &span[i], (int)(span.size() - i), tok0, frame, n_heads, group,
                                     uniform(1, 300), max_slots, &a);
      CHECK(done >= 1 && done <= (int)(span.size() - i), "sequences covered");
      CHECK(a.n_pass <= rv::kMaxPasses && a.n_pass - a.n_inner == done, "passes");
      CHECK(a.E > 0 && (int64_t)a.chunks * a.E >= a.total - a.pos_first &&
                (a.chunks == 0 || (int64_t)(a.chunks - 1) * a.E < a.total - a.pos_first), "chunks");
      // the segments, as the kernel walks them
      std::set<std::vector<int>> tiles_done;
      std::map<int, std::vector<int>> slot_of;       // sub-slot -> pass, unit
      std::map<std::vector<int>, int> segments;      // pass, unit, chunk -> slot, or -1: final
      auto last_below = [&](int x) {
        int i = -1;
        while (i + 1 < a.n_pass && a.pass[i + 1].pos0 <= x) ++i;
        return i;
      };
      std::vector<int> order;
      for (int j = 0; j < rv::seq_grid(a); ++j)
        for (int x = 0; x < a.n_queues; ++x)
          if (rv::seq_chunk_of(a, x, j) >= 0) order.push_back(rv::seq_chunk_of(a, x, j));
      std::vector<int> sorted = order;
      std::sort(sorted.begin(), sorted.end());
      const int places = a.rounds > 0 ? std::max(a.width, a.chunks) : a.chunks;
      for (int c = 0; c < places; ++c) CHECK(c < (int)sorted.size() && sorted[c] == c, "chunk %d", c);
      CHECK((int)sorted.size() == places, "chunks taken");
      for (int c : order) {
        for (int r = 0; r < a.rounds && c < a.width; ++r) {
          int ip = -1;
          while (ip + 1 < a.n_pass && a.unit0[ip + 1] <= r * a.width + c) ++ip;
          const rv::SeqPass& p = a.pass[ip];
          const int unit = r * a.width + c - a.unit0[ip];
          CHECK(unit < n_heads * p.q_tiles && ip >= a.n_inner && p.parent < 0, "a unit of no pass");
          for (int t = 0; t < rv::seq_tiles(p); ++t) CHECK(tiles_done.insert({ip, unit, t}).second, "a tile taken twice");
          segments[{ip, unit, -1}] = -1;
        }
        if (c >= a.chunks) continue;
        const int begin = a.pos_first + c * a.E, end = std::min(begin + a.E, a.total);
        int ip = last_below(begin);
        for (int pos = begin; pos < end;) {
          const rv::SeqPass& p = a.pass[ip];
          const int T = rv::seq_tiles(p), units = n_heads * p.q_tiles;
          int unit = 0, end_unit = 0;
          const int t0 = T == 0 ? 0 : rv::seq_first_tile(p, T, pos - p.pos0, &unit);
          if (T == 0 || unit >= units) {
            if (++ip >= a.n_pass) break;
            pos = std::max(pos, a.pass[ip].pos0);
            continue;
          }
          const int end_tile = rv::seq_first_tile(p, T, end - p.pos0, &end_unit);
          const int t1 = end_unit > unit ? T : end_tile;
          if (end_unit < unit || t1 <= t0) break;
          const bool shared = ip < a.n_inner || p.parent >= 0;
          CHECK(t0 >= 0 && t0 < t1 && unit >= 0 && unit < units, "a segment outside its unit");
          for (int t = t0; t < t1; ++t) {
            CHECK(tiles_done.insert({ip, unit, t}).second, "a tile taken twice");
            CHECK(rv::seq_chunk_at(a, rv::seq_pos(p, unit, t)) == c, "a tile of another chunk");
          }
          int slot = -1;
          if (shared || t0 > 0 || t1 < T) {
            slot = rv::seq_slot(p, shared, unit, c, rv::seq_chunk_at(a, rv::seq_pos(p, unit, 0)));
            for (int q = slot; q < slot + p.tile_rows / rv::kSubRows; ++q) {
              CHECK(q >= 0 && (q < max_slots || done == 1), "slot %d", q);
              CHECK(slot_of.emplace(q, std::vector<int>{ip, unit, c}).second, "slot %d used twice", q);
            }
          }
          segments[{ip, unit, c}] = slot;
          pos = t1 < T ? end : rv::seq_pos(p, unit + 1, 0);
        }
      }
      int merge = 0, pos = 0, all_units = 0;
      for (int k = 0; k < a.n_pass; ++k) {
        const rv::SeqPass& p = a.pass[k];
        const int T = rv::seq_tiles(p), units = n_heads * p.q_tiles;
        CHECK(p.pos0 == pos && a.pos0[k] == pos && p.cost > 0, "first position");
        CHECK(p.unit0 == all_units && a.unit0[k] == all_units, "first unit");
        all_units += units;
        pos += units * (p.fixed + T * p.cost);
        CHECK((int64_t)p.q_tiles * p.tile_rows >= (int64_t)p.n_tok * group, "query tiles");
        CHECK(p.parent < a.n_inner && (k < a.n_inner ? p.parent < k : true), "parent");
        bool parts = T == 0;
        for (int u = 0; u < units; ++u) {
          for (int t = 0; t < T; ++t) CHECK(tiles_done.count({k, u, t}), "a tile left out");
          if (T == 0) continue;
          // as the merge finds them
          const bool shared = k < a.n_inner || p.parent >= 0;
          if (rv::seq_whole(a, p, u)) {
            CHECK(segments.count({k, u, -1}), "a whole unit left out");
            continue;
          }
          const int c0 = rv::seq_chunk_at(a, rv::seq_pos(p, u, 0));
          const int n = rv::seq_chunk_at(a, rv::seq_pos(p, u, T - 1)) - c0 + 1;
          parts = parts || shared || n > 1;
          for (int c = c0; c < c0 + n; ++c) {
            CHECK(segments.count({k, u, c}), "a segment left out");
            const int want = !shared && n == 1 ? -1 : rv::seq_slot(p, shared, u, c0, c0) + (c - c0) * rv::seq_slot_step(p, shared);
            CHECK((segments[{k, u, c}]) == want, "the merge reads another slot");
          }
        }
        if (k >= a.n_inner) {
          CHECK(a.merge0[k] == merge, "first merge workgroup");
          if (parts) merge += (p.n_tok * group + p.merge_rows - 1) / p.merge_rows * n_heads;
          // (16 rows of a merge workgroup are in one query tile)
          CHECK(p.merge_rows == rv::kMergeOne || (p.merge_rows == rv::kMergeFew && p.parent < 0), "merge rows");
        }
      }
      CHECK(pos == a.total && merge == a.merge_blocks, "workgroups");
      for (int k = 0; k < done; ++k) {  // the pages from the leaf up are the sequence's, in order
        const rv::SeqSpan& s = span[i + k];
        const rv::SeqPass& leaf = a.pass[a.n_inner + k];
        CHECK(leaf.tok0 == tok0 && leaf.n_tok == s.n_tok && leaf.frame == (frame ? s.n_tok : 0), "leaf");
        int end = book.pages(s.seq);
        if (leaf.n_pages > 0) CHECK(leaf.last_rows == book.len(s.seq) - (int64_t)(end - 1) * 64, "last rows");
        for (int j = a.n_inner + k; j >= 0; j = a.pass[j].parent) {
          const rv::SeqPass& p = a.pass[j];
          CHECK(p.tok0 <= tok0 && tok0 + s.n_tok <= p.tok0 + p.n_tok, "tokens of a pass");
          if (j < a.n_inner) CHECK(p.last_rows == 64, "a shared page is full");
          end -= p.n_pages;
          for (int q = 0; q < p.n_pages && end >= 0; ++q)
            CHECK(book.list(s.seq)[end + q] == (book.list(0) - book.entry0(0))[p.entry0 + q], "page of a pass");
        }
        CHECK(end == 0, "pages covered");
        tok0 += s.n_tok;
      }
      i += done;
    }
  }
};

void check_turns() {
  uint64_t f[rv::kMaxFreqs];
  rv::rotation_turns(1.0, 32, f);
  // 2^64 / (2 pi) = 2.93589050328200122...e18
  CHECK(f[0] >= 2935890503282001220ull && f[0] <= 2935890503282001232ull && f[31] == f[0], "turns %llu",
        (unsigned long long)f[0]);
  rv::rotation_turns(10000.0, 16, f);
  CHECK(f[8] > f[0] / 100 - 2 && f[8] < f[0] / 100 + 2 && f[16] == 0, "turns of a lower frequency");
}
}  // namespace

int main() {
  check_turns();
  for (int round = 0; round < 60; ++round) {
    World w(uniform(1, 120), uniform(1, 24), uniform(0, 3) ? 1500 : uniform(1, 200));
    for (int step = 0; step < 120; ++step) {
      const int what = uniform(0, 9);
      if (what <= 1) {
        const int s = w.book.open();
        CHECK((s < 0) == ((int)w.rows.size() == w.max_seqs), "open");
        if (s >= 0) CHECK(w.rows.emplace(s, std::vector<int>()).second, "an open sequence given again");
      } else if (what <= 3 && !w.rows.empty()) {
        const int parent = std::next(w.rows.begin(), uniform(0, (int)w.rows.size() - 1))->first;
        const auto was = w.rows[parent];
        const int n = uniform(0, 3) ? (int)was.size() : uniform(0, (int)was.size());
        for (int i = uniform(1, 4); i > 0 && w.book.can_open() > 0; --i) {
          const int c = w.book.open();
          w.book.fork(c, parent, n);
          w.rows[c] = std::vector<int>(was.begin(), was.begin() + n);
        }
      } else if (what <= 6) {
        w.append(w.some(6));
      } else if (what == 7) {
        w.compact(w.some(3));
      } else if (what == 8) {
        for (int s : w.some(1)) {
          w.rows[s].resize(uniform(0, (int)w.rows[s].size()));
          w.book.truncate(s, w.rows[s].size());
        }
      } else {
        for (int s : w.some(2)) {
          w.book.close(s);
          w.rows.erase(s);
        }
      }
      w.verify();
      if (step % 10 == 9) w.plan(uniform(0, 1), uniform(1, 16), uniform(1, 4));
    }
  }
  if (g_fail) {
    std::fprintf(stderr, "%d checks failed\n", g_fail);
    return 1;
  }
  std::printf("sequence logic OK\n");
  return 0;
}
