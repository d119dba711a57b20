// Host checks of the plans of an attention over sequences: what they read, and the largest ones.
#include <algorithm>
#include <climits>
#include <cstdarg>
#include <cstdio>
#include <vector>

#include "../../paper_2609_23286_amd/csrc/rv_ops.h"

namespace {
int g_fail = 0;
__attribute__((format(printf, 2, 3))) void check(bool ok, const char* fmt, ...) {
  if (ok || ++g_fail >= 20) return;
  va_list ap;
  va_start(ap, fmt);
  std::vfprintf(stderr, fmt, ap);
  va_end(ap);
  std::fputc('\n', stderr);
}

using rv::PageBook;

int grown(PageBook& book, int parent, int64_t keep, int64_t rows) {  // a fork of `keep` rows, `rows` appended
  const int s = book.open();
  if (parent >= 0) book.fork(s, parent, keep);
  book.append(s, rows);
  book.release_dropped();
  return s;
}

rv::SeqArgs plan(const PageBook& book, const std::vector<int>& seqs, int tokens, bool frame, int n_heads, int group,
                 int* done) {
  std::vector<rv::SeqSpan> span;
  for (int s : seqs) span.push_back({s, tokens});
  rv::SeqArgs a{};
  a.n_queues = 8;
  *done = rv::plan_seqs(book, span.data(), (int)span.size(), 0, frame, n_heads, group, 256, 8192, &a);
  return a;
}

// Key tiles of pages that a head's units of all passes go over.
int64_t tiles(const rv::SeqArgs& a) {
  int64_t n = 0;
  for (int i = 0; i < a.n_pass; ++i) n += (int64_t)a.pass[i].q_tiles * a.pass[i].n_pages;
  return n;
}

// Branches below a root of `levels` short shared stretches, one inside the other, `per` leaves to a branch: however short
// what they all have in common, a branch's own pages are read once for its leaves, and the root's no more often than
// once a branch (or in passes of their own, for no more).
void check_short_roots() {
  struct Tree { int branches, per, levels; int64_t stretch, trunk; int tokens, group; };
  std::vector<Tree> trees;
  for (int64_t root = 0; root <= 512; root += 64)
    for (int tokens : {1, 5}) {
      trees.push_back({2, 8, 1, root, 20000, tokens, 1});
      trees.push_back({3, 4, 1, root, 6000, tokens, 4});
      trees.push_back({4, 4, 2, root, 9000, tokens, 1});
      trees.push_back({5, 3, 4, root / 2, 5000, tokens, 2});
    }
  for (const Tree& t : trees) {
    PageBook book;
    check(book.init(20000, 200, 1000), "init");
    // (levels: branch b leaves the root after min(b + 1, levels) stretches)
    const int root = grown(book, -1, 0, t.levels * t.stretch);
    std::vector<int> with, without;
    int64_t root_pages = 0;
    for (int b = 0; b < t.branches; ++b) {
      const int64_t keep = std::min(b + 1, t.levels) * t.stretch;
      const int trunk = grown(book, root, keep, t.trunk), bare = grown(book, -1, 0, t.trunk);
      root_pages += (keep + 63) / 64;
      for (int k = 0; k < t.per; ++k) {
        with.push_back(grown(book, trunk, keep + t.trunk, 20 * k));
        without.push_back(grown(book, bare, t.trunk, 20 * k));
      }
    }
    int n, m;
    const rv::SeqArgs a = plan(book, with, t.tokens, true, 16, t.group, &n);
    const rv::SeqArgs b = plan(book, without, t.tokens, true, 16, t.group, &m);
    check(n == (int)with.size() && m == (int)without.size(), "one launch");
    // a trunk behind a root that ends inside a page may take a page more, in each leaf's and the branch's passes
    const int64_t most = tiles(b) + root_pages + t.branches * (t.per + 1);
    check(tiles(a) <= most, "%d branches of %d, root of %d x %lld rows, %d tokens: %lld tiles, at most %lld (%d inner passes)",
          t.branches, t.per, t.levels, (long long)t.stretch, t.tokens, (long long)tiles(a), (long long)most, a.n_inner);
  }
}
// The largest sequences that fit are planned whole and within 32 bits, alone and several together; larger ones do not fit.
void check_largest() {
  struct Size { int tokens, n_heads, group; bool frame; };
  for (const Size& z : {Size{16384, 1, 1024, false}, Size{16384, 16, 8, true}, Size{16384, 1024, 1, false},
                        Size{1041, 16, 1, true}, Size{1, 2, 4, false}, Size{129, 3, 1, true}}) {
    const int64_t q_rows = (int64_t)z.tokens * z.group, units = (q_rows + 127) / 128 * z.n_heads;
    const int64_t frame = z.frame ? (z.tokens + 63) / 64 : 0, most = ((int64_t)1 << 28) / units;
    const int64_t pages = (most * units < (int64_t)1 << 28 ? most : most - 1) - 4 - frame;  // units (pages + frame + 4) < 2^28
    check(rv::seq_fits(pages * 64, z.tokens, z.frame, z.n_heads, z.group), "%d tokens over %lld pages fit", z.tokens, (long long)pages);
    check(!rv::seq_fits(pages * 64 + 1, z.tokens, z.frame, z.n_heads, z.group), "%d tokens over %lld pages and a row do not", z.tokens,
          (long long)pages);
    if (pages > 4000000) continue;  // (more than a device holds)
    PageBook book;
    check(book.init((int)pages * 2, 2, (int)pages), "init");
    const std::vector<int> seqs = {grown(book, -1, 0, pages * 64), grown(book, -1, 0, pages * 64 - 1)};
    for (int n = 1; n <= 2; ++n) {
      int done;
      const rv::SeqArgs a = plan(book, std::vector<int>(seqs.begin(), seqs.begin() + n), z.tokens, z.frame, z.n_heads, z.group, &done);
      check(done >= 1 && a.n_inner == 0 && a.n_pass == done, "sequences planned");
      int64_t pos = 0;
      for (int i = 0; i < done; ++i) {
        const rv::SeqPass& p = a.pass[i];
        check(p.n_pages == pages && p.pos0 == pos, "pass %d", i);
        pos += (int64_t)p.q_tiles * z.n_heads * (p.fixed + (int64_t)rv::seq_tiles(p) * p.cost);
      }
      check(pos == a.total && a.total > 0 && a.E > 0 && a.pos_first >= 0 && (int64_t)a.pos_first + (int64_t)a.chunks * a.E < INT32_MAX,
            "positions within 32 bits");
    }
  }
}
// The merge launch stays within what a grid holds, however many rows the batch has.
void check_merge_grid() {
  PageBook book;
  check(book.init(200, 60, 10), "init");
  std::vector<int> seqs;
  for (int i = 0; i < 50; ++i) seqs.push_back(grown(book, -1, 0, 128));
  for (int tokens : {16384, 5000, 1}) {
    std::vector<rv::SeqSpan> span;
    for (int s : seqs) span.push_back({s, tokens});
    span.push_back({seqs[0], 1});  // (few queries: the others' units are cut)
    int tok0 = 0;
    for (size_t i = 0; i < span.size();) {
      rv::SeqArgs a{};
      a.n_queues = 8;
      const int done = rv::plan_seqs(book, &span[i], (int)(span.size() - i), tok0, false, 1024, 1, 256, 8192, &a);
      check(done >= 1, "sequences planned");
      check(a.merge_blocks <= rv::kMaxGridBlocks, "%d sequences of %d tokens: %d workgroups join", done, tokens, a.merge_blocks);
      for (int k = 0; k < done; ++k) tok0 += span[i + k].n_tok;
      i += done;
    }
  }
}
// Common pages are a pass of their own where that was measured to be clearly faster, and only there.
void check_worth() {
  struct Batch { int seqs, tokens, n_heads, group, pages; bool pass; };
  for (const Batch& b : {Batch{4, 1041, 16, 1, 160, false}, Batch{16, 1041, 16, 1, 160, false}, Batch{4, 1041, 16, 1, 24, false},
                         Batch{12, 200, 16, 1, 80, false}, Batch{4, 300, 16, 1, 48, false}, Batch{8, 40, 16, 1, 8, false},
                         Batch{48, 5, 16, 1, 8, false}, Batch{40, 17, 2, 8, 12, false}, Batch{48, 5, 16, 1, 24, true},
                         Batch{16, 1, 16, 1, 24, true}, Batch{16, 1, 4, 4, 80, true}, Batch{8, 40, 16, 1, 80, true},
                         Batch{8, 130, 16, 1, 160, true}, Batch{2, 1, 16, 1, 80, true}, Batch{40, 17, 2, 8, 160, true}}) {
    PageBook book;
    check(book.init(2000, 60, 400), "init");
    const int root = grown(book, -1, 0, b.pages * 64);
    std::vector<int> seqs;
    for (int i = 0; i < b.seqs; ++i) seqs.push_back(grown(book, root, b.pages * 64, 300));
    int done;
    const rv::SeqArgs a = plan(book, seqs, b.tokens, false, b.n_heads, b.group, &done);
    check(done == b.seqs && (a.n_inner > 0) == b.pass, "%d sequences of %d tokens over %d pages: %d shared passes", b.seqs,
          b.tokens, b.pages, a.n_inner);
  }
}
}  // namespace

int main() {
  check_short_roots();
  check_worth();
  check_largest();
  check_merge_grid();
  if (g_fail) {
    std::fprintf(stderr, "%d checks failed\n", g_fail);
    return 1;
  }
  std::printf("sequence plans OK\n");
  return 0;
}
