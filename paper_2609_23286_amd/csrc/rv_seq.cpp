// rv_seq.cpp -- host-side planning of the operators around a frame's attention: rotation
// frequencies, the page pool's bookkeeping and the passes of an attention over several
// sequences.  No device calls here, so this file also builds with a host compiler alone.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
#include <new>

#include "rv_ops.h"

namespace rv {

void rotation_turns(double base, int n_freqs, uint64_t* out) {
  // base^(-i / n) as the product of the powers at i's bits: six roundings of 64 bits at most
  const long double two_pi = 6.283185307179586476925286766559005768L;
  long double bit[5];
  for (int b = 0; b < 5; ++b) bit[b] = powl((long double)base, -(long double)(1 << b) / n_freqs);
  for (int i = 0; i < kMaxFreqs; ++i) {
    long double f = 1 / two_pi;  // (so the turns stay below 0.16)
    for (int b = 0; b < 5; ++b)
      if (i >> b & 1) f *= bit[b];
    out[i] = i < n_freqs ? (uint64_t)(f * 18446744073709551616.0L + 0.5L) : 0;
  }
}

// ---- page pool --------------------------------------------------------------------------

namespace {
template <class T>
bool alloc(T** p, int64_t n) {
  *p = new (std::nothrow) T[(size_t)std::max<int64_t>(n, 1)]();
  return *p != nullptr;
}
}  // namespace

PageBook::~PageBook() {
  delete[] table_;
  delete[] refs_;
  delete[] free_;
  delete[] closed_;
  delete[] dropped_;
  delete[] moved_;
  delete[] old_pages_;
  delete[] len_;
  delete[] stamp_;
  delete[] open_;
  delete[] side_;
}

bool PageBook::init(int n_pages, int max_seqs, int width) {
  n_pages_ = n_pages;
  max_seqs_ = max_seqs;
  width_ = width;
  const bool ok = alloc(&table_, 2 * (int64_t)max_seqs * width) && alloc(&refs_, n_pages) && alloc(&free_, n_pages) &&
                  alloc(&closed_, max_seqs) && alloc(&dropped_, max_seqs) && alloc(&moved_, max_seqs) &&
                  alloc(&old_pages_, max_seqs) && alloc(&len_, max_seqs) && alloc(&stamp_, max_seqs) &&
                  alloc(&open_, max_seqs) && alloc(&side_, max_seqs);
  if (!ok) return false;
  // the lowest page and the lowest sequence go first
  for (int i = 0; i < n_pages; ++i) free_[i] = n_pages - 1 - i;
  for (int i = 0; i < max_seqs; ++i) closed_[i] = max_seqs - 1 - i;
  n_free_ = n_pages;
  n_closed_ = max_seqs;
  return true;
}

bool PageBook::first_in_batch(int s) {
  if (stamp_[s] == batch_) return false;
  stamp_[s] = batch_;
  return true;
}

int PageBook::take() {
  const int p = free_[--n_free_];
  refs_[p] = 1;
  return p;
}

int PageBook::open() {
  if (n_closed_ == 0) return -1;
  const int s = closed_[--n_closed_];
  open_[s] = 1;
  len_[s] = 0;
  return s;
}

void PageBook::close(int s) {
  truncate(s, 0);
  open_[s] = 0;
  closed_[n_closed_++] = s;
}

void PageBook::fork(int child, int s, int64_t n_rows) {
  len_[child] = n_rows;
  const int n = pages(child);
  const int32_t from = entry0(s), to = entry0(child);
  for (int i = 0; i < n; ++i) {
    table_[to + i] = table_[from + i];
    ++refs_[table_[from + i]];
  }
}

void PageBook::truncate(int s, int64_t n_rows) {
  const int have = pages(s);
  len_[s] = n_rows;
  for (int i = have - 1; i >= pages(s); --i) drop(page(s, i));  // (so that they are taken in this order again)
}

bool PageBook::append_copies(int s, int64_t n) const {
  return n > 0 && len_[s] % kPageRows != 0 && refs_[page(s, pages(s) - 1)] > 1;
}

int PageBook::append_pages(int s, int64_t n) const {
  return (int)(ceil_div64(len_[s] + n, kPageRows) - pages(s)) + (append_copies(s, n) ? 1 : 0);
}

int PageBook::append(int s, int64_t n) {
  const int have = pages(s);
  const bool copies = append_copies(s, n);
  len_[s] += n;
  int old = -1;
  if (copies) {
    old = page(s, have - 1);
    dropped_[n_dropped_++] = old;
    table_[entry0(s) + have - 1] = take();
  }
  for (int i = have; i < pages(s); ++i) table_[entry0(s) + i] = take();
  return old;
}

bool PageBook::in_a_row(int s, int from) const {
  const int32_t* x = list(s);
  for (int i = from + 1, n = pages(s); i < n; ++i)
    if (x[i] != x[i - 1] + 1) return false;
  return true;
}

int PageBook::compact_pages(int64_t first, int64_t n_rows) const {
  return (int)(ceil_div64(n_rows, kPageRows) - first / kPageRows);
}

void PageBook::compact(int s, int64_t first, int64_t n_rows) {
  const int keep = (int)(first / kPageRows);
  moved_[n_moved_++] = s;
  old_pages_[s] = pages(s);
  const int32_t from = entry0(s);
  side_[s] ^= 1;
  len_[s] = n_rows;
  const int32_t to = entry0(s);
  for (int i = 0; i < keep; ++i) {
    table_[to + i] = table_[from + i];
    ++refs_[table_[from + i]];
  }
  for (int i = keep; i < pages(s); ++i) table_[to + i] = take();
}

void PageBook::release_dropped() {
  while (n_dropped_ > 0) drop(dropped_[--n_dropped_]);
  while (n_moved_ > 0) {
    const int s = moved_[--n_moved_];
    const int32_t old = (2 * s + (side_[s] ^ 1)) * width_;
    for (int i = old_pages_[s] - 1; i >= 0; --i) drop(table_[old + i]);
  }
}

// ---- attention of several sequences ----------------------------------------------------

namespace {

// Full pages that sequences a and b have in common from their start.
int common_pages(const PageBook& book, int a, int b) {
  const int n = (int)(std::min(book.len(a), book.len(b)) / kPageRows);
  if (n == 0) return 0;
  const int32_t *x = book.list(a), *y = book.list(b);
  constexpr int kStep = 128;
  int i = 0;
  while (i + kStep <= n && memcmp(x + i, y + i, kStep * sizeof(int32_t)) == 0) i += kStep;
  while (i < n && x[i] == y[i]) ++i;
  return i;
}

// Positions of a key tile and, once, of a unit: for a workgroup's 128 rows, and for 32 (where the waves take tiles
// side by side).  (Fixed shares of 8 to 24 and 6 to 20, tile costs of 1 to 4 for the narrow units and shortest
// chunks of 8 to 32 measured on twelve batches, from two single tokens to 16 frames: these were within 4 % of the
// best of each but one, where narrow tiles of cost 1 and units of 20 were 5 % faster; without fixed shares long
// batches lost 10 to 40 %.)
constexpr int kWideCost = 4, kWideFixed = 16, kNarrowCost = 2, kNarrowFixed = 16;
constexpr int kMinChunk = 20;     // positions
// (a sequence that fits takes no more positions than a plan may have)
static_assert(kWideCost * kMaxSeqTiles <= INT32_MAX / 2 + 1 && kWideFixed <= kWideCost * kSeqTilesMore &&
              kNarrowCost <= kWideCost && kNarrowFixed <= kWideCost * kSeqTilesMore, "positions");
// (no chunk between a unit's first and last is without a tile of it)
static_assert(kMinChunk >= kWideFixed + kWideCost && kMinChunk >= kNarrowFixed + kNarrowCost, "chunk length");
// Where all units have one length, they are cut into equal pieces, so that the query tiles of a head go over the
// same keys, unless chunks that run from one unit into the next are shorter by more than this many tiles; and
// they are left whole where pieces would be shorter by no more than this.  (1041 queries of 16 heads: over 2000,
// 5000 and 10,000 rows three pieces 36, 49 and 76 us, running chunks 44, 56 and 79; over 20,000 the same; over 52,000
// 319 and 300.  Over 64 rows whole units 22.3 us, three pieces 24.6; over 1000 rows 35 and 31.)
constexpr int kStartTiles = 16;
// Positions that 32 rows of a unit's partial result take as long as, written and joined.  (Pages from which a shared pass
// was the faster one, measured, and those by the rule: 48 sequences of 5 tokens of 16 heads 14, 13; 16 of a token 13, 12;
// 8 of 40 tokens 24 to 36, 45; 8 of 130 about 75, 72; 4 of 300 about 240, 221; 12 of 200 about 250, 173.  Away from there:
// 48 of 5 over 8 pages 29 us shared and 25 apart, over 48 31 and 91; 4 frames of 1041 over 160 pages 282 and 224.)
constexpr int kPartialCost = 20;
// Up to which the merge takes a row in 16 lanes, four segments at a time, and above it a wave a row, 16 at a time.
// (Over 5000 rows of 16 heads, with 16 lanes and with a wave: three segments 47 and 54 us, six 32.5 and 34.8, eight 27.1
// and 28.7, ten 26.0 both, sixteen 24.4 and 24.0, 31 19.7 and 18.8; over 20,000 rows the same order.)
constexpr int kFewSegments = 12;

// First position of unit u of all passes' units.
int first_pos(const SeqArgs& a, int64_t u) {
  int i = a.n_pass - 1;
  while (i > 0 && a.unit0[i] > u) --i;
  return seq_pos(a.pass[i], (int)(u - a.unit0[i]), 0);
}

// Rounds of whole units, one to each of `width` workgroups: as many as the units fill, unless the one whose units are
// the longest would work kWholeMore percent longer than with all units cut into equal chunks.  (16 frames of 1041
// tokens over 5100 to 6000 rows of their own: whole units 570 us, chunks 684; over 750 to 6000 rows 410 and 461.  4
// frames, a round of 3.5 of them: over 4200 to 6000 rows, 10 % longer, 154 and 159; 3000 to 6000, 19 %, 148 and 147;
// 600 to 6000, 40 %, 145 and 116.)
constexpr int kWholeMore = 15;
int whole_rounds(const SeqArgs& a, int64_t units, int64_t total, int width) {
  const int rounds = (int)(units / width);
  if (rounds == 0) return 0;
  const int64_t cut = (int64_t)rounds * width, rest = cut < units ? total - first_pos(a, cut) : 0;
  int64_t most = 0;  // of a workgroup's whole units; workgroups between two places where a pass begins have the same
  for (int i = 0; i < a.n_pass; ++i) {
    int64_t sum = 0;
    for (int64_t u = a.unit0[i] % width; u < cut; u += width)
      sum += (u + 1 < units ? first_pos(a, u + 1) : total) - first_pos(a, u);
    most = std::max(most, sum);
  }
  return (most + ceil_div64(rest, width)) * 100 <= ceil_div64(total, width) * (100 + kWholeMore) ? rounds : 0;
}

struct Builder {
  const PageBook& book;
  const SeqSpan* spans;
  const int* tok;      // tokens before sequence i
  const int* common;   // pages in common of sequences i and i + 1
  int n_heads, group;
  bool frame;
  SeqArgs* a;
  SeqPass leaf[kMaxPasses];
  int n_leaf, n_inner;
  bool overflow;

  int64_t tiles(int64_t n_tok) const { return ceil_div64(n_tok * group, tile_rows(n_tok)); }
  int tile_rows(int64_t n_tok) const { return seq_tile_rows(n_tok * group); }
  // Positions that a page takes with all the queries of n_tok tokens, and 32-row slots of their partial results.
  int64_t page_cost(int64_t n_tok) const { return tiles(n_tok) * (tile_rows(n_tok) == kSubRows ? kNarrowCost : kWideCost); }
  int64_t slots(int64_t n_tok) const { return tiles(n_tok) * (tile_rows(n_tok) / kSubRows); }

  SeqPass make(int i, int j, int p0, int p1, int parent) const {
    SeqPass p{};
    p.tok0 = tok[i];
    p.n_tok = tok[j] - tok[i];
    p.entry0 = book.entry0(spans[i].seq) + p0;
    p.n_pages = p1 - p0;
    p.last_rows = kPageRows;
    p.parent = parent;
    p.tile_rows = tile_rows(p.n_tok);
    p.q_tiles = (int)tiles(p.n_tok);
    return p;
  }

  // Sequences [i, j), whose first p0 pages the passes above cover.
  void build(int i, int j, int p0, int parent) {
    if (overflow) return;
    if (j - i == 1) {
      if (n_leaf + n_inner >= kMaxPasses) {
        overflow = true;
        return;
      }
      const int s = spans[i].seq;
      SeqPass p = make(i, j, p0, book.pages(s), parent);
      if (p.n_pages > 0) p.last_rows = (int)(book.len(s) - (int64_t)(book.pages(s) - 1) * kPageRows);
      p.frame = frame ? p.n_tok : 0;
      leaf[n_leaf++] = p;
      return;
    }
    int shared = common[i];
    for (int k = i + 1; k + 1 < j; ++k) shared = std::min(shared, common[k]);
    const int64_t joint_tok = tok[j] - tok[i];
    int64_t saved = -page_cost(joint_tok), parts = slots(joint_tok);
    for (int k = i; k < j; ++k) {
      saved += page_cost(spans[k].n_tok);
      parts += slots(spans[k].n_tok);
    }
    // Worth a pass if it saves more positions than the partial results take that every unit then writes and the
    // merge reads.
    if (saved * (shared - p0) > kPartialCost * parts) {
      if (n_leaf + n_inner >= kMaxPasses) {
        overflow = true;
        return;
      }
      a->pass[n_inner] = make(i, j, p0, shared, parent);
      parent = n_inner++;
      p0 = shared;
    }
    // Neighbours that have more in common go on together; pages that were not worth a pass above begin theirs.
    for (int k = i; k < j;) {
      int e = k + 1;
      while (e < j && common[e - 1] > shared) ++e;
      build(k, e, p0, parent);
      k = e;
    }
  }
};

}  // namespace

bool seq_fits(int64_t rows, int n_tok, bool frame, int n_heads, int group) {
  const int64_t q_rows = (int64_t)n_tok * group, units = ceil_div64(q_rows, seq_tile_rows(q_rows)) * n_heads;
  const int64_t T = ceil_div64(rows, kPageRows) + (frame ? ceil_div64(n_tok, kAttnBK) : 0);
  return units * (T + kSeqTilesMore) < kMaxSeqTiles;
}

int plan_seqs(const PageBook& book, const SeqSpan* spans, int n, int tok0, bool frame, int n_heads, int group,
              int n_cus, int64_t max_slots, SeqArgs* a) {
  n = std::min(n, kMaxPasses - 1);
  int tok[kMaxPasses + 1], common[kMaxPasses] = {};
  tok[0] = tok0;
  for (int i = 0; i < n; ++i) tok[i + 1] = tok[i] + spans[i].n_tok;
  for (int i = 0; i + 1 < n; ++i) common[i] = common_pages(book, spans[i].seq, spans[i + 1].seq);
  for (;; n = (n + 1) / 2) {
    Builder b{book, spans, tok, common, n_heads, group, frame, a, {}, 0, 0, false};
    for (int k = 0; k < n;) {
      int e = k + 1;
      while (e < n && common[e - 1] > 0) ++e;
      b.build(k, e, 0, -1);
      k = e;
    }
    if (b.overflow) continue;
    a->n_inner = b.n_inner;
    a->n_pass = b.n_inner + b.n_leaf;
    std::copy(b.leaf, b.leaf + b.n_leaf, a->pass + b.n_inner);
    int64_t pos = 0, units = 0;
    int64_t longest = 0, shortest = INT64_MAX;  // positions of a unit
    bool fits = true, wide = a->n_inner == 0;  // wide: leaves of 128-row tiles with keys, and nothing else
    for (int i = 0; i < a->n_pass; ++i) {
      SeqPass& p = a->pass[i];
      const bool narrow = p.tile_rows == kSubRows;
      const int64_t T = seq_tiles(p);
      p.cost = narrow ? kNarrowCost : kWideCost;
      p.fixed = T == 0 ? 0 : narrow ? kNarrowFixed : kWideFixed;
      a->pos0[i] = p.pos0 = (int)std::min<int64_t>(pos, INT32_MAX);
      a->unit0[i] = p.unit0 = (int)std::min<int64_t>(units, INT32_MAX);
      const int64_t per = p.fixed + T * p.cost;
      pos += (int64_t)p.q_tiles * n_heads * per;
      units += (int64_t)p.q_tiles * n_heads;
      longest = std::max(longest, per);
      shortest = std::min(shortest, per);
      wide = wide && !narrow && T > 0;
    }
    if (n > 1 && (pos > INT32_MAX / 2 || units > INT32_MAX / 2)) continue;
    // The device's workgroup slots.  (With inner passes an XCD's two shares are rounded up each: a workgroup more
    // than its slots would wait for a whole chunk.)
    const int at_once = std::max(1, kAttnWgPerCu * n_cus - (a->n_inner > 0 ? a->n_queues : 0));
    a->rounds = wide ? whole_rounds(*a, units, pos, at_once) : 0;
    a->width = at_once;
    a->total = (int)pos;
    const int first = a->rounds * at_once;  // the first unit that is cut
    a->pos_first = first == 0 ? 0 : first < units ? first_pos(*a, first) : a->total;
    a->E = (int)std::max<int64_t>(kMinChunk, ceil_div64(a->total - a->pos_first, at_once));
    if (wide && longest == shortest && first < units) {
      // units of one length in equal pieces: a tile takes `pieces` positions and a chunk as many as a unit has tiles
      const int64_t T = seq_tiles(a->pass[0]), even = ceil_div64((units - first) * T, at_once);
      int64_t pieces = std::min<int64_t>(at_once / (units - first), std::max<int64_t>(1, T * kWideCost / kMinChunk));
      if (T - ceil_div64(T, pieces) <= kStartTiles) pieces = 1;
      if (units * T * pieces <= INT32_MAX / 2 && ceil_div64(T, pieces) <= even + kStartTiles) {
        for (int i = 0; i < a->n_pass; ++i) {
          SeqPass& p = a->pass[i];
          p.cost = (int)pieces;
          p.fixed = 0;
          a->pos0[i] = p.pos0 = (int)(p.unit0 * T * pieces);
        }
        a->total = (int)(units * T * pieces);
        a->pos_first = (int)(first * T * pieces);
        a->E = (int)T;
      }
    }
    a->chunks = (int)ceil_div64(a->total - a->pos_first, a->E);
    const int leaf0 = a->n_inner < a->n_pass ? a->pass[a->n_inner].pos0 : a->total;
    a->inner_chunks = (int)ceil_div64(leaf0, a->E);
    const int X = a->n_queues, rest = (a->rounds > 0 ? std::max(a->width, a->chunks) : a->chunks) - a->inner_chunks;
    a->inner = {a->inner_chunks / X, a->inner_chunks % X};
    a->leaves = {rest / X, rest % X};
    int64_t slots = (2 * (int64_t)a->chunks + 1) * kSubsPerTile, merge = 0;
    for (int i = 0; i < a->n_pass; ++i) {
      SeqPass& p = a->pass[i];
      const int n_units = p.q_tiles * n_heads, T = seq_tiles(p);
      const bool leaf = i >= a->n_inner, shared = !leaf || p.parent >= 0;
      if (shared && T > 0) {
        const int c0 = seq_chunk_at(*a, p.pos0), c1 = seq_chunk_at(*a, seq_pos(p, n_units - 1, T - 1));
        p.slot0 = (int)(slots - (int64_t)c0 * (p.tile_rows / kSubRows));
        slots += (int64_t)(n_units + c1 - c0) * (p.tile_rows / kSubRows);
        fits = fits && slots <= max_slots;
      }
      a->merge0[i] = (int)merge;
      if (!leaf) continue;
      // merged: sums in parts, or none at all
      int most = T == 0 ? 2 : 1;
      // chunks that a unit can lie in (in equal pieces: that each does)
      const int64_t bound = T == 0 ? 0 : p.fixed == 0 ? p.cost : ceil_div64(seq_pos(p, 0, T - 1) - p.pos0, a->E) + 1;
      for (int u = 0; u < n_units && most < bound; ++u)
        if (!seq_whole(*a, p, u))
          most = std::max(most, seq_chunk_at(*a, seq_pos(p, u, T - 1)) - seq_chunk_at(*a, seq_pos(p, u, 0)) + 1);
      p.merge_rows = shared || most > kFewSegments ? kMergeOne : kMergeFew;
      if (shared || most > 1) merge += ceil_div64((int64_t)p.n_tok * group, p.merge_rows) * n_heads;
    }
    a->merge_blocks = (int)merge;
    // (one sequence's join takes 16384 x 1024 / 4 workgroups at most)
    if (n == 1 || (fits && slots <= max_slots && merge <= kMaxGridBlocks)) return n;
  }
}

}  // namespace rv
