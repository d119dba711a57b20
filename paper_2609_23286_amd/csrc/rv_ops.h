// rv_ops.h -- argument blocks and host-side planning of the operators around a frame's
// attention (not installed): the projection's norms and rotation, the page pool, and the
// attention of several sequences over shared pages.  Plain C++ with no HIP dependency, as
// rv_plan.h.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/rv.h"
#include "rv_plan.h"

namespace rv {

// Workgroups of 256 threads a launch may have: a grid holds fewer than 2^32 threads.
constexpr int kMaxGridBlocks = 1 << 23;

// ---- projection outputs to frame tensors ------------------------------------------------

constexpr int kMaxFreqs = kHeadDim / 2;
constexpr int kPrepThreads = 256;
constexpr int kPrepRows = 8;       // heads a wave takes at a time
constexpr int kPrepMaxTokens = 8;  // tokens a wave takes at a time

// Source and gradient rows are [n_tokens] rows of `stride` elements, head h at column 64 h.
struct PrepArgs {
  const void *q, *k, *v;        // bf16 or fp32 (v may be NULL)
  int64_t q_stride, k_stride, v_stride;
  const int32_t* pos;           // [n_tokens][axes]
  uint16_t *Q, *K, *V;          // [n][Hq][64]; row j of kv head h at K / V + j kv_row + h kv_head
  int64_t kv_row, kv_head;
  const float *qw, *qb, *kw, *kb;  // [64] or NULL
  const uint16_t *dQ, *dK, *dV;    // backward: [n][H][64] (dV may be NULL)
  void *dq, *dk, *dv;
  int64_t dq_stride, dk_stride, dv_stride;
  float* part;                     // backward: [blocks][4][64] weight and bias sums
  float *dqw, *dqb, *dkw, *dkb;    // [64] or NULL
  int n_tokens, n_q_heads, n_kv_heads;
  int norm;
  float eps;
  int tokens_per_wave;
  int blocks;
  uint64_t freq[kMaxFreqs];     // turns a position, in 2^-64 turns
};

// The turns one position step rotates pair i of an axis block by, base^(-i / n_freqs) / (2 pi),
// as a fraction of 2^64: the product with a position wraps modulo whole turns, so the phase of
// any 32-bit position is exact to 2^-32 turns.
void rotation_turns(double base, int n_freqs, uint64_t* out);

// ---- page pool --------------------------------------------------------------------------

constexpr int kPageRows = RV_PAGE_ROWS;
static_assert(kPageRows == kAttnBK, "a page is one key tile of the attention");

// A run of page-table entries: entry dst + i becomes page src + i, or (copy) entry src + i.
struct TableRun {
  int32_t dst, src, count, copy;
};
constexpr int kMaxRuns = 240;
constexpr int kPageBlockRows = 32;  // rows (of one head) a workgroup of the row-moving kernels takes
struct TableArgs {
  int32_t* table;
  int n;
  TableRun run[kMaxRuns];
};

// Rows written to sequences: sequence i's rows start at `start`, `n` of them from row src_row of
// the packed frame.  The page that holds row `start` and the one after it are given here; the pages after
// that follow the second in number (their entries are written here), or were entered by an earlier launch.
struct AppendSeq {
  int32_t block0;     // its first workgroup
  int32_t entry0;     // table entry of the page that holds row `start`
  int32_t page[2];
  int32_t write0, writes;  // entries written here: those of pages write0 .. write0 + writes - 1 of the ones touched
  int32_t in_a_row;   // the pages after the second are given by its number
  int32_t cow;        // page whose rows before `start` are copied to page[0], or -1
  int32_t offset;     // start % 64
  int32_t n;
  int32_t src_row;
};
constexpr int kMaxAppend = 64;
struct AppendArgs {
  uint16_t *K, *V;    // pages [H][n_pages][64][64]
  int32_t* table;
  const uint16_t *srcK, *srcV;  // row j of head h: src + (src_row + j) H 64 + h 64
  const int32_t* idx;           // NULL, or per sequence [H][n]: row j of head h is frame token
                                //   idx[h][j] (sequence i's block starts at H src_row)
  int idx_tokens;               // ... of a frame of this many tokens, sequence i's at i idx_tokens
  int n_heads, n_pages, n_seqs, blocks;
  AppendSeq seq[kMaxAppend];
};

// Rows copied out of sequences into [H][n][64] blocks.
struct GatherSeq {
  int32_t block0;
  int32_t entry0;     // table entry of the page that holds row `first`
  int32_t offset;     // first % 64
  int32_t n;
  int64_t dst_row;    // sum of H n over earlier sequences
};
constexpr int kMaxGather = 128;
struct GatherArgs {
  const uint16_t *K, *V;
  const int32_t* table;
  uint16_t *dstK, *dstV;  // either may be NULL
  int n_heads, n_pages, n_seqs, blocks;
  GatherSeq seq[kMaxGather];
};

// Rows of sequences gathered into new pages: row i >= offset of head h comes from row
// keep[h][i - offset] of the old table row, row i < offset (the rows kept in place at the head
// of the first new page) from old row base + i.
struct CompactSeq {
  int32_t block0;
  int32_t old0, new0;  // first entries of the old table row and of the first new page
  int32_t base;        // row of the sequence that the first new page starts at
  int32_t offset;
  int32_t n;           // kept rows after `offset`
  int32_t lo, hi;      // rows that `keep` may name: [lo, hi)
  int32_t page0;       // new pages are page0, page0 + 1, ..., and the new table row is written here (the
                       //   `base` / 64 entries before them copied); -1: an earlier launch wrote it
  int64_t keep0;       // sum of H n over earlier sequences
};
constexpr int kMaxCompact = 64;
struct CompactArgs {
  uint16_t *K, *V;
  int32_t* table;
  const int32_t* keep;
  int n_heads, n_pages, n_seqs, blocks;
  CompactSeq seq[kMaxCompact];
};

// A kernel's arguments hold at most 4 KB.
static_assert(sizeof(TableArgs) <= 4096 && sizeof(AppendArgs) <= 4096 && sizeof(GatherArgs) <= 4096 &&
              sizeof(CompactArgs) <= 4096, "kernel arguments");

// Which sequence holds which pages, on the host.  Every array is allocated by init(), so no later
// call allocates.  Entries of sequence s lie at row(s) * width; a compaction builds the new list in
// the sequence's other row, so that the old one stays readable on the device meanwhile.
class PageBook {
 public:
  PageBook() = default;
  ~PageBook();
  PageBook(const PageBook&) = delete;
  PageBook& operator=(const PageBook&) = delete;
  bool init(int n_pages, int max_seqs, int width);  // false: no memory

  int width() const { return width_; }
  int max_seqs() const { return max_seqs_; }
  int free_pages() const { return n_free_; }
  bool is_open(int s) const { return s >= 0 && s < max_seqs_ && open_[s]; }
  int64_t len(int s) const { return len_[s]; }
  int pages(int s) const { return (int)((len_[s] + kPageRows - 1) / kPageRows); }
  int32_t entry0(int s) const { return (2 * s + side_[s]) * width_; }
  int32_t page(int s, int i) const { return table_[entry0(s) + i]; }
  const int32_t* list(int s) const { return table_ + entry0(s); }
  bool in_a_row(int s, int from) const;  // pages from index `from` on are consecutive numbers
  int users(int page) const { return refs_[page]; }
  // True once for every sequence of a batch: begin_batch() first.
  void begin_batch() { ++batch_; }
  bool first_in_batch(int s);

  int open();                             // a new, empty sequence, or -1
  int can_open() const { return n_closed_; }
  void close(int s);
  void fork(int child, int s, int64_t n_rows);
  void truncate(int s, int64_t n_rows);

  // Pages that appending n rows takes, the copy of a shared last page included.
  int append_pages(int s, int64_t n) const;
  bool append_copies(int s, int64_t n) const;  // whether the last page is shared and has to be copied
  // Gives s the pages of n more rows.  A page that was copied is dropped by release_dropped(), so
  // that nothing of this batch is written to a page that it still reads.  Returns that page or -1.
  int append(int s, int64_t n);
  // Gives s a new list: its pages before row `first`, then new ones up to `n_rows` rows, in its
  // other table row.  The old pages are dropped by release_dropped().
  int compact_pages(int64_t first, int64_t n_rows) const;
  void compact(int s, int64_t first, int64_t n_rows);
  void release_dropped();

 private:
  int take();
  void drop(int page) { if (--refs_[page] == 0) free_[n_free_++] = page; }
  int n_pages_ = 0, max_seqs_ = 0, width_ = 0, n_free_ = 0, n_closed_ = 0, n_dropped_ = 0, n_moved_ = 0;
  int64_t batch_ = 0;
  int32_t *table_ = nullptr, *refs_ = nullptr, *free_ = nullptr, *closed_ = nullptr;
  int32_t *dropped_ = nullptr;  // pages that appends copied
  int32_t *moved_ = nullptr, *old_pages_ = nullptr;  // compacted sequences, and how many pages each had
  int64_t *len_ = nullptr, *stamp_ = nullptr;
  uint8_t *open_ = nullptr, *side_ = nullptr;
};

// ---- attention of several sequences ----------------------------------------------------

// A pass: queries of consecutive tokens over a range of pages that all of them attend to (and,
// for one sequence's own pass, the frame keys of its tokens).  Passes form a forest: a sequence's
// context is its own pass (a leaf) and the passes above it.
//
// A unit is one query tile of one kv head of a pass; its work is the pass's key tiles, each of
// `cost` positions, and `fixed` more before its second.  Units are numbered through all passes.  Where they are
// more than the device's workgroup slots, the first `rounds` times `width` may be dealt out whole, one of a
// round to each workgroup, so that neighbours (query tiles of a head) go over the same keys at the same time.
// The positions of the others, one unit after another from pos_first on, are cut into chunks of E, one workgroup
// each: a tile belongs to the chunk that its first position lies in.
struct SeqPass {
  int32_t pos0;       // first position
  int32_t unit0;      // first unit
  int32_t tok0, n_tok;
  int32_t entry0;     // table entry of the first page
  int32_t n_pages;
  int32_t last_rows;  // valid rows of the last page
  int32_t frame;      // frame keys: n_tok or 0
  int32_t parent;     // pass above, or -1
  int32_t q_tiles;    // query tiles of tile_rows rows
  int32_t tile_rows;  // 128, or 32 where the pass has few queries
  int32_t cost;       // positions of a key tile
  int32_t fixed;      // positions of a unit's start and end
  int32_t slot0;      // shared passes (inner ones, and leaves below one): slot of unit 0 and chunk 0
  int32_t merge_rows; // leaves: rows a merge workgroup takes
};
constexpr int kMaxPasses = 52;
constexpr int kSubRows = 32;  // rows of a partial slot of this launch
constexpr int kSubFloats = kSubRows * kHeadDim + 2 * kSubRows;  // fp32 rows, references, row sums
constexpr int kSubsPerTile = kAttnBQ / kSubRows;
constexpr int kMergeOne = 4, kMergeFew = 16;  // rows a merge workgroup takes: a wave one, or four
struct SeqShares {
  int32_t each, more;  // chunks an XCD, and XCDs that take one more
};
struct SeqArgs {
  const uint16_t *Q, *K, *V;      // packed frames [tokens][Hq or H][64]; K, V NULL without frame keys
  const uint16_t *pageK, *pageV;  // [H][n_pages][64][64]
  const int32_t* table;
  uint16_t* out;
  float* lse;
  float* part;
  int n_heads, n_pages, group;    // kv heads, pages of the pool, query heads to each kv head
  int n_pass, n_inner;            // passes; the first n_inner are not leaves
  int rounds, width;              // whole units to a workgroup, and workgroups that take them
  int pos_first, total, E, chunks;  // positions of the units that are cut: [pos_first, total), chunks of E
  int inner_chunks;               // chunks that begin in an inner pass
  SeqShares inner, leaves;        // the XCDs' shares of them and of the others (and places in a round)
  int n_queues;                   // XCDs that the workgroups are dealt over
  int merge_blocks;
  int32_t pos0[kMaxPasses];    // the passes' first positions and units, again (a workgroup finds its pass by them)
  int32_t unit0[kMaxPasses];
  int32_t merge0[kMaxPasses];  // leaves: first workgroup of the merge launch
  SeqPass pass[kMaxPasses];
};
static_assert(sizeof(SeqArgs) <= 4096, "kernel arguments");

RV_HD inline int seq_tiles(const SeqPass& p) { return p.n_pages + (p.frame + kAttnBK - 1) / kAttnBK; }
// First position of a unit's tile.
RV_HD inline int seq_pos(const SeqPass& p, int unit, int tile) {
  return p.pos0 + unit * (p.fixed + seq_tiles(p) * p.cost) + (tile > 0 ? p.fixed + tile * p.cost : 0);
}
// The first tile (returned) and unit whose position is at or after pos0 + off; the unit may be past the last.
RV_HD inline int seq_first_tile(const SeqPass& p, int T, int off, int* unit) {
  const int per = p.fixed + T * p.cost, u = off / per, rest = off - u * per;
  int t = rest <= 0 ? 0 : rest <= p.fixed + p.cost ? 1 : (rest - p.fixed + p.cost - 1) / p.cost;
  *unit = t < T ? u : u + 1;
  return t < T ? t : 0;
}
// The chunk (and place in a round) of workgroup (x, j), or -1.  Workgroups are dealt to the XCDs in turn, x first;
// consecutive chunks (query tiles of a head) go to one XCD, and each XCD gets its share of the inner passes' chunks,
// which are bound by arithmetic, and of the leaves', which are bound by memory.
RV_HD inline int seq_share0(const SeqShares& s, int x) { return x * s.each + (x < s.more ? x : s.more); }
template <class A>
RV_HD inline int seq_chunk_of(const A& a, int x, int j) {
  const int ni = a.inner.each + (x < a.inner.more ? 1 : 0), nl = a.leaves.each + (x < a.leaves.more ? 1 : 0);
  if (j < ni) return seq_share0(a.inner, x) + j;
  return j - ni < nl ? a.inner_chunks + seq_share0(a.leaves, x) + j - ni : -1;
}
template <class A>
RV_HD inline int seq_grid(const A& a) {  // workgroups an XCD
  return a.inner.each + (a.inner.more > 0) + a.leaves.each + (a.leaves.more > 0);
}

template <class A>
RV_HD inline int seq_chunk_at(const A& a, int pos) { return (pos - a.pos_first) / a.E; }
// Whether a unit was dealt out whole.
template <class A>
RV_HD inline bool seq_whole(const A& a, const SeqPass& p, int unit) { return p.unit0 + unit < a.rounds * a.width; }

// Partial slot of the segment of unit `unit` that chunk c takes, where c0 is the unit's first chunk.
// Shared passes: a slot for each unit and chunk (their sum grows with each segment).  Other
// units write partial results only where they are cut, and a unit of n chunks takes the n slots from
// 2 c0 + 1 on; the next one begins in chunk c0 + n - 1 at the earliest.
RV_HD inline int seq_slot_step(const SeqPass& p, bool shared) { return shared ? p.tile_rows / kSubRows : kSubsPerTile; }
RV_HD inline int seq_slot(const SeqPass& p, bool shared, int unit, int c, int c0) {
  return shared ? p.slot0 + (unit + c) * seq_slot_step(p, true) : (c0 + c + 1) * kSubsPerTile;
}

struct SeqSpan {  // one sequence of a batch, as the plan sees it
  int seq;
  int n_tok;
};

// Rows of a query tile of a pass of q_rows (token, query head of the group) rows.
RV_HD inline int seq_tile_rows(int64_t q_rows) { return q_rows <= kSubRows ? kSubRows : kAttnBQ; }

// Whether one sequence's queries fit a launch, whose positions are 32-bit numbers: its units, each of its key tiles
// and kSeqTilesMore, come to fewer than kMaxSeqTiles.
constexpr int64_t kMaxSeqTiles = (int64_t)1 << 28, kSeqTilesMore = 4;
bool seq_fits(int64_t rows, int n_tok, bool frame, int n_heads, int group);

// Plans one launch for sequences [0, n) of a batch (tokens packed in order, the first at tok0), each of which
// fits: fills a's passes, returns how many of the sequences it covers (>= 1).
int plan_seqs(const PageBook& book, const SeqSpan* spans, int n, int tok0, bool frame, int n_heads, int group,
              int n_cus, int64_t max_slots, SeqArgs* a);

inline int64_t ceil_div64(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace rv
