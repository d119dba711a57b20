// rv_pool.cpp -- librv host side of the page pool and the attention over its sequences: argument
// checks, the page lists, and launches.
#include <algorithm>
#include <climits>
#include <mutex>
#include <new>

#include "rv_host.h"

struct rv_pool_s {
  int device = 0;
  int n_heads = 0, n_pages = 0;
  int64_t max_rows = 0;
  uint16_t* K = nullptr;
  uint16_t* V = nullptr;
  int32_t* table = nullptr;
  rv::PageBook book;
  std::mutex mu;
};

namespace {

using rv::fail;
using rv::kPageRows;
typedef std::lock_guard<std::mutex> Lock;

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Page-table entries to be written, sent in launches of kMaxRuns runs.
class Runs {
 public:
  explicit Runs(rv_pool p, hipStream_t s) : s_(s) {
    a_.table = p->table;
    a_.n = 0;
  }
  hipError_t add(int32_t dst, int32_t src, int32_t count, bool copy) {
    if (count <= 0) return hipSuccess;
    if (a_.n > 0 && !copy) {
      rv::TableRun& l = a_.run[a_.n - 1];
      if (!l.copy && l.dst + l.count == dst && l.src + l.count == src) {
        l.count += count;
        return hipSuccess;
      }
    }
    if (a_.n == rv::kMaxRuns) {
      const hipError_t e = flush();
      if (e != hipSuccess) return e;
    }
    a_.run[a_.n++] = rv::TableRun{dst, src, count, copy ? 1 : 0};
    return hipSuccess;
  }
  hipError_t flush() {
    const hipError_t e = rv::launch_table(a_, s_);
    a_.n = 0;
    return e;
  }

 private:
  rv::TableArgs a_;
  hipStream_t s_;
};

rv_status check_pool(rv_pool p) {
  if (!p) return fail(RV_ERR_INVALID, "pool is NULL");
  return rv::check_current(p->device, "pool");
}

// Open sequences; `once`: each named once.
rv_status check_seqs(rv_pool p, int n, const int* seqs, bool once) {
  if (n < 0) return fail(RV_ERR_INVALID, "the number of sequences must be >= 0 (got %d)", n);
  if (n > 0 && !seqs) return fail(RV_ERR_INVALID, "seqs is NULL");
  if (once) p->book.begin_batch();
  for (int i = 0; i < n; ++i) {
    if (!p->book.is_open(seqs[i])) return fail(RV_ERR_INVALID, "sequence %d is not open", seqs[i]);
    if (once && !p->book.first_in_batch(seqs[i])) return fail(RV_ERR_INVALID, "sequence %d is named twice", seqs[i]);
  }
  return RV_OK;
}

int64_t blocks_of(int64_t rows) { return rv::ceil_div64(rows, rv::kPageBlockRows); }

// Whether appending n_rows[i] rows (all `same` where n_rows is NULL) to the sequences can go ahead.
rv_status check_append(rv_pool p, int n, const int* seqs, const int* n_rows, int same, int64_t* total) {
  int64_t pages = 0;
  *total = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t r = n_rows ? n_rows[i] : same;
    if (r < 0) return fail(RV_ERR_INVALID, "sequence %d: n_rows must be >= 0", seqs[i]);
    if (p->book.len(seqs[i]) + r > p->max_rows)
      return fail(RV_ERR_CAPACITY, "sequence %d would exceed max_rows", seqs[i]);
    if (blocks_of((r + kPageRows) * p->n_heads) > rv::kMaxGridBlocks)
      return fail(RV_ERR_INVALID, "sequence %d: too many rows for one call", seqs[i]);
    pages += p->book.append_pages(seqs[i], r);
    *total += r;
  }
  if (*total > INT32_MAX) return fail(RV_ERR_INVALID, "too many rows for one call");
  if (pages > p->book.free_pages())
    return fail(RV_ERR_CAPACITY, "the rows take %lld pages, %d are free", (long long)pages, p->book.free_pages());
  return RV_OK;
}

// Appends (the checks have passed).  idx as in AppendArgs.
rv_status append(rv_pool p, int n, const int* seqs, const void* K, const void* V, const int* n_rows, int same,
                 const int32_t* idx, int idx_tokens, hipStream_t s) {
  rv::PageBook& book = p->book;
  rv::AppendArgs a{};
  a.K = p->K;
  a.V = p->V;
  a.table = p->table;
  a.srcK = (const uint16_t*)K;
  a.srcV = (const uint16_t*)V;
  a.idx = idx;
  a.idx_tokens = idx_tokens;
  a.n_heads = p->n_heads;
  a.n_pages = p->n_pages;
  Runs runs(p, s);
  hipError_t err = hipSuccess;
  auto flush = [&]() {
    if (err == hipSuccess) err = runs.flush();
    if (err == hipSuccess) err = rv::launch_append(a, s);
    a.n_seqs = a.blocks = 0;
  };
  int src_row = 0;
  // (a failed launch stops the launches, not the lists: they stay in line with themselves)
  for (int i = 0; i < n; ++i) {
    const int r = n_rows ? n_rows[i] : same;
    if (r == 0) continue;
    const int64_t start = book.len(seqs[i]);
    const int old = book.append(seqs[i], r);
    const int first = (int)(start / kPageRows), end = book.pages(seqs[i]);
    rv::AppendSeq d{};
    d.entry0 = book.entry0(seqs[i]) + first;
    d.offset = (int)(start % kPageRows);
    d.cow = old;
    d.page[0] = book.page(seqs[i], first);
    d.page[1] = first + 1 < end ? book.page(seqs[i], first + 1) : d.page[0];
    // entries to write: of the first page where it is new or a copy, and of all after it
    d.write0 = d.offset == 0 || old >= 0 ? 0 : 1;
    d.in_a_row = book.in_a_row(seqs[i], first + 1) ? 1 : 0;
    d.writes = (d.in_a_row ? end - first : std::min(end - first, 2)) - d.write0;
    d.n = r;
    d.src_row = src_row;
    src_row += r;
    const int64_t blocks = blocks_of((int64_t)(r + (old >= 0 ? d.offset : 0)) * p->n_heads);
    if (a.n_seqs == rv::kMaxAppend || a.blocks + blocks > rv::kMaxGridBlocks) flush();
    for (int k = first + 2; !d.in_a_row && k < end && err == hipSuccess; ++k)
      err = runs.add(d.entry0 + (k - first), book.page(seqs[i], k), 1, false);
    d.block0 = a.blocks;
    a.blocks += (int)blocks;
    a.seq[a.n_seqs++] = d;
  }
  flush();
  book.release_dropped();
  RV_HIP(err, "append launch");
  return RV_OK;
}

}  // namespace

extern "C" {

rv_status rv_pool_create(int n_heads, int head_dim, int n_pages, int max_seqs, int64_t max_rows, rv_pool* out) {
  if (!out) return fail(RV_ERR_INVALID, "out is NULL");
  *out = nullptr;
  if (n_heads < 1 || n_heads > 1024) return fail(RV_ERR_INVALID, "n_heads must be in [1, 1024] (got %d)", n_heads);
  if (head_dim != rv::kHeadDim) return fail(RV_ERR_INVALID, "head_dim must be 64 (got %d)", head_dim);
  if (n_pages < 1 || max_seqs < 1 || max_rows < 1 || max_rows > (int64_t)1 << 30)
    return fail(RV_ERR_INVALID, "need n_pages >= 1, max_seqs >= 1 and max_rows in [1, 2^30]");
  const int64_t width = rv::ceil_div64(max_rows, kPageRows), entries = 2 * width * max_seqs;
  if (entries > INT32_MAX) return fail(RV_ERR_INVALID, "max_seqs sequences of max_rows rows need too large a page table");
  rv_status st = rv::setup_sequences();
  if (st != RV_OK) return st;
  rv_pool p = new (std::nothrow) rv_pool_s;
  if (!p) return fail(RV_ERR_OOM, "host allocation failed");
  p->n_heads = n_heads;
  p->n_pages = n_pages;
  p->max_rows = max_rows;
  const size_t bytes = (size_t)n_pages * n_heads * kPageRows * rv::kHeadDim * 2;
  hipError_t e = hipGetDevice(&p->device);
  if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&p->K), bytes);
  if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&p->V), bytes);
  if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&p->table), (size_t)entries * sizeof(int32_t));
  if (e == hipSuccess) e = hipMemset(p->table, 0, (size_t)entries * sizeof(int32_t));
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    st = rv::hip_fail(e, "page pool allocation");
  } else if (!p->book.init(n_pages, max_seqs, (int)width)) {  // (after the device's: a size it has room for)
    st = fail(RV_ERR_OOM, "host allocation failed");
  }
  if (st != RV_OK) {
    (void)hipGetLastError();
    (void)hipFree(p->K);
    (void)hipFree(p->V);
    (void)hipFree(p->table);
    delete p;
    return st;
  }
  *out = p;
  return RV_OK;
}

rv_status rv_pool_destroy(rv_pool p) {
  if (!p) return RV_OK;
  int prev = 0;
  (void)hipGetDevice(&prev);
  (void)hipSetDevice(p->device);
  (void)hipDeviceSynchronize();
  (void)hipFree(p->K);
  (void)hipFree(p->V);
  (void)hipFree(p->table);
  (void)hipSetDevice(prev);
  delete p;
  return RV_OK;
}

int rv_pool_free_pages(rv_pool p) {
  if (!p) return -1;
  Lock lk(p->mu);
  return p->book.free_pages();
}

rv_status rv_pool_open(rv_pool p, int* seq) {
  if (!p || !seq) return fail(RV_ERR_INVALID, "NULL argument");
  Lock lk(p->mu);
  const int s = p->book.open();
  if (s < 0) return fail(RV_ERR_CAPACITY, "all %d sequences are open", p->book.max_seqs());
  *seq = s;
  return RV_OK;
}

int64_t rv_pool_len(rv_pool p, int seq) {
  if (!p) return -1;
  Lock lk(p->mu);
  return p->book.is_open(seq) ? p->book.len(seq) : -1;
}

rv_status rv_pool_fork(rv_pool p, int seq, int64_t n_rows, int n, int* children, void* stream) {
  rv_status st = check_pool(p);
  if (st != RV_OK) return st;
  Lock lk(p->mu);
  if ((st = check_seqs(p, 1, &seq, false)) != RV_OK) return st;
  if (n < 0 || (n > 0 && !children)) return fail(RV_ERR_INVALID, "need n >= 0 and room for the children");
  if (n_rows < 0 || n_rows > p->book.len(seq))
    return fail(RV_ERR_INVALID, "n_rows must be in [0, length %lld] (got %lld)", (long long)p->book.len(seq),
                (long long)n_rows);
  if (n > p->book.can_open()) return fail(RV_ERR_CAPACITY, "%d sequences can be opened, not %d", p->book.can_open(), n);
  Runs runs(p, (hipStream_t)stream);
  hipError_t e = hipSuccess;
  for (int i = 0; i < n; ++i) {
    const int c = p->book.open();
    p->book.fork(c, seq, n_rows);
    children[i] = c;
    if (e == hipSuccess) e = runs.add(p->book.entry0(c), p->book.entry0(seq), p->book.pages(c), true);
  }
  if (e == hipSuccess) e = runs.flush();
  RV_HIP(e, "fork launch");
  return RV_OK;
}

rv_status rv_pool_close(rv_pool p, int n, const int* seqs) {
  if (!p) return fail(RV_ERR_INVALID, "pool is NULL");
  Lock lk(p->mu);
  rv_status st = check_seqs(p, n, seqs, true);
  if (st != RV_OK) return st;
  for (int i = 0; i < n; ++i) p->book.close(seqs[i]);
  return RV_OK;
}

rv_status rv_pool_truncate(rv_pool p, int seq, int64_t n_rows) {
  if (!p) return fail(RV_ERR_INVALID, "pool is NULL");
  Lock lk(p->mu);
  rv_status st = check_seqs(p, 1, &seq, false);
  if (st != RV_OK) return st;
  if (n_rows < 0 || n_rows > p->book.len(seq))
    return fail(RV_ERR_INVALID, "n_rows must be in [0, length %lld] (got %lld)", (long long)p->book.len(seq),
                (long long)n_rows);
  p->book.truncate(seq, n_rows);
  return RV_OK;
}

rv_status rv_pool_append(rv_pool p, int n, const int* seqs, const void* K, const void* V, const int* n_rows,
                         void* stream) {
  rv_status st = check_pool(p);
  if (st != RV_OK) return st;
  Lock lk(p->mu);
  if ((st = check_seqs(p, n, seqs, true)) != RV_OK) return st;
  if (n > 0 && !n_rows) return fail(RV_ERR_INVALID, "n_rows is NULL");
  int64_t total;
  if ((st = check_append(p, n, seqs, n_rows, 0, &total)) != RV_OK) return st;
  if (total == 0) return RV_OK;
  if (!K || !V) return fail(RV_ERR_INVALID, "K and V are required");
  if (!aligned(K) || !aligned(V)) return fail(RV_ERR_INVALID, "K and V must be 16-byte aligned");
  return append(p, n, seqs, K, V, n_rows, 0, nullptr, 0, (hipStream_t)stream);
}

rv_status rv_pool_gather(rv_pool p, int n, const int* seqs, const int64_t* first, const int64_t* n_rows, void* K,
                         void* V, void* stream) {
  rv_status st = check_pool(p);
  if (st != RV_OK) return st;
  Lock lk(p->mu);
  if ((st = check_seqs(p, n, seqs, false)) != RV_OK) return st;
  if (n > 0 && !n_rows) return fail(RV_ERR_INVALID, "n_rows is NULL");
  if (!aligned(K) || !aligned(V)) return fail(RV_ERR_INVALID, "K and V must be 16-byte aligned");
  for (int i = 0; i < n; ++i) {
    const int64_t f = first ? first[i] : 0, len = p->book.len(seqs[i]);
    if (f < 0 || n_rows[i] < 0 || f > len || n_rows[i] > len - f)
      return fail(RV_ERR_INVALID, "sequence %d: rows %lld .. + %lld of %lld", seqs[i], (long long)f,
                  (long long)n_rows[i], (long long)len);
    if (blocks_of(n_rows[i] * p->n_heads) > rv::kMaxGridBlocks)
      return fail(RV_ERR_INVALID, "sequence %d: too many rows for one call", seqs[i]);
  }
  if (!K && !V) return RV_OK;
  rv::GatherArgs a{};
  a.K = p->K;
  a.V = p->V;
  a.table = p->table;
  a.dstK = (uint16_t*)K;
  a.dstV = (uint16_t*)V;
  a.n_heads = p->n_heads;
  a.n_pages = p->n_pages;
  int64_t dst_row = 0;
  for (int i = 0; i < n; ++i) {
    if (n_rows[i] == 0) continue;
    const int64_t f = first ? first[i] : 0, blocks = blocks_of(n_rows[i] * p->n_heads);
    if (a.n_seqs == rv::kMaxGather || a.blocks + blocks > rv::kMaxGridBlocks) {
      RV_HIP(rv::launch_gather(a, (hipStream_t)stream), "gather launch");
      a.n_seqs = a.blocks = 0;
    }
    a.seq[a.n_seqs++] = rv::GatherSeq{a.blocks, (int32_t)(p->book.entry0(seqs[i]) + f / kPageRows),
                                      (int32_t)(f % kPageRows), (int32_t)n_rows[i], dst_row};
    a.blocks += (int)blocks;
    dst_row += n_rows[i] * p->n_heads;
  }
  RV_HIP(rv::launch_gather(a, (hipStream_t)stream), "gather launch");
  return RV_OK;
}

rv_status rv_pool_compact(rv_pool p, int n, const int* seqs, const int64_t* first, const int64_t* n_keep,
                          const int32_t* keep, void* stream) {
  rv_status st = check_pool(p);
  if (st != RV_OK) return st;
  Lock lk(p->mu);
  if ((st = check_seqs(p, n, seqs, true)) != RV_OK) return st;
  if (n > 0 && !n_keep) return fail(RV_ERR_INVALID, "n_keep is NULL");
  rv::PageBook& book = p->book;
  int64_t pages = 0, total = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t f = first ? first[i] : 0, len = book.len(seqs[i]);
    if (f < 0 || f > len) return fail(RV_ERR_INVALID, "sequence %d: first must be in [0, length %lld]", seqs[i],
                                      (long long)len);
    if (n_keep[i] < 0) return fail(RV_ERR_INVALID, "sequence %d: n_keep must be >= 0", seqs[i]);
    if (n_keep[i] > p->max_rows - f) return fail(RV_ERR_CAPACITY, "sequence %d would exceed max_rows", seqs[i]);
    if (blocks_of((n_keep[i] + kPageRows) * p->n_heads) > rv::kMaxGridBlocks)
      return fail(RV_ERR_INVALID, "sequence %d: too many rows for one call", seqs[i]);
    if (n_keep[i] > 0) pages += book.compact_pages(f, f + n_keep[i]);
    total += n_keep[i];
  }
  if (total > 0 && !keep) return fail(RV_ERR_INVALID, "keep is NULL");
  if (pages > book.free_pages())
    return fail(RV_ERR_CAPACITY, "the kept rows take %lld pages, %d are free", (long long)pages, book.free_pages());

  hipStream_t s = (hipStream_t)stream;
  rv::CompactArgs a{};
  a.K = p->K;
  a.V = p->V;
  a.table = p->table;
  a.keep = keep;
  a.n_heads = p->n_heads;
  a.n_pages = p->n_pages;
  Runs runs(p, s);
  hipError_t err = hipSuccess;
  auto flush = [&]() {
    if (err == hipSuccess) err = runs.flush();
    if (err == hipSuccess) err = rv::launch_compact(a, s);
    a.n_seqs = a.blocks = 0;
  };
  int64_t keep0 = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t f = first ? first[i] : 0, len = book.len(seqs[i]);
    if (n_keep[i] == 0) {  // nothing to gather: the pages before `first` stay as they are
      book.truncate(seqs[i], f);
      continue;
    }
    rv::CompactSeq d{};
    const int leading = (int)(f / kPageRows);
    d.old0 = book.entry0(seqs[i]);
    book.compact(seqs[i], f, f + n_keep[i]);
    const int32_t new0 = book.entry0(seqs[i]);
    d.new0 = new0 + leading;
    d.base = leading * kPageRows;
    d.offset = (int)(f % kPageRows);
    d.n = (int32_t)n_keep[i];
    d.lo = (int32_t)f;
    d.hi = (int32_t)len;
    d.keep0 = keep0;
    keep0 += n_keep[i] * p->n_heads;
    const int64_t blocks = blocks_of((int64_t)(d.offset + d.n) * p->n_heads);
    if (a.n_seqs == rv::kMaxCompact || a.blocks + blocks > rv::kMaxGridBlocks) flush();
    d.page0 = book.in_a_row(seqs[i], leading) ? book.page(seqs[i], leading) : -1;
    if (d.page0 < 0) {
      if (err == hipSuccess) err = runs.add(new0, d.old0, leading, true);
      for (int k = leading; k < book.pages(seqs[i]) && err == hipSuccess; ++k)
        err = runs.add(new0 + k, book.page(seqs[i], k), 1, false);
    }
    d.block0 = a.blocks;
    a.blocks += (int)blocks;
    a.seq[a.n_seqs++] = d;
  }
  flush();
  book.release_dropped();
  RV_HIP(err, "compact launch");
  return RV_OK;
}

rv_status rv_attend_seqs(rv_pool p, int n, const int* seqs, const int* n_tokens, const void* Q, const void* K,
                         const void* V, int n_q_heads, void* out, float* lse, void* stream) {
  rv_status st = check_pool(p);
  if (st != RV_OK) return st;
  Lock lk(p->mu);
  if ((st = check_seqs(p, n, seqs, false)) != RV_OK) return st;
  if (n_q_heads < 1 || n_q_heads > 1024 || n_q_heads % p->n_heads != 0)
    return fail(RV_ERR_INVALID, "n_q_heads must be a multiple of %d, at most 1024 (got %d)", p->n_heads, n_q_heads);
  if (n > 0 && !n_tokens) return fail(RV_ERR_INVALID, "n_tokens is NULL");
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (n_tokens[i] < 0 || n_tokens[i] > rv::kMaxTokens)
      return fail(RV_ERR_INVALID, "n_tokens must be in [0, %d] (got %d)", rv::kMaxTokens, n_tokens[i]);
    total += n_tokens[i];
  }
  if (total > INT32_MAX / 2) return fail(RV_ERR_INVALID, "too many tokens for one call");
  if (!K != !V) return fail(RV_ERR_INVALID, "K and V must both be given or both be NULL");
  if (total == 0) return RV_OK;
  for (int i = 0; i < n; ++i)  // (all of them before the first launch)
    if (!rv::seq_fits(p->book.len(seqs[i]), n_tokens[i], K != nullptr, p->n_heads, n_q_heads / p->n_heads))
      return fail(RV_ERR_INVALID, "sequence %d: too many tokens over too many rows for one call", seqs[i]);
  if (!Q || !out || !lse) return fail(RV_ERR_INVALID, "Q, out and lse are required");
  if (!aligned(Q) || !aligned(K) || !aligned(V) || !aligned(out))
    return fail(RV_ERR_INVALID, "Q, K, V and out must be 16-byte aligned");
  rv::DeviceContext ctx;
  if ((st = rv::device_context(&ctx)) != RV_OK) return st;
  rv::SeqArgs a{};
  a.Q = (const uint16_t*)Q;
  a.K = (const uint16_t*)K;
  a.V = (const uint16_t*)V;
  a.pageK = p->K;
  a.pageV = p->V;
  a.table = p->table;
  a.out = (uint16_t*)out;
  a.lse = lse;
  a.part = ctx.seq_part;
  a.n_heads = p->n_heads;
  a.n_pages = p->n_pages;
  a.group = n_q_heads / p->n_heads;
  a.n_queues = ctx.n_queues;
  int tok0 = 0;
  for (int i = 0; i < n;) {
    rv::SeqSpan span[rv::kMaxPasses];
    int at[rv::kMaxPasses], m = 0;  // the next sequences with queries, and where each is in the batch
    for (int k = i; k < n && m < rv::kMaxPasses - 1; ++k)
      if (n_tokens[k] > 0) {
        span[m] = rv::SeqSpan{seqs[k], n_tokens[k]};
        at[m++] = k;
      }
    if (m == 0) break;
    const int done = rv::plan_seqs(p->book, span, m, tok0, K != nullptr, p->n_heads, a.group, ctx.n_cus,
                                   (int64_t)(ctx.seq_floats / rv::kSubFloats), &a);
    RV_HIP(rv::launch_attend_seqs(a, (hipStream_t)stream), "attention launch");
    for (int k = 0; k < done; ++k) tok0 += span[k].n_tok;
    i = at[done - 1] + 1;
  }
  return RV_OK;
}

rv_status rv_admit_seqs(rv_pool p, int n, const int* seqs, const void* Q, const void* K, const void* V,
                        const float* lse, int n_tokens, const rv_qsub* qs, int budget, float* saliency_out,
                        int32_t* idx_out, void* stream) {
  rv_status st = check_pool(p);
  if (st != RV_OK) return st;
  Lock lk(p->mu);
  if (n > 4096) return fail(RV_ERR_INVALID, "at most 4096 sequences a call");
  if ((st = check_seqs(p, n, seqs, true)) != RV_OK) return st;
  if (n_tokens < 1 || n_tokens > rv::kMaxTokens)
    return fail(RV_ERR_INVALID, "n_tokens must be in [1, %d] (got %d)", rv::kMaxTokens, n_tokens);
  if (budget < 0 || budget > n_tokens)
    return fail(RV_ERR_INVALID, "budget must be in [0, n_tokens] (got %d)", budget);
  if (const char* why = rv::qsub_problem(qs, n_tokens)) return fail(RV_ERR_INVALID, "%s", why);
  if (n == 0) return RV_OK;
  if (!Q || !K || !V || !lse || !saliency_out || (budget > 0 && !idx_out))
    return fail(RV_ERR_INVALID, "Q, K, V, lse, saliency_out and idx_out are required");
  if (!aligned(Q) || !aligned(K) || !aligned(V)) return fail(RV_ERR_INVALID, "Q, K and V must be 16-byte aligned");
  int64_t total;
  if ((st = check_append(p, n, seqs, nullptr, budget, &total)) != RV_OK) return st;
  rv::DeviceContext ctx;
  if ((st = rv::device_context(&ctx)) != RV_OK) return st;
  const int H = p->n_heads;
  rv::AdmitArgs b{};
  b.n_tokens = n_tokens;
  b.n_heads = H;
  b.budget = budget;
  b.mode = rv::kModeBoth;
  b.sal_xcds = ctx.n_queues;
  rv::set_qsub(&b, *qs);
  rv::plan_saliency(&b, std::min(n, rv::kMaxLayersPerLaunch) * H, ctx.n_cus, ctx.max_lds);
  if (rv::admit_lds_bytes(b) > (size_t)rv::admit_max_dynamic_lds(ctx.max_lds))
    return fail(RV_ERR_INVALID, "frame too large for the admission workgroup's LDS");
  const int64_t frame = (int64_t)n_tokens * H;
  for (int i0 = 0; i0 < n; i0 += rv::kMaxLayersPerLaunch) {
    b.n_layers = std::min(rv::kMaxLayersPerLaunch, n - i0);
    for (int i = 0; i < b.n_layers; ++i) {
      rv::AdmitLayer& L = b.layer[i];
      L.Q = (const uint16_t*)Q + (i0 + i) * frame * rv::kHeadDim;
      L.K = (const uint16_t*)K + (i0 + i) * frame * rv::kHeadDim;
      L.kv_row = (int64_t)H * rv::kHeadDim;
      L.kv_head = rv::kHeadDim;
      L.lse = lse + (i0 + i) * frame;
      L.sal = saliency_out + (i0 + i) * frame;
      L.idx = idx_out ? idx_out + (int64_t)(i0 + i) * H * budget : nullptr;
    }
    RV_HIP(rv::launch_admit(b, ctx.max_lds, (hipStream_t)stream), "admit launch");
  }
  if (budget == 0) return RV_OK;
  return append(p, n, seqs, K, V, nullptr, budget, idx_out, n_tokens, (hipStream_t)stream);
}

}  // extern "C"
