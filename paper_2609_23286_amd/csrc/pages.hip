// pages.hip -- rows into, out of and within the pages of a pool, gfx950.
//
// A page is 64 rows of every head; its rows of head h are [64][64] bf16 at page number `page` of the head's own
// array, for K and the same for V ([H][n_pages][64][64]: with all heads of a page together halving two memories of
// 52,000 rows took 162 us instead of 152).  A sequence's pages are listed in its row of the device's page table.  All
// kernels here move 16-byte chunks, eight lanes to a row's 128 bytes, so that every access is whole cache lines
// whatever rows are picked; they are bound by memory, and read and write past the caches' reuse (nontemporal: 184
// -> 162 us for the same).  Those 152 us move 852 MB (the kept rows to new pages and out again) at 5.6 TB/s, as much
// as a large copy reaches.  A workgroup finds its sequence by its first-block number.
#include "rv_internal.h"
#include "rv_ops.h"

namespace rv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int D = kHeadDim;
constexpr int NT = 256;
constexpr int kRowsPerBlock = NT / 8;
static_assert(kRowsPerBlock == kPageBlockRows, "the host counts workgroups by it");

// The last i < n whose block0 is at or below the workgroup's number (block0 ascends).
template <class S>
__device__ __forceinline__ int my_seq(const S* seq, int n) {
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int i = 0; i < n; i += 64)
    count += __popcll(__ballot(i + lane < n && seq[min(i + lane, n - 1)].block0 <= (int)blockIdx.x));
  return __builtin_amdgcn_readfirstlane(count - 1);
}

__device__ __forceinline__ int64_t page_at(int page, int n_pages, int h, int row) {
  return (((int64_t)h * n_pages + page) * kPageRows + row) * D;
}

__global__ __launch_bounds__(64) void table_kernel(TableArgs a) {
  const TableRun& r = a.run[blockIdx.x];
  for (int i = threadIdx.x; i < r.count; i += 64)
    a.table[r.dst + i] = r.copy ? a.table[r.src + i] : r.src + i;
}

// Frame rows [n][H][64] (or the picked ones of each head) to the sequences' pages.  Row i of a
// sequence, i < offset, is a row before `start` in its first page: copied where that page is copied.
__global__ __launch_bounds__(NT) void append_kernel(AppendArgs a) {
  const AppendSeq& s = a.seq[my_seq(a.seq, a.n_seqs)];
  const int H = a.n_heads, block = (int)blockIdx.x - s.block0;
  if (block == 0)
    for (int i = s.write0 + threadIdx.x; i < s.write0 + s.writes; i += NT)
      a.table[s.entry0 + i] = i == 0 ? s.page[0] : s.page[1] + i - 1;
  const int64_t r = (int64_t)block * kRowsPerBlock + (threadIdx.x >> 3);
  const int e = 8 * (threadIdx.x & 7);
  const int skip = s.cow >= 0 ? 0 : s.offset;  // rows of the first page that stay
  const int64_t rows = (int64_t)(s.offset + s.n - skip) * H;
  if (r >= rows) return;
  const int i = skip + (int)(r / H), h = (int)(r % H), p = i / kPageRows;
  const int page = p == 0 ? s.page[0] : p == 1 || s.in_a_row ? s.page[1] + p - 1 : a.table[s.entry0 + p];
  const int64_t to = page_at(page, a.n_pages, h, i % kPageRows) + e;
  u32x4 k, v;
  if (i < s.offset) {
    const int64_t from = page_at(s.cow, a.n_pages, h, i) + e;
    k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.K + from));
    v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.V + from));
  } else {
    const int j = i - s.offset;
    int64_t row = (int64_t)s.src_row + j;
    if (a.idx) {
      const int pick = a.idx[(int64_t)s.src_row * H + (int64_t)h * s.n + j];
      row = (int64_t)(s.src_row / s.n) * a.idx_tokens + min(max(pick, 0), a.idx_tokens - 1);
    }
    const int64_t from = (row * H + h) * D + e;
    k = *reinterpret_cast<const u32x4*>(a.srcK + from);
    v = *reinterpret_cast<const u32x4*>(a.srcV + from);
  }
  __builtin_nontemporal_store(k, reinterpret_cast<u32x4*>(a.K + to));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(a.V + to));
}

// Rows of sequences to [H][n][64] blocks.
__global__ __launch_bounds__(NT) void gather_kernel(GatherArgs a) {
  const GatherSeq& s = a.seq[my_seq(a.seq, a.n_seqs)];
  const int H = a.n_heads;
  const int64_t r = (int64_t)((int)blockIdx.x - s.block0) * kRowsPerBlock + (threadIdx.x >> 3);
  const int e = 8 * (threadIdx.x & 7);
  if (r >= (int64_t)s.n * H) return;
  const int h = (int)(r / s.n), i = s.offset + (int)(r - (int64_t)h * s.n);
  const int64_t from = page_at(a.table[s.entry0 + i / kPageRows], a.n_pages, h, i % kPageRows) + e;
  const int64_t to = (s.dst_row + r) * D + e;
  if (a.dstK) __builtin_nontemporal_store(__builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.K + from)), reinterpret_cast<u32x4*>(a.dstK + to));
  if (a.dstV) __builtin_nontemporal_store(__builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.V + from)), reinterpret_cast<u32x4*>(a.dstV + to));
}

// The kept rows of a sequence to its new pages.
__global__ __launch_bounds__(NT) void compact_kernel(CompactArgs a) {
  const CompactSeq& s = a.seq[my_seq(a.seq, a.n_seqs)];
  const int H = a.n_heads, block = (int)blockIdx.x - s.block0;
  const int64_t r = (int64_t)block * kRowsPerBlock + (threadIdx.x >> 3);
  const int e = 8 * (threadIdx.x & 7);
  const int per_head = s.offset + s.n, leading = s.base / kPageRows;
  if (block == 0 && s.page0 >= 0)
    for (int i = (int)threadIdx.x - leading; i < (per_head + kPageRows - 1) / kPageRows; i += NT)
      a.table[s.new0 + i] = i < 0 ? a.table[s.old0 + leading + i] : s.page0 + i;
  if (r >= (int64_t)per_head * H) return;
  const int h = (int)(r / per_head), i = (int)(r - (int64_t)h * per_head);
  int row = s.base + i;
  if (i >= s.offset) {
    row = a.keep[s.keep0 + (int64_t)h * s.n + (i - s.offset)];
    if (row < s.lo || row >= s.hi) row = -1;
  }
  u32x4 k = {0, 0, 0, 0}, v = k;
  if (row >= 0) {
    const int64_t from = page_at(a.table[s.old0 + row / kPageRows], a.n_pages, h, row % kPageRows) + e;
    k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.K + from));
    v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.V + from));
  }
  const int page = s.page0 >= 0 ? s.page0 + i / kPageRows : a.table[s.new0 + i / kPageRows];
  const int64_t to = page_at(page, a.n_pages, h, i % kPageRows) + e;
  __builtin_nontemporal_store(k, reinterpret_cast<u32x4*>(a.K + to));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(a.V + to));
}

}  // namespace

hipError_t launch_table(const TableArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(table_kernel, dim3((unsigned)a.n), dim3(64), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  if (a.blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)a.blocks), dim3(NT), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_gather(const GatherArgs& a, hipStream_t s) {
  if (a.blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(gather_kernel, dim3((unsigned)a.blocks), dim3(NT), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs& a, hipStream_t s) {
  if (a.blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(compact_kernel, dim3((unsigned)a.blocks), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace rv
