// attend_seqs.hip -- attention of several sequences' queries over paged rows, gfx950.
//
// As attend.hip for one frame (z = q k / 8, LSE = log sum exp z, o = sum exp(z - LSE) v), with the
// context of a query made of passes: a pass is a range of pages that a run of sequences has in
// common, with the queries of all of them as one list of rows (token, query head of the group), so
// that shared keys and values are read once for all.  A workgroup takes one query tile of one
// kv head over one piece of a pass's key tiles; a page is one tile.  Softmax sums of disjoint key
// sets combine exactly, so each piece writes its normalised output with its reference and row sum, and
// the merge launch joins, per query, the pieces of its sequence's pass and of the passes above
// it, in a fixed order.
#include <type_traits>

#include "attn_tile.h"
#include "rv_ops.h"

namespace rv {
namespace {

// The last i in [i0, n) whose value is at or below x (they ascend).
template <class F>
__device__ __forceinline__ int last_at_or_below(int i0, int n, int x, F value) {
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int i = i0; i < n; i += 64) count += __popcll(__ballot(i + lane < n && value(min(i + lane, n - 1)) <= x));
  return uniform(i0 + count - 1);
}

// The key tiles of a workgroup's pass: pages, then frame rows.
struct SeqCursor {
  const char *pk, *pv;   // this head's rows of page 0
  const char *fk, *fv;   // this head's rows of the pass's first token
  int64_t page_bytes;    // bytes between pages
  int64_t frame_bytes;   // bytes between frame tiles
  const int32_t* entry;  // the pass's table entries
  int pages;             // this lane's entry: of tile base + lane
  int base;
  int n_pages, n_tiles;
  int last_rows, frame_rows;  // valid rows of the last page and of the last frame tile
  uint32_t r, g0, g1;    // this thread's row (and row + 32) of a tile, byte offsets in the rows
  uint32_t frame_row;    // bytes between frame rows

  __device__ __forceinline__ int valid(int t) const {
    int v = BK;
    if (t == n_tiles - 1) v = frame_rows;
    if (t == n_pages - 1) v = last_rows;
    return v;
  }
  __device__ __forceinline__ void fetch_entries(int t) {  // of tiles t .. t + 63
    base = t;
    pages = entry[min(t + (int)(threadIdx.x & 63), n_pages - 1)];
  }
  // Tile t's K and V into a ring stage (the wave's rows of it).  Rows past the tile's last valid one
  // are read as that one: pages hold anything there, and their weights are zero only for numbers.
  __device__ __forceinline__ void load(int t, uint16_t* st) {
    const uint32_t last = (uint32_t)valid(t) - 1;
    const char *k, *v;
    uint32_t row;
    if (t < n_pages) {
      if (t - base >= 64) fetch_entries(t);
      const int64_t at = (int64_t)__builtin_amdgcn_readlane(pages, t - base) * page_bytes;
      k = pk + at;
      v = pv + at;
      row = D * 2;
    } else {
      const int64_t at = (t - n_pages) * frame_bytes;
      k = fk + at;
      v = fv + at;
      row = frame_row;
    }
    const uint32_t o0 = min(r, last) * row + g0, o1 = min(r + 32, last) * row + g1;
    lds_load16(k + o0, st);
    lds_load16(k + o1, st + 32 * D);
    lds_load16(v + o0, st + TILE);
    lds_load16(v + o1, st + TILE + 32 * D);
  }
};

__global__ __launch_bounds__(kAttnThreads, 2) void seq_fwd_kernel(SeqArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[NSTAGE * STAGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int H = a.n_heads, G = a.group;
  const int ip = last_at_or_below(0, a.n_pass, (int)blockIdx.x, [&](int i) { return a.pass[i].block0; });
  const SeqPass& p = a.pass[ip];
  // workgroups of a pass: head fastest, so that (the workgroups being dealt to the XCDs in turn) a
  // head's query tiles share an L2; then query tiles; then pieces
  const int b = (int)blockIdx.x - p.block0;
  const int h = uniform(b % H), qt = uniform(b / H % p.q_tiles), piece = uniform(b / H / p.q_tiles);
  const int n_tiles = p.n_pages + (p.frame + BK - 1) / BK;
  const int t0 = uniform((int)((int64_t)piece * n_tiles / p.pieces));
  const int t1 = uniform((int)((int64_t)(piece + 1) * n_tiles / p.pieces));
  const int rows = p.n_tok * G;

  SeqCursor tc;
  tc.pk = reinterpret_cast<const char*>(a.pageK + (int64_t)h * TILE);
  tc.pv = reinterpret_cast<const char*>(a.pageV + (int64_t)h * TILE);
  tc.fk = reinterpret_cast<const char*>(a.K + ((int64_t)p.tok0 * H + h) * D);
  tc.fv = reinterpret_cast<const char*>(a.V + ((int64_t)p.tok0 * H + h) * D);
  tc.page_bytes = (int64_t)H * TILE * 2;
  tc.frame_row = 2u * (uint32_t)(H * D);
  tc.frame_bytes = (int64_t)BK * tc.frame_row;
  tc.entry = a.table + p.entry0;
  tc.n_pages = p.n_pages;
  tc.n_tiles = n_tiles;
  tc.last_rows = p.last_rows;
  tc.frame_rows = p.frame > 0 ? p.frame - (n_tiles - p.n_pages - 1) * BK : p.last_rows;
  tc.r = tid >> 3;
  tc.g0 = 16u * ((tid & 7) ^ sw(tid >> 3));
  tc.g1 = 16u * ((tid & 7) ^ sw((tid >> 3) + 32));
  tc.base = t0;
  if (t0 < p.n_pages) tc.fetch_entries(t0);
  uint16_t* const ldsw = lds + wave * 8 * D;

  const int q0 = qt * BQ + wave * 32;  // this wave's first row of the pass
  const bool active = q0 < rows;
  bf16x8 qf[4];
  {
    const int r = min(q0 + l32, rows - 1);
    const uint16_t* qp = a.Q + (((int64_t)p.tok0 + r / G) * H * G + h * G + r % G) * D + half * 8;
#pragma unroll
    for (int ds = 0; ds < 4; ++ds) qf[ds] = *reinterpret_cast<const bf16x8*>(qp + ds * 16);
  }
  SoftmaxState sm;
  sm.m = kNegBig;
  sm.l = 0.f;
  sm.o0 = f32x16{};
  sm.o1 = f32x16{};

  // The ring of attend.hip: two tiles computed per barrier while the next two stream in.
  auto step = [&](auto phase, auto first, int t) {
    constexpr int P = decltype(phase)::value;
    if (t + 2 < t1) tc.load(t + 2, ldsw + (P + 2) % NSTAGE * STAGE);
    if (t + 3 < t1) tc.load(t + 3, ldsw + (P + 3) % NSTAGE * STAGE);
    if (active) {
      tile_compute<decltype(first)::value>(lds + P * STAGE, qf, lane, tc.valid(t), sm);
      if (t + 1 < t1) tile_compute<false>(lds + (P + 1) * STAGE, qf, lane, tc.valid(t + 1), sm);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  tc.load(t0, ldsw);
  if (t0 + 1 < t1) tc.load(t0 + 1, ldsw + STAGE);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  step(StageConst<0>{}, std::true_type{}, t0);
  for (int t = t0 + 2; t < t1; t = uniform(t + 4)) {
    step(StageConst<2>{}, std::false_type{}, t);
    if (t + 2 >= t1) break;
    step(StageConst<0>{}, std::false_type{}, t + 2);
  }

  // Rows through LDS, as whole 128-byte rows (the ring is free: the last step ended in a barrier).
  if (!active) return;  // uniform in the wave; no barrier follows
  const float l_tot = half_sum(sm.l);
  constexpr int kOutStageRow = D + 8;
  uint16_t* const st = lds + wave * 32 * kOutStageRow;
  {
    const float inv = 1.f / l_tot;
    uint16_t* sp = st + l32 * kOutStageRow + 4 * half;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      *reinterpret_cast<uint2*>(sp + 8 * j) =
          to_bf16x4(sm.o0[4 * j] * inv, sm.o0[4 * j + 1] * inv, sm.o0[4 * j + 2] * inv, sm.o0[4 * j + 3] * inv);
      *reinterpret_cast<uint2*>(sp + 32 + 8 * j) =
          to_bf16x4(sm.o1[4 * j] * inv, sm.o1[4 * j + 1] * inv, sm.o1[4 * j + 2] * inv, sm.o1[4 * j + 3] * inv);
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const int r8 = lane >> 3, c8 = (lane & 7) * 8;
  if (p.slot0 < 0) {
    if (half == 0 && q0 + l32 < rows) {
      const int r = q0 + l32;
      a.lse[(int64_t)p.tok0 * H * G + (int64_t)(h * G + r % G) * p.n_tok + r / G] = (sm.m + __log2f(l_tot)) * kLn2;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = q0 + 8 * i + r8;
      if (r < rows)
        *reinterpret_cast<uint4*>(a.out + (((int64_t)p.tok0 + r / G) * H * G + h * G + r % G) * D + c8) =
            *reinterpret_cast<const uint4*>(st + (8 * i + r8) * kOutStageRow + c8);
    }
    return;
  }
  const int sub = ((h * p.q_tiles + qt) * p.pieces + piece) * (BQ / kSubRows) + wave;
  float* const ps = a.part + (int64_t)(p.slot0 + sub) * kSubFloats;
  if (half == 0) {
    ps[kSubRows * D / 2 + l32] = sm.m;
    ps[kSubRows * D / 2 + kSubRows + l32] = l_tot;
  }
  uint16_t* const po = reinterpret_cast<uint16_t*>(ps);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (q0 + 8 * i + r8 < rows)
      *reinterpret_cast<uint4*>(po + (8 * i + r8) * D + c8) =
          *reinterpret_cast<const uint4*>(st + (8 * i + r8) * kOutStageRow + c8);
}

// Joins the pieces of 32 rows of one sequence and kv head, eight threads a row.
__global__ __launch_bounds__(256) void seq_merge_kernel(SeqArgs a) {
  const int H = a.n_heads, G = a.group;
  const int ip = last_at_or_below(a.n_inner, a.n_pass, (int)blockIdx.x, [&](int i) { return a.pass[i].merge0; });
  const SeqPass& leaf = a.pass[ip];
  const int b = (int)blockIdx.x - leaf.merge0;
  const int h = uniform(b % H), rb = uniform(b / H);
  const int row = rb * kSubRows + (threadIdx.x >> 3), d8 = (threadIdx.x & 7) * 8;
  if (row >= leaf.n_tok * G) return;
  constexpr int kBatch = 8;  // pieces whose loads are in flight together
  float mmax = kNegBig, L = 0.f;
  float acc[8] = {};
  for (int i = ip; i >= 0; i = a.pass[i].parent) {
    const SeqPass& p = a.pass[i];
    const int r = (leaf.tok0 - p.tok0) * G + row, per_tile = p.tile_rows / kSubRows;
    const int qt = r / p.tile_rows, sub = r % p.tile_rows / kSubRows, rr = r % kSubRows;
    const float* const first =
        a.part + ((int64_t)p.slot0 + (int64_t)(h * p.q_tiles + qt) * p.pieces * per_tile + sub) * kSubFloats;
    for (int j0 = 0; j0 < p.pieces; j0 += kBatch) {
      float mv[kBatch], lv[kBatch];
      uint4 v[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float* ps = first + (int64_t)min(j0 + j, p.pieces - 1) * per_tile * kSubFloats;
        mv[j] = ps[kSubRows * D / 2 + rr];
        lv[j] = ps[kSubRows * D / 2 + kSubRows + rr];
        v[j] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(ps) + rr * D + d8);
      }
      float m_new = mmax;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) m_new = fmaxf(m_new, mv[j]);  // clamped copies repeat a real one
      const float scale = __builtin_amdgcn_exp2f(mmax - m_new);
      L *= scale;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= scale;
      mmax = m_new;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float w = j0 + j < p.pieces ? __builtin_amdgcn_exp2f(mv[j] - mmax) * lv[j] : 0.f;
        L += w;
        const uint32_t wd[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[2 * e] = fmaf(w, __uint_as_float(wd[e] << 16), acc[2 * e]);
          acc[2 * e + 1] = fmaf(w, __uint_as_float(wd[e] & 0xFFFF0000u), acc[2 * e + 1]);
        }
      }
    }
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;  // no key at all: zeros, and a log-sum-exp of -inf
  const int tok = row / G, head = h * G + row % G;
  const uint2 lo = to_bf16x4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  const uint2 hi = to_bf16x4(acc[4] * inv, acc[5] * inv, acc[6] * inv, acc[7] * inv);
  *reinterpret_cast<uint4*>(a.out + (((int64_t)leaf.tok0 + tok) * H * G + head) * D + d8) =
      make_uint4(lo.x, lo.y, hi.x, hi.y);
  if (d8 == 0)
    a.lse[(int64_t)leaf.tok0 * H * G + (int64_t)head * leaf.n_tok + tok] =
        L > 0.f ? (mmax + __log2f(L)) * kLn2 : -__builtin_inff();
}

}  // namespace

hipError_t launch_attend_seqs(const SeqArgs& a, hipStream_t s) {
  if (a.blocks > 0) {
    hipLaunchKernelGGL(seq_fwd_kernel, dim3((unsigned)a.blocks), dim3(kAttnThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.merge_blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(seq_merge_kernel, dim3((unsigned)a.merge_blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rv
