// attend_seqs.hip -- attention of several sequences' queries over paged rows, gfx950.
//
// As attend.hip for one frame (z = q k / 8, LSE = log sum exp z, o = sum exp(z - LSE) v), with the
// context of a query made of passes: a pass is a range of pages that a run of sequences has in
// common, with the queries of all of them as one list of rows (token, query head of the group), so
// that shared keys and values are read once for all.  The key tiles (a page is one) of all
// units -- a query tile of one kv head of a pass -- are one list, cut into equal chunks, a workgroup
// each.  Softmax sums of disjoint key sets combine exactly, so a segment of a unit writes its
// sums with their reference, and the merge launch joins, per query, the segments of its sequence's
// pass and of the passes above it, in a fixed order.
//
// A query tile has 128 rows, 32 a wave, over key tiles that the workgroup loads together (as attend.hip's core), or
// 32 where a pass has no more, each wave taking key tiles of its own and no barrier among them.  What bounds them:
// many queries, the core's stalls (attend.hip): four sequences' frames of 1041 tokens over 5000 shared rows and 100 to
// 430 of their own 146 us, 736 TFLOP/s; one frame over 52,000 rows 271 us.  Few queries, memory, and over shared rows
// both: 48 sequences of 5 tokens over 52,000 shared rows and 242 to 1041 of their own 105 us (at a large copy's rate
// the bytes, 340 MB, are 66; at the core's rate the 240 rows over the shared pages are 60 and the others' bytes 25).
// A token each of 16 sequences over 10,000 rows of its own, 655 MB: 118 us, 5.6 TB/s; over 9990 shared rows, latency:
// 18 us, 13 of them the forward launch (3.6 until a workgroup has its place, 2 for the first keys, the rest two or
// three tiles and the write of the sums), 5 the merge.
#include <type_traits>

#include "attn_tile.h"
#include "rv_ops.h"

namespace rv {
namespace {

// The last i in [i0, n) with values[i] <= x (they ascend, and the first is not above x).  The load waits for no
// other one: every lane's element is there, whatever i0 and n.
static_assert(kMaxPasses <= 64, "a lane each");
__device__ __forceinline__ int last_at_or_below(const int32_t (&values)[kMaxPasses], int i0, int n, int x) {
  const int lane = threadIdx.x & 63, v = values[min(lane, kMaxPasses - 1)];
  return uniform(63 - __builtin_clzll(__ballot(lane >= i0 && lane < n && v <= x) | 1));
}

// The key tiles of a workgroup's pass: pages, then frame rows.
struct SeqCursor {
  const char *pk, *pv;   // this head's rows of page 0
  const char *fk, *fv;   // this head's rows of the pass's first token
  const int32_t* entry;  // the pass's table entries
  int n_pages, n_tiles;
  int last_rows, frame_rows;  // valid rows of the last page and of the last frame tile
  uint32_t frame_row;    // bytes between frame rows

  __device__ __forceinline__ int valid(int t) const {
    int v = BK;
    if (t == n_tiles - 1) v = frame_rows;
    if (t == n_pages - 1) v = last_rows;
    return v;
  }
};

__device__ __forceinline__ const char* uniform_ptr(const char* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)x), hi = (uint32_t)uniform((int)(uint32_t)(x >> 32));
  return reinterpret_cast<const char*>((uint64_t)hi << 32 | lo);
}

// Where a tile's rows lie (uniform).
struct TileRows {
  const char *k, *v;
  uint32_t row;   // bytes between rows
  uint32_t last;  // last valid row: rows past it are read as that one (pages hold anything there,
                  // and a weight of zero makes zero only of numbers)
};

// The tiles a wave loads, in turn: index i is tile first + i step (modulo the segment).  Their page numbers are
// held a lane each and fetched 64 at a time, so that no tile's addresses wait for memory (a scalar load of the
// entry for each tile cost a tenth of the forward launch).
struct TileOrder {
  int first, step;
  int up, wrap;   // indices from `up` on go back by `wrap` tiles
  int base = 0;   // index of lane 0's page
  int pages;      // this lane's page number
  __device__ __forceinline__ int at(int i) const { return first + i * step - (i >= up ? wrap : 0); }
  __device__ __forceinline__ void fetch(const SeqCursor& tc, int i) {
    base = i;
    pages = tc.n_pages > 0 ? tc.entry[max(0, min(at(i + (int)(threadIdx.x & 63)), tc.n_pages - 1))] : 0;
    // (Read here, so that the wait for it stands here: at its use the compiler would wait, for every tile, for all
    // the loads of the tiles before: 3 % of a frame over 52,000 rows.)
    asm volatile("" : "+v"(pages));
  }
  __device__ __forceinline__ TileRows rows(const SeqCursor& tc, int i) {
    const int t = at(i);
    TileRows r;
    r.last = (uint32_t)tc.valid(t) - 1;
    if (t < tc.n_pages) {  // uniform
      if (i - base >= 64) fetch(tc, i);
      const int64_t at = (int64_t)__builtin_amdgcn_readlane(pages, i - base) * (TILE * 2);
      r.k = tc.pk + at;
      r.v = tc.pv + at;
      r.row = D * 2;
    } else {
      const int64_t at = (int64_t)(t - tc.n_pages) * BK * tc.frame_row;
      r.k = tc.fk + at;
      r.v = tc.fv + at;
      r.row = tc.frame_row;
    }
    r.k = uniform_ptr(r.k);
    r.v = uniform_ptr(r.v);
    return r;
  }
};

// Lane l's 16 bytes at base + off go to LDS byte lds + 16 l.  (Assembly: the compiler would wait for
// every such load in flight before each LDS read.  No register is written.  The wait states are
// those a scalar that a vector instruction wrote needs before a load reads it.)
__device__ __forceinline__ void lds_load16_asm(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(lds) : "memory");
}

// A tile's K and V into a ring stage by the whole workgroup: `st` is the LDS byte of the stage plus this wave's row
// block (rows 8w .. 8w + 7; the second load of each fills rows 32 + 8w ..).
__device__ __forceinline__ void load_tile(const TileRows& ts, uint32_t st) {
  const uint32_t r = threadIdx.x >> 3, c = threadIdx.x & 7;
  const uint32_t o0 = min(r, ts.last) * ts.row + 16u * (c ^ sw(r));
  const uint32_t o1 = min(r + 32, ts.last) * ts.row + 16u * (c ^ sw(r + 32));
  lds_load16_asm(ts.k, o0, st);
  lds_load16_asm(ts.k, o1, st + 32 * D * 2);
  lds_load16_asm(ts.v, o0, st + TILE * 2);
  lds_load16_asm(ts.v, o1, st + TILE * 2 + 32 * D * 2);
}

constexpr int kHalf = 32;  // keys of a wave's stage

// ---- 32 queries over 32 keys ------------------------------------------------------------------

// Scores: entry r is key 8 (r / 4) + 4 half + r % 4.
__device__ __forceinline__ f32x16 score(const uint16_t* keys, const bf16x8 (&qf)[4], int lane) {
  f32x16 z = {};
#pragma unroll
  for (int ds = 0; ds < 4; ++ds)
    z = mfma32(*reinterpret_cast<const bf16x8*>(&keys[swz(lane & 31, ds * 2 + (lane >> 5))]), qf[ds], z);
  return z;
}
// Keys >= valid get -1e30 (arithmetically: lane masks would take the scalar registers).
__device__ __forceinline__ void mask_scores(f32x16& z, int lane, int valid) {
  const float fv = (float)(valid - 4 * (lane >> 5) - 1);
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = fmaf(__saturatef((float)(8 * (r >> 2) + (r & 3)) - fv), kNegBig, z[r]);
}
// p = 2^(z log2(e) / 8 - m), rounded to bf16 as the value product's operand (the values are bf16, and the matrix
// instruction takes both operands in one type): outputs are 0.0021 to 0.0024 of their size from the exact ones, 0.0017
// of it by their own rounding.  Returns this lane's share of their sum, of the unrounded ones (summed after rounding,
// two to an instruction, the log-sum-exp of 63 keys was 2e-4 off).
__device__ __forceinline__ float exponentials(const f32x16& z, float m, bf16x8 (&p)[2]) {
  float sum = -0.f;  // -0 + x == x: the first add folds away
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    const float e0 = __builtin_amdgcn_exp2f(fmaf(z[r], kScaleLog2, -m));
    const float e1 = __builtin_amdgcn_exp2f(fmaf(z[r + 1], kScaleLog2, -m));
    sum += e0 + e1;
    p[r >> 3][r & 7] = (__bf16)e0;
    p[r >> 3][(r & 7) + 1] = (__bf16)e1;
  }
  return sum;
}

// 32 keys and values in LDS.  The running reference follows tile_compute's rule: where some lane's sum reaches 2^64
// (every p is infinite while the reference is unset) it is raised to the keys' maximum and p formed again.
__device__ __forceinline__ void compute(const uint16_t* keys, const uint16_t* values, const bf16x8 (&qf)[4], int lane,
                                        int valid, SoftmaxState& sm) {
  f32x16 z = score(keys, qf, lane);
  if (__builtin_expect(valid < kHalf, 0)) mask_scores(z, lane, valid);
  // V^T fragments through transposing reads, as in tile_compute
  bf16x8 vf[2][2], p[2];
  const int g = lane >> 4, i16 = lane & 15, rr = i16 >> 2, jj = i16 & 3, hh = g >> 1;
  const int col = 16 * (g & 1) + 4 * jj;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int db = 0; db < 2; ++db) {
      const int row = ks * 16 + 4 * hh + rr, lcol = db * 32 + col;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(values + swz(row, lcol >> 3) + (lcol & 7)));
      const i16x4 hi =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(values + swz(row + 8, lcol >> 3) + (lcol & 7)));
      vf[ks][db] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  float sum = exponentials(z, sm.m, p);
  if (__builtin_expect(__any(!(sum < kOverflowGuard)), 0)) {
    float mx = z[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, z[r]);
    const float m_new = fmaxf(sm.m, half_max(mx) * kScaleLog2);
    const float alpha = __builtin_amdgcn_exp2f(sm.m - m_new);
    sm.l *= alpha;
    sm.o0 *= alpha;
    sm.o1 *= alpha;
    sm.m = m_new;
    sum = exponentials(z, m_new, p);
  }
  sm.l += sum;
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    sm.o0 = mfma32(vf[ks][0], p[ks], sm.o0);
    sm.o1 = mfma32(vf[ks][1], p[ks], sm.o1);
  }
}

// ---- few queries: every wave takes tiles of its own -------------------------------------------

constexpr int kHalfStage = 2 * kHalf * D;   // K rows then V rows: 8 KB
constexpr int kHalfLoads = 8;               // load instructions of a stage
static_assert(2 * 4 * kHalfStage == NSTAGE * STAGE, "four waves' two stages fill the same LDS");

// Half hk (32 keys) of a tile into a wave's stage at LDS byte `st`, 8 rows an instruction.
__device__ __forceinline__ void load_half(const TileRows& ts, int hk, uint32_t st, int lane) {
  const uint32_t r0 = lane >> 3, c = lane & 7;
  if (ts.last == BK - 1) {  // uniform: two thread offsets (the swizzle alternates) beside scalar bases
    const uint32_t o = r0 * ts.row, o0 = o + 16u * (c ^ sw(r0)), o1 = o + 16u * (c ^ sw(r0 + 8));
    const int64_t at = (int64_t)(kHalf * hk) * ts.row, step = 8 * (int64_t)ts.row;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lds_load16_asm(ts.k + at + i * step, i & 1 ? o1 : o0, st + i * 8 * D * 2);
      lds_load16_asm(ts.v + at + i * step, i & 1 ? o1 : o0, st + kHalf * D * 2 + i * 8 * D * 2);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t r = 8 * i + r0;
      const uint32_t off = min(r + kHalf * hk, ts.last) * ts.row + 16u * (c ^ sw(r));
      lds_load16_asm(ts.k, off, st + i * 8 * D * 2);
      lds_load16_asm(ts.v, off, st + kHalf * D * 2 + i * 8 * D * 2);
    }
  }
}

// ---- results ----------------------------------------------------------------------------------

// A wave's 32 output rows staged in LDS as fp32, stride kRowStride (16-byte aligned; the 32 rows' pieces
// spread over the banks).
constexpr int kRowStride = D + 4;
__device__ __forceinline__ void stage_rows(const SoftmaxState& sm, float* st, int lane) {
  float* sp = st + (lane & 31) * kRowStride + 4 * (lane >> 5);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    *reinterpret_cast<float4*>(sp + 8 * j) =
        make_float4(sm.o0[4 * j], sm.o0[4 * j + 1], sm.o0[4 * j + 2], sm.o0[4 * j + 3]);
    *reinterpret_cast<float4*>(sp + 32 + 8 * j) =
        make_float4(sm.o1[4 * j], sm.o1[4 * j + 1], sm.o1[4 * j + 2], sm.o1[4 * j + 3]);
  }
}

// Eight elements d8 .. of an output row (unnormalised, row sum l, reference m): final, or into the
// workgroup's partial slot (fp32: rounding it to bf16 would cost as much again as the output's own rounding).
__device__ __forceinline__ void write_row(const SeqArgs& a, const SeqPass& p, int h, int r, int d8, const float (&o)[8],
                                          float m, float l, float* slot) {
  if (!slot) {
    const int G = a.group, HG = a.n_heads * G, tok = r / G, head = h * G + r % G;
    const float inv = 1.f / l;
    const uint2 lo = to_bf16x4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    const uint2 hi = to_bf16x4(o[4] * inv, o[5] * inv, o[6] * inv, o[7] * inv);
    *reinterpret_cast<uint4*>(a.out + (((int64_t)p.tok0 + tok) * HG + head) * D + d8) =
        make_uint4(lo.x, lo.y, hi.x, hi.y);
    if (d8 == 0) a.lse[(int64_t)p.tok0 * HG + (int64_t)head * p.n_tok + tok] = (m + __log2f(l)) * kLn2;
    return;
  }
  const int rr = r % kSubRows;
  float* const row = slot + rr * D + d8;
  *reinterpret_cast<float4*>(row) = make_float4(o[0], o[1], o[2], o[3]);
  *reinterpret_cast<float4*>(row + 4) = make_float4(o[4], o[5], o[6], o[7]);
  if (d8 == 0) {
    slot[kSubRows * D + rr] = m;
    slot[kSubRows * D + kSubRows + rr] = l;
  }
}

// A segment: tiles t0 .. t1 - 1 of one unit, taken in the order ts .. t1 - 1, t0 .. ts - 1.
struct Segment {
  int h, qt, t0, t1, ts;
  float* slots;   // partial slots of the segment, or NULL: it is the whole unit, and final
};

__device__ __forceinline__ void load_queries(const SeqArgs& a, const SeqPass& p, int h, int q0, int lane, bf16x8 (&qf)[4]) {
  const int G = a.group, r = min(q0 + (lane & 31), p.n_tok * G - 1);
  const uint16_t* qp = a.Q + (((int64_t)p.tok0 + r / G) * a.n_heads * G + h * G + r % G) * D + (lane >> 5) * 8;
#pragma unroll
  for (int ds = 0; ds < 4; ++ds) qf[ds] = *reinterpret_cast<const bf16x8*>(qp + ds * 16);
}

// Few queries: the waves share them and take every fourth tile each, half a tile at a time through
// two stages of their own, without barriers; the loads of the next half run under this one's work.
__device__ __forceinline__ void narrow_segment(const SeqArgs& a, const SeqPass& p, const SeqCursor& tc, const Segment& g,
                                               uint16_t* lds, float (*s_m)[kSubRows], float (*s_l)[kSubRows]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int q0 = g.qt * kSubRows;
  bf16x8 qf[4];
  load_queries(a, p, g.h, q0, lane, qf);
  SoftmaxState sm;
  sm.m = kNegBig;
  sm.l = 0.f;
  sm.o0 = f32x16{};
  sm.o1 = f32x16{};
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_void*)(lds + wave * 2 * kHalfStage);
  const uint16_t* const st0 = lds + wave * 2 * kHalfStage;
  const uint16_t* const st1 = st0 + kHalfStage;
  const int n = g.t1 - g.t0 > wave ? (g.t1 - g.t0 - wave + 3) / 4 : 0;  // tiles of this wave
  TileOrder order{g.t0 + wave, 4, 1 << 30, 0};
  TileRows next{};
  if (n > 0) {
    order.fetch(tc, 0);
    next = order.rows(tc, 0);
  }
  // (the queries pass through a wait here: the compiler's own for them would wait for the tiles too)
  asm volatile("s_waitcnt vmcnt(0)" : "+v"(qf[0]), "+v"(qf[1]), "+v"(qf[2]), "+v"(qf[3])::"memory");
  if (n > 0) {
    load_half(next, 0, ring, lane);
    load_half(next, 1, ring + kHalfStage * 2, lane);
  }
  for (int i = 0; i < n; i = uniform(i + 1)) {
    const int valid = tc.valid(order.at(i));
    const bool more = i + 1 < n;
    if (more) next = order.rows(tc, i + 1);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kHalfLoads) : "memory");
    compute(st0, st0 + kHalf * D, qf, lane, valid, sm);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) {
      load_half(next, 0, ring, lane);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kHalfLoads) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    if (valid > kHalf) compute(st1, st1 + kHalf * D, qf, lane, valid - kHalf, sm);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load_half(next, 1, ring + kHalfStage * 2, lane);
  }
  // The four waves' sums meet in LDS.
  const float l_tot = half_sum(sm.l);
  __syncthreads();
  float* const st = reinterpret_cast<float*>(lds);
  stage_rows(sm, st + wave * kSubRows * kRowStride, lane);
  if (half == 0) {
    s_m[wave][l32] = sm.m;
    s_l[wave][l32] = l_tot;
  }
  __syncthreads();
  const int rr = tid >> 3, d8 = (tid & 7) * 8, r = q0 + rr;
  if (r < p.n_tok * a.group) {
    float m = s_m[0][rr];
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, s_m[w][rr]);
    float l = 0.f, o[8] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][rr] - m);
      l = fmaf(f, s_l[w][rr], l);
      const float* x = st + (w * kSubRows + rr) * kRowStride + d8;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf(f, x[e], o[e]);
    }
    write_row(a, p, g.h, r, d8, o, m, l, g.slots);
  }
  __syncthreads();  // (the LDS is the next segment's)
}

// Many queries: 32 to a wave, and a ring of four tiles, two computed per barrier while the next two stream in.
__device__ __forceinline__ void wide_segment(const SeqArgs& a, const SeqPass& p, const SeqCursor& tc, const Segment& g,
                                             uint16_t* lds, float (*s_m)[kSubRows], float (*s_l)[kSubRows]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  const int q0 = g.qt * BQ + wave * 32, rows = p.n_tok * a.group, t0 = g.t0, t1 = g.t1;
  bf16x8 qf[4];
  load_queries(a, p, g.h, q0, lane, qf);
  SoftmaxState sm;
  sm.m = kNegBig;
  sm.l = 0.f;
  sm.o0 = f32x16{};
  sm.o1 = f32x16{};
  const bool active = q0 < rows;
  const int n = t1 - t0;
  TileOrder order{g.ts, 1, t1 - g.ts, n};
  order.fetch(tc, 0);
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_void*)lds + wave * 8 * D * 2;
  constexpr uint32_t kStageBytes = STAGE * 2;
  load_tile(order.rows(tc, 0), ring);
  if (n > 1) load_tile(order.rows(tc, 1), ring + kStageBytes);
  // (the queries pass through the wait: the compiler's own for them would wait for tiles in the loop)
  asm volatile("s_waitcnt vmcnt(0)" : "+v"(qf[0]), "+v"(qf[1]), "+v"(qf[2]), "+v"(qf[3])::"memory");
  __syncthreads();
  auto step = [&](auto phase, auto first, int i) {
    constexpr int P = decltype(phase)::value;
    if (i + 2 < n) load_tile(order.rows(tc, i + 2), ring + (P + 2) % NSTAGE * kStageBytes);
    if (i + 3 < n) load_tile(order.rows(tc, i + 3), ring + (P + 3) % NSTAGE * kStageBytes);
    if (active) {
      tile_compute<decltype(first)::value>(lds + P * STAGE, qf, lane, tc.valid(order.at(i)), sm);
      if (i + 1 < n) tile_compute<false>(lds + (P + 1) * STAGE, qf, lane, tc.valid(order.at(i + 1)), sm);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  step(StageConst<0>{}, std::true_type{}, 0);
  for (int i = 2; i < n; i = uniform(i + 4)) {
    step(StageConst<2>{}, std::false_type{}, i);
    if (i + 2 >= n) break;
    step(StageConst<0>{}, std::false_type{}, i + 2);
  }

  // Rows through LDS, so that whole rows are written (the ring is free: the last step ended in a barrier).
  if (active) {  // uniform in the wave
    const float l_tot = half_sum(sm.l);
    float* const st = reinterpret_cast<float*>(lds) + wave * kSubRows * kRowStride;
    stage_rows(sm, st, lane);
    if (half == 0) {
      s_m[wave][l32] = sm.m;
      s_l[wave][l32] = l_tot;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (g.slots) {
      // all 32 rows (those past the last query's are never read), 1 KB of them a store
      float* const slot = g.slots + wave * kSubFloats;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int rr = 4 * i + (lane >> 4), d4 = (lane & 15) * 4;
        *reinterpret_cast<float4*>(slot + rr * D + d4) = *reinterpret_cast<const float4*>(st + rr * kRowStride + d4);
      }
      slot[kSubRows * D + lane] = half ? s_l[wave][l32] : s_m[wave][l32];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int rr = 8 * i + (lane >> 3), d8 = (lane & 7) * 8;
        if (q0 + rr >= rows) continue;
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = st[rr * kRowStride + d8 + e];
        write_row(a, p, g.h, q0 + rr, d8, o, s_m[wave][rr], s_l[wave][rr], nullptr);
      }
    }
  }
  __syncthreads();  // (the LDS is the next segment's)
}

__global__ __launch_bounds__(kAttnThreads, 2) void seq_fwd_kernel(SeqArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[NSTAGE * STAGE];
  __shared__ float s_m[4][kSubRows], s_l[4][kSubRows];
  const int c = uniform(seq_chunk_of(a, (int)blockIdx.x, (int)blockIdx.y));
  if (c < 0) return;
  const int H = a.n_heads;
  // A whole unit of each round, then the chunk's segments.
  const int begin = a.pos_first + c * a.E, end = c < a.chunks ? min(begin + a.E, a.total) : 0;
  int round = c < a.width ? 0 : a.rounds;
  int pos = begin;  // the chunk's positions from here on are still to be done
  int ip = round < a.rounds ? 0 : last_at_or_below(a.pos0, 0, a.n_pass, begin);
  int done = 0;     // tiles this workgroup has taken of its chunk
  while (round < a.rounds || pos < end) {
    const bool whole = round < a.rounds;
    int unit;
    Segment g;
    if (whole) {
      const int u = uniform(round * a.width + c);
      ip = last_at_or_below(a.unit0, 0, a.n_pass, u);
      unit = u - a.unit0[ip];
      g.t0 = 0;
      g.t1 = seq_tiles(a.pass[ip]);
      g.slots = nullptr;
    } else {
      const SeqPass& p = a.pass[ip];
      const int T = seq_tiles(p), units = H * p.q_tiles;
      unit = 0;
      const int t0 = T == 0 ? 0 : uniform(seq_first_tile(p, T, pos - p.pos0, &unit));
      unit = uniform(unit);
      if (T == 0 || unit >= units) {
        if (++ip >= a.n_pass) break;
        pos = max(pos, a.pos0[ip]);  // (the chunk may begin inside the last tile before it)
        continue;
      }
      int end_unit = 0;
      const int end_tile = uniform(seq_first_tile(p, T, end - p.pos0, &end_unit));
      const int t1 = uniform(end_unit) > unit ? T : end_tile;
      if (uniform(end_unit) < unit || t1 <= t0) break;  // the last positions belong to a tile that began before
      const bool shared = ip < a.n_inner || p.parent >= 0;
      g.t0 = t0;
      g.t1 = t1;
      g.slots = !shared && t0 == 0 && t1 == T
                    ? nullptr
                    : a.part + (int64_t)seq_slot(p, shared, unit, c, uniform(seq_chunk_at(a, seq_pos(p, unit, 0)))) *
                                   kSubFloats;
    }
    const SeqPass& p = a.pass[ip];
    const int T = seq_tiles(p);
    // query tiles of a head are neighbours
    g.h = uniform(unit / p.q_tiles);
    g.qt = unit - g.h * p.q_tiles;
    SeqCursor tc;
    tc.pk = reinterpret_cast<const char*>(a.pageK + (int64_t)g.h * a.n_pages * TILE);
    tc.pv = reinterpret_cast<const char*>(a.pageV + (int64_t)g.h * a.n_pages * TILE);
    tc.fk = reinterpret_cast<const char*>(a.K + ((int64_t)p.tok0 * H + g.h) * D);
    tc.fv = reinterpret_cast<const char*>(a.V + ((int64_t)p.tok0 * H + g.h) * D);
    tc.frame_row = 2u * (uint32_t)(H * D);
    tc.entry = a.table + p.entry0;
    tc.n_pages = p.n_pages;
    tc.n_tiles = T;
    tc.last_rows = p.last_rows;
    tc.frame_rows = p.frame > 0 ? p.frame - (T - p.n_pages - 1) * BK : p.last_rows;
    if (p.tile_rows == kSubRows) {
      narrow_segment(a, p, tc, g, lds, s_m, s_l);
    } else {
      // The sums over a segment's keys take any order.  The chunks of a head cover different keys; the one that has
      // worked for i tiles takes tile i modulo the chunk's length (or the unit's, where that is less) if its segment
      // holds it, so that they are at the same few tiles at a time and find them in their XCD's L2.  (In key order
      // each fetched its keys from beyond it, and that was the bound: 1041 queries over 52,000 rows 342 -> 322 us.)
      const int per = uniform(max(1, min(a.E / p.cost, T)));
      const int ahead = uniform((done - g.t0) % per);
      g.ts = g.t0 + (ahead < 0 ? ahead + per : ahead);
      if (whole || g.ts >= g.t1) g.ts = g.t0;
      wide_segment(a, p, tc, g, lds, s_m, s_l);
    }
    if (whole) {
      if (++round == a.rounds && pos < end) ip = last_at_or_below(a.pos0, 0, a.n_pass, begin);
    } else {
      done += g.t1 - g.t0;
      pos = g.t1 < T ? end : seq_pos(p, unit + 1, 0);
    }
  }
}

// Joins the segments of a sequence's rows, 16 lanes a row's 64 elements.  Where a row has many segments
// a wave takes one row and its four groups of lanes every fourth segment each (kOne); where it has few, each
// group takes a row of its own.
// (Bound by latency: a launch of 5 to 6 us, 1.4 of which an empty one takes; the sums are fp32, 14 MB of them for a
// frame in three pieces.)
template <bool kOne>
__device__ __forceinline__ void merge_rows(const SeqArgs& a, const SeqPass& leaf, int ip, int h, int row) {
  const int G = a.group, lane = threadIdx.x & 63;
  const int grp = kOne ? lane >> 4 : 0, d4 = (lane & 15) * 4;
  constexpr int kStep = kOne ? 4 : 1;
  constexpr int kBatch = 4;             // segments a lane has in flight together
  constexpr int kLevels = 3;            // passes whose segments are taken as one list
  float mmax = kNegBig, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = ip; i >= 0;) {
    // segments [count[k], count[k + 1]) of the list are level k's, `stride` slots apart; `in_slot`: the row
    int first[kLevels], stride[kLevels], in_slot[kLevels], count[kLevels + 1];
    count[0] = 0;
#pragma unroll
    for (int k = 0; k < kLevels; ++k) {
      first[k] = stride[k] = in_slot[k] = 0;
      count[k + 1] = count[k];
      if (i < 0) continue;  // (uniform in the wave)
      const SeqPass& p = a.pass[i];
      const int T = seq_tiles(p);
      const bool shared = i < a.n_inner || p.parent >= 0;
      i = uniform(p.parent);
      if (T == 0) continue;
      const int r = (leaf.tok0 - p.tok0) * G + row;
      const int qt = uniform(r / p.tile_rows), unit = h * p.q_tiles + qt;
      if (seq_whole(a, p, unit)) return;  // written by the forward launch
      const int c0 = uniform(seq_chunk_at(a, seq_pos(p, unit, 0)));
      const int n = uniform(seq_chunk_at(a, seq_pos(p, unit, T - 1))) - c0 + 1;  // its chunks
      if (!shared && n == 1) return;  // written by the forward launch
      stride[k] = seq_slot_step(p, shared);
      first[k] = seq_slot(p, shared, unit, c0, c0) + r % p.tile_rows / kSubRows - count[k] * stride[k];
      in_slot[k] = r % kSubRows;
      count[k + 1] = count[k] + n;
    }
    const int n = count[kLevels];
    for (int j0 = grp; j0 < n; j0 += kStep * kBatch) {
      float mv[kBatch], lv[kBatch];
      float4 v[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int x = min(j0 + kStep * j, n - 1);
        int slot = first[0] + x * stride[0], rr = in_slot[0];
#pragma unroll
        for (int k = 1; k < kLevels; ++k)
          if (x >= count[k]) slot = first[k] + x * stride[k], rr = in_slot[k];
        const float* ps = a.part + (int64_t)slot * kSubFloats;
        mv[j] = ps[kSubRows * D + rr];
        lv[j] = ps[kSubRows * D + kSubRows + rr];
        v[j] = *reinterpret_cast<const float4*>(ps + rr * D + d4);
      }
      float m_new = mmax;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) m_new = fmaxf(m_new, mv[j]);  // clamped copies repeat a real one
      const float scale = __builtin_amdgcn_exp2f(mmax - m_new);
      L *= scale;
      acc.x *= scale, acc.y *= scale, acc.z *= scale, acc.w *= scale;
      mmax = m_new;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float w = j0 + kStep * j < n ? __builtin_amdgcn_exp2f(mv[j] - mmax) : 0.f;
        L = fmaf(w, lv[j], L);
        acc.x = fmaf(w, v[j].x, acc.x);
        acc.y = fmaf(w, v[j].y, acc.y);
        acc.z = fmaf(w, v[j].z, acc.z);
        acc.w = fmaf(w, v[j].w, acc.w);
      }
    }
  }
  if (kOne) {
#pragma unroll
    for (int mask = 16; mask < 64; mask <<= 1) {
      const float m2 = __shfl_xor(mmax, mask), m_new = fmaxf(mmax, m2);
      const float f = __builtin_amdgcn_exp2f(mmax - m_new), f2 = __builtin_amdgcn_exp2f(m2 - m_new);
      L = f * L + f2 * __shfl_xor(L, mask);
      acc.x = f * acc.x + f2 * __shfl_xor(acc.x, mask);
      acc.y = f * acc.y + f2 * __shfl_xor(acc.y, mask);
      acc.z = f * acc.z + f2 * __shfl_xor(acc.z, mask);
      acc.w = f * acc.w + f2 * __shfl_xor(acc.w, mask);
      mmax = m_new;
    }
    if (grp != 0) return;
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;  // no key at all: zeros, and a log-sum-exp of -inf
  const int HG = a.n_heads * G, tok = row / G, head = h * G + row % G;
  *reinterpret_cast<uint2*>(a.out + (((int64_t)leaf.tok0 + tok) * HG + head) * D + d4) =
      to_bf16x4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  if (d4 == 0)
    a.lse[(int64_t)leaf.tok0 * HG + (int64_t)head * leaf.n_tok + tok] =
        L > 0.f ? (mmax + __log2f(L)) * kLn2 : -__builtin_inff();
}

__global__ __launch_bounds__(256) void seq_merge_kernel(SeqArgs a) {
  const int H = a.n_heads, wave = threadIdx.x >> 6;
  const int ip = last_at_or_below(a.merge0, a.n_inner, a.n_pass, (int)blockIdx.x);
  const SeqPass& leaf = a.pass[ip];
  const int b = (int)blockIdx.x - a.merge0[ip];
  const int h = uniform(b % H), row0 = uniform(b / H * leaf.merge_rows), rows = leaf.n_tok * a.group;
  if (leaf.merge_rows == kMergeOne) {
    if (row0 + wave < rows) merge_rows<true>(a, leaf, ip, h, uniform(row0 + wave));
  } else {
    const int row = row0 + (int)(threadIdx.x >> 4);  // (a block's 16 rows lie in one query tile)
    if (row < rows) merge_rows<false>(a, leaf, ip, h, row);
  }
}

}  // namespace

hipError_t launch_attend_seqs(const SeqArgs& a, hipStream_t s) {
  if (seq_grid(a) > 0) {
    hipLaunchKernelGGL(seq_fwd_kernel, dim3((unsigned)a.n_queues, (unsigned)seq_grid(a)), dim3(kAttnThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.merge_blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(seq_merge_kernel, dim3((unsigned)a.merge_blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rv
