// attn_tile.h -- the attention kernels' common ground, gfx950: the LDS tile layout, cross-lane
// and bf16 helpers, and one 64-key tile of online-softmax attention for a wave's 32 queries.
#pragma once

#include "rv_internal.h"

namespace rv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int BQ = kAttnBQ;
constexpr int BK = kAttnBK;
constexpr int D = kHeadDim;
constexpr int TILE = BK * D;                    // one K or V tile: 64 rows x 128 bytes
constexpr int STAGE = 2 * TILE;                 // K tile then V tile
constexpr int NSTAGE = 4;                       // LDS ring: two tiles computed, two in flight
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kScaleLog2 = 1.44269504088896341f * 0.125f;  // log2(e) / sqrt(64)
constexpr float kOverflowGuard = 18446744073709551616.0f;  // 2^64
constexpr float kNegBig = -1.0e30f;

typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

template <int P>
struct StageConst {
  static constexpr int value = P;
};

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ uint2 to_bf16x4(float a, float b, float c, float d) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 v = {(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
  return __builtin_bit_cast(uint2, v);
}

__device__ __forceinline__ int hw_xcc_id() { return __builtin_amdgcn_s_getreg((3 << 11) | 20) & 15; }

// Partner value of the other 32-lane half (lane l <-> l ^ 32): v_permlane32_swap returns
// the two halves exchanged between its operands, so the pair holds {own, partner} in
// some order on every lane; sums and maxima over the pair need no lane test.
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// LDS tile layout: 64 rows of 128 bytes, no padding.  The 16-byte chunk c of row r is
// stored at chunk c ^ sw(r), sw(r) = (2 (r & 3) | (r >> 2) & 1) ^ 2 ((r >> 3) & 1), which
// takes 8 distinct values on every 8 aligned rows and, with the row's parity, 16 distinct
// (parity, chunk) pairs on every 16: the 16-byte K reads (one row per lane, 8 or 16
// lanes a cycle) and the transposing V reads (4 rows x 32 bytes per 16 lanes, the rows'
// 32-byte pieces on disjoint chunk pairs) are free of bank conflicts whether the LDS
// serves 128 or 256 bytes a cycle.
__device__ __forceinline__ int sw(int row) { return attn_tile_swizzle(row); }
__device__ __forceinline__ int swz(int row, int chunk) { return row * D + ((chunk ^ sw(row)) << 3); }

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ void lds_load16(const char* g, uint16_t* lds_wave_base) {
  __builtin_amdgcn_global_load_lds((const void*)g, (lds_void*)lds_wave_base, 16, 0, 0);
}

struct SoftmaxState {
  float m;      // running max of z * log2(e) / 8
  float l;      // this lane's share of the row sum
  f32x16 o0;    // O^T rows d = 0..31 for this lane's query (accumulator layout)
  f32x16 o1;    // d = 32..63
};

// One 64-key tile for this wave's 32 queries.  kFirst: the segment's first tile, whose
// running reference is still unset, so its maximum is taken directly (the exact path of
// a later tile, without the rescale of an empty state).
template <bool kFirst>
__device__ __forceinline__ void tile_compute(const uint16_t* stage, const bf16x8 (&qf)[4], int lane, int valid,
                                             SoftmaxState& sm) {
  const int l32 = lane & 31, half = lane >> 5;
  // Wave priority 1 from the score MFMAs through the softmax, 0 for the value product: of
  // the two waves sharing a SIMD, the one in the first part of its tile issues first, which
  // keeps the pair out of step so that one's MFMAs run under the other's vector work
  // (about +1 % per stream over a uniform priority).  Priority changes no result.
  __builtin_amdgcn_s_setprio(1);
  f32x16 s0 = {}, s1 = {};
#pragma unroll
  for (int ds = 0; ds < 4; ++ds) {
    const bf16x8 ka = *reinterpret_cast<const bf16x8*>(&stage[swz(l32, ds * 2 + half)]);
    const bf16x8 kb = *reinterpret_cast<const bf16x8*>(&stage[swz(32 + l32, ds * 2 + half)]);
    s0 = mfma32(ka, qf[ds], s0);
    s1 = mfma32(kb, qf[ds], s1);
  }
  // accumulator entry r of this lane: key 8*(r/4) + 4*half + r%4 (+32 in s1)
  if (__builtin_expect(valid < BK, 0)) {
    // keys >= valid get -1e30: sat(key + 1 - valid) is 1 exactly for them, 0 otherwise
    // (arithmetic masking keeps the 32 lane masks out of scalar registers)
    const float fv = (float)(valid - 4 * half - 1);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float key = (float)(8 * (r >> 2) + (r & 3));
      s0[r] = fmaf(__saturatef(key - fv), kNegBig, s0[r]);
      s1[r] = fmaf(__saturatef(key + 32.0f - fv), kNegBig, s1[r]);
    }
  }
  // P = 2^(z*log2e/8 - m) against the running reference m.  Softmax does not depend on
  // the reference, so the tile maximum is only needed when some p could overflow: a
  // lane whose tile sum reaches 2^64 (or inf; every p starts as inf while m is unset)
  // makes the wave take the exact path -- raise m to the tile maximum, rescale the
  // accumulators, recompute P.  Terms far below the reference underflow to 0, exactly
  // as they would relative to the true maximum.
  bf16x8 p[4];
  float rsum = -0.f;  // -0 + x == x: the first add folds away
  auto exact = [&]() {
    float mx = fmaxf(s0[0], s1[0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, fmaxf(s0[r], s1[r]));
    const float m_new = fmaxf(sm.m, half_max(mx) * kScaleLog2);
    if (!kFirst) {
      const float alpha = __builtin_amdgcn_exp2f(sm.m - m_new);
      sm.l *= alpha;
      sm.o0 *= alpha;
      sm.o1 *= alpha;
    }
    sm.m = m_new;
    rsum = -0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s0[r], kScaleLog2, -sm.m));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s1[r], kScaleLog2, -sm.m));
      rsum += e0 + e1;
      p[r >> 3][r & 7] = (__bf16)e0;
      p[2 + (r >> 3)][r & 7] = (__bf16)e1;
    }
  };
  if (kFirst) {
    exact();
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e0 = __builtin_amdgcn_exp2f(fmaf(s0[r], kScaleLog2, -sm.m));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(s1[r], kScaleLog2, -sm.m));
      rsum += e0 + e1;
      p[r >> 3][r & 7] = (__bf16)e0;
      p[2 + (r >> 3)][r & 7] = (__bf16)e1;
    }
    if (__any(!(rsum < kOverflowGuard))) exact();
  }
  sm.l += rsum;
  __builtin_amdgcn_s_setprio(0);

  // V^T operand through transposing LDS reads.  Within each 16-lane group, lane i
  // receives element i%4 of the 8-byte chunk addressed by lane 4r + i/4 (r = 0..3), so
  // lane 4r + j points at row (key) r, columns d0 + 4j .. +3: lane i then holds
  // V[key r][d0 + i] for the 4 keys.  Keys follow the P^T slot order: for k-step ks and
  // lane half hh, slots 0..3 are keys ks*16 + 4hh + r, slots 4..7 keys ks*16 + 8 + 4hh + r.
  const uint16_t* vt = stage + TILE;
  const int g = lane >> 4, i16 = lane & 15, rr = i16 >> 2, jj = i16 & 3, hh = g >> 1;
  const int col = 16 * (g & 1) + 4 * jj;  // logical column (elements) within a 32-dim block
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const int row = ks * 16 + 4 * hh + rr;
#pragma unroll
    for (int db = 0; db < 2; ++db) {
      const int lcol = db * 32 + col;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(vt + swz(row, lcol >> 3) + (lcol & 7)));
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(vt + swz(row + 8, lcol >> 3) + (lcol & 7)));
      const i16x8 w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      const bf16x8 va = __builtin_bit_cast(bf16x8, w);
      if (db == 0)
        sm.o0 = mfma32(va, p[ks], sm.o0);
      else
        sm.o1 = mfma32(va, p[ks], sm.o1);
    }
  }
}

}  // namespace
}  // namespace rv
