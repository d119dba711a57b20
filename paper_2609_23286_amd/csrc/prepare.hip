// prepare.hip -- projection outputs to frame tensors, gfx950: the norm of every query and key
// head and the rotation by the token's position, and their gradients.
//
// Layout.  Four lanes hold a head's 64 elements, 16 each, as two 8-element chunks a and b that
// are the rotation's two halves: with two axes lane j holds chunks {0,1,4,5}[j] and the chunk two
// further on, with one axis (and none) chunks j and j + 4.  So a pair's two elements lie in one
// lane, the norm's sums are 16 adds and two exchanges in a quad, and 16 heads fill a wave.  A wave
// takes `tokens_per_wave` consecutive tokens: their heads are one list of rows (token, head), 16 to
// an iteration, queries first, then keys; the values are copied.
//
// Angles.  A token's position gives 32 distinct (axis, frequency) pairs whatever its head count, so
// each lane of the wave forms one pair's sine and cosine and the heads read them from LDS.  The
// phase is the low 64 bits of position x turns-per-position (2^-64 turns a unit): whole
// turns vanish in the wrap, which is exact however far the position.
#include "rv_internal.h"
#include "rv_ops.h"

namespace rv {
namespace {

constexpr int D = kHeadDim;
constexpr int NT = kPrepThreads;
constexpr int NW = NT / 64;
constexpr int kAngles = kMaxFreqs;  // per token: axes x frequencies

struct Pair16 {   // a lane's 16 elements: a[i] and b[i] turn together
  float a[8], b[8];
};

// x = 2 pi phase / 2^32 within an eighth of a turn, by the Taylor series of sine (to x^9, the next
// term is below 2^-29) and cosine (to x^10, 2^-32), and the quadrant's exchange and signs.
__device__ __forceinline__ float2 sin_cos_turns(uint32_t phase) {
  const uint32_t quad = (phase + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(phase - (quad << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float t = x * x;
  const float s = x * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), 1.f);
  const float c = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const float sv = (quad & 1) ? c : s, cv = (quad & 1) ? s : c;
  return make_float2((quad & 2) ? -sv : sv, ((quad + 1) & 2) ? -cv : cv);
}

template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&x)[8]) {
  if (F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
    p[0] = make_float4(x[0], x[1], x[2], x[3]);
    p[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 p0 = {(__bf16)x[0], (__bf16)x[1]}, p1 = {(__bf16)x[2], (__bf16)x[3]};
    const bf16x2 p2 = {(__bf16)x[4], (__bf16)x[5]}, p3 = {(__bf16)x[6], (__bf16)x[7]};
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + at) =
        make_uint4(__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1), __builtin_bit_cast(uint32_t, p2),
                   __builtin_bit_cast(uint32_t, p3));
  }
}

// A lane's 16 elements as they are in memory, so that loads can be issued well before their use.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool F32>
struct Raw16 {
  u32x4 a0, b0, a1, b1;  // (the second pair: fp32)
};

template <bool F32>
__device__ __forceinline__ Raw16<F32> load_raw(const void* base, int64_t at, int a, int b) {
  constexpr int S = F32 ? 4 : 2;
  const char* p = static_cast<const char*>(base) + at * S;
  Raw16<F32> r;
  r.a0 = *reinterpret_cast<const u32x4*>(p + a * S);
  r.b0 = *reinterpret_cast<const u32x4*>(p + b * S);
  if (F32) {
    r.a1 = *reinterpret_cast<const u32x4*>(p + a * S + 16);
    r.b1 = *reinterpret_cast<const u32x4*>(p + b * S + 16);
  }
  return r;
}

template <bool F32>
__device__ __forceinline__ void unpack(const Raw16<F32>& r, Pair16& x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F32) {
      x.a[i] = __uint_as_float(r.a0[i]), x.a[4 + i] = __uint_as_float(r.a1[i]);
      x.b[i] = __uint_as_float(r.b0[i]), x.b[4 + i] = __uint_as_float(r.b1[i]);
    } else {
      x.a[2 * i] = __uint_as_float(r.a0[i] << 16), x.a[2 * i + 1] = __uint_as_float(r.a0[i] & 0xFFFF0000u);
      x.b[2 * i] = __uint_as_float(r.b0[i] << 16), x.b[2 * i + 1] = __uint_as_float(r.b0[i] & 0xFFFF0000u);
    }
  }
}

template <int CTRL>
__device__ __forceinline__ float quad_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
// Sum over the four lanes of a head.
__device__ __forceinline__ float head_sum(float x) { return quad_add<0x4E>(quad_add<0xB1>(x)); }

// The angles of tokens t0 .. t0 + n - 1, into the wave's table: [token][axis][frequency].
template <int AXES>
__device__ __forceinline__ void fill_angles(const PrepArgs& a, int t0, int n, int lane, float2* table) {
  constexpr int per_axis = AXES == 2 ? 16 : 32;
  for (int i = lane; i < n * kAngles; i += 64) {
    const int t = i / kAngles, axis = AXES == 2 ? (i % kAngles) / per_axis : 0;
    const int64_t pos = a.pos[(int64_t)(t0 + t) * AXES + axis];
    table[i] = sin_cos_turns((uint32_t)(((uint64_t)pos * a.freq[i % per_axis]) >> 32));
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Where a lane's two chunks lie, and its angles in a token's table.
template <int AXES>
struct LaneMap {
  int a, b, angle;
  __device__ explicit LaneMap(int j) {
    a = 8 * (AXES == 2 ? (j & 1) + 4 * (j >> 1) : j);
    b = a + (AXES == 2 ? 16 : 32);
    angle = 8 * j;  // two axes: axis j / 2, frequencies 8 (j % 2) ..; one: frequencies 8 j ..
  }
};

// Turns every pair by its angle (backward: by minus its angle).
template <int AXES, bool BACK>
__device__ __forceinline__ void rotate(const float2* angles, Pair16& x) {
  if (AXES == 0) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 sc = angles[i];
    const float s = BACK ? -sc.x : sc.x, p = x.a[i], q = x.b[i];
    x.a[i] = p * sc.y - q * s;
    x.b[i] = q * sc.y + p * s;
  }
}

// x to its normed form g r; returns r.
__device__ __forceinline__ float normalise(int norm, float eps, Pair16& x) {
  if (norm == RV_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x.a[i] + x.b[i];
    const float mean = head_sum(s) * (1.f / D);
#pragma unroll
    for (int i = 0; i < 8; ++i) x.a[i] -= mean, x.b[i] -= mean;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(x.a[i], x.a[i], fmaf(x.b[i], x.b[i], s));
  const float r = 1.f / sqrtf(head_sum(s) * (1.f / D) + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x.a[i] *= r, x.b[i] *= r;
  return r;
}

// A weight or bias vector's elements at the lane's chunks; the default where there is none (by address: a branch
// around the loads would wait for them).
__device__ const float kOnes[D] = {1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1,
                                   1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1,
                                   1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1};
__device__ const float kZeros[D] = {};
__device__ __forceinline__ void load_vec(const float* p, const float* dflt, int a, int b, Pair16& x) {
  unpack(load_raw<true>(p ? p : dflt, 0, a, b), x);
}

// One part (queries or keys) of the forward pass: rows r, r + 16, ... of n * H, the first already loaded; the
// next row's elements are requested before this one's are worked on.
template <bool F32, int AXES>
__device__ __forceinline__ void prepare_part(const PrepArgs& a, const LaneMap<AXES>& m, const float2* angles, int t0, int n,
                                             int lane, int H, const void* src, int64_t stride, uint16_t* dst, int64_t dst_row,
                                             int64_t dst_head, const float* weight, const float* bias_p, Raw16<F32> raw) {
  Pair16 w, bias;
  if (a.norm != RV_NORM_NONE) {
    load_vec(weight, kOnes, m.a, m.b, w);
    load_vec(bias_p, kZeros, m.a, m.b, bias);
  }
  for (int r = lane >> 2; r < n * H; r += 16) {
    const int t = n == 1 ? 0 : r / H, h = r - t * H;
    Pair16 x;
    unpack(raw, x);
    if (r + 16 < n * H) {
      const int t2 = n == 1 ? 0 : (r + 16) / H, h2 = r + 16 - t2 * H;
      raw = load_raw<F32>(src, (int64_t)(t0 + t2) * stride + h2 * D, m.a, m.b);
    }
    if (a.norm != RV_NORM_NONE) {
      normalise(a.norm, a.eps, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x.a[i] = fmaf(x.a[i], w.a[i], bias.a[i]);
        x.b[i] = fmaf(x.b[i], w.b[i], bias.b[i]);
      }
    }
    rotate<AXES, false>(angles + t * kAngles + m.angle, x);
    const int64_t to = (int64_t)(t0 + t) * dst_row + h * dst_head;
    store8<false>(dst, to + m.a, x.a);
    store8<false>(dst, to + m.b, x.b);
  }
}

template <bool F32, int AXES>
__global__ __launch_bounds__(NT) void prepare_kernel(PrepArgs a) {
  __shared__ float2 s_angles[NW][kPrepMaxTokens * kAngles];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t first = ((int64_t)blockIdx.x * NW + wave) * a.tokens_per_wave;
  if (first >= a.n_tokens) return;  // uniform in the wave; no barrier follows
  const int t0 = (int)first, n = min(a.tokens_per_wave, a.n_tokens - t0);
  float2* const angles = s_angles[wave];
  const LaneMap<AXES> m(lane & 3);
  // The first rows of all three parts are requested at once, before anything waits.
  const int Hq = a.n_q_heads, Hk = a.n_kv_heads, r = lane >> 2;
  const int tq = n == 1 ? 0 : r / Hq, tk = n == 1 ? 0 : r / Hk;
  Raw16<F32> q{}, k{};
  if (r < n * Hq) q = load_raw<F32>(a.q, (int64_t)(t0 + tq) * a.q_stride + (r - tq * Hq) * D, m.a, m.b);
  if (r < n * Hk) k = load_raw<F32>(a.k, (int64_t)(t0 + tk) * a.k_stride + (r - tk * Hk) * D, m.a, m.b);
  if (a.V) {  // (values in the same pattern: a lane's two chunks of a row)
    Raw16<F32> v{};
    if (r < n * Hk) v = load_raw<F32>(a.v, (int64_t)(t0 + tk) * a.v_stride + (r - tk * Hk) * D, m.a, m.b);
    if (AXES > 0) fill_angles<AXES>(a, t0, n, lane, angles);
    for (int i = r; i < n * Hk; i += 16) {
      const int t = n == 1 ? 0 : i / Hk, h = i - t * Hk;
      Pair16 x;
      unpack(v, x);
      if (i + 16 < n * Hk) {
        const int t2 = n == 1 ? 0 : (i + 16) / Hk, h2 = i + 16 - t2 * Hk;
        v = load_raw<F32>(a.v, (int64_t)(t0 + t2) * a.v_stride + h2 * D, m.a, m.b);
      }
      const int64_t to = (int64_t)(t0 + t) * a.kv_row + h * a.kv_head;
      store8<false>(a.V, to + m.a, x.a);
      store8<false>(a.V, to + m.b, x.b);
    }
  } else if (AXES > 0) {
    fill_angles<AXES>(a, t0, n, lane, angles);
  }
  prepare_part<F32, AXES>(a, m, angles, t0, n, lane, Hq, a.q, a.q_stride, a.Q, (int64_t)Hq * D, D, a.qw, a.qb, q);
  prepare_part<F32, AXES>(a, m, angles, t0, n, lane, Hk, a.k, a.k_stride, a.K, a.kv_row, a.kv_head, a.kw, a.kb, k);
}

// Gradients.  dy is the incoming gradient turned back; with n the normed input, dw = sum dy n,
// db = sum dy, and dx = r (e - [layer] mean(e) - n mean(e n)), e = dy w.  A lane adds up dw and db of
// its 16 columns over its rows.
struct Sums {
  Pair16 dw, db;
};

template <bool F32, int AXES>
__device__ __forceinline__ void backward_part(const PrepArgs& a, const LaneMap<AXES>& m, const float2* angles, int t0, int n,
                                              int lane, int H, const void* src, int64_t stride, const uint16_t* grad,
                                              void* dst, int64_t dst_stride, const Pair16& w, Raw16<F32> raw,
                                              Raw16<false> graw, Sums& sum) {
  for (int r = lane >> 2; r < n * H; r += 16) {
    const int t = n == 1 ? 0 : r / H, h = r - t * H;
    Pair16 g, x;
    unpack(graw, g);
    unpack(raw, x);
    if (r + 16 < n * H) {
      const int t2 = n == 1 ? 0 : (r + 16) / H, h2 = r + 16 - t2 * H;
      graw = load_raw<false>(grad, ((int64_t)(t0 + t2) * H + h2) * D, m.a, m.b);
      if (a.norm != RV_NORM_NONE) raw = load_raw<F32>(src, (int64_t)(t0 + t2) * stride + h2 * D, m.a, m.b);
    }
    rotate<AXES, true>(angles + t * kAngles + m.angle, g);
    if (a.norm != RV_NORM_NONE) {
      const float rs = normalise(a.norm, a.eps, x);
      float se = 0.f, sn = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum.dw.a[i] = fmaf(g.a[i], x.a[i], sum.dw.a[i]);
        sum.dw.b[i] = fmaf(g.b[i], x.b[i], sum.dw.b[i]);
        sum.db.a[i] += g.a[i];
        sum.db.b[i] += g.b[i];
        g.a[i] *= w.a[i];
        g.b[i] *= w.b[i];
        se += g.a[i] + g.b[i];
        sn = fmaf(g.a[i], x.a[i], fmaf(g.b[i], x.b[i], sn));
      }
      const float mn = head_sum(sn) * (1.f / D);
      const float me = a.norm == RV_NORM_LAYER ? head_sum(se) * (1.f / D) : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g.a[i] = rs * (g.a[i] - me - x.a[i] * mn);
        g.b[i] = rs * (g.b[i] - me - x.b[i] * mn);
      }
    }
    const int64_t to = (int64_t)(t0 + t) * dst_stride + h * D;
    store8<F32>(dst, to + m.a, g.a);
    store8<F32>(dst, to + m.b, g.b);
  }
}

// Sum over the wave's 16 rows of head elements (lanes that differ in bits 2 to 5), of two values at a
// time: lanes of the upper half go on with the second value, so that 64 sums take 60 exchanges rather than 256.
__device__ __forceinline__ float fold32(float x, float y) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float fold16(float x, float y) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int CTRL>
__device__ __forceinline__ float from_lane(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float fold8(float x, float y, bool upper) {  // row_ror:8 is the lane 8 away
  const float keep = upper ? y : x, give = upper ? x : y;
  return keep + from_lane<0x128>(give);
}
__device__ __forceinline__ float fold4(float x, float y, bool upper) {  // half-row mirror, quad reversed: 4 away
  const float keep = upper ? y : x, give = upper ? x : y;
  return keep + from_lane<0x1B>(from_lane<0x141>(give));
}

// The block's sums go to part[block][q dw, q db, k dw, k db][64].
template <bool F32, int AXES>
__global__ __launch_bounds__(NT) void prepare_bwd_kernel(PrepArgs a) {
  __shared__ float2 s_angles[NW][kPrepMaxTokens * kAngles];
  __shared__ float s_sum[NW][4 * D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float2* const angles = s_angles[wave];
  const LaneMap<AXES> m(lane & 3);
  Sums sums[2] = {};
  Pair16 w[2];
  if (a.norm != RV_NORM_NONE) {
    load_vec(a.qw, kOnes, m.a, m.b, w[0]);
    load_vec(a.kw, kOnes, m.a, m.b, w[1]);
  }
  const int Hq = a.n_q_heads, Hk = a.n_kv_heads, r = lane >> 2;
  const int64_t step = (int64_t)gridDim.x * NW * a.tokens_per_wave;
  for (int64_t first = ((int64_t)blockIdx.x * NW + wave) * a.tokens_per_wave; first < a.n_tokens; first += step) {
    const int t0 = (int)first, n = (int)min((int64_t)a.tokens_per_wave, a.n_tokens - first);
    // The first rows of all parts are requested at once, before anything waits.
    const int tq = n == 1 ? 0 : r / Hq, tk = n == 1 ? 0 : r / Hk;
    const int hq = r - tq * Hq, hk = r - tk * Hk;
    Raw16<F32> q{}, k{};
    Raw16<false> gq{}, gk{}, gv{};
    if (r < n * Hq) {
      gq = load_raw<false>(a.dQ, ((int64_t)(t0 + tq) * Hq + hq) * D, m.a, m.b);
      if (a.norm != RV_NORM_NONE) q = load_raw<F32>(a.q, (int64_t)(t0 + tq) * a.q_stride + hq * D, m.a, m.b);
    }
    if (r < n * Hk) {
      gk = load_raw<false>(a.dK, ((int64_t)(t0 + tk) * Hk + hk) * D, m.a, m.b);
      if (a.norm != RV_NORM_NONE) k = load_raw<F32>(a.k, (int64_t)(t0 + tk) * a.k_stride + hk * D, m.a, m.b);
      if (a.dv) gv = load_raw<false>(a.dV, ((int64_t)(t0 + tk) * Hk + hk) * D, m.a, m.b);
    }
    if (AXES > 0) {
      __builtin_amdgcn_wave_barrier();  // (the last tokens' angles have been read)
      fill_angles<AXES>(a, t0, n, lane, angles);
    }
    backward_part<F32, AXES>(a, m, angles, t0, n, lane, Hq, a.q, a.q_stride, a.dQ, a.dq, a.dq_stride, w[0], q, gq, sums[0]);
    backward_part<F32, AXES>(a, m, angles, t0, n, lane, Hk, a.k, a.k_stride, a.dK, a.dk, a.dk_stride, w[1], k, gk, sums[1]);
    if (a.dv) {
      for (int i = r; i < n * Hk; i += 16) {
        const int t = n == 1 ? 0 : i / Hk, h = i - t * Hk;
        Pair16 x;
        unpack(gv, x);
        if (i + 16 < n * Hk) {
          const int t2 = n == 1 ? 0 : (i + 16) / Hk, h2 = i + 16 - t2 * Hk;
          gv = load_raw<false>(a.dV, ((int64_t)(t0 + t2) * Hk + h2) * D, m.a, m.b);
        }
        const int64_t to = (int64_t)(t0 + t) * a.dv_stride + h * D;
        store8<F32>(a.dv, to + m.a, x.a);
        store8<F32>(a.dv, to + m.b, x.b);
      }
    }
  }
  if (!a.part) return;
  // Over the wave's 16 rows.  v[i], i = 8 c + e: element e of the lane's a (even c) or b (odd c) of q dw, q db,
  // k dw, k db (c / 2).
  float v[64];
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      v[32 * p + e] = sums[p].dw.a[e];
      v[32 * p + 8 + e] = sums[p].dw.b[e];
      v[32 * p + 16 + e] = sums[p].db.a[e];
      v[32 * p + 24 + e] = sums[p].db.b[e];
    }
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = fold32(v[i], v[i + 32]);  // lanes 32 ..: k's
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = fold16(v[i], v[i + 16]);  // lanes 16 .. of each half: db
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fold8(v[i], v[i + 8], lane & 8);  // lanes 8 .. of each row: b
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = fold4(v[i], v[i + 4], lane & 4);  // lanes 4 .. of each half row: elements 4 ..
  {
    const int col = (lane & 8 ? m.b : m.a) + (lane & 4), vec = 2 * (lane >> 5) + (lane >> 4 & 1);
    *reinterpret_cast<float4*>(&s_sum[wave][vec * D + col]) = make_float4(v[0], v[1], v[2], v[3]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 4 * D; i += NT) {
    float t = 0.f;
#pragma unroll
    for (int u = 0; u < NW; ++u) t += s_sum[u][i];
    a.part[(int64_t)blockIdx.x * 4 * D + i] = t;
  }
}

// The blocks' sums to the four gradients: a workgroup adds up 8 of the 256 columns, 32 threads a column.
constexpr int kSumCols = 8, kSumGroups = 32;
__global__ __launch_bounds__(kSumCols* kSumGroups) void prepare_sum_kernel(const float* part, int blocks, float* qw, float* qb,
                                                                          float* kw, float* kb) {
  __shared__ float s[kSumGroups][kSumCols + 1];
  const int c = threadIdx.x % kSumCols, g = threadIdx.x / kSumCols, col = blockIdx.x * kSumCols + c;
  float v = 0.f;
#pragma unroll 8
  for (int b = g; b < blocks; b += kSumGroups) v += part[(int64_t)b * 4 * D + col];
  s[g][c] = v;
  __syncthreads();
  if (threadIdx.x >= kSumCols) return;
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < kSumGroups; ++i) t += s[i][threadIdx.x];
  float* const out[4] = {qw, qb, kw, kb};
  float* o = out[col / D];
  if (o) o[col % D] = t;
}

template <bool F32>
hipError_t launch(const PrepArgs& a, int axes, bool back, hipStream_t s) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.blocks), dim3(NT), 0, s, a);
    return hipGetLastError();
  };
  if (back)
    return axes == 2   ? go(prepare_bwd_kernel<F32, 2>)
           : axes == 1 ? go(prepare_bwd_kernel<F32, 1>)
                       : go(prepare_bwd_kernel<F32, 0>);
  return axes == 2   ? go(prepare_kernel<F32, 2>)
         : axes == 1 ? go(prepare_kernel<F32, 1>)
                     : go(prepare_kernel<F32, 0>);
}

}  // namespace

hipError_t launch_prepare(const PrepArgs& a, bool f32, int axes, bool back, hipStream_t s) {
  if (a.n_tokens > 0) {
    const hipError_t e = f32 ? launch<true>(a, axes, back, s) : launch<false>(a, axes, back, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dqw && !a.dqb && !a.dkw && !a.dkb) return hipSuccess;
  hipLaunchKernelGGL(prepare_sum_kernel, dim3(4 * D / kSumCols), dim3(kSumCols * kSumGroups), 0, s, a.part, a.n_tokens > 0 ? a.blocks : 0, a.dqw,
                     a.dqb, a.dkw, a.dkb);
  return hipGetLastError();
}

}  // namespace rv
