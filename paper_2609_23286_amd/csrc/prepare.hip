// prepare.hip -- projection outputs to frame tensors, gfx950: the norm of every query and key
// head and the rotation by the token's position, and their gradients.
//
// Layout.  Eight lanes hold a head's 64 elements, 8 each, as two pieces of 4, chosen so that every
// access is 16 bytes a lane and whole lines a row: of bf16 rows a lane's pieces are neighbours, of fp32 rows
// (128 bytes to an instruction) 32 elements apart.  The partner of an element in its rotation pair
// lies in lane j ^ 2 (with fp32 rows and one axis: in the lane itself); where that needs it, the lane
// number's bits 1 and 2 change places.  The multiply-add reads the partner through a lane exchange, and the
// norm's sums are 8 adds and three exchanges.  Eight heads fill a wave.  A wave takes a token (or a few, where
// they have fewer than eight heads): its rows (token, head) of queries, of keys and of values are requested at
// once, eight to an instruction.  Forward, a lane holds 67 to 109 registers, so that the four to seven waves a SIMD
// cover the latency of memory, which bounds it; backward 161 to 214, two or three waves, each with more rows on their
// way.  Results are written past the caches' reuse (nontemporal: 8328 tokens of 16 heads 24.5 -> 19.6 us when it was
// taken; now 18.5 us, 5.5 TB/s, from fp32 25.7 us, 6.0 TB/s; the attention that follows takes the same time).
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
constexpr int E = 8;               // elements a lane
constexpr int R = 64 * E / D;      // rows (heads) a wave takes at a time
static_assert(R == kPrepRows, "the host sizes a wave's tokens by it");

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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Where a lane's two pieces of 4 elements lie in a head (WIDE: the rows that count are fp32).
template <bool WIDE>
struct Cols {
  int a, b;
};
template <bool WIDE, int AXES>
__device__ __forceinline__ Cols<WIDE> lane_cols(int lane) {
  const int j = lane & 7, turned = (j & 1) | (j & 2) << 1 | (j & 4) >> 1;
  if (WIDE) {
    const int c = AXES == 2 ? turned : j;
    return {4 * c, D / 2 + 4 * c};
  }
  const int c = AXES == 1 ? turned : j;
  return {E * c, E * c + 4};
}

// A lane's 8 elements as they are in memory, so that loads can be issued well before their use.
template <bool F32>
struct Raw {
  u32x4 lo, hi;  // (hi: fp32)
};
template <bool F32, bool WIDE>
__device__ __forceinline__ Raw<F32> load_raw(const void* base, int64_t at, Cols<WIDE> c) {
  const char* p = static_cast<const char*>(base) + at * (F32 ? 4 : 2);
  Raw<F32> r;
  if (F32) {
    r.lo = *reinterpret_cast<const u32x4*>(p + c.a * 4);
    r.hi = *reinterpret_cast<const u32x4*>(p + c.b * 4);
  } else if (WIDE) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p + c.a * 2), y = *reinterpret_cast<const u32x2*>(p + c.b * 2);
    r.lo = u32x4{x[0], x[1], y[0], y[1]};
  } else {
    r.lo = *reinterpret_cast<const u32x4*>(p + c.a * 2);
  }
  return r;
}
template <bool F32>
__device__ __forceinline__ void unpack(const Raw<F32>& r, float (&x)[E]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F32) {
      x[i] = __uint_as_float(r.lo[i]), x[4 + i] = __uint_as_float(r.hi[i]);
    } else {
      x[2 * i] = __uint_as_float(r.lo[i] << 16), x[2 * i + 1] = __uint_as_float(r.lo[i] & 0xFFFF0000u);
    }
  }
}

template <bool F32, bool WIDE>
__device__ __forceinline__ void store8(void* base, int64_t at, Cols<WIDE> c, const float (&x)[E]) {
  if (F32) {
    float* p = static_cast<float*>(base) + at;
    __builtin_nontemporal_store((f32x4{x[0], x[1], x[2], x[3]}), reinterpret_cast<f32x4*>(p + c.a));
    __builtin_nontemporal_store((f32x4{x[4], x[5], x[6], x[7]}), reinterpret_cast<f32x4*>(p + c.b));
    return;
  }
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 p0 = {(__bf16)x[0], (__bf16)x[1]}, p1 = {(__bf16)x[2], (__bf16)x[3]};
  const bf16x2 p2 = {(__bf16)x[4], (__bf16)x[5]}, p3 = {(__bf16)x[6], (__bf16)x[7]};
  const u32x4 v = {__builtin_bit_cast(uint32_t, p0), __builtin_bit_cast(uint32_t, p1), __builtin_bit_cast(uint32_t, p2),
                   __builtin_bit_cast(uint32_t, p3)};
  uint16_t* p = static_cast<uint16_t*>(base) + at;
  if (WIDE) {
    __builtin_nontemporal_store((u32x2{v[0], v[1]}), reinterpret_cast<u32x2*>(p + c.a));
    __builtin_nontemporal_store((u32x2{v[2], v[3]}), reinterpret_cast<u32x2*>(p + c.b));
  } else {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p + c.a));
  }
}

template <int CTRL>
__device__ __forceinline__ float from_lane(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;  // lanes exchanged within a quad
constexpr int kMirror8 = 0x141;            // lane 7 - j of the eight
constexpr int kRotate8 = 0x128;            // the lane 8 away, of 16
// Sum over the eight lanes of a row.
__device__ __forceinline__ float row_sum(float x) {
  x += from_lane<kXor1>(x);
  x += from_lane<kXor2>(x);
  return x + from_lane<kMirror8>(x);
}

// The angles of tokens t0 .. t0 + n - 1, into the wave's table: [token][element] (sine, cosine), the sine
// with the sign its element's partner takes it with.  A lane forms items lane, lane + 64, ...; the position of
// the first is loaded ahead (loads return in order: behind the rows' loads it would wait for them).
template <int AXES>
struct Angles {
  static constexpr int kBlock = D / (AXES > 0 ? AXES : 1), kFreqs = kBlock / 2;
  int32_t first = 0;
  __device__ __forceinline__ int32_t position(const PrepArgs& a, int t0, int i) const {
    return a.pos[(int64_t)(t0 + i / kMaxFreqs) * AXES + i % kMaxFreqs / kFreqs];
  }
  __device__ __forceinline__ void start(const PrepArgs& a, int t0, int n, int lane) {
    if (AXES > 0 && lane < n * kMaxFreqs) first = position(a, t0, lane);
  }
  __device__ __forceinline__ void fill(const PrepArgs& a, int t0, int n, int lane, float2* table) {
    if (AXES == 0) return;
    for (int i = lane; i < n * kMaxFreqs; i += 64) {
      const int64_t pos = i == lane ? first : position(a, t0, i);
      const int f = i % kFreqs;
      const float2 sc = sin_cos_turns((uint32_t)(((uint64_t)pos * a.freq[f]) >> 32));
      float2* const e = table + i / kMaxFreqs * D + i % kMaxFreqs / kFreqs * kBlock + f;
      e[0] = make_float2(-sc.x, sc.y);
      e[kFreqs] = sc;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
};

// Turns every pair by its angle (BACK: by minus its angle).
template <bool WIDE, int AXES, bool BACK>
__device__ __forceinline__ void rotate(const float2* angles, Cols<WIDE> c, float (&x)[E]) {
  if (AXES == 0) return;
  float y[E];
#pragma unroll
  for (int i = 0; i < E; ++i) y[i] = WIDE && AXES == 1 ? x[i ^ 4] : from_lane<kXor2>(x[i]);
#pragma unroll
  for (int i = 0; i < E; i += 2) {
    const float4 sc = *reinterpret_cast<const float4*>(angles + (i < 4 ? c.a : c.b) + (i & 3));
    x[i] = x[i] * sc.y + y[i] * (BACK ? -sc.x : sc.x);
    x[i + 1] = x[i + 1] * sc.w + y[i + 1] * (BACK ? -sc.z : sc.z);
  }
}

// x to its normed form g r; returns r.
__device__ __forceinline__ float normalise(int norm, float eps, float (&x)[E]) {
  if (norm == RV_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) s += x[i];
    const float mean = row_sum(s) * (1.f / D);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] -= mean;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) s = fmaf(x[i], x[i], s);
  const float r = 1.f / sqrtf(row_sum(s) * (1.f / D) + eps);
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] *= r;
  return r;
}

// The weights and biases, q w, q b, k w, k b, in LDS (a load of them among the rows' would wait for those):
// thread i holds element i % 64 of vector i / 64.  The default stands in for one that there is not, by its address.
__device__ const float kOnes[D] = {1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1,
                                   1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1,
                                   1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1};
__device__ const float kZeros[D] = {};
__device__ __forceinline__ float own_weight(const PrepArgs& a) {
  const int v = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float* p = v == 0 ? a.qw : v == 1 ? a.qb : v == 2 ? a.kw : a.kb;
  if (!p) p = v & 1 ? kZeros : kOnes;
  return p[threadIdx.x & 63];
}
template <bool WIDE>
__device__ __forceinline__ void read_vec(const float* vec, Cols<WIDE> c, float (&x)[E]) {
  const float4 lo = *reinterpret_cast<const float4*>(vec + c.a), hi = *reinterpret_cast<const float4*>(vec + c.b);
  x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w, x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
}

// The rows of one part (queries, keys or values) of a wave's tokens: row r is head r % H of token t0 + r / H.
// ONE: a wave has a single token (its rows then lie at a scalar base).
template <bool ONE>
struct Rows {
  int t0, n, H;
  __device__ __forceinline__ int count() const { return ONE ? H : n * H; }
  __device__ __forceinline__ int token(int r) const { return ONE ? 0 : r / H; }
  // element offset of row r where tokens are `row` elements apart and heads `head`
  __device__ __forceinline__ int64_t at(int r, int64_t row, int64_t head) const {
    if (ONE) return t0 * row + r * head;
    const int t = token(r);
    return (int64_t)(t0 + t) * row + (r - t * H) * head;
  }
};

// The first rows of a part, kFirst to a lane, requested together; later ones as the earlier are done.
constexpr int kFirst = 2;
template <bool F32, bool WIDE, bool ONE>
struct Ahead {
  Raw<F32> raw[kFirst];
  __device__ __forceinline__ void start(const void* src, const Rows<ONE>& p, int r, int64_t row, int64_t head, Cols<WIDE> c) {
#pragma unroll
    for (int k = 0; k < kFirst; ++k)
      if (r + k * R < p.count()) raw[k] = load_raw<F32, WIDE>(src, p.at(r + k * R, row, head), c);
  }
  // Row r's elements; row r + kFirst R takes their place.
  __device__ __forceinline__ void next(const void* src, const Rows<ONE>& p, int r, int64_t row, int64_t head,
                                       Cols<WIDE> c, float (&x)[E]) {
    unpack(raw[0], x);
#pragma unroll
    for (int k = 0; k + 1 < kFirst; ++k) raw[k] = raw[k + 1];
    if (r + kFirst * R < p.count()) raw[kFirst - 1] = load_raw<F32, WIDE>(src, p.at(r + kFirst * R, row, head), c);
  }
};

template <bool F32, int AXES, bool ONE>
__device__ __forceinline__ void prepare_part(const PrepArgs& a, const Rows<ONE>& p, const float2* angles, int lane, const void* src,
                                             int64_t stride, uint16_t* dst, int64_t dst_row, int64_t dst_head,
                                             const float* vecs, Ahead<F32, F32, ONE>& ahead) {
  const Cols<F32> c = lane_cols<F32, AXES>(lane);
  for (int r = lane / 8; r < p.count(); r += R) {
    float x[E];
    ahead.next(src, p, r, stride, D, c, x);
    if (a.norm != RV_NORM_NONE) {
      float w[E], b[E];
      read_vec(vecs, c, w);
      read_vec(vecs + D, c, b);
      normalise(a.norm, a.eps, x);
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = fmaf(x[i], w[i], b[i]);
    }
    rotate<F32, AXES, false>(angles + p.token(r) * D, c, x);
    store8<false, F32>(dst, p.at(r, dst_row, dst_head), c, x);
  }
}

template <bool F32, int AXES, bool ONE>
__global__ __launch_bounds__(NT) void prepare_kernel(PrepArgs a) {
  __shared__ __attribute__((aligned(16))) float2 s_angles[NW][kPrepMaxTokens * D];
  __shared__ __attribute__((aligned(16))) float s_vec[4 * D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t first = ((int64_t)blockIdx.x * NW + wave) * a.tokens_per_wave;
  const int t0 = (int)min(first, (int64_t)a.n_tokens), n = min(a.tokens_per_wave, a.n_tokens - t0);  // n: 0 past the end
  const Cols<F32> c = lane_cols<F32, AXES>(lane);
  const int r = lane / 8;
  float2* const angles = s_angles[wave];
  const Rows<ONE> pq{t0, n, a.n_q_heads}, pk{t0, n, a.n_kv_heads};
  const bool norm = a.norm != RV_NORM_NONE;
  Angles<AXES> ang;
  Ahead<F32, F32, ONE> q, k, v;
  float vec = 0.f;
  if (norm) vec = own_weight(a);
  if (n > 0) {
    ang.start(a, t0, n, lane);
    q.start(a.q, pq, r, a.q_stride, D, c);
    k.start(a.k, pk, r, a.k_stride, D, c);
    if (a.V) v.start(a.v, pk, r, a.v_stride, D, c);
  }
  if (norm) {
    s_vec[threadIdx.x] = vec;
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (the rows stay on their way)
  }
  if (n <= 0) return;
  ang.fill(a, t0, n, lane, angles);
  prepare_part<F32, AXES, ONE>(a, pq, angles, lane, a.q, a.q_stride, a.Q, (int64_t)pq.H * D, D, s_vec, q);
  prepare_part<F32, AXES, ONE>(a, pk, angles, lane, a.k, a.k_stride, a.K, a.kv_row, a.kv_head, s_vec + 2 * D, k);
  if (!a.V) return;
  for (int i = r; i < pk.count(); i += R) {
    float x[E];
    v.next(a.v, pk, i, a.v_stride, D, c, x);
    store8<false, F32>(a.V, pk.at(i, a.kv_row, a.kv_head), c, x);
  }
}

// Gradients.  dy is the incoming gradient turned back; with n the normed input, dw = sum dy n,
// db = sum dy, and dx = r (e - [layer] mean(e) - n mean(e n)), e = dy w.  A lane adds up dw and db of
// its 8 columns over its rows.
struct Sums {
  float dw[E], db[E];
};

template <bool F32, int AXES, bool ONE>
__device__ __forceinline__ void backward_part(const PrepArgs& a, const Rows<ONE>& p, const float2* angles, int lane, const void* src,
                                              int64_t stride, const uint16_t* grad, void* dst, int64_t dst_stride,
                                              const float* vecs, Ahead<F32, F32, ONE>& ahead, Ahead<false, F32, ONE>& grads, Sums& sum) {
  const Cols<F32> c = lane_cols<F32, AXES>(lane);
  for (int r = lane / 8; r < p.count(); r += R) {
    float g[E];
    grads.next(grad, p, r, (int64_t)p.H * D, D, c, g);
    rotate<F32, AXES, true>(angles + p.token(r) * D, c, g);
    if (a.norm != RV_NORM_NONE) {
      float x[E], w[E];
      ahead.next(src, p, r, stride, D, c, x);
      read_vec(vecs, c, w);
      const float rs = normalise(a.norm, a.eps, x);
      float se = 0.f, sn = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        sum.dw[i] = fmaf(g[i], x[i], sum.dw[i]);
        sum.db[i] += g[i];
        g[i] *= w[i];
        se += g[i];
        sn = fmaf(g[i], x[i], sn);
      }
      const float mn = row_sum(sn) * (1.f / D);
      const float me = a.norm == RV_NORM_LAYER ? row_sum(se) * (1.f / D) : 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i) g[i] = rs * (g[i] - me - x[i] * mn);
    }
    store8<F32, F32>(dst, p.at(r, dst_stride, D), c, g);
  }
}

// Sums over the wave's 8 rows of head elements (lanes that differ in bits 3 to 5), of two values at a
// time: lanes of the upper half go on with the second value, so that 32 sums take 28 exchanges rather than 96.
__device__ __forceinline__ float fold32(float x, float y) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float fold16(float x, float y) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float fold8(float x, float y, bool upper) {
  const float keep = upper ? y : x, give = upper ? x : y;
  return keep + from_lane<kRotate8>(give);
}

// The block's sums go to part[block][q dw, q db, k dw, k db][64].
template <bool F32, int AXES, bool ONE>
__global__ __launch_bounds__(NT) void prepare_bwd_kernel(PrepArgs a) {
  __shared__ __attribute__((aligned(16))) float2 s_angles[NW][kPrepMaxTokens * D];
  __shared__ __attribute__((aligned(16))) float s_sum[NW][4 * D];
  __shared__ __attribute__((aligned(16))) float s_vec[4 * D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Cols<F32> c = lane_cols<F32, AXES>(lane);
  const int r = lane / 8;
  float2* const angles = s_angles[wave];
  Sums sq = {}, sk = {};
  if (a.norm != RV_NORM_NONE) {
    s_vec[threadIdx.x] = own_weight(a);
    __syncthreads();
  }
  const int64_t step = (int64_t)gridDim.x * NW * a.tokens_per_wave;
  for (int64_t first = ((int64_t)blockIdx.x * NW + wave) * a.tokens_per_wave; first < a.n_tokens; first += step) {
    const int t0 = (int)first, n = (int)min((int64_t)a.tokens_per_wave, a.n_tokens - first);
    const Rows<ONE> pq{t0, n, a.n_q_heads}, pk{t0, n, a.n_kv_heads};
    Angles<AXES> ang;
    Ahead<F32, F32, ONE> q, k;
    Ahead<false, F32, ONE> gq, gk, gv;
    ang.start(a, t0, n, lane);
    gq.start(a.dQ, pq, r, (int64_t)pq.H * D, D, c);
    gk.start(a.dK, pk, r, (int64_t)pk.H * D, D, c);
    if (a.norm != RV_NORM_NONE) {
      q.start(a.q, pq, r, a.q_stride, D, c);
      k.start(a.k, pk, r, a.k_stride, D, c);
    }
    if (a.dv) gv.start(a.dV, pk, r, (int64_t)pk.H * D, D, c);
    __builtin_amdgcn_wave_barrier();  // (the last tokens' angles have been read)
    ang.fill(a, t0, n, lane, angles);
    backward_part<F32, AXES, ONE>(a, pq, angles, lane, a.q, a.q_stride, a.dQ, a.dq, a.dq_stride, s_vec, q, gq, sq);
    backward_part<F32, AXES, ONE>(a, pk, angles, lane, a.k, a.k_stride, a.dK, a.dk, a.dk_stride, s_vec + 2 * D, k, gk, sk);
    if (a.dv) {
      for (int i = r; i < pk.count(); i += R) {
        float x[E];
        gv.next(a.dV, pk, i, (int64_t)pk.H * D, D, c, x);
        store8<F32, F32>(a.dv, pk.at(i, a.dv_stride, D), c, x);
      }
    }
  }
  if (!a.part) return;
  // Over the wave's rows, then over the waves.
  float v[32];
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = sq.dw[i], v[8 + i] = sq.db[i], v[16 + i] = sk.dw[i], v[24 + i] = sk.db[i];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = fold32(v[i], v[i + 16]);  // lanes 32 ..: the keys'
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fold16(v[i], v[i + 8]);  // lanes 16 .. of each half: db
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = fold8(v[i], v[i + 4], lane & 8);  // lanes 8 .. of each 16: elements 4 ..
  const int vec = 2 * (lane >> 5) + (lane >> 4 & 1), col = (lane & 8) ? c.b : c.a;
  *reinterpret_cast<float4*>(&s_sum[wave][vec * D + col]) = make_float4(v[0], v[1], v[2], v[3]);
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

template <bool F32, bool ONE>
hipError_t launch(const PrepArgs& a, int axes, bool back, hipStream_t s) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.blocks), dim3(NT), 0, s, a);
    return hipGetLastError();
  };
  if (back)
    return axes == 2   ? go(prepare_bwd_kernel<F32, 2, ONE>)
           : axes == 1 ? go(prepare_bwd_kernel<F32, 1, ONE>)
                       : go(prepare_bwd_kernel<F32, 0, ONE>);
  return axes == 2   ? go(prepare_kernel<F32, 2, ONE>)
         : axes == 1 ? go(prepare_kernel<F32, 1, ONE>)
                     : go(prepare_kernel<F32, 0, ONE>);
}

}  // namespace

hipError_t launch_prepare(const PrepArgs& a, bool f32, int axes, bool back, hipStream_t s) {
  if (a.n_tokens > 0) {
    const bool one = a.tokens_per_wave == 1;
    const hipError_t e = f32 ? (one ? launch<true, true>(a, axes, back, s) : launch<true, false>(a, axes, back, s))
                             : (one ? launch<false, true>(a, axes, back, s) : launch<false, false>(a, axes, back, s));
    if (e != hipSuccess) return e;
  }
  if (!a.dqw && !a.dqb && !a.dkw && !a.dkb) return hipSuccess;
  hipLaunchKernelGGL(prepare_sum_kernel, dim3(4 * D / kSumCols), dim3(kSumCols * kSumGroups), 0, s, a.part, a.n_tokens > 0 ? a.blocks : 0, a.dqw,
                     a.dqb, a.dkw, a.dkb);
  return hipGetLastError();
}

}  // namespace rv
