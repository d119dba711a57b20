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
__device__ __forceinline__ void load8(const void* base, int64_t at, float (&x)[8]) {
  if (F32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
    const float4 lo = p[0], hi = p[1];
    x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w, x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&x)[8]) {
  if (F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
    p[0] = make_float4(x[0], x[1], x[2], x[3]);
    p[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
    *reinterpret_cast<bf16x8*>(static_cast<uint16_t*>(base) + at) = v;
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

__device__ __forceinline__ void load_vec(const float* p, float dflt, int a, int b, Pair16& x) {
  if (p) {
    load8<true>(p, a, x.a);
    load8<true>(p, b, x.b);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x.a[i] = x.b[i] = dflt;
  }
}

// Bytes of the forward pass at 8328 tokens of 16 heads and what it takes: see the launcher.
template <bool F32, int AXES>
__global__ __launch_bounds__(NT) void prepare_kernel(PrepArgs a) {
  __shared__ float2 s_angles[NW][kPrepMaxTokens * kAngles];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t first = ((int64_t)blockIdx.x * NW + wave) * a.tokens_per_wave;
  if (first >= a.n_tokens) return;  // uniform in the wave; no barrier follows
  const int t0 = (int)first, n = min(a.tokens_per_wave, a.n_tokens - t0);
  float2* const angles = s_angles[wave];
  if (AXES > 0) fill_angles<AXES>(a, t0, n, lane, angles);
  const LaneMap<AXES> m(lane & 3);
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    const int H = part ? a.n_kv_heads : a.n_q_heads;
    const void* src = part ? a.k : a.q;
    const int64_t stride = part ? a.k_stride : a.q_stride;
    Pair16 w, bias;
    if (a.norm != RV_NORM_NONE) {
      load_vec(part ? a.kw : a.qw, 1.f, m.a, m.b, w);
      load_vec(part ? a.kb : a.qb, 0.f, m.a, m.b, bias);
    }
    for (int r = lane >> 2; r < n * H; r += 16) {
      const int t = r / H, h = r - t * H;
      const int64_t at = (int64_t)(t0 + t) * stride + h * D;
      Pair16 x;
      load8<F32>(src, at + m.a, x.a);
      load8<F32>(src, at + m.b, x.b);
      if (a.norm != RV_NORM_NONE) {
        normalise(a.norm, a.eps, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x.a[i] = fmaf(x.a[i], w.a[i], bias.a[i]);
          x.b[i] = fmaf(x.b[i], w.b[i], bias.b[i]);
        }
      }
      rotate<AXES, false>(angles + t * kAngles + m.angle, x);
      const int64_t to = part ? (int64_t)(t0 + t) * a.kv_row + h * a.kv_head
                              : ((int64_t)(t0 + t) * H + h) * D;
      store8<false>(part ? a.K : a.Q, to + m.a, x.a);
      store8<false>(part ? a.K : a.Q, to + m.b, x.b);
    }
  }
  if (a.V) {
    const int H = a.n_kv_heads;
    for (int c = lane; c < n * H * 8; c += 64) {
      const int r = c >> 3, t = r / H, h = r - t * H, e = 8 * (c & 7);
      float x[8];
      load8<F32>(a.v, (int64_t)(t0 + t) * a.v_stride + h * D + e, x);
      store8<false>(a.V, (int64_t)(t0 + t) * a.kv_row + h * a.kv_head + e, x);
    }
  }
}

// Gradients.  dy is the incoming gradient turned back; with n the normed input, dw = sum dy n,
// db = sum dy, and dx = r (e - [layer] mean(e) - n mean(e n)), e = dy w.  A lane adds up dw and db of
// its 16 columns over its rows; the block's sums go to part[block][q dw, q db, k dw, k db][64].
template <bool F32, int AXES>
__global__ __launch_bounds__(NT) void prepare_bwd_kernel(PrepArgs a) {
  __shared__ float2 s_angles[NW][kPrepMaxTokens * kAngles];
  __shared__ float s_sum[NW][4 * D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float2* const angles = s_angles[wave];
  const LaneMap<AXES> m(lane & 3);
  Pair16 dw[2] = {}, db[2] = {};
  const int64_t step = (int64_t)gridDim.x * NW * a.tokens_per_wave;
  for (int64_t first = ((int64_t)blockIdx.x * NW + wave) * a.tokens_per_wave; first < a.n_tokens; first += step) {
    const int t0 = (int)first, n = (int)min((int64_t)a.tokens_per_wave, a.n_tokens - first);
    if (AXES > 0) {
      __builtin_amdgcn_wave_barrier();  // (the last tokens' angles have been read)
      fill_angles<AXES>(a, t0, n, lane, angles);
    }
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const int H = part ? a.n_kv_heads : a.n_q_heads;
      const void* src = part ? a.k : a.q;
      void* dst = part ? a.dk : a.dq;
      const uint16_t* grad = part ? a.dK : a.dQ;
      const int64_t stride = part ? a.k_stride : a.q_stride, dst_stride = part ? a.dk_stride : a.dq_stride;
      Pair16 w;
      if (a.norm != RV_NORM_NONE) load_vec(part ? a.kw : a.qw, 1.f, m.a, m.b, w);
      for (int r = lane >> 2; r < n * H; r += 16) {
        const int t = r / H, h = r - t * H;
        Pair16 g;
        const int64_t from = ((int64_t)(t0 + t) * H + h) * D;
        load8<false>(grad, from + m.a, g.a);
        load8<false>(grad, from + m.b, g.b);
        Pair16 x;
        if (a.norm != RV_NORM_NONE) {
          const int64_t at = (int64_t)(t0 + t) * stride + h * D;
          load8<F32>(src, at + m.a, x.a);
          load8<F32>(src, at + m.b, x.b);
        }
        rotate<AXES, true>(angles + t * kAngles + m.angle, g);
        if (a.norm != RV_NORM_NONE) {
          const float rs = normalise(a.norm, a.eps, x);
          float se = 0.f, sn = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            dw[part].a[i] = fmaf(g.a[i], x.a[i], dw[part].a[i]);
            dw[part].b[i] = fmaf(g.b[i], x.b[i], dw[part].b[i]);
            db[part].a[i] += g.a[i];
            db[part].b[i] += g.b[i];
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
    if (a.dv) {
      const int H = a.n_kv_heads;
      for (int c = lane; c < n * H * 8; c += 64) {
        const int r = c >> 3, t = r / H, h = r - t * H, e = 8 * (c & 7);
        float x[8];
        load8<false>(a.dV, (int64_t)(t0 + t) * H * D + h * D + e, x);
        store8<F32>(a.dv, (int64_t)(t0 + t) * a.dv_stride + h * D + e, x);
      }
    }
  }
  if (!a.part) return;
  // Over the wave's 16 rows, then over the waves.
  float* const sum = s_sum[wave];
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[4] = {dw[part].a[i], dw[part].b[i], db[part].a[i], db[part].b[i]};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int mask = 4; mask < 64; mask <<= 1) v[k] += __shfl_xor(v[k], mask);
      }
      if (lane < 4) {
        sum[(2 * part) * D + m.a + i] = v[0];
        sum[(2 * part) * D + m.b + i] = v[1];
        sum[(2 * part + 1) * D + m.a + i] = v[2];
        sum[(2 * part + 1) * D + m.b + i] = v[3];
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 4 * D; i += NT) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += s_sum[w][i];
    a.part[(int64_t)blockIdx.x * 4 * D + i] = v;
  }
}

// The blocks' sums to the four gradients: a workgroup adds up 16 of the 256 columns, 16 threads a
// column.
__global__ __launch_bounds__(256) void prepare_sum_kernel(const float* part, int blocks, float* qw, float* qb, float* kw,
                                                          float* kb) {
  __shared__ float s[16][17];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float v = 0.f;
#pragma unroll 8
  for (int b = g; b < blocks; b += 16) v += part[(int64_t)b * 4 * D + col];
  s[g][c] = v;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) t += s[i][threadIdx.x];
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
  hipLaunchKernelGGL(prepare_sum_kernel, dim3(4 * D / 16), dim3(256), 0, s, a.part, a.n_tokens > 0 ? a.blocks : 0, a.dqw,
                     a.dqb, a.dkw, a.dkb);
  return hipGetLastError();
}

}  // namespace rv
