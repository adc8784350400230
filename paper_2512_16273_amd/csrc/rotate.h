// tslt_rotate and its gradients: the norm of every head's row and the rotation of its first channels by the token's positions.
//
// With r = 1 / sqrt(mean x^2 + eps), x^ = w x r, and of every pair y = (u cos - v sin, v cos + u sin).  Backwards, g the gradient of y turned back by
// the same angles and h = w g:  dx = r (h - x r mean(h x r)),  dw = sum over rows of g x r.
//
// A row is D / 16 lanes wide: each has two runs of eight channels, of which one holds the partners of the other (of pairs half the rotated
// channels apart; neighbours are partners inside a run), so that nothing but a row's sums crosses lanes.  The angles of a token are those of all its
// heads: a workgroup takes kTokens tokens, computes their cosines and sines once, a lane an angle, and then all of their rows.
//
// Bound by memory, and forwards almost as much by vector instructions (250 for the 16 channels of a lane: sums of squares in fp64, two products with r and the weight,
// the turn, two addresses).  bfloat16, 40 heads of 128: prompts of 4 x 4001 tokens, three axes, a third of which count, 26.7 us (3.8 TB/s), 64 x 21 tokens 9.1; backwards 8 x 2048 tokens 102 us
// (4.9 TB/s, what a copy reaches), 5 of them the weights' second launch.  One token 2.9 on the device, 5.1 a call: the launch, its position, its row.
#pragma once
#include "rows.h"

namespace tslt {

struct RotateParams {
  RowsView q, k, out_q, out_k;           // k.data null: no keys (heads is 0 then)
  RowsView grad_q, grad_k;               // backward
  int64_t tokens;                        // B * n
  int n, heads_q, heads;
  const int32_t* position;
  int64_t position_seq;
  const int32_t* base;
  const float* freq;
  const int32_t* axis;
  int axes, pairs;
  bool adjacent, norm;
  float eps;
  const float *q_weight, *k_weight;
  const int32_t* count;
  int32_t* status;
  float* part;                           // [workgroups][2][D]: their shares of the weights' gradients; null: not asked for
  float *out_q_weight, *out_k_weight;
  int parts;
};

// Sum over the W lanes of a row (4, 8 or 16, aligned); all of them get it.
template <int W> __device__ __forceinline__ double row_sum(double v) {
  v += dpp_f64<0xB1>(0.0, v);                            // quad_perm 1 0 3 2, then 2 3 0 1
  v += dpp_f64<0x4E>(0.0, v);
  if constexpr (W >= 8) v += dpp_f64<0x141>(0.0, v);     // the other quad of eight lanes, mirrored
  if constexpr (W >= 16) v += dpp_f64<0x140>(0.0, v);    // the other eight of sixteen
  return v;
}

// Cosine and sine of position * freq.  The product of a whole number and an fp32 number in fp64 is off by 2^-53 of itself; it is brought into
// a quarter turn around 0 there, and the rest is the functions' series up to x^11 (what they leave out is below 2^-33 up to pi / 4).
__device__ __forceinline__ float2 turn_by(int64_t position, float freq) {
  const double turns = double(position) * double(freq) * 0.15915494309189533577;
  const double part = turns - __builtin_rint(turns);
  const double quarter = __builtin_rint(4.0 * part);
  const float x = float((part - 0.25 * quarter) * 6.283185307179586477), x2 = x * x;
  float s = -1.0f / 39916800.0f;
  s = fmaf(s, x2, 1.0f / 362880.0f);
  s = fmaf(s, x2, -1.0f / 5040.0f);
  s = fmaf(s, x2, 1.0f / 120.0f);
  s = fmaf(s, x2, -1.0f / 6.0f);
  s = fmaf(s * x2, x, x);
  float c = -1.0f / 3628800.0f;
  c = fmaf(c, x2, 1.0f / 40320.0f);
  c = fmaf(c, x2, -1.0f / 720.0f);
  c = fmaf(c, x2, 1.0f / 24.0f);
  c = fmaf(c, x2, -0.5f);
  c = fmaf(c, x2, 1.0f);
  const int quadrant = int(quarter) & 3;
  const float a = quadrant & 1 ? s : c, b = quadrant & 1 ? c : s;
  return make_float2(quadrant == 1 || quadrant == 2 ? -a : a, quadrant >= 2 ? -b : b);
}

// What the rows of a workgroup's tokens need, in LDS.
template <int D, int kTokens> struct RotateShared {
  float2 turn[kTokens * (D / 2)];        // [token][pair]
  float weight[2 * D];                   // queries', keys'
  int seq[kTokens], at[kTokens];         // sequence and place of a token; -1: there is none
  int bad_axis;
};
template <int D, int kTokens> __device__ __forceinline__ void rotate_weights(const RotateParams& p, RotateShared<D, kTokens>& sh) {
  for (int i = threadIdx.x; i < 2 * D; i += kBlock) {
    const float* w = i < D ? p.q_weight : p.k_weight;
    sh.weight[i] = w ? as_global(w)[i < D ? i : i - D] : 1.0f;
  }
  if (threadIdx.x == 0) sh.bad_axis = 0;
}
// Behind a barrier on both sides.  Sequences' status: by whoever has their first token.
template <int D, int kTokens> __device__ __forceinline__ void rotate_turns(const RotateParams& p, int64_t t0, RotateShared<D, kTokens>& sh) {
  const int tid = threadIdx.x;
  bool bad = false;
  for (int e = tid; e < kTokens * max(p.pairs, 1); e += kBlock) {
    const int tok = p.pairs ? e / p.pairs : e, j = p.pairs ? e - tok * p.pairs : 0;      // (without a rotation an entry is a token)
    const int64_t t = t0 + tok;
    const uint32_t seq = uint32_t(t < p.tokens ? t : 0) / uint32_t(p.n);
    const int i = int(uint32_t(t < p.tokens ? t : 0) - seq * uint32_t(p.n));
    const bool there = t < p.tokens && i < counted(p.count, seq, p.n);
    if (j == 0) {
      sh.seq[tok] = t < p.tokens ? int(seq) : -1;
      sh.at[tok] = there ? i : -1 - i;
    }
    if (p.pairs == 0) continue;
    const int named = p.axis ? as_global(p.axis)[j] : 0, axis = min(max(named, 0), p.axes - 1);
    bad |= named != axis;
    if (!there) continue;
    int64_t position = p.base ? as_global(p.base)[seq] : 0;
    position += p.position ? as_global(p.position)[seq * p.position_seq + int64_t(i) * p.axes + axis] : i;
    sh.turn[tok * p.pairs + j] = turn_by(position, as_global(p.freq)[j]);
  }
  if (bad) sh.bad_axis = 1;
  __syncthreads();
  if (p.status && tid < kTokens && sh.seq[tid] >= 0 && (sh.at[tid] == 0 || sh.at[tid] == -1)) {
    const int64_t b = sh.seq[tid];
    const bool odd = p.count && as_global(p.count)[b] != counted(p.count, b, p.n);
    p.status[b] = odd || sh.bad_axis ? kBadIndex : 0;
  }
}

// A lane's two runs of eight channels, and what it has of a row's turns.
template <int D> struct RowLanes {
  static constexpr int kLanes = D / 16;
  int a, b;                              // first channels
  int pair_a, pair_b;                    // first pairs; -1: not rotated
  __device__ __forceinline__ RowLanes(const RotateParams& p, int lane) {
    const int rotated = p.pairs / 8, rest = lane - rotated;
    a = 8 * (rest < 0 ? lane : 2 * rotated + 2 * rest);
    b = 8 * (rest < 0 ? lane + rotated : 2 * rotated + 2 * rest + 1);
    pair_a = rest >= 0 ? -1 : p.adjacent ? a / 2 : a;
    pair_b = b / 2;
  }
  // kBack: by the opposite angle.
  template <bool kBack> __device__ __forceinline__ void rotate(const float2* turn, bool adjacent, float (&u)[8], float (&v)[8]) const {
    if (pair_a < 0) return;
    if (!adjacent) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = turn[pair_a + e].x, s = kBack ? -turn[pair_a + e].y : turn[pair_a + e].y, x = u[e], y = v[e];
        u[e] = fmaf(x, c, -(y * s));
        v[e] = fmaf(y, c, x * s);
      }
      return;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 t = turn[(half ? pair_b : pair_a) + e];
        float(&w)[8] = half ? v : u;
        const float c = t.x, s = kBack ? -t.y : t.y, x = w[2 * e], y = w[2 * e + 1];
        w[2 * e] = fmaf(x, c, -(y * s));
        w[2 * e + 1] = fmaf(y, c, x * s);
      }
  }
};

// 1 / sqrt(mean x^2 + eps) of a row, in fp64: squares of large numbers do not overflow, those of small ones do not vanish.
template <int D> __device__ __forceinline__ float inverse_rms(const float (&u)[8], const float (&v)[8], float eps) {
  double sum = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sum = fma(double(u[e]), double(u[e]), sum);
    sum = fma(double(v[e]), double(v[e]), sum);
  }
  return float(rsqrt(row_sum<D / 16>(sum) * (1.0 / D) + double(eps)));
}

__device__ __forceinline__ int64_t row_of(const RowsView& r, int64_t seq, int at, int head) { return seq * r.seq + at * r.token + head * r.head; }

template <typename T, int D, int kTokens>
__global__ __launch_bounds__(kBlock) void rotate_kernel(const RotateParams p) {
  __shared__ RotateShared<D, kTokens> sh;
  constexpr int kLanes = RowLanes<D>::kLanes, kRows = kBlock / kLanes;
  const int tid = threadIdx.x, heads = p.heads_q + p.heads;
  const RowLanes<D> mine(p, tid % kLanes);
  rotate_weights(p, sh);
  __syncthreads();
  rotate_turns(p, int64_t(blockIdx.x) * kTokens, sh);
  for (int unit = tid / kLanes; unit < kTokens * heads; unit += kRows) {
    const int tok = unit / heads, head = unit - tok * heads;
    if (sh.seq[tok] < 0 || sh.at[tok] < 0) continue;
    const bool key = head >= p.heads_q;
    const int h = key ? head - p.heads_q : head;
    const RowsView &from = key ? p.k : p.q, &to = key ? p.out_k : p.out_q;
    const int64_t at = row_of(from, sh.seq[tok], sh.at[tok], h), out = row_of(to, sh.seq[tok], sh.at[tok], h);
    Eight<T> x, y;
    x.load(from.data, at + mine.a);
    y.load(from.data, at + mine.b);
    float u[8], v[8];
    x.get(u);
    y.get(v);
    if (p.norm) {
      const float r = inverse_rms<D>(u, v, p.eps);
      const float* w = sh.weight + (key ? D : 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = u[e] * r * w[mine.a + e];
        v[e] = v[e] * r * w[mine.b + e];
      }
    }
    mine.template rotate<false>(sh.turn + tok * p.pairs, p.adjacent, u, v);
    x.set(u);
    y.set(v);
    x.store(to.data, out + mine.a);
    y.store(to.data, out + mine.b);
  }
}

// Workgroups go through the tokens, kTokens at a time, and keep their share of the weights' gradients in registers.
template <typename T, int D, int kTokens>
__global__ __launch_bounds__(kBlock) void rotate_backward_kernel(const RotateParams p) {
  __shared__ RotateShared<D, kTokens> sh;
  __shared__ float share[16][kBlock];
  constexpr int kLanes = RowLanes<D>::kLanes, kRows = kBlock / kLanes;
  const int tid = threadIdx.x;
  const RowLanes<D> mine(p, tid % kLanes);
  float sum[2][16] = {};
  rotate_weights(p, sh);
  for (int64_t t0 = int64_t(blockIdx.x) * kTokens; t0 < p.tokens; t0 += int64_t(gridDim.x) * kTokens) {
    __syncthreads();
    rotate_turns(p, t0, sh);
#pragma unroll
    for (int key = 0; key < 2; ++key) {
      const int heads = key ? p.heads : p.heads_q;
      const RowsView &g_rows = key ? p.grad_k : p.grad_q, &x_rows = key ? p.k : p.q, &to = key ? p.out_k : p.out_q;
      for (int unit = tid / kLanes; unit < kTokens * heads; unit += kRows) {
        const int tok = unit / heads, h = unit - tok * heads, seq = sh.seq[tok];
        if (seq < 0) continue;
        const bool there = sh.at[tok] >= 0;
        const int i = there ? sh.at[tok] : -1 - sh.at[tok];
        const int64_t out = row_of(to, seq, i, h);
        Eight<T> gu, gv;
        float u[8] = {}, v[8] = {};
        if (there) {
          const int64_t g_at = row_of(g_rows, seq, i, h);
          gu.load(g_rows.data, g_at + mine.a);
          gv.load(g_rows.data, g_at + mine.b);
          gu.get(u);
          gv.get(v);
          mine.template rotate<true>(sh.turn + tok * p.pairs, p.adjacent, u, v);
          if (p.norm) {
            const int64_t x_at = row_of(x_rows, seq, i, h);
            Eight<T> xu, xv;
            float x[8], y[8];
            xu.load(x_rows.data, x_at + mine.a);
            xv.load(x_rows.data, x_at + mine.b);
            xu.get(x);
            xv.get(y);
            const float r = inverse_rms<D>(x, y, p.eps);
            const float* w = sh.weight + (key ? D : 0);
            double dot = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[e] *= r;
              y[e] *= r;
              sum[key][e] = fmaf(u[e], x[e], sum[key][e]);
              sum[key][8 + e] = fmaf(v[e], y[e], sum[key][8 + e]);
              u[e] *= w[mine.a + e];
              v[e] *= w[mine.b + e];
              dot = fma(double(u[e]), double(x[e]), dot);
              dot = fma(double(v[e]), double(y[e]), dot);
            }
            const float mean = float(row_sum<kLanes>(dot) * (1.0 / D));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              u[e] = r * fmaf(-x[e], mean, u[e]);
              v[e] = r * fmaf(-y[e], mean, v[e]);
            }
          }
        }
        gu.set(u);
        gv.set(v);
        gu.store(to.data, out + mine.a);
        gv.store(to.data, out + mine.b);
      }
    }
  }
  if (!p.part) return;
  // the rows of a workgroup together: run a lane's, channel e of its sixteen
#pragma unroll
  for (int key = 0; key < 2; ++key) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 16; ++e) share[e][tid] = sum[key][e];
    __syncthreads();
    if (tid < D) {
      const int lane = tid % kLanes, e = tid / kLanes;
      double all = 0.0;
#pragma unroll 8
      for (int row = 0; row < kRows; ++row) all += share[e][row * kLanes + lane];
      const RowLanes<D> its(p, lane);
      p.part[(int64_t(blockIdx.x) * 2 + key) * D + (e < 8 ? its.a + e : its.b + e - 8)] = float(all);
    }
  }
}

// The workgroups' shares together: eight of the 2 D channels to a workgroup, 32 of its lanes to each.
template <int D> __global__ __launch_bounds__(kBlock) void rotate_weights_kernel(const RotateParams p) {
  __shared__ double share[32][8];
  const int lane = threadIdx.x & 7, group = threadIdx.x >> 3, channel = blockIdx.x * 8 + lane;
  double all = 0.0;
#pragma unroll 8
  for (int i = group; i < p.parts; i += 32) all += as_global(p.part)[int64_t(i) * (2 * D) + channel];
  share[group][lane] = all;
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int g = 1; g < 32; ++g) all += share[g][lane];
  float* out = channel < D ? p.out_q_weight : p.out_k_weight;
  if (out) out[channel < D ? channel : channel - D] = float(all);
}

}  // namespace tslt
