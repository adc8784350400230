// tslt_adapt: out = base + scale (x A^T) B^T, of every sequence its own A and B, in two launches.
//
// The first makes h = x A^T.  A workgroup has 16 tokens of one sequence, whose four waves share the channels, or 64, 16 a wave; where that makes few workgroups the
// channels are cut too, and each cut leaves its sums.  The second adds those up, and has of 16 or 64 tokens 256 channels of the result, 64 a wave.
//
// Tokens are the columns of the matrix instructions and what is learned the rows, 16 bytes a lane straight from memory: a lane has of the first one's results
// four ranks in a row, and of the second one's eight (four of fp32) channels in a row, as the rows of the second are dealt out to two instructions so.
//
// h enters the second in two terms of the rows' type, as if it were twice as many ranks: 16 bits of it for bfloat16, 22 for binary16 (whose range it is
// brought to by a power of two a token), where the result keeps 8 and 11.  So the products of 16 ranks are one instruction of 32.
#pragma once
#include "rows.h"

namespace tslt {

struct AdaptParams {
  RowsView x, base, out;
  int K, N, R, n;
  int64_t B, n_adapters;
  const void *a, *b;
  const int32_t *adapter, *rank, *count;
  const float* scale;
  int32_t* status;
  int tiles;                             // of a sequence's tokens
  int chunks;                            // of the ranks (first launch), of the result's channels (second)
  int cuts;                              // of the channels of x
  float* h;                              // [cuts][B * n][R]
  bool copy;                             // out is not base
};

typedef float f32x4 __attribute__((ext_vector_type(4)));

// 16 bytes a lane of each operand: 32 channels of 16-bit rows, 16 of fp32 ones.
template <typename T> struct Product;
template <> struct Product<Bf16> {
  static constexpr int kChannels = 32;
  static __device__ __forceinline__ f32x4 add(u32x4 a, u32x4 b, f32x4 c) {
    typedef __bf16 V __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
};
template <> struct Product<F16> {
  static constexpr int kChannels = 32;
  static __device__ __forceinline__ f32x4 add(u32x4 a, u32x4 b, f32x4 c) {
    typedef _Float16 V __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
};
template <> struct Product<float> {
  static constexpr int kChannels = 16;
  static __device__ __forceinline__ f32x4 add(u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(as_f32(a[i]), as_f32(b[i]), c, 0, 0, 0);
    return c;
  }
};

// A sequence's adapter (-1: none) and how many of its ranks count.
__device__ __forceinline__ int adapter_of(const AdaptParams& p, int64_t b, int& rank, bool& odd) {
  const int named = as_global(p.adapter)[b];
  odd = named < -1 || named >= p.n_adapters;
  const int a = odd ? -1 : named;
  rank = a < 0 ? 0 : p.rank ? min(max(as_global(p.rank)[a], 0), p.R) : p.R;
  return a;
}

// h of kTokenTiles * 16 tokens and kRankTiles * 16 ranks.
template <typename T, int kTokenTiles, int kRankTiles>
__global__ __launch_bounds__(kBlock) void adapt_down_kernel(const AdaptParams p) {
  constexpr int kBytes = ElemTraits<T>::kBytes, kLane = 16 / kBytes, kStep = Product<T>::kChannels;
  constexpr bool kShare = kTokenTiles == 1;              // the waves share the channels
  __shared__ f32x4 part[kShare ? 3 : 1][kShare ? kRankTiles : 1][64];
  const int wave = wave_id(), lane = lane_id(), r = lane & 15, g = lane >> 4;
  uint32_t block = blockIdx.x;
  const int cut = int(block % uint32_t(p.cuts));
  block /= uint32_t(p.cuts);
  const int chunk = int(block % uint32_t(p.chunks));
  block /= uint32_t(p.chunks);
  const uint32_t b = block / uint32_t(p.tiles);
  const int tile = int(block - b * uint32_t(p.tiles)), tokens = counted(p.count, b, p.n);
  const int t0 = tile * (16 * kTokenTiles) + (kShare ? 0 : 16 * wave), rank0 = chunk * (16 * kRankTiles);
  int rank;
  bool odd;
  const int a = adapter_of(p, b, rank, odd);
  if (tile * (16 * kTokenTiles) >= tokens || rank0 >= rank) return;
  const int tiles = min((rank - rank0 + 15) / 16, kRankTiles);
  // this cut's steps, and the wave's of them
  const int steps = (p.K + kStep - 1) / kStep, each = (steps + p.cuts - 1) / p.cuts, begin = cut * each, end = min(begin + each, steps);
  const char* x = reinterpret_cast<const char*>(p.x.data) + (int64_t(b) * p.x.seq + min(t0 + r, tokens - 1) * p.x.token) * kBytes;
  const char* rows = reinterpret_cast<const char*>(p.a) + ((int64_t(a) * p.R + rank0 + r) * p.K) * kBytes;
  f32x4 sum[kRankTiles];
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j) sum[j] = f32x4{0, 0, 0, 0};
  constexpr int kAheadSteps = 4, kEvery = kShare ? 4 : 1;
  for (int s0 = begin + (kShare ? wave : 0); s0 < end; s0 += kEvery * kAheadSteps) {
    u32x4 xs[kAheadSteps], as[kAheadSteps][kRankTiles];
#pragma unroll
    for (int u = 0; u < kAheadSteps; ++u) {
      const int s = s0 + u * kEvery, k = s * kStep + g * kLane;
      const bool there = s < end && k < p.K;             // (K is a multiple of a lane's channels)
      xs[u] = there ? load16(x + int64_t(k) * kBytes) : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < kRankTiles; ++j) as[u][j] = there && j < tiles ? load16(rows + (int64_t(16 * j) * p.K + k) * kBytes) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < kAheadSteps; ++u)
#pragma unroll
      for (int j = 0; j < kRankTiles; ++j) sum[j] = Product<T>::add(as[u][j], xs[u], sum[j]);
  }
  if constexpr (kShare) {
    if (wave > 0)
#pragma unroll
      for (int j = 0; j < kRankTiles; ++j) part[wave - 1][j][lane] = sum[j];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int j = 0; j < kRankTiles; ++j)
#pragma unroll
      for (int w = 0; w < 3; ++w) sum[j] += part[w][j][lane];
  }
  if (t0 + r >= tokens) return;
  float* to = p.h + ((int64_t(cut) * p.B + b) * p.n + t0 + r) * p.R + rank0 + 4 * g;
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j)
    if (j < tiles) *reinterpret_cast<f32x4*>(to + 16 * j) = sum[j];
}

// Two terms of eight numbers as operands.
template <typename T> struct Terms;
template <> struct Terms<Bf16> { typedef __bf16 E; };
template <> struct Terms<F16> { typedef _Float16 E; };

constexpr int kRanksTogether = 64;       // of h in LDS

template <typename T, int kTokenTiles> struct AdaptShared {
  // 16-bit rows: of each 16 ranks [g][token][8], g = 0, 1 the first terms of ranks 8 g .., g = 2, 3 the second of ranks 8 (g - 2) ..; fp32: [g][token][4]
  u32x4 h[kRanksTogether / 16][4][16 * kTokenTiles];
  float factor[16 * kTokenTiles];
};

// Ranks rank0 .. rank0 + 63 of the tokens' h into LDS; behind a barrier on both sides.
template <typename T, int kTokenTiles>
__device__ __forceinline__ void adapt_place(const AdaptParams& p, const float* h, int64_t cut_stride, int tokens, int rank0, int rank, AdaptShared<T, kTokenTiles>& sh) {
  const int q = threadIdx.x & 15;                        // four ranks: 4 q ..
#pragma unroll
  for (int it = 0; it < kTokenTiles; ++it) {
    const int token = it * 16 + (threadIdx.x >> 4), at = rank0 + 4 * q;
    f32x4 v{0, 0, 0, 0};
    if (token < tokens && at < rank) {
      const float* from = h + int64_t(token) * p.R + at;
      for (int c = 0; c < p.cuts; ++c) v += *(const f32x4 __attribute__((address_space(1)))*)(from + c * cut_stride);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (at + i >= rank) v[i] = 0.0f;
    }
    if constexpr (sizeof(T) == 4) {
      sh.h[q >> 2][q & 3][token] = __builtin_bit_cast(u32x4, v);
    } else {
      typedef typename Terms<T>::E E;
      typedef E E4 __attribute__((ext_vector_type(4)));
      E4 first, second;
      const float up = sizeof(E) == 2 && __is_same(E, _Float16) ? sh.factor[token] : 1.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float w = v[i] * up;
        first[i] = E(w);
        second[i] = E(w - float(first[i]));
      }
      uint64_t* to = reinterpret_cast<uint64_t*>(&sh.h[q >> 2][(q & 3) >> 1][token]) + (q & 1);
      *to = __builtin_bit_cast(uint64_t, first);
      reinterpret_cast<uint64_t*>(&sh.h[q >> 2][2 + ((q & 3) >> 1)][token])[q & 1] = __builtin_bit_cast(uint64_t, second);
    }
  }
}

// A power of two for each token that brings its largest h to 2^13 .. 2^14 (binary16 rows).
template <int kTokenTiles>
__device__ __forceinline__ void adapt_range(const AdaptParams& p, const float* h, int64_t cut_stride, int tokens, int rank, float* factor) {
  const int q = threadIdx.x & 15;
#pragma unroll
  for (int it = 0; it < kTokenTiles; ++it) {
    const int token = it * 16 + (threadIdx.x >> 4);
    uint32_t most = 0;                                   // magnitudes as whole numbers: NaN is the largest
    for (int at = 4 * q; at < rank; at += 64) {
      if (token >= tokens) break;
      f32x4 v{0, 0, 0, 0};
      for (int c = 0; c < p.cuts; ++c) v += *(const f32x4 __attribute__((address_space(1)))*)(h + int64_t(token) * p.R + at + c * cut_stride);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (at + i < rank) most = max(most, as_u32(v[i]) & 0x7FFFFFFFu);
    }
#pragma unroll
    for (int w = 1; w < 16; w *= 2) most = max(most, uint32_t(__shfl_xor(int(most), w, 16)));
    const int e = int(most >> 23) - 127;                 // 2^e <= largest
    if (q == 0) factor[token] = as_f32(uint32_t(127 + min(max(13 - e, -126), 100)) << 23);
  }
}

// 16 bytes of a row of the result, at any alignment of its elements; its last `elements`, if they are fewer.
template <typename T> __device__ __forceinline__ u32x4 load_part(const char* p, int elements) {
  constexpr int kLane = 16 / ElemTraits<T>::kBytes;
  if (elements >= kLane) return load16_any(p);
  u32x4 v{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kLane; ++i)
    if (i < elements) {
      if constexpr (sizeof(T) == 4) v[i] = as_global(reinterpret_cast<const uint32_t*>(p))[i];
      else v[i >> 1] |= uint32_t(as_global(reinterpret_cast<const uint16_t*>(p))[i]) << (16 * (i & 1));
    }
  return v;
}
template <typename T> __device__ __forceinline__ void store_part(char* p, u32x4 v, int elements) {
  constexpr int kLane = 16 / ElemTraits<T>::kBytes;
  if (elements >= kLane) return store16_any(p, v);
#pragma unroll
  for (int i = 0; i < kLane; ++i)
    if (i < elements) {
      if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(p)[i] = v[i];
      else reinterpret_cast<uint16_t*>(p)[i] = uint16_t(v[i >> 1] >> (16 * (i & 1)));
    }
}

// Ranks from..from + 7 (or 3) of 16 bytes, those that count.
template <typename T> __device__ __forceinline__ u32x4 mask_ranks(u32x4 v, int from, int rank) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = from + i < rank ? v[i] : 0;
    else v[i] &= (from + 2 * i < rank ? 0xFFFFu : 0u) | (from + 2 * i + 1 < rank ? 0xFFFF0000u : 0u);
  }
  return v;
}

template <typename T, int kTokenTiles>
__global__ __launch_bounds__(kBlock) void adapt_up_kernel(const AdaptParams p) {
  constexpr int kBytes = ElemTraits<T>::kBytes, kLane = 16 / kBytes;       // kLane: a lane's channels in a row
  constexpr int kSets = kLane / 4, kGroups = 4 / kSets;                      // instructions that make those, groups of them: 64 channels
  __shared__ AdaptShared<T, kTokenTiles> sh;
  const int wave = wave_id(), lane = lane_id(), r = lane & 15, g = lane >> 4;
  uint32_t block = blockIdx.x;
  const int chunk = int(block % uint32_t(p.chunks));
  block /= uint32_t(p.chunks);
  const uint32_t b = block / uint32_t(p.tiles);
  const int tile = int(block - b * uint32_t(p.tiles)), t0 = tile * (16 * kTokenTiles), tokens = counted(p.count, b, p.n) - t0;
  int rank;
  bool odd;
  const int a = adapter_of(p, b, rank, odd);
  if (tile == 0 && chunk == 0 && threadIdx.x == 0 && p.status)
    p.status[b] = odd || (p.count && as_global(p.count)[b] != counted(p.count, b, p.n)) ? kBadIndex : 0;
  if (tokens <= 0) return;
  const int n0 = chunk * 256 + wave * 64;                // the wave's first channel
  const bool any = n0 < p.N;
  const char* base = reinterpret_cast<const char*>(p.base.data) + (int64_t(b) * p.base.seq + t0 * p.base.token) * kBytes;
  char* out = reinterpret_cast<char*>(const_cast<void*>(p.out.data)) + (int64_t(b) * p.out.seq + t0 * p.out.token) * kBytes;
  if (rank == 0) {                                       // nothing to add
    if (!p.copy || !any) return;
    for (int t = r; t < min(tokens, 16 * kTokenTiles); t += 16)
#pragma unroll
      for (int q = 0; q < kGroups; ++q) {
        const int c = n0 + (q * 4 + g) * kLane;
        if (c < p.N) store_part<T>(out + (t * p.out.token + c) * kBytes, load_part<T>(base + (t * p.base.token + c) * kBytes, p.N - c), p.N - c);
      }
    return;
  }
  const float* h = p.h + (int64_t(b) * p.n + t0) * p.R;
  const int64_t cut_stride = p.B * p.n * int64_t(p.R);
  u32x4 held[kTokenTiles][kGroups];                      // base
#pragma unroll
  for (int t = 0; t < kTokenTiles; ++t)
#pragma unroll
    for (int q = 0; q < kGroups; ++q) {
      const int c = n0 + (q * 4 + g) * kLane, token = 16 * t + r;
      held[t][q] = c < p.N && token < tokens ? load_part<T>(base + (token * p.base.token + c) * kBytes, p.N - c) : u32x4{0, 0, 0, 0};
    }
  if constexpr (__is_same(T, F16)) {
    adapt_range<kTokenTiles>(p, h, cut_stride, tokens, rank, sh.factor);
    __syncthreads();
  }
  f32x4 sum[kTokenTiles][4];
#pragma unroll
  for (int t = 0; t < kTokenTiles; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[t][j] = f32x4{0, 0, 0, 0};
  // Row r of instruction j: channel of the lane's run 4 j' + i, so that a lane's results lie in a row.
  const char* rows = reinterpret_cast<const char*>(p.b) + int64_t(a) * p.N * p.R * kBytes;
  for (int rank0 = 0; rank0 < rank; rank0 += kRanksTogether) {
    if (rank0 > 0) __syncthreads();
    adapt_place<T, kTokenTiles>(p, h, cut_stride, tokens, rank0, rank, sh);
    __syncthreads();
    if (!any) continue;
    for (int s = 0; s < kRanksTogether / 16 && rank0 + 16 * s < rank; ++s) {
      const int from = rank0 + 16 * s + (sizeof(T) == 4 ? 4 * g : 8 * (g & 1));
      u32x4 w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = n0 + (j / kSets) * (4 * kLane) + (r >> 2) * kLane + 4 * (j % kSets) + (r & 3);
        w[j] = c < p.N && from < rank ? load16(rows + (int64_t(c) * p.R + from) * kBytes) : u32x4{0, 0, 0, 0};
        if (from + kLane > rank) w[j] = mask_ranks<T>(w[j], from, rank);
      }
#pragma unroll
      for (int t = 0; t < kTokenTiles; ++t) {
        const u32x4 hs = sh.h[s][g][16 * t + r];
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[t][j] = Product<T>::add(w[j], hs, sum[t][j]);
      }
    }
  }
  if (!any) return;
  const float scale = p.scale ? as_global(p.scale)[a] : 1.0f;
#pragma unroll
  for (int t = 0; t < kTokenTiles; ++t) {
    const int token = 16 * t + r;
    if (token >= tokens) continue;
    const float f = __is_same(T, F16) ? scale / sh.factor[token] : scale;
#pragma unroll
    for (int q = 0; q < kGroups; ++q) {
      const int c = n0 + (q * 4 + g) * kLane;
      if (c >= p.N) continue;
      u32x4 made;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) made[i] = as_u32(fmaf(sum[t][q][i], f, as_f32(held[t][q][i])));
      } else {
        float v[8];
        unpack<T>(make_uint4(held[t][q][0], held[t][q][1], held[t][q][2], held[t][q][3]), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(sum[t][2 * q + (i >> 2)][i & 3], f, v[i]);
        Eight<T> e;
        e.set(v);
        made = e.w;
      }
      store_part<T>(out + (token * p.out.token + c) * kBytes, made, p.N - c);
    }
  }
}

}  // namespace tslt
