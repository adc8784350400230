// tslt_adapt: out = base + scale (x A^T) B^T, of every sequence its own A and B, in two launches.
//
// The first makes h = x A^T.  A workgroup has 16 tokens of one sequence, whose four waves share the channels, or 64, 16 a wave; where that makes few workgroups the
// channels are cut too, and each cut leaves its sums.  The second adds those up, and has of 16 or 64 tokens runs of 256 channels of the result.
//
// Tokens are the columns of the matrix instructions and what is learned the rows, 16 bytes a lane straight from memory: a lane has of the first one's results
// four ranks in a row, and of the second one's eight (four of fp32) channels in a row, as the rows of the second are dealt out to two instructions so.
//
// h enters the second in two terms of the rows' type, as if it were twice as many ranks: 16 bits of it for bfloat16, 22 for binary16 (whose range it is
// brought to by a power of two a token), where the result keeps 8 and 11.
//
// Bound by trips to memory that follow one another (count and adapter, its rank, rows and h, B) more than by bytes.  One token, 4096 to 4096 channels, rank 16: 3.5 and 5.3 us; 256 x 9 tokens to 6144, 48
// adapters 9.1 and 15.4 (49 MB: 10 at a copy's rate); 4 x 2001 binary16 tokens, rank 64, 21 and 66 (267 MB: 54).  With A straight from memory for every wave the first of
// these was 43, its loads' addresses the bound; with one run of channels a workgroup, and none asked for ahead, the second was 114.  Without its products, its loads of B, or
// its stores (which are no kernels) the second is some 16, 17 and 26 us faster: no one of them bounds it alone.
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
  int tiles, up_tiles;                   // of a sequence's tokens, in the first launch and the second
  int chunks;                            // of the ranks
  int cuts;                              // of the channels of x
  int splits;                            // workgroups that share the result's channels
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

// Where a workgroup of the first launch stands: its cut of the channels, its ranks, its tokens.
struct DownBlock {
  int cut, rank0, rank, a, tile, tokens;
  uint32_t b;
  __device__ __forceinline__ DownBlock(const AdaptParams& p, int rank_tiles) {
    uint32_t block = blockIdx.x;
    cut = int(block % uint32_t(p.cuts));
    block /= uint32_t(p.cuts);
    rank0 = int(block % uint32_t(p.chunks)) * (16 * rank_tiles);
    block /= uint32_t(p.chunks);
    b = block / uint32_t(p.tiles);
    tile = int(block - b * uint32_t(p.tiles));
    tokens = counted(p.count, b, p.n);
    bool odd;
    a = adapter_of(p, b, rank, odd);
  }
};

// h of 16 tokens and kRankTiles * 16 ranks: the four waves share the channels.
template <typename T, int kRankTiles>
__global__ __launch_bounds__(kBlock) void adapt_down_few_kernel(const AdaptParams p) {
  constexpr int kBytes = ElemTraits<T>::kBytes, kLane = 16 / kBytes, kStep = Product<T>::kChannels;
  __shared__ f32x4 part[3][kRankTiles][64];
  const int wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, g = lane >> 4;
  const DownBlock at(p, kRankTiles);
  const int t0 = at.tile * 16, rank0 = at.rank0;
  if (t0 >= at.tokens || rank0 >= at.rank) return;
  const int tiles = min((at.rank - rank0 + 15) / 16, kRankTiles);
  const int steps = (p.K + kStep - 1) / kStep, each = (steps + p.cuts - 1) / p.cuts, begin = at.cut * each, end = min(begin + each, steps);
  const char* x = reinterpret_cast<const char*>(p.x.data) + (int64_t(at.b) * p.x.seq + min(t0 + r, at.tokens - 1) * p.x.token) * kBytes;
  const char* rows = reinterpret_cast<const char*>(p.a) + ((int64_t(at.a) * p.R + rank0 + r) * p.K) * kBytes;
  f32x4 sum[kRankTiles];
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j) sum[j] = f32x4{0, 0, 0, 0};
  constexpr int kSteps = 4;
  for (int s0 = begin + wave; s0 < end; s0 += 4 * kSteps) {
    u32x4 xs[kSteps], as[kSteps][kRankTiles];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int s = s0 + u * 4, k = s * kStep + g * kLane;
      const bool there = s < end && k < p.K;             // (K is a multiple of a lane's channels)
      xs[u] = there ? load16(x + int64_t(k) * kBytes) : u32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < kRankTiles; ++j) as[u][j] = there && j < tiles ? load16(rows + (int64_t(16 * j) * p.K + k) * kBytes) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < kSteps; ++u)
#pragma unroll
      for (int j = 0; j < kRankTiles; ++j) sum[j] = Product<T>::add(as[u][j], xs[u], sum[j]);
  }
  if (wave > 0)
#pragma unroll
    for (int j = 0; j < kRankTiles; ++j) part[wave - 1][j][lane] = sum[j];
  __syncthreads();
  if (wave > 0 || t0 + r >= at.tokens) return;
  float* to = p.h + ((int64_t(at.cut) * p.B + at.b) * p.n + t0 + r) * p.R + rank0 + 4 * g;
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j) {
#pragma unroll
    for (int w = 0; w < 3; ++w) sum[j] += part[w][j][lane];
    if (j < tiles) *reinterpret_cast<f32x4*>(to + 16 * j) = sum[j];
  }
}

// h of 64 tokens, 16 a wave: A goes through LDS, 128 bytes of each rank at a time, as all four waves take it.  Its 16-byte pieces are dealt out there so that
// the 16 ranks of an operand lie in different banks.
template <typename T, int kRankTiles>
__global__ __launch_bounds__(kBlock) void adapt_down_many_kernel(const AdaptParams p) {
  constexpr int kBytes = ElemTraits<T>::kBytes, kLane = 16 / kBytes, kRound = 128 / kBytes;      // channels of a lane, of a round
  constexpr int kPieces = kRankTiles * 16 * 8, kMine = (kPieces + kBlock - 1) / kBlock;
  __shared__ u32x4 piece[2][kPieces];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, g = lane >> 4;
  const DownBlock at(p, kRankTiles);
  const int t0 = at.tile * 64 + 16 * wave, rank0 = at.rank0;
  if (at.tile * 64 >= at.tokens || rank0 >= at.rank) return;
  const int tiles = min((at.rank - rank0 + 15) / 16, kRankTiles);
  const int rounds = (p.K + kRound - 1) / kRound, each = (rounds + p.cuts - 1) / p.cuts, begin = at.cut * each, end = min(begin + each, rounds);
  const char* x = reinterpret_cast<const char*>(p.x.data) + (int64_t(at.b) * p.x.seq + min(t0 + r, at.tokens - 1) * p.x.token) * kBytes;
  const char* rows = reinterpret_cast<const char*>(p.a) + ((int64_t(at.a) * p.R + rank0) * p.K) * kBytes;
  f32x4 sum[kRankTiles];
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j) sum[j] = f32x4{0, 0, 0, 0};
  u32x4 xs[2], as[kMine];
  const auto ask = [&](int round) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int q = tid + i * kBlock, k = round * kRound + (q & 7) * kLane;
      as[i] = round < end && q < 128 * tiles && k < p.K ? load16(rows + (int64_t(q >> 3) * p.K + k) * kBytes) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k = round * kRound + (4 * u + g) * kLane;
      xs[u] = round < end && k < p.K ? load16(x + int64_t(k) * kBytes) : u32x4{0, 0, 0, 0};
    }
  };
  ask(begin);
  for (int round = begin; round < end; ++round) {
    u32x4* now = piece[round & 1];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int q = tid + i * kBlock, row = q >> 3;
      if (kPieces % kBlock == 0 || q < kPieces) now[row * 8 + ((q & 7) ^ (row >> 1 & 7))] = as[i];
    }
    const u32x4 xn[2] = {xs[0], xs[1]};
    ask(round + 1);
    __syncthreads();                                     // (what is read below is written again behind the next one)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < kRankTiles; ++j) {
        const int row = 16 * j + r;
        sum[j] = Product<T>::add(now[row * 8 + ((4 * u + g) ^ (row >> 1 & 7))], xn[u], sum[j]);
      }
  }
  if (t0 + r >= at.tokens) return;
  float* to = p.h + ((int64_t(at.cut) * p.B + at.b) * p.n + t0 + r) * p.R + rank0 + 4 * g;
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j)
    if (j < tiles) *reinterpret_cast<f32x4*>(to + 16 * j) = sum[j];
}

// Two terms of eight numbers as operands.
template <typename T> struct Terms;
template <> struct Terms<Bf16> { typedef __bf16 E; };
template <> struct Terms<F16> { typedef _Float16 E; };

// How h lies in LDS and meets B.  A set is the ranks of 16 bytes of four lanes, 32 of 16-bit rows and 16 of fp32 ones: one instruction (of fp32, four) for each
// term.  Of 16 ranks in all (kPacked), both terms are one instruction of 32: g = 0, 1 the first terms of ranks 8 g .. 8 g + 7, g = 2, 3 the second ones of ranks 8 (g - 2) ..
template <typename T, bool kPacked> struct Sets {
  static constexpr int kTerms = sizeof(T) == 4 || kPacked ? 1 : 2, kRanks = sizeof(T) == 4 || kPacked ? 16 : 32;
};
// [set][term][g][token] 16 bytes; two sets are taken together.
constexpr int adapt_lds_bytes(int ranks, int token_tiles, bool packed) { return (packed ? 16 : (ranks + 31) / 32 * 32) * 4 * 16 * token_tiles; }

// Behind a barrier on both sides.  Sixteen lanes have a token.
template <typename T, int kTokenTiles, bool kPacked>
__device__ __forceinline__ void adapt_place(const AdaptParams& p, const float* h, int64_t cut_stride, int tokens, int rank, u32x4* to, float* factor) {
  constexpr int kTokens = 16 * kTokenTiles;
  const int q = threadIdx.x & 15;                        // four ranks of 64: 4 q ..
  const auto load = [&](int token, int at) {
    f32x4 v{0, 0, 0, 0};
    if (token < tokens && at < rank) {
      const float* from = h + int64_t(token) * p.R + at;
      for (int c = 0; c < p.cuts; ++c) v += *(const f32x4 __attribute__((address_space(1)))*)(from + c * cut_stride);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (at + i >= rank) v[i] = 0.0f;
    }
    return v;
  };
  f32x4 first[kTokenTiles];
#pragma unroll
  for (int it = 0; it < kTokenTiles; ++it) first[it] = load(it * 16 + (threadIdx.x >> 4), 4 * q);
#pragma unroll
  for (int it = 0; it < kTokenTiles; ++it) {
    const int token = it * 16 + (threadIdx.x >> 4);
    float up = 1.0f;
    if constexpr (__is_same(T, F16)) {
      // a power of two that brings the token's largest h to 2^13 .. 2^14 (magnitudes as whole numbers: NaN is the largest)
      uint32_t most = 0;
      for (int at = 4 * q; at < rank; at += 64) {
        const f32x4 v = at < 64 ? first[it] : load(token, at);
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, as_u32(v[i]) & 0x7FFFFFFFu);
      }
#pragma unroll
      for (int w = 1; w < 16; w *= 2) most = max(most, uint32_t(__shfl_xor(int(most), w, 16)));
      const int e = int(most >> 23) - 127;               // 2^e <= largest
      up = as_f32(uint32_t(127 + min(max(13 - e, -126), 100)) << 23);
      if (q == 0) factor[token] = up;
    }
    // (zeros up to a whole set)
    constexpr int kRanks = Sets<T, kPacked>::kRanks, kTerms = Sets<T, kPacked>::kTerms;
    for (int at = 4 * q; at < (rank + kRanks - 1) / kRanks * kRanks; at += 64) {
      const f32x4 v = at < 64 ? first[it] : load(token, at);
      u32x4* set = to + at / kRanks * (4 * kTerms * kTokens) + token;
      const int within = at % kRanks;
      if constexpr (sizeof(T) == 4) {
        set[(within >> 2) * kTokens] = __builtin_bit_cast(u32x4, v);
      } else {
        typedef typename Terms<T>::E E;
        typedef E E4 __attribute__((ext_vector_type(4)));
        E4 term[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = v[i] * up;
          term[0][i] = E(w);
          term[1][i] = E(w - float(term[0][i]));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          reinterpret_cast<uint64_t*>(set + ((kPacked ? 2 : 4) * i + (within >> 3)) * kTokens)[within >> 2 & 1] = __builtin_bit_cast(uint64_t, term[i]);
      }
    }
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

constexpr int kUpWaves = 2;

// A workgroup has 16 or 64 tokens and every p.splits-th run of 256 channels of the result, 64 a wave.  Two sets of ranks at a time; B of the next ones, and then the next run's base, are asked
// for before the present ones' products (in that order: loads come back in the order in which they were asked for, and B is nearer).
template <typename T, int kTokenTiles, bool kPacked>
__global__ __launch_bounds__(kBlock, kUpWaves) void adapt_up_kernel(const AdaptParams p) {
  constexpr int kBytes = ElemTraits<T>::kBytes, kLane = 16 / kBytes;       // kLane: a lane's channels in a row
  constexpr int kRows = kLane / 4, kGroups = 4 / kRows;                      // instructions that make those, groups of them: 64 channels
  constexpr int kTokens = 16 * kTokenTiles, kRanks = Sets<T, kPacked>::kRanks, kTerms = Sets<T, kPacked>::kTerms, kTogether = kPacked ? 1 : 2;
  extern __shared__ u32x4 placed[];
  __shared__ float factor[kTokens];
  const int wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, g = lane >> 4;
  uint32_t block = blockIdx.x;
  const int split = int(block % uint32_t(p.splits));
  block /= uint32_t(p.splits);
  const uint32_t b = block / uint32_t(p.up_tiles);
  const int tile = int(block - b * uint32_t(p.up_tiles)), t0 = tile * kTokens;
  int rank;
  bool odd;
  const int a = adapter_of(p, b, rank, odd), tokens = counted(p.count, b, p.n) - t0;
  if (tile == 0 && split == 0 && threadIdx.x == 0 && p.status)
    p.status[b] = odd || (p.count && as_global(p.count)[b] != counted(p.count, b, p.n)) ? kBadIndex : 0;
  if (tokens <= 0) return;
  const char* base = reinterpret_cast<const char*>(p.base.data) + (int64_t(b) * p.base.seq + t0 * p.base.token) * kBytes;
  char* out = reinterpret_cast<char*>(const_cast<void*>(p.out.data)) + (int64_t(b) * p.out.seq + t0 * p.out.token) * kBytes;
  const int first = split * 256 + wave * 64, stride = p.splits * 256;      // the wave's first channel of each run
  if (rank == 0) {                                       // nothing to add
    if (!p.copy) return;
    for (int n0 = first; n0 < p.N; n0 += stride)
      for (int t = r; t < min(tokens, kTokens); t += 16)
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
          const int c = n0 + (q * 4 + g) * kLane;
          if (c < p.N) store_part<T>(out + (t * p.out.token + c) * kBytes, load_part<T>(base + (t * p.base.token + c) * kBytes, p.N - c), p.N - c);
        }
    return;
  }
  // A lane's place in the rows of base and out, and in those of B: row r of instruction j is a channel of the lane's run, so that its results lie in a row.  What is the
  // same for all lanes is added in scalar registers.
  const char* lane_base[kTokenTiles];                    // (lanes behind the last token read that one's)
#pragma unroll
  for (int t = 0; t < kTokenTiles; ++t) lane_base[t] = base + (min(16 * t + r, tokens - 1) * p.base.token + g * kLane) * kBytes;
  char* lane_out = out + (r * p.out.token + g * kLane) * kBytes;
  const char* rows = reinterpret_cast<const char*>(p.b) + int64_t(a) * p.N * p.R * kBytes;
  const int lane_rank = kLane * (kPacked && sizeof(T) == 2 ? g & 1 : g), lane_channel = (r >> 2) * kLane + (r & 3);
  const uint32_t lane_row = uint32_t((lane_channel * p.R + lane_rank) * kBytes);
  u32x4 next[kTokenTiles][kGroups];                      // base
  const auto ask = [&](int n0) {
#pragma unroll
    for (int t = 0; t < kTokenTiles; ++t)
#pragma unroll
      for (int q = 0; q < kGroups; ++q) {
        const char* at = lane_base[t] + n0 * kBytes + q * 64;
        const int c = n0 + (q * 4 + g) * kLane;
        if (n0 + 64 <= p.N) next[t][q] = load16_any(at);
        else next[t][q] = c < p.N ? load_part<T>(at, p.N - c) : u32x4{0, 0, 0, 0};
      }
  };
  u32x4 w[kTogether][4];
  const auto ask_rows = [&](int n0, int rank0) {
    if (n0 + 64 <= p.N && rank0 + kTogether * kRanks <= rank) {
#pragma unroll
      for (int s = 0; s < kTogether; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[s][j] = load16(rows + (int64_t(n0 + (j / kRows) * (4 * kLane) + 4 * (j % kRows)) * p.R + rank0 + s * kRanks) * kBytes + lane_row);
      return;
    }
#pragma unroll
    for (int s = 0; s < kTogether; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = n0 + (j / kRows) * (4 * kLane) + lane_channel + 4 * (j % kRows), from = rank0 + s * kRanks + lane_rank;
        w[s][j] = c < p.N && from < rank ? load16(rows + (int64_t(c) * p.R + from) * kBytes) : u32x4{0, 0, 0, 0};
      }
  };
  ask_rows(first, 0);
  ask(first);
  const float scale = p.scale ? as_global(p.scale)[a] : 1.0f;
  adapt_place<T, kTokenTiles, kPacked>(p, p.h + (int64_t(b) * p.n + t0) * p.R, p.B * p.n * int64_t(p.R), tokens, rank, placed, factor);
  __syncthreads();
  for (int n0 = first; n0 < p.N; n0 += stride) {
    u32x4 held[kTokenTiles][kGroups];
    f32x4 sum[kTokenTiles][4];
#pragma unroll
    for (int t = 0; t < kTokenTiles; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[t][j] = f32x4{0, 0, 0, 0};
    for (int rank0 = 0; rank0 < rank; rank0 += kTogether * kRanks) {
      u32x4 v[kTogether][4];
#pragma unroll
      for (int s = 0; s < kTogether; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[s][j] = w[s][j];
      if (rank0 + kTogether * kRanks > rank)             // (not where they are asked for: that would wait for them)
#pragma unroll
        for (int s = 0; s < kTogether; ++s)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[s][j] = mask_ranks<T>(v[s][j], rank0 + s * kRanks + lane_rank, rank);
      const bool last = rank0 + kTogether * kRanks >= rank;
      ask_rows(last ? n0 + stride : n0, last ? 0 : rank0 + kTogether * kRanks);
      if (last) {
#pragma unroll
        for (int t = 0; t < kTokenTiles; ++t)
#pragma unroll
          for (int q = 0; q < kGroups; ++q) held[t][q] = next[t][q];
        ask(n0 + stride);
      }
#pragma unroll
      for (int s = 0; s < kTogether; ++s) {
        if (s > 0 && rank0 + s * kRanks >= rank) continue;
        const u32x4* set = placed + (rank0 / kRanks + s) * (4 * kTerms * kTokens);
#pragma unroll
        for (int e = 0; e < kTerms; ++e)
#pragma unroll
          for (int t = 0; t < kTokenTiles; ++t) {
            const u32x4 hs = set[(e * 4 + g) * kTokens + 16 * t + r];
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[t][j] = Product<T>::add(v[s][j], hs, sum[t][j]);
          }
      }
    }
#pragma unroll
    for (int t = 0; t < kTokenTiles; ++t) {
      if (16 * t + r >= tokens) continue;
      const float f = __is_same(T, F16) ? scale / factor[16 * t + r] : scale;
      char* to = lane_out + (16 * t * p.out.token + n0) * kBytes;
#pragma unroll
      for (int q = 0; q < kGroups; ++q) {
        u32x4 made;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) made[i] = as_u32(fmaf(sum[t][q][i], f, as_f32(held[t][q][i])));
        } else {
          float x[8];
          unpack<T>(make_uint4(held[t][q][0], held[t][q][1], held[t][q][2], held[t][q][3]), x);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = fmaf(sum[t][2 * q + (i >> 2)][i & 3], f, x[i]);
          Eight<T> e;
          e.set(x);
          made = e.w;
        }
        const int c = n0 + (q * 4 + g) * kLane;
        if (n0 + 64 <= p.N) store16_any(to + q * 64, made);
        else if (c < p.N) store_part<T>(to + q * 64, made, p.N - c);
      }
    }
  }
}

}  // namespace tslt
