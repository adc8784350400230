// Attention weight of every cached token, accumulated (tslt_cache_weigh):
//
//   w'_j = decay * w_j + sum over rows i of exp(s_ij - lse_i)
//
// A wave takes pages of a head one after the other, the next two's keys on their way while this one's meet the rows; the rows, RT tiles of 16, stay in
// registers where they are no more, and else pass by every page, RT tiles at a time.  A token's weight is added to by one wave alone, so that
// nothing is exchanged between waves (but for the sums of four that share a page, in an order that does not change).  Bound by the bytes of the keys where the rows are few, by the products and the exponentials where they are many.
// Where there are fewer pages than workgroups fit the GPU and many rows, a workgroup's four waves share a page and its rows.
// All pages of all sequences and heads are dealt out to one round of waves in equal shares, as sequences differ in length and the host does not know
// how (32 sequences of 1000 to 16000 tokens, 8 heads, 36 rows: 97 us with as many workgroups to each head of each sequence, 78 so: 298 MB that it
// cannot do without at 3.8 TB/s, 351 moved, 20 GFLOP; matrix units are busy an eighth of the time: a tile's products and its exponentials take turns).
#pragma once
#include "cache.h"

namespace tslt {

struct WeighParams {
  CacheView c;
  RowsView q;
  int64_t B;
  int n, group, heads_q;
  const int32_t* count;
  const float* lse;                        // [B][n][heads_q]
  float scale2, decay;
  const float* weight;                     // [B][heads][width * 64]
  float* out_weight;
  int32_t* status;
};

// The lane whose number differs in bit 0, 1, 2 or 3 (kHalf = 1, 2, 4, 8): its value.
template <int kHalf> __device__ __forceinline__ float across(float x) {
  const int v = int(as_u32(x));
  int y;
  if constexpr (kHalf == 1) y = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false);         // quad_perm 1 0 3 2
  else if constexpr (kHalf == 2) y = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false);    // quad_perm 2 3 0 1
  else if constexpr (kHalf == 8) y = __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false);   // row_ror 8
  else y = __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false), 0x1B, 0xF, 0xF, false);   // 7 - i, then 3 - i: 4 apart
  return as_f32(uint32_t(y));
}
// Sixteen lanes' sums of sixteen tokens: each exchange halves the tokens that a lane goes on with; lane 16 g + r ends with token r's.
template <int kHalf> __device__ __forceinline__ void fold(float (&sum)[16], int r) {
  const bool up = (r & kHalf) != 0;
#pragma unroll
  for (int i = 0; i < kHalf; ++i) {
    const float mine = up ? sum[kHalf + i] : sum[i], other = up ? sum[i] : sum[kHalf + i];
    sum[i] = mine + across<kHalf>(other);
  }
}

// Most tiles of rows that there are registers for (none spills; 16 bits, D = 128, four tiles: 253 of 256).
template <typename T, int D> constexpr int weigh_tiles() { return sizeof(T) == 2 ? (D == 256 ? 2 : 4) : D == 64 ? 2 : 1; }

// Pages of a sequence.
__device__ __forceinline__ int sequence_pages(const CacheView& c, int64_t b) {
  bool bad;
  return (cached_tokens(c, b, bad) + kPage - 1) / kPage;
}
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return int64_t(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(int(x >> 32)))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(int(x))));
}

// Pages first .. first + count - 1 of one head.  kWaves = 4: for a whole workgroup, whose waves have every fourth RT tiles of rows each, the next ones on their
// way, and hand each other their sums; turn: pages that the workgroup has done.
template <typename T, int D, int RT, int kWaves> __device__ __forceinline__ void weigh_pages(const WeighParams& p, int64_t b, int h, int first, int count, int wave, uint32_t& turn) {
  constexpr bool kTwo = kWaves > 1 && weigh_tiles<T, D>() >= 2 * RT;      // room for the next rows
  __shared__ float parts[kWaves > 1 ? 2 : 1][kWaves][kPage];
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  bool bad;
  const int len = cached_tokens(p.c, b, bad);
  const int32_t* table = p.c.pages + b * p.c.width;
  const int there = counted(p.count, b, p.n);
  const int rows = there * p.group, blocks = (rows + 16 * RT - 1) / (16 * RT);
  const int64_t weights = (b * p.c.heads + h) * p.c.width * kPage;

  Queries<T, D, RT> qs[kTwo ? 2 : 1];
  float offs[kTwo ? 2 : 1][RT];
  const auto load_rows = [&](int from, Queries<T, D, RT>& q, float (&off)[RT]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = min(from + rt * 16 + r, rows - 1), token = row / p.group, head = h * p.group + row % p.group;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) Operand<T>::load(p.q.data, b * p.q.seq + token * p.q.token + head * p.q.head + Tile::channel(i, g), q.v[rt][i]);
      const float lse = as_global(p.lse)[(b * p.n + token) * p.heads_q + head];
      // (a row that saw nothing gives nothing, and neither does one that is not there)
      off[rt] = from + rt * 16 + r < rows && lse != -INFINITY ? lse * -1.4426950408889634f : -INFINITY;
    }
  };

  for (int base = 0; base < count; base += 64) {
    // Up to 64 entries of the table with the scales of their pages, one a lane.
    const int some = min(64, count - base);
    int page = -1;
    float scale = 1.0f;
    if (lane < some) page = as_global(table)[first + base + lane];
    if (page < 0 || page >= p.c.n_pages) page = -1;
    else scale = as_global(p.c.scales)[(int64_t(page) * p.c.heads + h) * 2];
    KeyTile<D> kt[2];
    float before[2];
    const auto load_keys = [&](KeyTile<D>& k, int i) { k.load(page_codes(p.c, max(0, __builtin_amdgcn_readlane(page, min(i, some - 1))), h, D), lane); };
    const auto load_weights = [&](int i) { return as_global(p.weight)[weights + int64_t(first + base + min(i, some - 1)) * kPage + lane]; };
    load_keys(kt[0], 0);
    before[0] = load_weights(0);
    load_keys(kt[1], 1);
    before[1] = load_weights(1);
    // (the rows are asked for behind the first pages: what their sums of weights are is looked at only when all are on their way)
    if (kWaves == 1 && blocks == 1 && base == 0) load_rows(0, qs[0], offs[0]);
    for (int i0 = 0; i0 < some; i0 += 2)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = i0 + u;
        if (i >= some) break;
        const int at_page = first + base + i, pg = __builtin_amdgcn_readlane(page, i);
        const int valid = min(kPage, len - at_page * kPage);
        const float had = before[u];
        float sum[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = 0;
        const float c = p.scale2 * as_f32(__builtin_amdgcn_readlane(as_u32(scale), i));
        const auto meet = [&](const Queries<T, D, RT>& q, const float (&off)[RT], bool last) {
          // (half of the tokens at a time, the scores of one tile: in registers, not those of all)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            typename Operand<T>::Vec keys[2][D / 32];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int j = 0; j < D / 32; ++j) keys[t][j] = kt[u].template operand<T>(2 * half + t, j);
            if (half == 1 && last) load_keys(kt[u], i + 2);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
              __builtin_amdgcn_sched_barrier(0);
              f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
              for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int e = 0; e < Operand<T>::kTerms; ++e)
#pragma unroll
                  for (int t = 0; t < 2; ++t) s[t] = mfma(keys[t][j], q.v[rt][j][e], s[t]);
              // (a row that saw nothing, and one that is not there, may hold anything: its scores are not looked at)
              if (off[rt] != -INFINITY) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[8 * half + e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][e & 3], c, off[rt]));
              }
            }
          }
        };
        const int last = (blocks - 1 - wave) / kWaves * kWaves + wave;       // the wave's last rows (below `wave`: it has none)
        if constexpr (kTwo) {
          if (wave < blocks) load_rows(wave * 16 * RT, qs[0], offs[0]);
          for (int two = wave; two < blocks; two += 2 * kWaves)
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              const int block = two + v * kWaves;
              if (block >= blocks) break;
              load_rows((block + kWaves) * 16 * RT, qs[v ^ 1], offs[v ^ 1]);
              meet(qs[v], offs[v], block == last);
            }
        } else {
          for (int block = wave; block < blocks; block += kWaves) {
            if (kWaves > 1 || blocks > 1) load_rows(block * 16 * RT, qs[0], offs[0]);
            meet(qs[0], offs[0], block == last);
          }
        }
        if (wave >= blocks) load_keys(kt[u], i + 2);
        before[u] = load_weights(i + 2);
        __builtin_amdgcn_sched_barrier(0);
        fold<8>(sum, r);
        fold<4>(sum, r);
        fold<2>(sum, r);
        fold<1>(sum, r);
        if constexpr (kWaves > 1) {
          // (a page's sums in the place of those two pages ago, which wave 0 has read before it came to the barrier of the page between)
          float(&part)[kWaves][kPage] = parts[turn++ & 1];
          part[wave][lane] = sum[0];
          __syncthreads();
          if (wave != 0) continue;
#pragma unroll
          for (int o = 1; o < kWaves; ++o) sum[0] += part[o][lane];
        }
        p.out_weight[weights + int64_t(at_page) * kPage + lane] = lane < valid ? had * p.decay + (pg < 0 ? 0.0f : sum[0]) : 0.0f;
      }
  }
}

template <typename T, int D, int RT, int kWaves> __global__ __launch_bounds__(256, D == 256 ? 1 : 2) void weigh_kernel(const WeighParams p) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), tid = int(threadIdx.x);
  const int64_t teams = int64_t(gridDim.x) * (4 / kWaves), me = kWaves > 1 ? int64_t(blockIdx.x) : int64_t(blockIdx.x) * 4 + wave;
  uint32_t turn = 0;
  // The wave's, or the workgroup's, share of all pages, counted sequence by sequence, head by head; then the sequence in which it begins.
  int64_t total = 0;
  for (int64_t b0 = 0; b0 < p.B; b0 += 64) {
    int64_t n = b0 + lane < p.B ? sequence_pages(p.c, b0 + lane) : 0;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) n += __shfl_xor(n, s);
    total += n;
  }
  total = uniform(total) * p.c.heads;
  const int64_t share = (total + teams - 1) / teams;
  int64_t left = min(share, total - me * share), skip = me * share;
  for (int64_t b0 = 0; b0 < p.B && left > 0; b0 += 64) {
    const int n = b0 + lane < p.B ? sequence_pages(p.c, b0 + lane) : 0;
    int64_t upto = int64_t(n) * p.c.heads;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int64_t y = __shfl_up(upto, s);
      if (lane >= s) upto += y;
    }
    const int64_t all = uniform(__shfl(upto, 63));
    while (left > 0 && skip < all) {
      const int k = __builtin_ctzll(ballot(upto > skip));            // the first sequence that reaches beyond
      const int pages = __builtin_amdgcn_readlane(n, k);
      const int64_t in = skip - (uniform(__shfl(upto, k)) - int64_t(pages) * p.c.heads);
      const int h = int(in / pages), page = int(in % pages), count = int(min<int64_t>(left, pages - page));
      weigh_pages<T, D, RT, kWaves>(p, b0 + k, h, page, count, kWaves > 1 ? wave : 0, turn);
      left -= count;
      skip += count;
    }
    skip -= all;
  }
  // Nothing lies behind a sequence's last page.
  for (int64_t row = me; row < p.B * p.c.heads; row += teams) {
    float* out = p.out_weight + row * p.c.width * kPage;
    for (int64_t i = int64_t(sequence_pages(p.c, row / p.c.heads)) * kPage + (kWaves > 1 ? tid : lane); i < p.c.width * kPage; i += 64 * kWaves) out[i] = 0;
  }
  if (p.status)
    for (int64_t b = blockIdx.x; b < p.B; b += gridDim.x) {
      bool bad;
      const int n_pages = (cached_tokens(p.c, b, bad) + kPage - 1) / kPage;
      for (int i = tid; i < n_pages; i += 256) {
        const int page = as_global(p.c.pages + b * p.c.width)[i];
        bad |= page < 0 || page >= p.c.n_pages;
      }
      bad = __syncthreads_or(bad) != 0;
      if (tid == 0) p.status[b] = sequence_status(p.count, b, p.n, bad);
    }
}

}  // namespace tslt
