// Attention weight of every cached token, accumulated (tslt_cache_weigh):
//
//   w'_j = decay * w_j + sum over rows i of exp(s_ij - lse_i)
//
// A wave takes the pages of a head one after the other, the next two's keys on their way while this one's meet the rows; the rows, RT tiles of 16, stay in
// registers where they are no more, and else pass by every page, RT tiles at a time.  A token's weight is added to by one wave alone, so that
// nothing is exchanged between waves.  Bound by the bytes of the keys where the rows are few, by the products and the exponentials where they are many.
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
  int strip, strips;                       // pages to a workgroup, workgroups along a sequence
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

template <typename T, int D, int RT> __global__ __launch_bounds__(256, D == 256 ? 1 : 2) void weigh_kernel(const WeighParams p) {
  constexpr int kTurns = 4;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  const int strip = int(blockIdx.x % uint32_t(p.strips));
  const int h = int(blockIdx.x / uint32_t(p.strips) % uint32_t(p.c.heads));
  const int64_t b = blockIdx.x / (uint32_t(p.strips) * uint32_t(p.c.heads));
  bool bad;
  const int len = cached_tokens(p.c, b, bad);
  const int n_pages = (len + kPage - 1) / kPage;
  const int32_t* table = p.c.pages + b * p.c.width;
  if (p.status && h == 0 && strip == 0) {
    for (int i = tid; i < n_pages; i += 256) {
      const int page = as_global(table)[i];
      bad |= page < 0 || page >= p.c.n_pages;
    }
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) p.status[b] = bad ? kBadPage : 0;
  }
  const int there = p.count ? min(max(as_global(p.count)[b], 0), p.n) : p.n;
  const int rows = there * p.group, blocks = (rows + 16 * RT - 1) / (16 * RT);
  const int64_t weights = (b * p.c.heads + h) * p.c.width * kPage;

  Queries<T, D, RT> q;
  float off[RT];
  const auto load_rows = [&](int first) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = min(first + rt * 16 + r, rows - 1), token = row / p.group, head = h * p.group + row % p.group;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) Operand<T>::load(p.q.data, b * p.q.seq + token * p.q.token + head * p.q.head + Tile::channel(i, g), q.v[rt][i]);
      const float lse = as_global(p.lse)[(b * p.n + token) * p.heads_q + head];
      // (a row that saw nothing gives nothing, and neither does one that is not there)
      off[rt] = first + rt * 16 + r < rows && lse != -INFINITY ? lse * -1.4426950408889634f : -INFINITY;
    }
  };

  const int from = strip * p.strip + wave, to = int(min(int64_t(strip + 1) * p.strip, p.c.width));
  for (int base = from; base < to; base += 64 * kTurns) {
    // Up to 64 entries of the table with the scales of their pages, one a lane.
    const int mine = base + kTurns * lane;
    int page = -1;
    float scale = 1.0f;
    if (mine < min(to, n_pages)) page = as_global(table)[mine];
    if (page < 0 || page >= p.c.n_pages) page = -1;
    else scale = as_global(p.c.scales)[(int64_t(page) * p.c.heads + h) * 2];
    const int some = min(64, (to - base + kTurns - 1) / kTurns);
    KeyTile<D> kt[2];
    const auto load_keys = [&](KeyTile<D>& k, int i) { k.load(page_codes(p.c, max(0, __builtin_amdgcn_readlane(page, min(i, some - 1))), h, D), lane); };
    float before[2];
    const auto load_weights = [&](int i) { return as_global(p.weight)[weights + int64_t(min(base + kTurns * i, to - 1)) * kPage + lane]; };
    load_keys(kt[0], 0);
    before[0] = load_weights(0);
    load_keys(kt[1], 1);
    before[1] = load_weights(1);
    // (the rows are asked for behind the first pages: what their sums of weights are is looked at only when all are on their way)
    if (blocks == 1 && base == from) load_rows(0);
    for (int i0 = 0; i0 < some; i0 += 2)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = i0 + u;
        if (i >= some) break;
        const int at_page = base + kTurns * i, pg = __builtin_amdgcn_readlane(page, i);
        const int valid = min(kPage, len - at_page * kPage);
        const int64_t at = weights + int64_t(at_page) * kPage + lane;
        const float had = before[u];
        float sum[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = 0;
        const float c = p.scale2 * as_f32(__builtin_amdgcn_readlane(as_u32(scale), i));
        typename Operand<T>::Vec keys[4][D / 32];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int j = 0; j < D / 32; ++j) keys[t][j] = kt[u].template operand<T>(t, j);
        load_keys(kt[u], i + 2);
        before[u] = load_weights(i + 2);
        for (int block = 0; block < blocks; ++block) {
          if (blocks > 1) load_rows(block * 16 * RT);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            __builtin_amdgcn_sched_barrier(0);           // (the scores of one tile in registers, not of several)
            f32x4 s[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) s[t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
              for (int e = 0; e < Operand<T>::kTerms; ++e)
#pragma unroll
                for (int t = 0; t < 4; ++t) s[t] = mfma(keys[t][j], q.v[rt][j][e], s[t]);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[e] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][e & 3], c, off[rt]));
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        fold<8>(sum, r);
        fold<4>(sum, r);
        fold<2>(sum, r);
        fold<1>(sum, r);
        p.out_weight[at] = lane < valid ? had * p.decay + (pg < 0 ? 0.0f : sum[0]) : 0.0f;
      }
  }
}
// Most tiles of rows that there are registers for.
template <typename T, int D> constexpr int weigh_tiles() { return sizeof(T) == 2 ? (D == 256 ? 2 : 4) : D == 64 ? 2 : 1; }

}  // namespace tslt
