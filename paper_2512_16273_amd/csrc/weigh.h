// Attention weight of every cached token, accumulated (tslt_cache_weigh):
//
//   w'_j = decay * w_j + sum over rows i of exp(s_ij - lse_i)
//
// One wave to a page of one head: its keys stay in the registers of the first product's operand and all rows that share the
// head pass by them, 16 at a time, so a page is read once and no weight is added to by two waves.  Bound by the bytes of the
// keys where the rows are few, by the exponentials and the products where they are many.
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

template <typename T, int D> __global__ __launch_bounds__(256) void weigh_kernel(const WeighParams p) {
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  const uint32_t groups = uint32_t((p.c.width + 3) / 4);
  const int at_page = int(blockIdx.x % groups) * 4 + wave;
  const int h = int(blockIdx.x / groups % uint32_t(p.c.heads));
  const int64_t b = blockIdx.x / (uint64_t(groups) * p.c.heads);
  bool bad;
  const int len = cached_tokens(p.c, b, bad);
  const int32_t* table = p.c.pages + b * p.c.width;
  if (p.status && h == 0 && blockIdx.x % groups == 0) {
    for (int i = tid; i < (len + kPage - 1) / kPage; i += 256) {
      const int page = as_global(table)[i];
      bad |= page < 0 || page >= p.c.n_pages;
    }
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) p.status[b] = bad ? kBadPage : 0;
  }
  if (at_page >= p.c.width) return;
  const int64_t at = ((b * p.c.heads + h) * p.c.width + at_page) * kPage + lane;
  const int valid = min(kPage, len - at_page * kPage);
  if (valid <= 0) {
    p.out_weight[at] = 0;
    return;
  }
  const float before = lane < valid ? as_global(p.weight)[at] * p.decay : 0.0f;
  const int page = __builtin_amdgcn_readfirstlane(as_global(table)[at_page]);
  if (page < 0 || page >= p.c.n_pages) {
    p.out_weight[at] = before;
    return;
  }
  const float k_scale = as_global(p.c.scales)[(int64_t(page) * p.c.heads + h) * 2];
  KeyTile<D> kt;
  kt.load(page_codes(p.c, page, h, D), lane);
  const int there = p.count ? min(max(as_global(p.count)[b], 0), p.n) : p.n;
  const int rows = there * p.group;
  const float c = p.scale2 * k_scale;
  float sum[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] = 0;
  for (int row0 = 0; row0 < rows; row0 += 16) {
    const int row = min(row0 + r, rows - 1), token = row / p.group, head = h * p.group + row % p.group;
    Queries<T, D, 1> q;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) Operand<T>::load(p.q.data, b * p.q.seq + token * p.q.token + head * p.q.head + Tile::channel(i, g), q.v[0][i]);
    const float lse = as_global(p.lse)[(b * p.n + token) * p.heads_q + head];
    // (a row that saw nothing gives nothing, and neither does one that is not there)
    const float off = row0 + r < rows && lse != -INFINITY ? lse * -1.4426950408889634f : -INFINITY;
    f32x4 s[1][4];
    key_products(kt, q, s);
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][i >> 2][i & 3], c, off));
  }
  // Sixteen rows' sums of sixteen tokens: each exchange halves the tokens that a lane goes on with; lane 16 g + r ends with token r.
#pragma unroll
  for (int half = 8; half > 0; half >>= 1) {
    const bool up = (r & half) != 0;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float mine = up ? sum[half + i] : sum[i], other = up ? sum[i] : sum[half + i];
      sum[i] = mine + __shfl_xor(other, half);
    }
  }
  p.out_weight[at] = lane < valid ? before + sum[0] : 0.0f;
}

}  // namespace tslt
