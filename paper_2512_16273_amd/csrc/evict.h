// The tokens of most weight moved to new pages (tslt_cache_evict).
//
// Two launches.  The first, a workgroup to a head of a sequence, finds which tokens stay: the weight of the least of them by three
// rounds of counting (11, 11 and 10 bits of a key that orders as the weights do), then the tokens above it and as many equal to it
// as are missing, the first ones, in ascending order.  The second, a workgroup to a new page, gathers their codes.  Bound
// by the latency of the counting where a cache is short, by the bytes moved where it is long.
#pragma once
#include "append.h"

namespace tslt {

struct EvictParams {
  CacheView c;
  int64_t B;
  const float* weight;                     // [B][heads][width * 64]
  int keep, recent;
  const int32_t* new_pages;                // [B][new_width]
  int64_t new_width;
  int32_t* out_length;
  int32_t* out_kept;                       // [B][heads][keep]
  float* out_weight;                       // [B][heads][new_width * 64]
  int32_t* status;
};

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64, kEvictBins = 2048;

// Larger weight, larger key; NaN below everything.
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? 0u : mono_key(w + 0.0f); }

__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const EvictParams p) {
  __shared__ uint32_t bins[kEvictBins];
  __shared__ uint32_t wave_sum[kEvictWaves], wave_above[kEvictWaves], wave_equal[kEvictWaves];
  __shared__ uint32_t found_bin, found_before;
  const int tid = int(threadIdx.x), lane = lane_id(), wave = wave_id();
  const int h = int(blockIdx.x % uint32_t(p.c.heads));
  const int64_t b = blockIdx.x / uint32_t(p.c.heads);
  bool bad;
  const int len = cached_tokens(p.c, b, bad);
  const int stay = min(len, p.keep), recent = min(p.recent, stay);
  const int from = len - recent, need = stay - recent;      // `need` of the first `from` tokens stay
  const float* weight = p.weight + (b * p.c.heads + h) * p.c.width * kPage;
  int32_t* kept = p.out_kept + (b * p.c.heads + h) * int64_t(p.keep);
  float* out = p.out_weight + (b * p.c.heads + h) * p.new_width * kPage;
  if (h == 0) {
    const int32_t* table = p.c.pages + b * p.c.width;
    for (int i = tid; i < (len + kPage - 1) / kPage; i += kEvictThreads) {
      const int page = as_global(table)[i];
      bad |= page < 0 || page >= p.c.n_pages;
    }
    for (int i = tid; i < (stay + kPage - 1) / kPage; i += kEvictThreads) {
      const int page = as_global(p.new_pages + b * p.new_width)[i];
      bad |= page < 0 || page >= p.c.n_pages;
    }
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) {
      p.out_length[b] = stay;
      if (p.status) p.status[b] = bad ? kBadPage : 0;
    }
  }

  uint32_t key = 0, ties = uint32_t(need);                  // tokens above `key`, and the first `ties` equal to it, stay
  if (need < from && need > 0) {
    uint32_t missing = uint32_t(need);
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, width = round == 2 ? 10 : 11;
      for (int i = tid; i < kEvictBins; i += kEvictThreads) bins[i] = 0;
      __syncthreads();
      for (int i = tid; i < from; i += kEvictThreads) {
        const uint32_t x = weight_key(as_global(weight)[i]);
        if (round == 0 || (x >> (shift + width)) == (key >> (shift + width))) atomicAdd(&bins[x >> shift & ((1u << width) - 1)], 1u);
      }
      __syncthreads();
      // the bin from the top in which the `missing`-th lies: thread t has bins 2 t and 2 t + 1 from the top
      const int top = kEvictBins - 1 - 2 * tid;
      const uint32_t c0 = bins[top], c1 = bins[top - 1];
      uint32_t inc = c0 + c1;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const uint32_t y = uint32_t(__shfl_up(int(inc), s));
        if (lane >= s) inc += y;
      }
      if (lane == 63) wave_sum[wave] = inc;
      __syncthreads();
      uint32_t before = inc - c0 - c1;
      for (int i = 0; i < wave; ++i) before += wave_sum[i];
      if (before < missing && before + c0 >= missing) { found_bin = uint32_t(top); found_before = before; }
      else if (before + c0 < missing && before + c0 + c1 >= missing) { found_bin = uint32_t(top - 1); found_before = before + c0; }
      __syncthreads();
      key |= found_bin << shift;
      missing -= found_before;
    }
    ties = missing;
  }
  // Each wave has a stretch of the tokens; how many of those before it stay says where its own go.
  const bool all = need == from;
  const int stretch = ((from + kEvictWaves - 1) / kEvictWaves + 63) / 64 * 64;
  const int lo = wave * stretch, hi = min(from, lo + stretch);
  if (need > 0) {
    uint32_t above = 0, equal = 0;
    if (!all)
      for (int i = lo + lane; i < hi; i += 64) {
        const uint32_t x = weight_key(as_global(weight)[i]);
        above += x > key;
        equal += x == key;
      }
    else if (hi > lo) equal = lane == 0 ? uint32_t(hi - lo) : 0u;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
      above += uint32_t(__shfl_xor(int(above), s));
      equal += uint32_t(__shfl_xor(int(equal), s));
    }
    if (lane == 0) { wave_above[wave] = above; wave_equal[wave] = equal; }
    __syncthreads();
    uint32_t n_above = 0, n_equal = 0;
    for (int i = 0; i < wave; ++i) { n_above += wave_above[i]; n_equal += wave_equal[i]; }
    const uint64_t below = (1ull << lane) - 1;
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const int i = i0 + lane;
      const float w = i < hi ? as_global(weight)[i] : 0.0f;
      const uint32_t x = weight_key(w);
      const uint64_t gt = ballot(i < hi && !all && x > key), eq = ballot(i < hi && (all || x == key));
      const uint32_t a = n_above + uint32_t(__popcll(gt & below)), e = n_equal + uint32_t(__popcll(eq & below));
      if ((gt >> lane & 1) || ((eq >> lane & 1) && e < ties)) {
        const uint32_t to = a + min(e, ties);
        kept[to] = i;
        out[to] = w;
      }
      n_above += uint32_t(__popcll(gt));
      n_equal += uint32_t(__popcll(eq));
    }
  }
  for (int i = tid; i < recent; i += kEvictThreads) {
    kept[need + i] = from + i;
    out[need + i] = as_global(weight)[from + i];
  }
  for (int64_t i = stay + tid; i < p.keep; i += kEvictThreads) kept[i] = -1;
  for (int64_t i = stay + tid; i < p.new_width * kPage; i += kEvictThreads) out[i] = 0;
}

template <int D> __global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p) {
  __shared__ int64_t source[kPage];        // where a slot's token's page and head begin, or -1
  __shared__ int token_of[kPage];          // its place in that page
  __shared__ float factor[2][kPage];       // its scales over the new page's
  const int tid = int(threadIdx.x);
  const uint32_t pages = uint32_t((p.keep + kPage - 1) / kPage);
  const int w = int(blockIdx.x % pages);
  const int h = int(blockIdx.x / pages % uint32_t(p.c.heads));
  const int64_t b = blockIdx.x / (uint64_t(pages) * p.c.heads);
  bool bad;
  const int stay = min(cached_tokens(p.c, b, bad), p.keep);
  if (w * kPage >= stay) return;
  const int to_page = as_global(p.new_pages + b * p.new_width)[w];
  if (to_page < 0 || to_page >= p.c.n_pages) return;
  const int64_t to = int64_t(to_page) * p.c.heads + h;
  if (tid < kPage) {
    const int slot = w * kPage + tid;
    int64_t at = -1;
    int token = 0;
    float s[2] = {0, 0};
    if (slot < stay) {
      token = as_global(p.out_kept + (b * p.c.heads + h) * int64_t(p.keep))[slot];
      const int page = as_global(p.c.pages + b * p.c.width)[token / kPage];
      if (page >= 0 && page < p.c.n_pages) {
        at = int64_t(page) * p.c.heads + h;
        s[0] = as_global(p.c.scales)[at * 2];
        s[1] = as_global(p.c.scales)[at * 2 + 1];
      }
    }
    source[tid] = at < 0 ? -1 : at * (2 * kPage * D);
    token_of[tid] = token % kPage;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      float most = s[part];
#pragma unroll
      for (int x = 32; x > 0; x >>= 1) most = fmaxf(most, __shfl_xor(most, x));
      if (most == 0.0f) most = as_f32(uint32_t(127 + kMinScaleExp) << 23);
      factor[part][tid] = at < 0 ? 1.0f : power_ratio(s[part], most);
      if (tid == 0) p.c.scales[to * 2 + part] = most;
    }
  }
  __syncthreads();
  uint8_t* codes = p.c.codes + to * (2 * kPage * D);
  for (int idx = tid; idx < kPage * D / 16; idx += 256) {
    const int slot = idx / (D / 16), d = idx % (D / 16) * 16;
    u32x4 x = {0, 0, 0, 0};
    if (source[slot] >= 0) {
      x = load16(p.c.codes + source[slot] + token_of[slot] * D + d);
      if (factor[0][slot] != 1.0f) x = rescaled(x, factor[0][slot]);
    }
    *reinterpret_cast<u32x4*>(codes + slot * D + d) = x;
  }
  for (int idx = tid; idx < 4 * D; idx += 256) {
    const int s0 = idx / D * 16, d = idx % D;
    u32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int64_t from = source[s0 + i];
      if (from < 0) continue;
      const int t = token_of[s0 + i];
      uint32_t code = as_global(p.c.codes)[from + kPage * D + (t >> 4) * (16 * D) + d * 16 + (t & 15)];
      if (factor[1][s0 + i] != 1.0f) code = rescaled(code, factor[1][s0 + i]) & 0xFFu;
      x[i >> 2] |= code << (8 * (i & 3));
    }
    *reinterpret_cast<u32x4*>(codes + kPage * D + s0 * D + d * 16) = x;
  }
}

}  // namespace tslt
