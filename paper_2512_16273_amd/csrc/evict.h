// The tokens of most weight moved to new pages (tslt_cache_evict).
//
// Two launches.  The first, a workgroup to a head of a sequence, finds which tokens stay: the weight of the least of them by three
// rounds of counting (11, 11 and 10 bits of a key that orders as the weights do), then the tokens above it and as many equal to it
// as are missing, the first ones, in ascending order.  The second, a workgroup to a new page, gathers their codes (moved by the first one's
// workgroups too, a head's 1024 tokens take 42 us in all, 16 so).  Bound
// by the latency of the counting where a cache is short (4096 tokens: 8 us of 16), by the bytes moved where it is long: 16 sequences of 9000 to 32768
// tokens, 8 heads of 128, to 16001, 280 us, 30 of them the counting; the move reads and writes 1.0 GB in 250, 4 TB/s, a copy 4.9.
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

// Larger weight, larger key; NaN below everything, and no token has key 0.
constexpr uint32_t kKeyNan = 1u, kKeyNoToken = 0u;
__device__ __forceinline__ uint32_t weight_key(float w) { return w != w ? kKeyNan : mono_key(w + 0.0f); }

// The keys of the weights that a wave has a stretch of: kHeld to a lane in registers, or (kHeld = 0) made from memory every time.  Places behind a
// stretch's last token (its last 256 are looked at together, and every stretch but the last may end inside them) have a key below every token's: as
// many tokens as are looked for there are, so the least key that stays is a token's and no such place is ever counted or kept.
template <int kHeld> struct Stretch {
  uint32_t key[kHeld > 0 ? kHeld : 1];
  const float* from;
  int lo, hi;                              // tokens of the stretch
  // (read whether or not there is one, the last one instead: so all are on their way at the same time)
  __device__ __forceinline__ float read(int i0) const { return as_global(from)[max(0, min(i0 + lane_id(), hi - 1))]; }
  __device__ __forceinline__ uint32_t made(float w, int i0) const { return lane_id() < hi - i0 ? weight_key(w) : kKeyNoToken; }
  __device__ __forceinline__ void load(const float* weight, int first, int last) {
    from = weight;
    lo = first;
    hi = last;
    if constexpr (kHeld > 0) {
      float w[kHeld];
#pragma unroll
      for (int i = 0; i < kHeld; ++i) w[i] = read(lo + i * 64);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) key[i] = made(w[i], lo + i * 64);
    }
  }
  // f(first token, keys) for the lane's places, four at a time; all lanes come along.
  template <typename F> __device__ __forceinline__ void each(const F& f) const {
    if constexpr (kHeld > 0) {
#pragma unroll
      for (int i = 0; i < kHeld; i += 4)
        if (lo + i * 64 < hi) f(lo + i * 64, reinterpret_cast<const uint32_t (&)[4]>(key[i]));
    } else {
      for (int i0 = lo; i0 < hi; i0 += 256) {
        float w[4];
        uint32_t x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = read(i0 + u * 64);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = made(w[u], i0 + u * 64);
        f(i0, x);
      }
    }
  }
};

template <int kHeld> __global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const EvictParams p) {
  __shared__ uint32_t bins[kEvictBins];
  __shared__ uint32_t wave_sum[kEvictWaves], wave_above[kEvictWaves], wave_equal[kEvictWaves];
  __shared__ uint32_t found_bin, found_before;
  const int tid = int(threadIdx.x), lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int h = int(blockIdx.x % uint32_t(p.c.heads));
  const int64_t b = blockIdx.x / uint32_t(p.c.heads);
  bool bad;
  const int len = cached_tokens(p.c, b, bad);
  const int stay = min(len, p.keep), recent = min(p.recent, stay);
  const int from = len - recent, need = stay - recent;      // `need` of the first `from` tokens stay
  const float* weight = p.weight + (b * p.c.heads + h) * p.c.width * kPage;
  int32_t* kept = p.out_kept + (b * p.c.heads + h) * int64_t(p.keep);
  float* out = p.out_weight + (b * p.c.heads + h) * p.new_width * kPage;
  const int stretch = ((from + kEvictWaves - 1) / kEvictWaves + 63) / 64 * 64;
  Stretch<kHeld> mine;
  mine.load(weight, min(from, wave * stretch), min(from, (wave + 1) * stretch));
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

  if (need == from) {
    for (int i = tid; i < need; i += kEvictThreads) {
      kept[i] = i;
      out[i] = as_global(weight)[i];
    }
  } else if (need > 0) {
    uint32_t key = 0, ties = uint32_t(need);                // tokens above `key`, and the first `ties` equal to it, stay
#pragma unroll
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, width = round == 2 ? 10 : 11;
      for (int i = tid; i < kEvictBins; i += kEvictThreads) bins[i] = 0;
      __syncthreads();
      mine.each([&](int, const uint32_t (&x)[4]) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (round == 0 || (x[u] ^ key) >> (shift + width) == 0) atomicAdd(&bins[x[u] >> shift & ((1u << width) - 1)], 1u);
      });
      __syncthreads();
      // the bin from the top in which the `ties`-th lies: thread t has bins 2 t and 2 t + 1 from the top
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
      if (before < ties && before + c0 >= ties) { found_bin = uint32_t(top); found_before = before; }
      else if (before + c0 < ties && before + c0 + c1 >= ties) { found_bin = uint32_t(top - 1); found_before = before + c0; }
      __syncthreads();
      key |= found_bin << shift;
      ties -= found_before;
    }
    // How many of those in the stretches before it stay says where a wave's own go.
    uint32_t above = 0, equal = 0;
    mine.each([&](int, const uint32_t (&x)[4]) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        above += uint32_t(__popcll(ballot(x[u] > key)));
        equal += uint32_t(__popcll(ballot(x[u] == key)));
      }
    });
    if (lane == 0) { wave_above[wave] = above; wave_equal[wave] = equal; }
    __syncthreads();
    uint32_t n_above = 0, n_equal = 0;
    for (int i = 0; i < wave; ++i) { n_above += wave_above[i]; n_equal += wave_equal[i]; }
    const auto before = [](uint64_t m) { return __builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), 0)); };
    mine.each([&](int i0, const uint32_t (&x)[4]) {
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = as_global(weight)[min(i0 + u * 64 + lane, from - 1)];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint64_t gt = ballot(x[u] > key), eq = ballot(x[u] == key);
        const uint32_t e = n_equal + before(eq);
        if (x[u] > key || (x[u] == key && e < ties)) {
          const uint32_t to = n_above + before(gt) + min(e, ties);
          kept[to] = i0 + u * 64 + lane;
          out[to] = w[u];
        }
        n_above += uint32_t(__popcll(gt));
        n_equal += uint32_t(__popcll(eq));
      }
    });
  }
  for (int i = tid; i < recent; i += kEvictThreads) {
    kept[need + i] = from + i;
    out[need + i] = as_global(weight)[from + i];
  }
  for (int64_t i = stay + tid; i < p.keep; i += kEvictThreads) kept[i] = -1;
  for (int64_t i = stay + tid; i < p.new_width * kPage; i += kEvictThreads) out[i] = 0;
}

// One of four words by a number that all lanes have in common.
__device__ __forceinline__ uint32_t word_of(u32x4 x, int i) { return i < 2 ? (i == 0 ? x[0] : x[1]) : (i == 2 ? x[2] : x[3]); }
__device__ __forceinline__ float lane_value(float x, int i) { return as_f32(__builtin_amdgcn_readlane(as_u32(x), i)); }

// A workgroup to a new page of a head, a wave to 16 of its tokens.  Where the tokens come from is known to all lanes alike, so a wave reads the runs of 16
// values that hold any of them, 16 bytes a lane and channel, and picks the bytes in registers; nothing goes through LDS and no wave waits for another.
template <int D> __global__ __launch_bounds__(256) void evict_move_kernel(const EvictParams p) {
  constexpr int kMine = D / 64;            // channels to a lane
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const uint32_t pages = uint32_t((p.keep + kPage - 1) / kPage);
  const int w = int(blockIdx.x % pages);
  const int h = int(blockIdx.x / pages % uint32_t(p.c.heads));
  const int64_t b = blockIdx.x / (uint64_t(pages) * p.c.heads);
  // Lane i: slot i of the page; its token (-1: there is none), the token's page and place there (-1: there is none), and the page's scales.
  int token = -1, page = -1;
  if (w * kPage + lane < p.keep) token = as_global(p.out_kept + (b * p.c.heads + h) * int64_t(p.keep))[w * kPage + lane];
  const int to_page = as_global(p.new_pages + b * p.new_width)[w];
  if (ballot(token >= 0) == 0 || to_page < 0 || to_page >= p.c.n_pages) return;
  const int64_t to = int64_t(to_page) * p.c.heads + h;
  float scale[2] = {0, 0}, most[2];
  if (token >= 0) {
    page = as_global(p.c.pages + b * p.c.width)[token / kPage];
    if (page < 0 || page >= p.c.n_pages) page = -1;
    else {
      const float* from = p.c.scales + (int64_t(page) * p.c.heads + h) * 2;
      scale[0] = as_global(from)[0];
      scale[1] = as_global(from)[1];
    }
  }
  token &= kPage - 1;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    most[part] = scale[part];
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) most[part] = fmaxf(most[part], __shfl_xor(most[part], x));
    if (most[part] == 0.0f) most[part] = as_f32(uint32_t(127 + kMinScaleExp) << 23);
    if (threadIdx.x == 0) p.c.scales[to * 2 + part] = most[part];
  }
  const float k_factor = page < 0 ? 1.0f : power_ratio(scale[0], most[0]), v_factor = page < 0 ? 1.0f : power_ratio(scale[1], most[1]);
  uint8_t* codes = p.c.codes + to * (2 * kPage * D);

  // Keys: 16 bytes a lane, of D / 16 lanes a token.
  constexpr int kKeyTurns = D / 64;
  u32x4 keys[kKeyTurns];
  float factor[kKeyTurns];
#pragma unroll
  for (int it = 0; it < kKeyTurns; ++it) {
    const int idx = it * 64 + lane, slot = wave * 16 + idx / (D / 16), d = idx % (D / 16) * 16;
    const int from = __shfl(page, slot), at = __shfl(token, slot);
    factor[it] = __shfl(k_factor, slot);
    keys[it] = u32x4{0, 0, 0, 0};
    if (from >= 0) keys[it] = load16(page_codes(p.c, from, h, D) + at * D + d);
  }
  // Values: the runs that slots 16 wave .. + 15 come from, one after the other, the next one on its way while this one's bytes are picked.
  const int first = wave * 16;
  const auto run_of = [&](int slot) {      // the run's first byte in the cache, or -1
    const int from = __builtin_amdgcn_readlane(page, slot), at = __builtin_amdgcn_readlane(token, slot);
    return from < 0 ? int64_t(-1) : (int64_t(from) * p.c.heads + h) * (2 * kPage * D) + kPage * D + (at >> 4) * (16 * D);
  };
  const auto load_run = [&](int64_t run, u32x4 (&x)[kMine]) {
#pragma unroll
    for (int k = 0; k < kMine; ++k) x[k] = run < 0 ? u32x4{0, 0, 0, 0} : load16(p.c.codes + run + (k * 64 + lane) * 16);
  };
  u32x4 x[kMine], next[kMine], o[kMine];
  uint32_t acc[kMine];
#pragma unroll
  for (int k = 0; k < kMine; ++k) { o[k] = u32x4{0, 0, 0, 0}; acc[k] = 0; }
  int64_t run = run_of(first);
  load_run(run, x);
  int slot = 0;
  while (slot < 16) {
    int end = slot + 1;                    // slots slot .. end - 1 come from this run
    int64_t next_run = -2;
    while (end < 16 && (next_run = run_of(first + end)) == run) ++end;
    if (end < 16) load_run(next_run, next);
    for (; slot < end; ++slot) {
      const int t = __builtin_amdgcn_readlane(token, first + slot) & 15;
      const float f = lane_value(v_factor, first + slot);
#pragma unroll
      for (int k = 0; k < kMine; ++k) {
        uint32_t y = word_of(x[k], t >> 2);
        if (f != 1.0f) y = rescaled(y, f);
        acc[k] = __builtin_amdgcn_alignbit(y >> (8 * (t & 3)), acc[k], 8);       // the byte on top of the three before it
        if ((slot & 3) == 3) o[k] = u32x4{o[k][1], o[k][2], o[k][3], acc[k]};
      }
    }
    run = next_run;
#pragma unroll
    for (int k = 0; k < kMine; ++k) x[k] = next[k];
  }
#pragma unroll
  for (int it = 0; it < kKeyTurns; ++it) {
    const int idx = it * 64 + lane;
    if (factor[it] != 1.0f) keys[it] = rescaled(keys[it], factor[it]);
    *reinterpret_cast<u32x4*>(codes + (first + idx / (D / 16)) * D + idx % (D / 16) * 16) = keys[it];
  }
#pragma unroll
  for (int k = 0; k < kMine; ++k) *reinterpret_cast<u32x4*>(codes + kPage * D + first * D + (k * 64 + lane) * 16) = o[k];
}

}  // namespace tslt
