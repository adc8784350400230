// Keys and values of new tokens into the 8-bit cache (tslt_cache_append).
//
// One workgroup (or, for the few tokens of a round, one of its waves) to a page that a sequence's new tokens touch and a head: it reads their keys and values, finds the page's scale
// (the least power of two that brings the largest finite magnitude to e4m3's 448, and no less than the page's old tokens have),
// and writes their codes; where the page's scale has to grow, its old tokens' codes too.  A page that a call begins is cleared
// behind its last token, so that no page of a sequence holds anything but its tokens and zeros.  Bound by memory for prompts, by the
// latency of one launch and three trips to memory for the tokens of a round: 8 sequences of 4001 binary16 tokens, 8 heads of 128, 53 us, 197 MB at
// 3.7 TB/s (a copy runs at 4.9); 256 sequences of 5 tokens on average, 14 us, of which the 16-byte runs of values, one token of 16 each, make
// several times the bytes that the tokens have; one token, 6 us.
#pragma once
#include "cache.h"
#include "handover.h"

namespace tslt {

struct AppendParams {
  CacheView c;
  RowsView k, v;
  int64_t B;
  int n;
  const int32_t* index;                    // [B][most], null: 0 .. most - 1
  const int32_t* count;                    // null: most
  int most;                                // tokens that a sequence appends at most
  int32_t* out_length;
  int32_t* status;
  int most_pages;                          // pages that `most` tokens can touch
};

// Two numbers as codes (the low or the high half of a word).  Infinite ones saturate, as the format has none; NaN stays.
__device__ __forceinline__ float finite_or_nan(float x) { return as_u32(x) << 1 == 0xFF000000u ? copysignf(448.0f, x) : x; }
__device__ __forceinline__ uint32_t as_codes(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(a), finite_or_nan(b), 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(c), finite_or_nan(d), lo, true));
}
// Four codes brought to another scale.
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float f) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
  return as_codes(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
}
__device__ __forceinline__ u32x4 rescaled(u32x4 w, float f) { return u32x4{rescaled(w[0], f), rescaled(w[1], f), rescaled(w[2], f), rescaled(w[3], f)}; }

// Bits of the least scale for a largest magnitude (as bits; not negative, finite): 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t scale_bits(uint32_t most) {
  const int e = int(most >> 23) - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);      // biased
  return uint32_t(max(e, 127 + kMinScaleExp)) << 23;
}
// Eight elements of a row, widened to fp32.
template <typename T> __device__ __forceinline__ void load8(const void* base, int64_t at, float (&x)[8]) {
  const T* p = reinterpret_cast<const T*>(base) + at;
  if constexpr (sizeof(T) == 4) {
    const u32x4 a = load16(p), b = load16(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = as_f32(a[i]); x[4 + i] = as_f32(b[i]); }
  } else {
    const u32x4 a = load16(p);
    unpack<T>(make_uint4(a[0], a[1], a[2], a[3]), x);
  }
}

// All threads of a team that share a page: what they have written to LDS is there.
template <int kTeam> __device__ __forceinline__ void team_sync() {
  if constexpr (kTeam == 64) wave_sync();
  else __syncthreads();
}

// kTeam threads to a page and head, 256 / kTeam heads to a workgroup; at most kMost new tokens a page (a call's tokens where they are fewer than that).
template <typename T, int D, int kTeam, int kMost> __global__ __launch_bounds__(256) void append_kernel(const AppendParams p) {
  constexpr int kChunks = D / 8, kTurns = kMost * kChunks / kTeam, kTeams = 256 / kTeam;
  constexpr int kPitch = D + 4;            // bytes from a token's codes to the next one's in LDS: rows start in different banks
  __shared__ __align__(16) uint8_t staged_all[kTeams][kMost * kPitch];
  __shared__ uint32_t most_of[2][4];
  const int tid = int(threadIdx.x), lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
  const int team = kTeam == 64 ? wave : 0, me = tid % kTeam;
  uint8_t* staged = staged_all[team];
  const uint32_t groups = uint32_t((p.c.heads + kTeams - 1) / kTeams);
  const int h0 = int(blockIdx.x % groups) * kTeams, h = h0 + team;
  const int w = int(blockIdx.x / groups % uint32_t(p.most_pages));
  const int64_t b = blockIdx.x / (groups * uint32_t(p.most_pages));
  bool bad_length;
  const int start = cached_tokens(p.c, b, bad_length);
  const int asked = p.count ? as_global(p.count)[b] : p.most;
  const int more = min(max(asked, 0), p.most);
  const int64_t end64 = min(int64_t(start) + more, p.c.width * kPage);
  const int end = int(end64);
  const int first = start / kPage;
  const int32_t* table = p.c.pages + b * p.c.width;
  const int32_t* index = p.index ? p.index + b * p.most : nullptr;

  if (h0 == 0 && w == 0) {
    int bits = bad_length || end64 < int64_t(start) + more ? kBadPage : 0;
    if (asked != more) bits |= kBadIndex;
    for (int i = first + tid; i * kPage < end; i += 256) {
      const int page = as_global(table)[i];
      if (page < 0 || page >= p.c.n_pages) bits |= kBadPage;
    }
    if (index)
      for (int i = tid; i < more; i += 256) {
        const int from = as_global(index)[i];
        if (from < 0 || from >= p.n) bits |= kBadIndex;
      }
    const int page_bits = __syncthreads_or(bits & kBadPage), index_bits = __syncthreads_or(bits & kBadIndex);
    if (tid == 0) {
      p.out_length[b] = end;
      if (p.status) p.status[b] = (page_bits ? kBadPage : 0) | (index_bits ? kBadIndex : 0);
    }
  }
  const int t0 = (first + w) * kPage;
  const int lo = max(start - t0, 0), hi = min(end - t0, kPage);        // the page's slots that get new tokens
  if (hi <= lo || h >= p.c.heads) return;                              // (where a team is less than a workgroup nothing waits for it behind this)
  const int page = as_global(table)[first + w];
  if (page < 0 || page >= p.c.n_pages) return;

  // New token `it * kTeam / kChunks + ..` of the page goes to slot lo + that.
  float k[kTurns][8], v[kTurns][8];
  uint32_t k_most = 0, v_most = 0;
#pragma unroll
  for (int it = 0; it < kTurns; ++it) {
    const int idx = it * kTeam + me, fresh = idx / kChunks, d = idx % kChunks * 8;
    int from = -1;
    if (fresh < hi - lo) {
      from = t0 + lo + fresh - start;
      if (index) from = as_global(index)[from];
    }
    if (from >= 0 && from < p.n) {
      load8<T>(p.k.data, b * p.k.seq + from * p.k.token + h * p.k.head + d, k[it]);
      load8<T>(p.v.data, b * p.v.seq + from * p.v.token + h * p.v.head + d, v[it]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) k[it][i] = v[it][i] = 0;
    }
  }
  float* scales = p.c.scales + (int64_t(page) * p.c.heads + h) * 2;
  float to[2], old[2];
#pragma unroll
  for (int part = 0; part < 2; ++part) old[part] = lo > 0 ? as_global(scales)[part] : 0.0f;
#pragma unroll
  for (int it = 0; it < kTurns; ++it)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = as_u32(k[it][i]) & 0x7FFFFFFFu, y = as_u32(v[it][i]) & 0x7FFFFFFFu;
      k_most = x < 0x7F800000u ? max(k_most, x) : k_most;
      v_most = y < 0x7F800000u ? max(v_most, y) : v_most;
    }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) {
    k_most = max(k_most, uint32_t(__shfl_xor(int(k_most), s)));
    v_most = max(v_most, uint32_t(__shfl_xor(int(v_most), s)));
  }
  if constexpr (kTeam > 64) {
    if (lane == 0) { most_of[0][wave] = k_most; most_of[1][wave] = v_most; }
    asm volatile("" ::"v"(old[0]), "v"(old[1]));         // (every thread has the old scales before any writes new ones)
    __syncthreads();
    k_most = max(max(most_of[0][0], most_of[0][1]), max(most_of[0][2], most_of[0][3]));
    v_most = max(max(most_of[1][0], most_of[1][1]), max(most_of[1][2], most_of[1][3]));
  }
  to[0] = fmaxf(as_f32(scale_bits(k_most)), old[0]);
  to[1] = fmaxf(as_f32(scale_bits(v_most)), old[1]);
  if (me < 2) scales[me] = me == 0 ? to[0] : to[1];
  const bool k_grows = lo > 0 && to[0] > old[0], v_grows = lo > 0 && to[1] > old[1];
  const float k_old = power_ratio(old[0], to[0]), v_old = power_ratio(old[1], to[1]);
  const float k_inv = power_ratio(1.0f, to[0]), v_inv = power_ratio(1.0f, to[1]);
  uint8_t* codes = p.c.codes + (int64_t(page) * p.c.heads + h) * (2 * kPage * D);
#pragma unroll
  for (int it = 0; it < kTurns; ++it) {
    const int idx = it * kTeam + me, fresh = idx / kChunks, d = idx % kChunks * 8;
    if (fresh < hi - lo) {
      float (&x)[8] = k[it], (&y)[8] = v[it];
      *reinterpret_cast<uint2*>(codes + (lo + fresh) * D + d) = make_uint2(as_codes(x[0] * k_inv, x[1] * k_inv, x[2] * k_inv, x[3] * k_inv),
                                                                           as_codes(x[4] * k_inv, x[5] * k_inv, x[6] * k_inv, x[7] * k_inv));
      uint32_t* s = reinterpret_cast<uint32_t*>(staged + fresh * kPitch + d);
      s[0] = as_codes(y[0] * v_inv, y[1] * v_inv, y[2] * v_inv, y[3] * v_inv);
      s[1] = as_codes(y[4] * v_inv, y[5] * v_inv, y[6] * v_inv, y[7] * v_inv);
    }
  }
  if (k_grows)
    for (int at = me * 16; at < lo * D; at += kTeam * 16) *reinterpret_cast<u32x4*>(codes + at) = rescaled(load16(codes + at), k_old);
  if (lo == 0)
    for (int at = hi * D + me * 16; at < kPage * D; at += kTeam * 16) *reinterpret_cast<u32x4*>(codes + at) = u32x4{0, 0, 0, 0};
  team_sync<kTeam>();
  // Values, 16 tokens of a channel at a time: those with a new token, all of a page that is begun or whose scale grows.
  const int from_run = v_grows || lo == 0 ? 0 : lo / 16, to_run = lo == 0 ? 4 : (hi + 15) / 16;
  for (int idx = from_run * D + me; idx < to_run * D; idx += kTeam) {
    const int d = idx % D, s0 = idx / D * 16;
    u32x4* at = reinterpret_cast<u32x4*>(codes + kPage * D + s0 * D + d * 16);
    u32x4 x = {0, 0, 0, 0};
    if (s0 < lo) {
      x = load16(at);
      if (v_grows) x = rescaled(x, v_old);
    }
    if (s0 + 16 > lo && s0 < hi) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int slot = s0 + i;
        if (slot < lo) continue;
        const uint32_t code = slot < hi ? staged[(slot - lo) * kPitch + d] : 0;
        x[i >> 2] = (x[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | code << (8 * (i & 3));
      }
    }
    *at = x;
  }
}

}  // namespace tslt
