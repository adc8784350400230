// Attention of a round's new tokens over the 8-bit cache and over each other (tslt_cache_attend).
//
//   s_ij = scale * q_i . k_j,  out_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = ln sum_j exp(s_ij)
//
// j runs over the cached tokens, all of which every query sees, and over those of the call's own tokens that its mask shows.
// A row is one query head of one token; the rows of one sequence that share a key/value head, n * group of them, meet the same
// keys, so the products are dense in tiles of 16 rows, and one pass keeps a running maximum m and sum l for each row.
//
// One wave takes 64 keys at a time against RT tiles of rows.  The scores come out with 16 keys of one row in each lane, which is how
// the second product wants its weights, so nothing is exchanged between lanes on the way.  Two kernels:
//   attend_stream_kernel, few rows: bound by memory.  Codes go from memory straight into the operand registers of the products (the
//     order in which the cache holds them is made for that).  Of a workgroup's four waves KS take pages in turn and 4 / KS have
//     rows of their own.
//   attend_rows_kernel, many rows: bound by the products and the exponentials.  A workgroup brings a page to LDS once, as operands, for
//     all of its waves, each with rows of its own.
// A sequence is cut into chunks of pages where its rows alone do not fill the GPU; whichever of its workgroups ends last joins them.
//
// Rounding.  Codes, and queries of 16 bits, enter the first product exactly; queries of 32 bits as three bfloat16 terms,
// exactly.  Sums are fp32.  A weight enters the second product as the sum of two bfloat16 terms, 16 bits, and of three, 24, in fp32
// calls; values enter it as bfloat16 times their page's scale, exactly.  (One bfloat16 term would be off by 2^-9, as much as the output's
// own rounding; one binary16 term by 2^-12, but it loses weights below 2^-30 of the largest, and where that one's value is 0 they are the result.)
// The running maximum is followed only when a row exceeds it by kLag powers of two: weights, in units of it, stay below 2^kLag.
#pragma once
#include "cache.h"
#include "handover.h"

namespace tslt {

constexpr float kLag = 8.0f;
constexpr float kNoMax = -3.4028235e38f;   // running maximum of a row that has met nothing yet

struct AttendParams {
  CacheView c;
  RowsView q, k, v;                        // k.data is null: no keys and values of new tokens
  int64_t B;
  int n, group, heads_q;
  const uint32_t* mask;                    // [B or 1][n][mask_words], null: token i sees tokens 0 .. i
  int64_t mask_seq;
  int mask_words;
  const int32_t* count;                    // null: n
  float scale2;                            // scale * log2 e
  void* out;
  float* lse;
  int32_t* status;
  int chunk, chunks, row_groups;           // pages to a workgroup, workgroups along a sequence, and along its rows
  uint64_t* words;                         // [B][heads][row_groups][chunks] tags of the chunks that are done
  uint64_t* part_ml;                       // [B][heads][chunks][rows] a chunk's maximum and sum (fp32 both), and
  uint64_t* part_o;                        // [B][heads][chunks][rows][D / 2] its sums of values, two to a word
  Tag tag;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float over_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float over_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}
template <typename T> __device__ __forceinline__ void store4(void* p, int64_t at, f32x4 v);
template <> __device__ __forceinline__ void store4<float>(void* p, int64_t at, f32x4 v) { *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p) + at) = v; }
template <> __device__ __forceinline__ void store4<F16>(void* p, int64_t at, f32x4 v) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<f16x4*>(reinterpret_cast<uint16_t*>(p) + at) = f16x4{_Float16(v[0]), _Float16(v[1]), _Float16(v[2]), _Float16(v[3])};
}
template <> __device__ __forceinline__ void store4<Bf16>(void* p, int64_t at, f32x4 v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4*>(reinterpret_cast<uint16_t*>(p) + at) = bf16x4{__bf16(v[0]), __bf16(v[1]), __bf16(v[2]), __bf16(v[3])};
}

// New tokens' keys and values, a tile of 64 in LDS.  16 bytes of keys are kPer channels of one token: chunk of channels c, token
// at place (token % 16) * 4 + token / 16 (the rows of one product next to each other), and that exclusive-or c % 16, so that neither
// the lanes that write a token's channels nor those that read a channel of 16 tokens meet in a bank.  16 bytes of values are kPer
// tokens of one channel.
template <typename T, int D> struct Fresh {
  static constexpr int kBytes = sizeof(T), kPer = 16 / kBytes;
  static constexpr int kKeyBytes = kPage * D * kBytes;
  static constexpr int kLds = 2 * kKeyBytes;
  static __device__ __forceinline__ int key_at(int chunk, int token) {
    const int place = (token & 15) * 4 + (token >> 4);
    return (chunk * kPage + (place ^ (chunk & 15))) * 16;
  }
  static __device__ __forceinline__ int value_at(int eight, int part, int d) { return kKeyBytes + ((eight * (8 / kPer) + part) * D + d) * 16; }
};
template <typename T> __device__ __forceinline__ bool not_finite(uint32_t bits);
template <> __device__ __forceinline__ bool not_finite<float>(uint32_t b) { return (b & 0x7F800000u) == 0x7F800000u; }
template <> __device__ __forceinline__ bool not_finite<Bf16>(uint32_t b) { return (b & 0x7F80u) == 0x7F80u; }
template <> __device__ __forceinline__ bool not_finite<F16>(uint32_t b) { return (b & 0x7C00u) == 0x7C00u; }

// An infinity or NaN in 16 bits.
template <typename T> __device__ __forceinline__ uint16_t odd_bits(float x);
template <> __device__ __forceinline__ uint16_t odd_bits<Bf16>(float x) { return x != x ? 0x7FC0u : uint16_t(as_u32(x) >> 16); }
template <> __device__ __forceinline__ uint16_t odd_bits<F16>(float x) { return x != x ? 0x7E00u : x > 0 ? 0x7C00u : 0xFC00u; }

struct FreshShared {
  int wanted[2];                           // the tile that a wave sees something of, of two tiles in turn
  int odd;                                 // a value that is not finite has been left out
};

// Brings 64 new tokens from j0 on to LDS, zeros where there are fewer.  A value that is not finite is left out (0), and that it was
// noted: a product would carry it to rows that do not see the token, as 0 times it (see add_odd_values).
template <typename T, int D, int NT>
__device__ __forceinline__ void stage_fresh(const AttendParams& p, int64_t b, int h, int j0, int there, uint8_t* lds, FreshShared& sh) {
  typedef Fresh<T, D> F;
  const int tid = int(threadIdx.x);
  const T* kp = reinterpret_cast<const T*>(p.k.data) + b * p.k.seq + h * p.k.head;
  const T* vp = reinterpret_cast<const T*>(p.v.data) + b * p.v.seq + h * p.v.head;
  constexpr int kChunks = D / F::kPer;
#pragma unroll 4
  for (int it = 0; it < kPage * kChunks / NT; ++it) {
    const int idx = it * NT + tid, chunk = idx % kChunks, token = idx / kChunks;
    u32x4 w = load16(kp + min(j0 + token, there - 1) * p.k.token + chunk * F::kPer);
    if (j0 + token >= there) w = u32x4{0, 0, 0, 0};
    *reinterpret_cast<u32x4*>(lds + F::key_at(chunk, token)) = w;
  }
  constexpr int kWide = F::kBytes == 4 ? 1 : 2;          // channels to a thread: a word
#pragma unroll 2
  for (int it = 0; it < (8 * (D / kWide) + NT - 1) / NT; ++it) {
    const int idx = it * NT + tid, at = idx % (D / kWide), eight = idx / (D / kWide);
    if (8 * (D / kWide) % NT != 0 && eight >= 8) continue;
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int token = j0 + eight * 8 + e;
      w[e] = *as_global(reinterpret_cast<const uint32_t*>(vp + min(token, there - 1) * p.v.token + at * kWide));
      if (token >= there) w[e] = 0;
    }
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (not_finite<T>(w[e])) { odd = true; w[e] = kWide == 1 ? 0 : w[e] & 0xFFFF0000u; }
      if (kWide == 2 && not_finite<T>(w[e] >> 16)) { odd = true; w[e] &= 0xFFFFu; }
    }
    if (odd) sh.odd = 1;
    if constexpr (kWide == 1) {
      *reinterpret_cast<u32x4*>(lds + F::value_at(eight, 0, at)) = u32x4{w[0], w[1], w[2], w[3]};
      *reinterpret_cast<u32x4*>(lds + F::value_at(eight, 1, at)) = u32x4{w[4], w[5], w[6], w[7]};
    } else {
      u32x4 a, c;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = (w[2 * e] & 0xFFFFu) | w[2 * e + 1] << 16;
        c[e] = w[2 * e] >> 16 | (w[2 * e + 1] & 0xFFFF0000u);
      }
      *reinterpret_cast<u32x4*>(lds + F::value_at(eight, 0, 2 * at)) = a;
      *reinterpret_cast<u32x4*>(lds + F::value_at(eight, 0, 2 * at + 1)) = c;
    }
  }
}

// What a wave keeps for its rows.  Lane l = 16 g + r: row r of each tile; of the sums, channels 16 t + 4 g .. + 3.
template <int D, int RT> struct RowState {
  f32x4 o[RT][D / 16];
  float m[RT], l[RT];
};

// The running maximum follows where a row of the tile exceeds it by more than 2^kLag.
template <int D, int RT> __device__ __forceinline__ void follow(RowState<D, RT>& st, int rt, float most) {
  if (ballot(most > st.m[rt] + kLag) == 0) return;
  const float m = over_groups_max(fmaxf(most, st.m[rt]));
  const float f = exp2_fast(st.m[rt] - m);
  st.m[rt] = m;
  st.l[rt] *= f;
#pragma unroll
  for (int d = 0; d < D / 16; ++d) st.o[rt][d] *= f;
}
// Of 16 bytes, one a token, those of the first `there` tokens: what lies behind them may be anything.
__device__ __forceinline__ u32x4 tokens_below(int there) {
  u32x4 keep;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int n = there - 4 * e;
    keep[e] = n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
  }
  return keep;
}

// A wave's tile of values, 64 tokens: of each 16 channels lane 16 g + r has channel r of tokens 16 g .. + 15.
template <int D> struct ValueTile {
  u32x4 w[D / 16];
  __device__ __forceinline__ void load(const uint8_t* values, int lane) {
    const uint8_t* p = values + (lane >> 4) * 16 * D + (lane & 15) * 16;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) w[d] = load16(p + d * 256);
  }
  __device__ __forceinline__ void cut(int there) {
    const u32x4 keep = tokens_below(there);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) w[d] &= keep;
  }
};

// Terms of a weight, and of a new token's value, in the second product; of terms a and b of a weight and a new value those with a + b < kSum.
template <typename T> struct Terms;
template <> struct Terms<Bf16> { static constexpr int kW = 2, kV = 1, kSum = 2; };
template <> struct Terms<F16> { static constexpr int kW = 2, kV = 2, kSum = 3; };       // (eleven bits: eight and three)
template <> struct Terms<float> { static constexpr int kW = 3, kV = 3, kSum = 3; };
template <int N> __device__ __forceinline__ void split_weight(float x, int i, bf16x8 (&w)[N]) {
  if constexpr (N == 3) {
    __bf16 a, b, c;
    split3(x, a, b, c);
    w[0][i] = a; w[1][i] = b; w[2][i] = c;
  } else {
    const float x0 = as_f32(as_u32(x) & 0xFFFF0000u);
    w[0][i] = __builtin_bit_cast(__bf16, uint16_t(as_u32(x0) >> 16));
    w[1][i] = __bf16(x - x0);
  }
}

// Scores of a cached page into weights and their sum.  `there` of its 64 tokens count.
template <typename T, int D, int RT>
__device__ __forceinline__ void page_weights(f32x4 (&s)[RT][4], RowState<D, RT>& st, float c, int there, int g, bf16x8 (&w)[RT][2][Terms<T>::kW]) {
  if (there < kPage) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (g * 16 + t * 4 + i >= there) s[rt][t][i] = -INFINITY;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float most = s[rt][0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) most = fmaxf(most, s[rt][i >> 2][i & 3]);
    follow(st, rt, most * c);
    float sum = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = exp2_fast(__builtin_fmaf(s[rt][i >> 2][i & 3], c, -st.m[rt]));
      sum += x;
      split_weight(x, i & 7, w[rt][i >> 3]);
    }
    st.l[rt] += sum;
  }
}

template <int D, int RT, int N>
__device__ __forceinline__ void page_values(const ValueTile<D>& v, const bf16x8 (&w)[RT][2][N], RowState<D, RT>& st, float scale) {
#pragma unroll
  for (int d = 0; d < D / 16; ++d)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bf16x8 a = codes_as_bf16(v.w[d][2 * k], v.w[d][2 * k + 1], scale);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < N; ++e) st.o[rt][d] = mfma(a, w[rt][k][e], st.o[rt][d]);
    }
}

// Eight new values (of one channel) as bfloat16 terms.
template <typename T> __device__ __forceinline__ void value_terms(u32x4 x, u32x4 y, bf16x8 (&a)[Terms<T>::kV]);
template <> __device__ __forceinline__ void value_terms<Bf16>(u32x4 x, u32x4, bf16x8 (&a)[1]) { a[0] = __builtin_bit_cast(bf16x8, x); }
template <> __device__ __forceinline__ void value_terms<F16>(u32x4 x, u32x4, bf16x8 (&a)[2]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) split_weight(i & 1 ? f16_hi(x[i >> 1]) : f16_lo(x[i >> 1]), i, a);
}
template <> __device__ __forceinline__ void value_terms<float>(u32x4 x, u32x4 y, bf16x8 (&a)[3]) { Operand<float>::split(x, y, a); }

// Which of 16 new tokens from `at` on token i sees, a bit each; `there` of them exist.
__device__ __forceinline__ uint32_t seen_of(const AttendParams& p, const uint32_t* mask, int i, int at, int there) {
  if (i >= there || at >= there) return 0;
  uint32_t bits;
  if (mask) bits = as_global(mask)[int64_t(i) * p.mask_words + (at >> 5)] >> (at & 31) & 0xFFFFu;
  else bits = i - at >= 15 ? 0xFFFFu : i < at ? 0u : (2u << (i - at)) - 1;
  return there - at < 16 ? bits & ((1u << (there - at)) - 1) : bits;
}

// The call's own tokens, all of them that the wave's rows see, tile after tile; the waves of a workgroup that share rows take turns.
template <typename T, int D, int RT, int KS, int NT>
__device__ __forceinline__ void attend_fresh(const AttendParams& p, int64_t b, int h, int first_row, int last_row, int there, int wave_k,
                                             const Queries<T, D, RT>& q, RowState<D, RT>& st, uint8_t* lds, FreshShared& sh) {
  typedef Fresh<T, D> F;
  typedef Terms<T> W;
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const uint32_t* mask = p.mask ? p.mask + b * p.mask_seq : nullptr;
  // (a token sees none behind itself where there is no mask: tiles behind the workgroup's last row's token are not looked at)
  const int reach = mask ? there : min(there, last_row / p.group + 1);
  for (int j0 = 0, turn = 0; j0 < reach; j0 += kPage, ++turn) {
    uint32_t seen[RT];
    bool any = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      seen[rt] = seen_of(p, mask, (first_row + rt * 16 + r) / p.group, j0 + g * 16, there);
      any |= seen[rt] != 0;
    }
    const bool wanted = ballot(any) != 0 && turn % KS == wave_k;
    if (ballot(any) != 0 && lane == 0) sh.wanted[turn & 1] = turn + 1;
    __syncthreads();                       // (also: what was staged before has been read)
    if (sh.wanted[turn & 1] != turn + 1) continue;
    stage_fresh<T, D, NT>(p, b, h, j0, there, lds, sh);
    __syncthreads();
    if (!wanted) continue;
    f32x4 s[RT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0, 0, 0, 0};
      const int token = (r >> 2) * 16 + t * 4 + (r & 3);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const int chunk = step_channel(i, g) / F::kPer;
        typename Operand<T>::Vec a[Operand<T>::kTerms];
        const u32x4 x = *reinterpret_cast<const u32x4*>(lds + F::key_at(chunk, token));
        if constexpr (sizeof(T) == 4) Operand<float>::split(x, *reinterpret_cast<const u32x4*>(lds + F::key_at(chunk + 1, token)), a);
        else a[0] = __builtin_bit_cast(typename Operand<T>::Vec, x);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int e = 0; e < Operand<T>::kTerms; ++e)
#pragma unroll
            for (int f = 0; f + e < Operand<T>::kTerms; ++f) s[rt][t] = mfma(a[e], q.v[rt][i][f], s[rt][t]);
        if constexpr (sizeof(T) == 4) __builtin_amdgcn_sched_barrier(0);       // (the terms of one step in registers, not of several)
      }
    }
    bf16x8 w[RT][2][W::kW];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float most = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[rt][i >> 2][i & 3] = (seen[rt] >> i & 1) ? s[rt][i >> 2][i & 3] * p.scale2 : -INFINITY;
        most = fmaxf(most, s[rt][i >> 2][i & 3]);
      }
      follow(st, rt, most);
      float sum = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = exp2_fast(s[rt][i >> 2][i & 3] - st.m[rt]);
        sum += x;
        split_weight(x, i & 7, w[rt][i >> 3]);
      }
      st.l[rt] += sum;
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bf16x8 a[W::kV];
        const int eight = g * 2 + k;
        const u32x4 x = *reinterpret_cast<const u32x4*>(lds + F::value_at(eight, 0, d * 16 + r));
        value_terms<T>(x, sizeof(T) == 4 ? *reinterpret_cast<const u32x4*>(lds + F::value_at(eight, 1, d * 16 + r)) : x, a);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int e = 0; e < W::kV; ++e)
#pragma unroll
            for (int f = 0; f < W::kW && f + e < W::kSum; ++f) st.o[rt][d] = mfma(a[e], w[rt][k][f], st.o[rt][d]);
        if constexpr (sizeof(T) == 4) __builtin_amdgcn_sched_barrier(0);
      }
  }
}

// Which part of the call a workgroup has.
struct Place {
  int64_t b;
  int h, rg, chunk, active;                // head, row group, chunk, and chunks of this sequence that hold anything
  int len, n_pages, there, rows;           // cached tokens and their pages, new tokens, rows of the head
  bool bad_length;
};
// False: there is nothing to do.  Workgroups go to the eight XCDs in turn; those that differ in their rows alone read the same pages: on one
// XCD, one after the other.
__device__ __forceinline__ bool place_of(const AttendParams& p, Place& at) {
  const uint32_t block = blockIdx.x, slot = block >> 3;
  const uint32_t unit = slot / uint32_t(p.row_groups) * 8 + (block & 7);
  if (unit >= uint64_t(p.B) * p.c.heads * p.chunks) return false;
  at.rg = int(slot % uint32_t(p.row_groups));
  at.chunk = int(unit % uint32_t(p.chunks));
  at.h = int(unit / uint32_t(p.chunks) % uint32_t(p.c.heads));
  at.b = int64_t(unit / (uint32_t(p.chunks) * uint32_t(p.c.heads)));
  at.len = cached_tokens(p.c, at.b, at.bad_length);
  at.n_pages = (at.len + kPage - 1) / kPage;
  at.active = max(1, (at.n_pages + p.chunk - 1) / p.chunk);
  at.there = p.count ? min(max(as_global(p.count)[at.b], 0), p.n) : p.n;
  at.rows = p.n * p.group;
  return at.chunk < at.active;
}
template <typename T, int D, int RT>
__device__ __forceinline__ void load_queries(const AttendParams& p, const Place& at, int first_row, Queries<T, D, RT>& q) {
  const int r = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = min(first_row + rt * 16 + r, at.rows - 1);
    const int64_t from = at.b * p.q.seq + int64_t(row / p.group) * p.q.token + int64_t(at.h * p.group + row % p.group) * p.q.head;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) Operand<T>::load(p.q.data, from + step_channel(i, g), q.v[rt][i]);
  }
}
template <int D, int RT> __device__ __forceinline__ void begin(RowState<D, RT>& st) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    st.m[rt] = kNoMax;
    st.l[rt] = 0;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) st.o[rt][d] = f32x4{0, 0, 0, 0};
  }
}
// Up to 64 entries of a sequence's table with the scales of their pages, one a lane: entries first, first + step, ...
struct PageList {
  int page;                                // -1: outside the cache
  float k_scale, v_scale;
  __device__ __forceinline__ bool load(const AttendParams& p, const Place& at, int first, int step, int some) {
    const int lane = lane_id();
    page = -1;
    k_scale = v_scale = 1.0f;
    if (lane < some) page = as_global(p.c.pages + at.b * p.c.width)[first + step * lane];
    const bool in = page >= 0 && page < p.c.n_pages;
    const bool bad = lane < some && !in;
    if (!in) page = -1;
    else {
      const float* sc = p.c.scales + (int64_t(page) * p.c.heads + at.h) * 2;
      k_scale = as_global(sc)[0];
      v_scale = as_global(sc)[1];
    }
    return bad;
  }
  __device__ __forceinline__ int page_at(int i) const { return __builtin_amdgcn_readlane(page, i); }
  __device__ __forceinline__ float k_at(int i) const { return as_f32(__builtin_amdgcn_readlane(as_u32(k_scale), i)); }
  __device__ __forceinline__ float v_at(int i) const { return as_f32(__builtin_amdgcn_readlane(as_u32(v_scale), i)); }
};

// A row's sums become its output (kLast: the sequence has no other chunk), or its part of it.  `from` channels on, four of them.
template <typename T, int D> __device__ __forceinline__ void give(const AttendParams& p, const Place& at, int row, int d, float m, float l, f32x4 o) {
  if (at.active > 1) {
    const int64_t part = ((at.b * p.c.heads + at.h) * p.chunks + at.chunk) * int64_t(at.rows) + row;
    if (d == 0) store_through(p.part_ml + part, uint64_t(as_u32(l)) << 32 | as_u32(m));
    store_through(p.part_o + part * (D / 2) + d / 2, uint64_t(as_u32(o[1])) << 32 | as_u32(o[0]));
    store_through(p.part_o + part * (D / 2) + d / 2 + 1, uint64_t(as_u32(o[3])) << 32 | as_u32(o[2]));
    return;
  }
  const int i = row / p.group;
  const bool none = i >= at.there || l == 0;
  const int64_t to = (at.b * p.n + i) * p.heads_q + at.h * p.group + row % p.group;
  if (d == 0) p.lse[to] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  store4<T>(p.out, to * D + d, none ? f32x4{0, 0, 0, 0} : o * (1.0f / l));
}

// Seen values that are not finite, to the rows that see them: a weight is positive, so that the sum becomes what they add up to alone.
// Called where there are such values, after the rows have been given without them.
template <typename T, int D, int NT, int kRows> __device__ __forceinline__ void add_odd_values(const AttendParams& p, const Place& at) {
  const uint32_t* mask = p.mask ? p.mask + at.b * p.mask_seq : nullptr;
  stores_arrived();
  __syncthreads();
#pragma unroll 1
  for (int idx = int(threadIdx.x); idx < kRows * (D / 2); idx += NT) {
    const int row = at.rg * kRows + idx / (D / 2), d = idx % (D / 2) * 2, i = row / p.group;
    if (row >= at.rows) break;
    float odd[2] = {0, 0};
    for (int j0 = 0; j0 < at.there; j0 += 16)
      for (uint32_t seen = seen_of(p, mask, i, j0, at.there); seen; seen &= seen - 1) {
        const T* from = reinterpret_cast<const T*>(p.v.data) + at.b * p.v.seq + at.h * p.v.head + (j0 + __builtin_ctz(seen)) * p.v.token;
        for (int e = 0; e < 2; ++e) {
          const float y = load_elem<T>(from, d + e);
          if (!__builtin_isfinite(y)) odd[e] += y;
        }
      }
    if (at.active > 1) {
      uint64_t* word = p.part_o + (((at.b * p.c.heads + at.h) * p.chunks + at.chunk) * int64_t(at.rows) + row) * (D / 2) + d / 2;
      const uint64_t x = load_through(word);
      store_through(word, uint64_t(as_u32(as_f32(uint32_t(x >> 32)) + odd[1])) << 32 | as_u32(as_f32(uint32_t(x)) + odd[0]));
    } else {
      const int64_t to = (at.b * p.n + i) * p.heads_q + at.h * p.group + row % p.group;
      for (int e = 0; e < 2; ++e)
        if (odd[e] != 0) {
          if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(p.out)[to * D + d + e] += odd[e];
          else reinterpret_cast<uint16_t*>(p.out)[to * D + d + e] = odd_bits<T>(odd[e]);
        }
    }
  }
}

// All threads of a workgroup that has given its rows: the last one of a sequence's chunks joins them, and says how the sequence's pages were.
template <typename T, int D, int NT, int kRows>
__device__ __forceinline__ void join_chunks(const AttendParams& p, Place at, bool bad, int& told) {
  const int tid = int(threadIdx.x);
  const bool speaks = p.status && at.h == 0 && at.rg == 0;
  if (at.active == 1) {
    if (!speaks) return;
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) p.status[at.b] = bad ? kBadPage : 0;
    return;
  }
  uint64_t* words = p.words + ((at.b * p.c.heads + at.h) * p.row_groups + at.rg) * int64_t(p.chunks);
  if (!all_arrived(words, at.chunk, at.active, p.tag, told)) return;
  if (wave_id() == 0) {
    const bool mine = claimed(words, at.active, p.tag);
    if (lane_id() == 0) told = mine ? 1 : 0;
  }
  __syncthreads();
  if (__builtin_amdgcn_readfirstlane(told) == 0) return;
  const int64_t part = (at.b * p.c.heads + at.h) * int64_t(p.chunks) * at.rows;
  const int chunks = at.active;
  at.active = 1;
  for (int idx = tid; idx < kRows * (D / 4); idx += NT) {
    const int row = at.rg * kRows + idx / (D / 4), d = idx % (D / 4) * 4;
    if (row >= at.rows) break;
    float m = kNoMax, l = 0;
    f32x4 o = {0, 0, 0, 0};
    for (int c0 = 0; c0 < chunks; c0 += 4) {             // four chunks' words asked for at a time
      uint64_t ml[4], x[4][2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t from = part + int64_t(min(c0 + u, chunks - 1)) * at.rows + row;
        ml[u] = load_through(p.part_ml + from);
        x[u][0] = load_through(p.part_o + from * (D / 2) + d / 2);
        x[u][1] = load_through(p.part_o + from * (D / 2) + d / 2 + 1);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (c0 + u < chunks) {
          const float mu = as_f32(uint32_t(ml[u])), most = fmaxf(m, mu);
          const float f = exp2_fast(m - most), fu = exp2_fast(mu - most);
          l = l * f + as_f32(uint32_t(ml[u] >> 32)) * fu;
          o = o * f + f32x4{as_f32(uint32_t(x[u][0])), as_f32(uint32_t(x[u][0] >> 32)), as_f32(uint32_t(x[u][1])), as_f32(uint32_t(x[u][1] >> 32))} * fu;
          m = most;
        }
    }
    give<T, D>(p, at, row, d, m, l, o);
  }
  if (speaks) {
    bad = at.bad_length;
    for (int i = tid; i < at.n_pages; i += NT) {
      const int page = as_global(p.c.pages + at.b * p.c.width)[i];
      bad |= page < 0 || page >= p.c.n_pages;
    }
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) p.status[at.b] = bad ? kBadPage : 0;
  }
}

template <typename T, int D, int RT, int KS> constexpr int stream_lds_bytes(bool fresh) {
  const int join = KS == 1 ? 0 : KS * 16 * RT * (4 / KS) * (D + 4) * 4, staged = fresh ? Fresh<T, D>::kLds : 0;
  return join > staged ? join : staged;
}

// Few rows.  KS of a workgroup's four waves share rows and take turns at the pages, 4 / KS have rows of their own.
template <typename T, int D, int RT, int KS>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend_stream_kernel(const AttendParams p) {
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ FreshShared sh;
  __shared__ float2 join_ml[KS][4 / KS * 16 * RT];
  __shared__ int told;
  constexpr int RS = 4 / KS, kRows = RS * 16 * RT;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  const int wave_k = wave % KS, wave_r = wave / KS;
  Place at;
  if (!place_of(p, at)) return;
  const int first_row = at.rg * kRows + wave_r * 16 * RT;
  Queries<T, D, RT> q;
  load_queries<T, D, RT>(p, at, first_row, q);
  RowState<D, RT> st;
  begin(st);

  const int from = at.chunk * p.chunk + wave_k, to = min((at.chunk + 1) * p.chunk, at.n_pages);
  const int turns = from < to ? (to - from + KS - 1) / KS : 0;
  bool bad = at.bad_length;
  for (int base = 0; base < turns; base += 64) {
    const int some = min(64, turns - base);
    PageList list;
    bad |= list.load(p, at, from + KS * base, KS, some);
    KeyTile<D> kt;
    ValueTile<D> vt;
    const uint8_t* codes = page_codes(p.c, max(0, list.page_at(0)), at.h, D);
    kt.load(codes, lane);
    vt.load(codes + kPage * D, lane);
    for (int i = 0; i < some; ++i) {
      const int valid = list.page_at(i) < 0 ? 0 : min(kPage, at.len - (from + KS * (base + i)) * kPage);
      f32x4 s[RT][4];
      key_products<T, D, RT>(kt, q, s);
      const uint8_t* next = page_codes(p.c, max(0, list.page_at(min(i + 1, some - 1))), at.h, D);
      if (i + 1 < some) kt.load(next, lane);
      bf16x8 w[RT][2][Terms<T>::kW];
      page_weights<T, D, RT>(s, st, p.scale2 * list.k_at(i), valid, g, w);
      if (valid < kPage) vt.cut(valid - g * 16);
      page_values(vt, w, st, list.v_at(i));
      if (i + 1 < some) vt.load(next + kPage * D, lane);
    }
  }
  const bool fresh = at.chunk == at.active - 1 && p.k.data && at.there > 0;
  if (fresh) {
    if (tid == 0) sh.wanted[0] = sh.wanted[1] = sh.odd = 0;
    __syncthreads();
    attend_fresh<T, D, RT, KS, 256>(p, at.b, at.h, first_row, min(at.rows, (at.rg + 1) * kRows) - 1, at.there, wave_k, q, st, lds, sh);
  }

  // Lane 16 g + r has its row's maximum, its group's part of the sum of weights, and its channels.
  if constexpr (KS == 1) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + rt * 16 + r;
      const float l = over_groups_sum(st.l[rt]);
      if (row >= at.rows) continue;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) give<T, D>(p, at, row, d * 16 + g * 4, st.m[rt], l, st.o[rt][d]);
    }
  } else {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float l = over_groups_sum(st.l[rt]);
      if (g == 0) join_ml[wave_k][wave_r * 16 * RT + rt * 16 + r] = make_float2(st.m[rt], l);
    }
    __syncthreads();                       // (also: what was staged of new tokens has been read)
    float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = wave_r * 16 * RT + rt * 16 + r;
      float m = st.m[rt];
#pragma unroll
      for (int k = 0; k < KS; ++k) m = fmaxf(m, join_ml[k][row].x);
      const float f = exp2_fast(st.m[rt] - m);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(sums + (wave_k * kRows + row) * (D + 4) + d * 16 + g * 4) = st.o[rt][d] * f;
    }
    __syncthreads();
    for (int idx = tid; idx < kRows * (D / 4); idx += 256) {
      const int local = idx / (D / 4), d = idx % (D / 4) * 4, row = at.rg * kRows + local;
      if (row >= at.rows) break;
      float m = kNoMax, l = 0;
#pragma unroll
      for (int k = 0; k < KS; ++k) m = fmaxf(m, join_ml[k][local].x);
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        l += join_ml[k][local].y * exp2_fast(join_ml[k][local].x - m);
        o += *reinterpret_cast<const f32x4*>(sums + (k * kRows + local) * (D + 4) + d);
      }
      give<T, D>(p, at, row, d, m, l, o);
    }
  }
  if (fresh && sh.odd) add_odd_values<T, D, 256, kRows>(p, at);
  join_chunks<T, D, 256, kRows>(p, at, bad, told);
}

// A page as operands in LDS: 16 bits a number, in the order of Fresh.  Bytes of one of the two that take turns.
template <int D> constexpr int page_lds_bytes() { return 2 * kPage * D * 2; }
template <typename T, int D> constexpr int rows_lds_bytes(bool fresh) {
  return 2 * page_lds_bytes<D>() > (fresh ? Fresh<T, D>::kLds : 0) ? 2 * page_lds_bytes<D>() : Fresh<T, D>::kLds;
}

// Many rows: NW waves with RT tiles of rows each.
template <typename T, int D, int RT, int NW>
__global__ __launch_bounds__(NW * 64, D == 256 && NW == 4 ? 1 : 2) void attend_rows_kernel(const AttendParams p) {
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ FreshShared sh;
  __shared__ int told;
  typedef Fresh<Bf16, D> F;                // (places in a tile of 16 bits)
  constexpr int NT = NW * 64, kRows = NW * 16 * RT, kLoads = kPage * D / 16 / NT;
  static_assert(kPage * D / 16 % NT == 0, "every thread has as many pieces of a page");
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  Place at;
  if (!place_of(p, at)) return;
  const int first_row = at.rg * kRows + wave * 16 * RT;
  Queries<T, D, RT> q;
  load_queries<T, D, RT>(p, at, first_row, q);
  RowState<D, RT> st;
  begin(st);

  const int from = at.chunk * p.chunk, to = min((at.chunk + 1) * p.chunk, at.n_pages);
  const int turns = max(0, to - from);
  bool bad = at.bad_length;
  for (int base = 0; base < turns; base += 64) {
    const int some = min(64, turns - base);
    PageList list;
    bad |= list.load(p, at, from + base, 1, some);
    u32x4 kw[kLoads], vw[kLoads];
    const uint8_t* codes = page_codes(p.c, max(0, list.page_at(0)), at.h, D);
#pragma unroll
    for (int it = 0; it < kLoads; ++it) {
      kw[it] = load16(codes + (it * NT + tid) * 16);
      vw[it] = load16(codes + kPage * D + (it * NT + tid) * 16);
    }
    for (int i = 0; i < some; ++i) {
      const int valid = list.page_at(i) < 0 ? 0 : min(kPage, at.len - (from + base + i) * kPage);
      uint8_t* tile = lds + (i & 1) * page_lds_bytes<D>();
      const float v_scale = list.v_at(i);
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        const int idx = it * NT + tid, key = idx / (D / 16), chunk = idx % (D / 16) * 2;
        *reinterpret_cast<u32x4*>(tile + F::key_at(chunk, key)) = __builtin_bit_cast(u32x4, Operand<T>::codes(kw[it][0], kw[it][1]));
        *reinterpret_cast<u32x4*>(tile + F::key_at(chunk + 1, key)) = __builtin_bit_cast(u32x4, Operand<T>::codes(kw[it][2], kw[it][3]));
        const int d = idx % D, eight = idx / D * 2;
        if (valid < kPage) vw[it] &= tokens_below(valid - eight * 8);
        *reinterpret_cast<u32x4*>(tile + F::value_at(eight, 0, d)) = __builtin_bit_cast(u32x4, codes_as_bf16(vw[it][0], vw[it][1], v_scale));
        *reinterpret_cast<u32x4*>(tile + F::value_at(eight + 1, 0, d)) = __builtin_bit_cast(u32x4, codes_as_bf16(vw[it][2], vw[it][3], v_scale));
      }
      if (i + 1 < some) {
        const uint8_t* next = page_codes(p.c, max(0, list.page_at(i + 1)), at.h, D);
#pragma unroll
        for (int it = 0; it < kLoads; ++it) {
          kw[it] = load16(next + (it * NT + tid) * 16);
          vw[it] = load16(next + kPage * D + (it * NT + tid) * 16);
        }
      }
      // (one barrier a page: whoever writes a tile again has passed the barrier that all reach after reading it)
      __syncthreads();
      if (first_row >= at.rows) continue;
      f32x4 s[RT][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0, 0, 0, 0};
        const int token = (r >> 2) * 16 + t * 4 + (r & 3);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          const auto a = __builtin_bit_cast(typename Operand<T>::Vec, *reinterpret_cast<const u32x4*>(tile + F::key_at(step_channel(j, g) / 8, token)));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int e = 0; e < Operand<T>::kTerms; ++e) s[rt][t] = mfma(a, q.v[rt][j][e], s[rt][t]);
        }
      }
      bf16x8 w[RT][2][Terms<T>::kW];
      page_weights<T, D, RT>(s, st, p.scale2 * list.k_at(i), valid, g, w);
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const auto a = *reinterpret_cast<const bf16x8*>(tile + F::value_at(g * 2 + k, 0, d * 16 + r));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int e = 0; e < Terms<T>::kW; ++e) st.o[rt][d] = mfma(a, w[rt][k][e], st.o[rt][d]);
        }
    }
    __syncthreads();                       // (the next list's first page, or a tile of new tokens, goes where this one's last ones are)
  }
  const bool fresh = at.chunk == at.active - 1 && p.k.data && at.there > 0;
  if (fresh) {
    if (tid == 0) sh.wanted[0] = sh.wanted[1] = sh.odd = 0;
    __syncthreads();
    attend_fresh<T, D, RT, 1, NT>(p, at.b, at.h, first_row, min(at.rows, (at.rg + 1) * kRows) - 1, at.there, 0, q, st, lds, sh);
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = first_row + rt * 16 + r;
    const float l = over_groups_sum(st.l[rt]);
    if (row >= at.rows) continue;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) give<T, D>(p, at, row, d * 16 + g * 4, st.m[rt], l, st.o[rt][d]);
  }
  if (fresh && sh.odd) add_odd_values<T, D, NT, kRows>(p, at);
  join_chunks<T, D, NT, kRows>(p, at, bad, told);
}

// The shapes of a type and head size: tiles of rows to a wave, so that nothing spills (two waves to a SIMD: 256 registers).
template <typename T, int D> struct AttendShapes { static constexpr int kRT = D == 64 || (sizeof(T) == 2 && D == 128) ? 2 : 1; };
// The launches, for each type of the call in a source file of its own (attend_launch.h, attend_*.hip).
template <typename T> hipError_t launch_attend(const AttendParams& p, int D, hipStream_t s);
// Which kernel `rows` that share a head go to, and the rows that one workgroup takes.
enum AttendKind { kStreamOne, kStreamTall, kStreamTwo, kRowsFour, kRowsEight };
struct AttendChoice { AttendKind kind; int rows; };
inline AttendChoice attend_choice(bool f32, int D, int64_t rows) {
  const bool tall = D == 64 || (!f32 && D == 128);      // two tiles of rows to a wave
  if (rows <= 16) return {kStreamOne, 16};
  if (tall && rows <= 32) return {kStreamTall, 32};
  if (rows <= (tall ? 64 : 32)) return {kStreamTwo, tall ? 64 : 32};
  if (tall) return {kRowsFour, 128};
  return rows <= 64 || (f32 && D == 256) ? AttendChoice{kRowsFour, 64} : AttendChoice{kRowsEight, 128};
}

}  // namespace tslt
