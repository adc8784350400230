// Attention of a round's new tokens over the 8-bit cache and over each other (tslt_cache_attend).
//
//   s_ij = scale * q_i . k_j,  out_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = ln sum_j exp(s_ij)
//
// j runs over the cached tokens, all of which every query sees, and over those of the call's own tokens that its mask shows.
// A row is one query head of one token; the rows of one sequence that share a key/value head, n * group of them, meet the same
// keys, so the products are dense in tiles of 16 rows, and one pass keeps a running maximum m and sum l for each row.
//
// One wave takes 64 keys at a time against tiles of 16 rows (see Tile), in two kernels:
//   attend_stream_kernel, few rows: bound by memory (4 sequences of 131000 tokens, 8 heads of 128, 4 rows: 174 us, 1029 MB at 5.9 TB/s; a large read runs at 7.0).  Codes go from memory straight into the operand registers of the products (the
//     order in which the cache holds them is made for that).  A workgroup's four waves have the same rows and take pages in turn.
//   attend_rows_kernel, many rows: bound by the products and the exponentials.  A workgroup brings a page to LDS once, as operands, for
//     all of its waves, each with rows of its own (2048 bfloat16 tokens on 16000, 32 heads of 128 on 8: 800 us, 571 GFLOP by the formula at 714
//     TFLOP/s, 1071 with the weights' second term; a large matrix product runs at 1200.  It is 3.6 vector instructions a product that keep it from that).
// A sequence is cut into chunks of pages where its rows alone do not fill the GPU; whichever of its workgroups ends last joins them.
//
// Rounding.  Codes, and queries of 16 bits, enter the first product exactly; queries of 32 bits as three bfloat16 terms,
// exactly.  Sums are fp32.  A weight enters the second product as the sum of two bfloat16 terms, 16 bits, and of three, 24, in fp32
// calls; values enter it as bfloat16 times their page's scale, exactly.  (One bfloat16 term would be off by 2^-9, as much as the output's
// own rounding; one binary16 term by 2^-12, but it loses weights below 2^-30 of the largest, and where that one's value is 0 they are the result.)
// The running maximum is followed only when a row exceeds it by kLag powers of two: weights, in units of it, stay below 2^kLag.  Sums of values are in
// units of 2^16, so that many weights that are not small yet and values near fp32's largest do not pass it before they are divided by the weights' sum:
// 65536 of them do where weights are 1, 256 where they are 2^kLag.  (A page's scale takes that in for nothing, exactly; of new tokens the weights do.)
#pragma once
#include "cache.h"
#include "handover.h"

namespace tslt {

constexpr float kLag = 8.0f;
constexpr float kUnit = 65536.0f;          // of sums of values
constexpr float kNoMax = -3.4028235e38f;   // running maximum of a row that has met nothing yet
// Scores (as powers of two) beyond which the maximum's own rounding, which a fused multiplication and subtraction does not share, is as much as a factor of
// 2 on a weight: there scores are rounded first, as the maximum is, so that the weight of its token is 1 (and not 0 or infinite from 2^31 on).
constexpr float kLarge = 16777216.0f;

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

// 64 tokens in LDS.  16 bytes of keys are kPer channels of one token.  A chunk's tokens lie in the order in which the lanes of a product read them,
// that exclusive-or a number of the chunk, so that of neither eight lanes that read a chunk of eight tokens nor eight that write eight chunks, or every
// other of sixteen, of one token two meet in a bank.  16 bytes of values are kPer tokens of one channel.
template <typename T, int D> struct Staged {
  static constexpr int kBytes = sizeof(T), kPer = 16 / kBytes;
  static constexpr int kKeyBytes = kPage * D * kBytes;
  static constexpr int kLds = 2 * kKeyBytes;
  static __device__ __forceinline__ int key_at(int chunk, int place) { return (chunk * kPage + (place ^ ((chunk & 7) ^ (chunk >> 3 & 1)))) * 16; }
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

// 64 new tokens from j0 on, on their way from memory to LDS in the registers of NT threads; zeros where there are fewer.  A value that is not finite is left out (0), and
// that it was noted: a product would carry it to rows that do not see the token, as 0 times it (see add_odd_values).
template <typename T, int D, int NT, bool kHold> struct FreshTile {
  typedef Staged<T, D> F;
  static constexpr int kWide = F::kBytes == 4 ? 1 : 2;   // channels of a value to a thread: a word
  static constexpr int kChunks = D / F::kPer, kKeys = kPage * kChunks / NT, kValues = (8 * (D / kWide) + NT - 1) / NT;
  static constexpr bool kAll = 8 * (D / kWide) % NT == 0;
  // 16 bits, many rows: the next tile is asked for before this one is met (46 sequences, 8 heads of 128, 319 tokens on some 30: 128 us without, 89 so).  fp32, whose rows and
  // terms leave no registers, and few rows, which seldom have a second tile: read when it is put there, a few at a time.
  static constexpr bool kHeld = kHold && F::kBytes == 2;
  u32x4 k[kHeld ? kKeys : 1];
  uint32_t v[kHeld ? kValues : 1][8];
  __device__ __forceinline__ static u32x4 keys(const AttendParams& p, int64_t b, int h, int j0, int there, int it) {
    const int idx = it * NT + int(threadIdx.x), chunk = idx % kChunks, token = idx / kChunks;
    return load16(reinterpret_cast<const T*>(p.k.data) + b * p.k.seq + h * p.k.head + min(j0 + token, there - 1) * p.k.token + chunk * F::kPer);
  }
  __device__ __forceinline__ static void values(const AttendParams& p, int64_t b, int h, int j0, int there, int it, uint32_t (&w)[8]) {
    const int idx = it * NT + int(threadIdx.x), at = idx % (D / kWide), eight = idx / (D / kWide) & 7;
    const T* vp = reinterpret_cast<const T*>(p.v.data) + b * p.v.seq + h * p.v.head;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = *as_global(reinterpret_cast<const uint32_t*>(vp + min(j0 + eight * 8 + e, there - 1) * p.v.token + at * kWide));
  }
  __device__ __forceinline__ void load(const AttendParams& p, int64_t b, int h, int j0, int there) {
    if constexpr (kHeld) {
#pragma unroll
      for (int it = 0; it < kKeys; ++it) k[it] = keys(p, b, h, j0, there, it);
#pragma unroll
      for (int it = 0; it < kValues; ++it) values(p, b, h, j0, there, it, v[it]);
    }
  }
  __device__ __forceinline__ void put(const AttendParams& p, int64_t b, int h, int j0, int there, uint8_t* lds, FreshShared& sh) const {
    const int tid = int(threadIdx.x);
    constexpr int kKeysAtOnce = kHeld ? kKeys : 4, kValuesAtOnce = kHeld ? kValues : 2;
#pragma unroll kKeysAtOnce
    for (int it = 0; it < kKeys; ++it) {
      const int idx = it * NT + tid, chunk = idx % kChunks, token = idx / kChunks;
      u32x4 w;
      if constexpr (kHeld) w = k[it];
      else w = keys(p, b, h, j0, there, it);
      *reinterpret_cast<u32x4*>(lds + F::key_at(chunk, Tile::place(token))) = j0 + token < there ? w : u32x4{0, 0, 0, 0};
    }
    bool odd = false;
#pragma unroll kValuesAtOnce
    for (int it = 0; it < kValues; ++it) {
      const int idx = it * NT + tid, at = idx % (D / kWide), eight = idx / (D / kWide);
      if (!kAll && eight >= 8) continue;
      uint32_t w[8];
      if constexpr (!kHeld) values(p, b, h, j0, there, it, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (kHeld) w[e] = v[it][e];
        if (j0 + eight * 8 + e >= there) w[e] = 0;
        if (not_finite<T>(w[e])) { odd = true; w[e] = kWide == 1 ? 0 : w[e] & 0xFFFF0000u; }
        if (kWide == 2 && not_finite<T>(w[e] >> 16)) { odd = true; w[e] &= 0xFFFFu; }
      }
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
    if (odd) sh.odd = 1;
  }
};

// What a wave keeps for its rows: of row r of each tile the running maximum, the lane's part of the sum of weights, and of channels 16 d + 4 g .. + 3 the sums.
template <int D, int RT> struct RowState {
  f32x4 o[RT][D / 16];
  float m[RT], l[RT];
  bool large;                              // of all lanes: a maximum has been beyond kLarge
};
template <int D, int RT> __device__ __forceinline__ void begin(RowState<D, RT>& st) {
  st.large = false;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    st.m[rt] = kNoMax;
    st.l[rt] = 0;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) st.o[rt][d] = f32x4{0, 0, 0, 0};
  }
}
// The running maximum follows where a row of the tile exceeds it by more than kLag.
template <int D, int RT> __device__ __forceinline__ void follow(RowState<D, RT>& st, int rt, float most) {
  if (ballot(most > st.m[rt] + kLag) == 0) return;
  const float m = over_groups_max(fmaxf(most, st.m[rt]));
  st.large |= ballot(fabsf(m) > kLarge) != 0;
  const float f = exp2_fast(st.m[rt] - m);
  st.m[rt] = m;
  st.l[rt] *= f;
#pragma unroll
  for (int d = 0; d < D / 16; ++d) st.o[rt][d] *= f;
}
__device__ __forceinline__ float most_of(const f32x4 (&s)[4]) {
  float most = s[0][0];
#pragma unroll
  for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i >> 2][i & 3]);
  return most;
}
// A page's scores without those of tokens from `there` on, which do not count, and the maximum.  Returns what a score is to be multiplied by.
template <int D, int RT> __device__ __forceinline__ float page_maximum(f32x4 (&s)[RT][4], RowState<D, RT>& st, float c, int there, int g) {
  if (there < kPage) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (g * 16 + i >= there) s[rt][i >> 2][i & 3] = -INFINITY;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) follow(st, rt, most_of(s[rt]) * c);
  if (!st.large) return c;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int t = 0; t < 4; ++t) s[rt][t] *= c;
  return 1.0f;
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

// 64 tokens' values in a wave: of channel 16 d + r the lane's 16 tokens.
template <int D> struct ValueTile {
  u32x4 w[D / 16];
  __device__ __forceinline__ void load(const uint8_t* values, int lane) {
    const uint8_t* p = values + (lane >> 4) * 16 * D + (lane & 15) * 16;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) w[d] = load16_once(p + d * 256);
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

// Vector instructions and matrix products stay in the order in which they are written down; memory's may move.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x3F4); }

// f(kFrom), f(kFrom + 1) .. f(kTo - 1), written out by a few at a time: the compiler gives up on a loop of many, and indexes registers by numbers that it does not
// know (fp32, D = 256, 700 tokens of 4 sequences on 100 to 900, 16 heads on 4: 6750 us so, 420 written out).
template <int kFrom, int kTo, typename F> __device__ __forceinline__ void in_parts(const F& f) {
#pragma unroll
  for (int n = kFrom; n < (kTo < kFrom + 16 ? kTo : kFrom + 16); ++n) f(n);
  if constexpr (kTo > kFrom + 16) in_parts<kFrom + 16, kTo>(f);
}
// A page's scores into weights, these and its values into the rows' sums, and beside that, the scores of the page after it, so that the products
// run while the exponentials are made.  keys(t, i): operand of instruction t and step i of the next page; values(d, k): of this page's channels 16 d ..
// and the k-th eight of the lane's 16 tokens; each is asked for kAhead operands before it is met.  The order is written out: a product, then a
// weight or none.  (A product leaves room for two vector instructions beside it: measured, two waves to a SIMD, 18.2 cycles alone, 20.6 with
// two, 23.9 with three, 30.6 with four.)
template <int kAhead, typename T, int D, int RT, typename Keys, typename Values>
__device__ __forceinline__ void page_round(const Queries<T, D, RT>& q, f32x4 (&s)[RT][4], RowState<D, RT>& st, float c, const Keys& keys, const Values& values) {
  constexpr int kTerms = Operand<T>::kTerms, kW = Terms<T>::kW, kRing = kAhead + 1;
  constexpr int kKeys = D / 32 * 4, kScores = kKeys * kTerms * RT;         // operands, and products with them
  constexpr int kHalf = D / 16, kValues = kHalf * kW * RT;                 // the same of half a page's values
  constexpr int kElements = 8 * RT;                                        // weights of half a page, a lane
  static_assert(kElements <= kScores && kElements <= kValues, "a weight to a product at most");
  f32x4 next[RT][4];
  bf16x8 w[RT][2][kW];
  float sum[RT] = {};                      // (a page's weights by themselves: a long sequence's sum takes an addition a page, not sixteen)
  const auto weight = [&](int k, int n) {
    const int rt = n >> 3, e = n & 7;
    const float x = exp2_fast(__builtin_fmaf(s[rt][2 * k + (e >> 2)][e & 3], c, -st.m[rt]));
    sum[rt] += x;
    split_weight(x, e, w[rt][k]);
  };
  typename Operand<T>::Vec key[kRing];
  bf16x8 value[kRing];
  const auto ask = [&](int f) {
    if (f < kKeys) key[f % kRing] = keys(f % 4, f / 4);
    else if (f < kKeys + 2 * kHalf) value[(f - kKeys) % kRing] = values((f - kKeys) % kHalf, (f - kKeys) / kHalf);
  };
#pragma unroll
  for (int f = 0; f < kAhead; ++f) ask(f);
  in_parts<0, kScores>([&](int n) __attribute__((always_inline)) {
    const int rt = n % RT, e = n / RT % kTerms, f = n / (RT * kTerms), t = f % 4, i = f / 4;
    if (n % (RT * kTerms) == 0) ask(f + kAhead);
    next[rt][t] = mfma(key[f % kRing], q.v[rt][i][e], i == 0 && e == 0 ? f32x4{0, 0, 0, 0} : next[rt][t]);
    if ((n + 1) * kElements / kScores > n * kElements / kScores) weight(0, n * kElements / kScores);
    keep_order();
  });
  in_parts<0, 2 * kValues>([&](int n) __attribute__((always_inline)) {
    const int k = n / kValues, rt = n % RT, e = n / RT % kW, f = n / (RT * kW), d = f % kHalf;
    if (n % (RT * kW) == 0) ask(kKeys + f + kAhead);
    st.o[rt][d] = mfma(value[f % kRing], w[rt][k][e], st.o[rt][d]);
    if (k == 0 && (n + 1) * kElements / kValues > n * kElements / kValues) weight(1, n * kElements / kValues);
    keep_order();
  });
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    st.l[rt] += sum[rt];
#pragma unroll
    for (int t = 0; t < 4; ++t) s[rt][t] = next[rt][t];
  }
}
// The same for the kernel whose waves read operands of their own: a page's weights, times `unit` for its values, then these.
template <typename T, int D, int RT>
__device__ __forceinline__ void page_weights(const f32x4 (&s)[RT][4], RowState<D, RT>& st, float c, float unit, bf16x8 (&w)[RT][2][Terms<T>::kW]) {
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float sum = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = exp2_fast(__builtin_fmaf(s[rt][i >> 2][i & 3], c, -st.m[rt]));
      sum += x;
      split_weight(x * unit, i & 7, w[rt][i >> 3]);
    }
    st.l[rt] += sum;
  }
}
template <int D, int RT, int W>
__device__ __forceinline__ void page_values(const ValueTile<D>& v, const bf16x8 (&w)[RT][2][W], RowState<D, RT>& st, float scale) {
#pragma unroll
  for (int d = 0; d < D / 16; ++d)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const bf16x8 a = codes_as_bf16(v.w[d][2 * k], v.w[d][2 * k + 1], scale);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < W; ++e) st.o[rt][d] = mfma(a, w[rt][k][e], st.o[rt][d]);
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

// The call's own tokens, all of them that the wave's rows see, tile after tile; `turns` waves that share rows take turns.
template <typename T, int D, int RT, int NT, bool kHold>
__device__ __forceinline__ void attend_fresh(const AttendParams& p, int64_t b, int h, int first_row, int last_row, int there, int turns, int my_turn,
                                             const Queries<T, D, RT>& q, RowState<D, RT>& st, uint8_t* lds, FreshShared& sh) {
  typedef Staged<T, D> F;
  typedef Terms<T> W;
  const int lane = lane_id(), r = lane & 15, g = lane >> 4;
  const uint32_t* mask = p.mask ? p.mask + b * p.mask_seq : nullptr;
  // (a token sees none behind itself where there is no mask: tiles behind the workgroup's last row's token are not looked at)
  const int reach = mask ? there : min(there, last_row / p.group + 1);
  FreshTile<T, D, NT, kHold> tile;
  tile.load(p, b, h, 0, there);
  for (int j0 = 0, turn = 0; j0 < reach; j0 += kPage, ++turn) {
    uint32_t seen[RT];                     // (a bit to each of the lane's scores)
    bool mine = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      seen[rt] = seen_of(p, mask, (first_row + rt * 16 + r) / p.group, j0 + g * 16, there);
      mine |= seen[rt] != 0;
    }
    const bool any = ballot(mine) != 0;
    if (any && lane == 0) sh.wanted[turn & 1] = turn + 1;
    __syncthreads();                       // (also: what was staged before has been read)
    const bool wanted = sh.wanted[turn & 1] == turn + 1;
    if (wanted) tile.put(p, b, h, j0, there, lds, sh);
    if (j0 + kPage < reach) tile.load(p, b, h, j0 + kPage, there);
    if (!wanted) continue;
    __syncthreads();
    if (!any || turn % turns != my_turn) continue;
    f32x4 s[RT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const int chunk = Tile::channel(i, g) / F::kPer, place = t * 16 + r;
        typename Operand<T>::Vec a[Operand<T>::kTerms];
        const u32x4 x = *reinterpret_cast<const u32x4*>(lds + F::key_at(chunk, place));
        if constexpr (sizeof(T) == 4) Operand<float>::split(x, *reinterpret_cast<const u32x4*>(lds + F::key_at(chunk + 1, place)), a);
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
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[rt][i >> 2][i & 3] = (seen[rt] >> i & 1) ? s[rt][i >> 2][i & 3] * p.scale2 : -INFINITY;
      follow(st, rt, most_of(s[rt]));
    }
    bf16x8 w[RT][2][W::kW];
    page_weights<T, D, RT>(s, st, 1.0f, 1.0f / kUnit, w);
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
  bool bad_length, none;                   // none: there is nothing to do
};
// What its number alone says.  Workgroups go to the eight XCDs in turn; those that differ in their rows alone read the same pages: on one
// XCD, one after the other, those of the last rows first, which see most of the new tokens.  A sequence's last chunk, which has the new tokens, comes first.
__device__ __forceinline__ Place place_of(const AttendParams& p) {
  Place at{};
  const uint32_t block = blockIdx.x, slot = block >> 3;
  const uint32_t unit = slot / uint32_t(p.row_groups) * 8 + (block & 7), heads = uint32_t(p.B * p.c.heads);
  at.none = unit >= uint64_t(heads) * p.chunks;
  at.rg = p.row_groups - 1 - int(slot % uint32_t(p.row_groups));
  at.h = int(unit % heads % uint32_t(p.c.heads));
  at.b = int64_t(unit % heads / uint32_t(p.c.heads));
  at.rows = p.n * p.group;
  at.chunk = int(unit / heads);            // (from the last one on, until the length is known)
  return at;
}
// The rest; false: the sequence has no such chunk.  What does not depend on lengths is asked for before this.
__device__ __forceinline__ bool place_in_sequence(const AttendParams& p, Place& at) {
  at.len = cached_tokens(p.c, at.b, at.bad_length);
  at.n_pages = (at.len + kPage - 1) / kPage;
  at.active = max(1, (at.n_pages + p.chunk - 1) / p.chunk);
  at.there = counted(p.count, at.b, p.n);
  at.chunk = at.active - 1 - at.chunk;
  return at.chunk >= 0;
}
template <typename T, int D, int RT> __device__ __forceinline__ void load_queries(const AttendParams& p, const Place& at, int first_row, Queries<T, D, RT>& q) {
  const int r = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = min(first_row + rt * 16 + r, at.rows - 1);
    const int64_t from = at.b * p.q.seq + int64_t(row / p.group) * p.q.token + int64_t(at.h * p.group + row % p.group) * p.q.head;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) Operand<T>::load(p.q.data, from + Tile::channel(i, g), q.v[rt][i]);
  }
}
// Up to 64 entries of a sequence's table with the scales of their pages, one a lane: entries first, first + step, ...
struct PageList {
  int page;                                // -1: outside the cache
  float k_scale, v_scale;                  // (for sums in units of kUnit)
  __device__ __forceinline__ void ask(const AttendParams& p, const Place& at, int first, int step, int some) {
    page = -1;
    if (lane_id() < some) page = as_global(p.c.pages + at.b * p.c.width)[first + step * lane_id()];
  }
  // Returns whether any is outside the cache; `asked`: ask() has been called, for these entries and perhaps ones behind them.
  __device__ __forceinline__ bool load(const AttendParams& p, const Place& at, int first, int step, int some, bool asked) {
    const int lane = lane_id();
    if (!asked) ask(p, at, first, step, some);
    if (lane >= some) page = -1;
    k_scale = v_scale = 1.0f;
    const bool in = page >= 0 && page < p.c.n_pages;
    const bool bad = lane < some && !in;
    if (!in) page = -1;
    else {
      const float* sc = p.c.scales + (int64_t(page) * p.c.heads + at.h) * 2;
      k_scale = as_global(sc)[0];
      v_scale = as_global(sc)[1] * (1.0f / kUnit);
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
  store4<T>(p.out, to * D + d, none ? f32x4{0, 0, 0, 0} : o * (kUnit / l));
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
          // (a row that is NaN without them stays NaN)
          if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(p.out)[to * D + d + e] += odd[e];
          else if (!__builtin_isnan(load_elem<T>(reinterpret_cast<const T*>(p.out), to * D + d + e))) reinterpret_cast<uint16_t*>(p.out)[to * D + d + e] = odd_bits<T>(odd[e]);
        }
    }
  }
}

// A chunk's maximum to another's units.  A weight is positive, however small: never 0, so that a sum which a chunk's seen values have made infinite stays so.
__device__ __forceinline__ float in_units(float x) { return fmaxf(exp2_fast(x), 1.4012985e-45f); }

// All threads of a workgroup that has given its rows: the last one of a sequence's chunks joins them, and says how the sequence's pages were.
template <typename T, int D, int NT, int kRows>
__device__ __forceinline__ void join_chunks(const AttendParams& p, Place at, bool bad, int (&told)[2]) {
  const int tid = int(threadIdx.x);
  const bool speaks = p.status && at.h == 0 && at.rg == 0;
  if (at.active == 1) {
    if (!speaks) return;
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) p.status[at.b] = sequence_status(p.count, at.b, p.n, bad);
    return;
  }
  uint64_t* words = p.words + ((at.b * p.c.heads + at.h) * p.row_groups + at.rg) * int64_t(p.chunks);
  if (!all_arrived(words, at.chunk, at.active, p.tag, told[0])) return;
  if (wave_id() == 0) {
    const bool mine = claimed(words, at.active, p.tag);
    if (lane_id() == 0) told[1] = mine ? 1 : 0;
  }
  __syncthreads();
  if (__builtin_amdgcn_readfirstlane(told[1]) == 0) return;
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
          const float f = in_units(m - most), fu = in_units(mu - most);
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
    if (tid == 0) p.status[at.b] = sequence_status(p.count, at.b, p.n, bad);
  }
}

constexpr int kStreamTurns = 4;            // waves of a workgroup that take pages in turn
// Most tiles of 16 rows that a wave has registers for with two waves to a SIMD (one for D = 256).
template <typename T, int D> constexpr int stream_most_tiles() { return D == 64 || (D == 128 && sizeof(T) == 2) ? 2 : 1; }
template <typename T, int D, int RT> constexpr int stream_lds_bytes(bool fresh) {
  const int join = kStreamTurns * 16 * RT * (D + 4) * 4, staged = fresh ? Staged<T, D>::kLds : 0;
  return join > staged ? join : staged;
}

// Few rows.
template <typename T, int D, int RT>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend_stream_kernel(const AttendParams p) {
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ FreshShared sh;
  __shared__ float2 join_ml[kStreamTurns][16 * RT];
  __shared__ int told[2];
  constexpr int KS = kStreamTurns, kRows = 16 * RT;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  Place at = place_of(p);
  if (at.none) return;
  const int first_row = at.rg * kRows;
  Queries<T, D, RT> q;
  load_queries(p, at, first_row, q);
  // (a sequence in one chunk: the wave's first pages, as far as the table goes)
  const bool early = p.chunks == 1;
  PageList list;
  if (early) list.ask(p, at, wave, KS, int(min<int64_t>(64, (p.c.width - wave + KS - 1) / KS)));
  if (!place_in_sequence(p, at)) return;
  RowState<D, RT> st;
  begin(st);

  const int from = at.chunk * p.chunk + wave, to = min((at.chunk + 1) * p.chunk, at.n_pages);
  const int turns = from < to ? (to - from + KS - 1) / KS : 0;
  bool bad = at.bad_length;
  for (int base = 0; base < turns; base += 64) {
    const int some = min(64, turns - base);
    bad |= list.load(p, at, from + KS * base, KS, some, early && base == 0);
    KeyTile<D> kt;
    ValueTile<D> vt;
    const uint8_t* codes = page_codes(p.c, max(0, list.page_at(0)), at.h, D);
    kt.load(codes, lane);
    vt.load(codes + kPage * D, lane);
    for (int i = 0; i < some; ++i) {
      const int valid = list.page_at(i) < 0 ? 0 : min(kPage, at.len - (from + KS * (base + i)) * kPage);
      f32x4 s[RT][4];
      key_products(kt, q, s);
      const uint8_t* next = page_codes(p.c, max(0, list.page_at(min(i + 1, some - 1))), at.h, D);
      if (i + 1 < some) kt.load(next, lane);
      const float c = page_maximum(s, st, p.scale2 * list.k_at(i), valid, g);
      bf16x8 w[RT][2][Terms<T>::kW];
      page_weights<T, D, RT>(s, st, c, 1.0f, w);
      if (valid < kPage) vt.cut(valid - g * 16);
      page_values(vt, w, st, list.v_at(i));
      if (i + 1 < some) vt.load(next + kPage * D, lane);
    }
  }
  const bool fresh = at.chunk == at.active - 1 && p.k.data && at.there > 0;
  if (fresh) {
    if (tid == 0) sh.wanted[0] = sh.wanted[1] = sh.odd = 0;
    __syncthreads();
    attend_fresh<T, D, RT, 256, false>(p, at.b, at.h, first_row, min(at.rows, first_row + kRows) - 1, at.there, KS, wave, q, st, lds, sh);
  }

  // The waves' parts meet in LDS.
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = over_groups_sum(st.l[rt]);
    if (g == 0) join_ml[wave][rt * 16 + r] = make_float2(st.m[rt], l);
  }
  __syncthreads();                         // (also: what was staged of new tokens has been read)
  float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = rt * 16 + r;
    float m = st.m[rt];
#pragma unroll
    for (int k = 0; k < KS; ++k) m = fmaxf(m, join_ml[k][row].x);
    const float f = exp2_fast(st.m[rt] - m);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(sums + (wave * kRows + row) * (D + 4) + d * 16 + g * 4) = st.o[rt][d] * f;
  }
  __syncthreads();
  for (int idx = tid; idx < kRows * (D / 4); idx += 256) {
    const int local = idx / (D / 4), d = idx % (D / 4) * 4, row = first_row + local;
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
  if (fresh && sh.odd) add_odd_values<T, D, 256, kRows>(p, at);
  join_chunks<T, D, 256, kRows>(p, at, bad, told);
}

// A page as operands in LDS: 16 bits a number.  Bytes of one of the two that take turns.
template <int D> constexpr int page_lds_bytes() { return 2 * kPage * D * 2; }
template <typename T, int D> constexpr int rows_lds_bytes(bool fresh) {
  return 2 * page_lds_bytes<D>() > (fresh ? Staged<T, D>::kLds : 0) ? 2 * page_lds_bytes<D>() : Staged<T, D>::kLds;
}
// Many rows: NW waves with RT tiles of rows each; kDeep pages on their way from memory, kAhead operands from LDS.
template <typename T, int D, int RT, int NW, int kDeep, int kAhead>
__global__ __launch_bounds__(NW * 64, D == 256 && NW == 4 ? 1 : 2) void attend_rows_kernel(const AttendParams p) {
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ FreshShared sh;
  __shared__ int told[2];
  typedef Staged<Bf16, D> F;               // (places in a tile of 16 bits)
  constexpr int NT = NW * 64, kRows = NW * 16 * RT, kLoads = kPage * D / 16 / NT;
  static_assert(kPage * D / 16 % NT == 0, "every thread has as many pieces of a page");
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  Place at = place_of(p);
  if (at.none) return;
  const int first_row = at.rg * kRows + wave * 16 * RT;
  Queries<T, D, RT> q;
  if (!place_in_sequence(p, at)) return;
  load_queries(p, at, first_row, q);
  RowState<D, RT> st;
  begin(st);

  const int from = at.chunk * p.chunk, to = min((at.chunk + 1) * p.chunk, at.n_pages);
  const int turns = max(0, to - from);
  bool bad = at.bad_length;
  for (int base = 0; base < turns; base += 64) {
    const int some = min(64, turns - base);
    PageList list;
    bad |= list.load(p, at, from + base, 1, some, false);
    // While page i's weights are made and meet its values, the scores of page i + 1 are: the products run beside the exponentials.  So
    // in LDS keys are a page ahead of values; in registers, on the way from memory, both are kDeep further.
    u32x4 kw[kDeep][kLoads], vw[kDeep][kLoads];
    const auto fetch = [&](u32x4 (&w)[kLoads], int i, int part) {
      const uint8_t* codes = page_codes(p.c, max(0, list.page_at(min(i, some - 1))), at.h, D) + part * kPage * D;
#pragma unroll
      for (int it = 0; it < kLoads; ++it) w[it] = load16(codes + (it * NT + tid) * 16);
    };
    const auto valid_of = [&](int i) { return list.page_at(i) < 0 ? 0 : min(kPage, at.len - (from + base + i) * kPage); };
    const auto put_keys = [&](const u32x4 (&w)[kLoads], int i) {
      uint8_t* tile = lds + (i & 1) * page_lds_bytes<D>();
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        const int idx = it * NT + tid, place = Tile::place(idx / (D / 16)), chunk = idx % (D / 16) * 2;
        *reinterpret_cast<u32x4*>(tile + F::key_at(chunk, place)) = __builtin_bit_cast(u32x4, Operand<T>::codes(w[it][0], w[it][1]));
        *reinterpret_cast<u32x4*>(tile + F::key_at(chunk + 1, place)) = __builtin_bit_cast(u32x4, Operand<T>::codes(w[it][2], w[it][3]));
      }
    };
    const auto put_values = [&](u32x4 (&w)[kLoads], int i) {
      uint8_t* tile = lds + (i & 1) * page_lds_bytes<D>();
      const float v_scale = list.v_at(i);
      const int valid = valid_of(i);
#pragma unroll
      for (int it = 0; it < kLoads; ++it) {
        const int idx = it * NT + tid, d = idx % D, eight = idx / D * 2;
        if (valid < kPage) w[it] &= tokens_below(valid - eight * 8);
        *reinterpret_cast<u32x4*>(tile + F::value_at(eight, 0, d)) = __builtin_bit_cast(u32x4, codes_as_bf16(w[it][0], w[it][1], v_scale));
        *reinterpret_cast<u32x4*>(tile + F::value_at(eight + 1, 0, d)) = __builtin_bit_cast(u32x4, codes_as_bf16(w[it][2], w[it][3], v_scale));
      }
    };
    const auto key_operand = [&](const uint8_t* tile, int t, int i) {
      return __builtin_bit_cast(typename Operand<T>::Vec, *reinterpret_cast<const u32x4*>(tile + F::key_at(Tile::channel(i, g) / 8, t * 16 + r)));
    };
    f32x4 s[RT][4];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      fetch(kw[u], u, 0);
      fetch(vw[u], u, 1);
    }
    put_keys(kw[0], 0);
    put_values(vw[0], 0);
    fetch(kw[0], kDeep, 0);
    fetch(vw[0], kDeep, 1);
    if (some > 1) put_keys(kw[1 % kDeep], 1);
    fetch(kw[1 % kDeep], kDeep + 1, 0);
    __syncthreads();
    if (first_row < at.rows) {
#pragma unroll
      for (int f = 0; f < D / 32 * 4; ++f) {
        const auto a = key_operand(lds, f % 4, f / 4);
#pragma unroll
        for (int e = 0; e < Operand<T>::kTerms; ++e)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[rt][f % 4] = mfma(a, q.v[rt][f / 4][e], f < 4 && e == 0 ? f32x4{0, 0, 0, 0} : s[rt][f % 4]);
      }
    }
    __syncthreads();                       // (the first page's keys have been read: the third's go there)
    for (int i0 = 0; i0 < some; i0 += kDeep)
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        const int i = i0 + u;
        if (i >= some) break;
        if (first_row < at.rows) {
          const float c = page_maximum(s, st, p.scale2 * list.k_at(i), valid_of(i), g);
          const uint8_t *tile = lds + (i & 1) * page_lds_bytes<D>(), *next_tile = lds + ((i + 1) & 1) * page_lds_bytes<D>();
          // (behind the last page: scores of what lies there, which are not used)
          page_round<kAhead>(q, s, st, c, [&](int t, int i) { return key_operand(next_tile, t, i); },
                             [&](int d, int k) { return *reinterpret_cast<const bf16x8*>(tile + F::value_at(g * 2 + k, 0, d * 16 + r)); });
        }
        if (i + 1 < some) put_values(vw[(u + 1) % kDeep], i + 1);
        if (i + 2 < some) put_keys(kw[(u + 2) % kDeep], i + 2);
        fetch(vw[(u + 1) % kDeep], i + 1 + kDeep, 1);
        fetch(kw[(u + 2) % kDeep], i + 2 + kDeep, 0);
        __syncthreads();                   // (of this page's tiles all is read, of the next one's all is written)
      }
  }
  const bool fresh = at.chunk == at.active - 1 && p.k.data && at.there > 0;
  if (fresh) {
    if (tid == 0) sh.wanted[0] = sh.wanted[1] = sh.odd = 0;
    __syncthreads();
    attend_fresh<T, D, RT, NT, true>(p, at.b, at.h, first_row, min(at.rows, (at.rg + 1) * kRows) - 1, at.there, 1, 0, q, st, lds, sh);
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

// Tiles of rows to a wave of the kernel for many rows, so that two waves to a SIMD have registers enough, one where D = 256 and four waves share a page.  (Not
// quite: 16 spill with bfloat16, D = 128, two tiles, 8 with fp32, D = 128, 64 rows, one with 16 bits, D = 256, eight waves.  They are addresses, written
// once and read outside of the loop over pages, in that over new tokens one or two a tile.)
template <typename T, int D> constexpr int rows_tiles() { return D == 64 || (D == 128 && sizeof(T) == 2) ? 2 : 1; }
// The launches, for each type of the call in a source file of its own (attend_launch.h, attend_*.hip).
template <typename T> hipError_t launch_attend(const AttendParams& p, int D, hipStream_t s);

// Which kernel `rows` that share a head go to (stream: the one for few), and the rows that one workgroup takes.
struct AttendChoice { bool stream; int rows; };
template <typename T, int D> constexpr AttendChoice attend_choice_of(int64_t rows) {
  if (rows <= 16 * stream_most_tiles<T, D>()) return {true, rows <= 16 ? 16 : 32};
  return {false, rows <= 64 || (sizeof(T) == 4 && D == 256) ? 64 : 128};
}
inline AttendChoice attend_choice(bool f32, int D, int64_t rows) {
  if (f32) return D == 64 ? attend_choice_of<float, 64>(rows) : D == 128 ? attend_choice_of<float, 128>(rows) : attend_choice_of<float, 256>(rows);
  return D == 64 ? attend_choice_of<F16, 64>(rows) : D == 128 ? attend_choice_of<F16, 128>(rows) : attend_choice_of<F16, 256>(rows);
}

}  // namespace tslt
