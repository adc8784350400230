// Attention of a round's new tokens over the 8-bit cache and over each other (tslt_cache_attend).
//
//   s_ij = scale * q_i . k_j,  out_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = ln sum_j exp(s_ij)
//
// j runs over the cached tokens, all of which every query sees, and over those of the call's own tokens that its mask shows.
// A row is one query head of one token; the rows of one sequence that share a key/value head, n * group of them, meet the same
// keys, so the products are dense in tiles of 16 rows, and one pass keeps a running maximum m and sum l for each row.
//
// One wave takes 64 keys at a time against RT tiles of rows, all in registers: codes go from memory into the operand registers of
// the products (the order in which the cache holds them is made for that), the scores come out with 16 keys of one row in
// each lane, which is how the second product wants its weights, so nothing is exchanged between lanes on the way.
// The four waves of a workgroup take different keys (KS of them) and different rows (4 / KS).
//
// Rounding.  Codes, and queries of 16 bits, enter the first product exactly; queries of 32 bits as three bfloat16 terms,
// exactly.  Sums are fp32.  A weight enters the second product as the sum of two bfloat16 terms, 16 bits, and of three, 24, in fp32
// calls; values enter it as bfloat16 times their page's scale, exactly.  (One bfloat16 term would be off by 2^-9, as much as the output's
// own rounding; one binary16 term by 2^-12, but it loses weights below 2^-30 of the largest, and where that one's value is 0 they are the result.)
// The running maximum is followed only when a row exceeds it by kLag powers of two: weights, in units of it, stay below 2^kLag.
#pragma once
#include "cache.h"

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
  float* part_o;                           // [B][heads][chunks][rows][D] sums of a chunk, and
  float2* part_ml;                         // [B][heads][chunks][rows] its maximum and sum
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

struct FreshShared {
  unsigned long long bad;                  // tokens of the tile with a value that is not finite
  int wanted[2];                           // waves that see something of the tile, of two tiles in turn
};

// Brings 64 new tokens from j0 on to LDS, zeros where there are fewer.  A value that is not finite is left out (0) and its token
// noted: a product would carry it to rows that do not see the token, as 0 times it.
template <typename T, int D>
__device__ __forceinline__ void stage_fresh(const AttendParams& p, int64_t b, int h, int j0, int there, uint8_t* lds, FreshShared& sh) {
  typedef Fresh<T, D> F;
  const int tid = int(threadIdx.x);
  const T* kp = reinterpret_cast<const T*>(p.k.data) + b * p.k.seq + h * p.k.head;
  const T* vp = reinterpret_cast<const T*>(p.v.data) + b * p.v.seq + h * p.v.head;
  constexpr int kChunks = D / F::kPer;
#pragma unroll
  for (int it = 0; it < kPage * kChunks / 256; ++it) {
    const int idx = it * 256 + tid, chunk = idx % kChunks, token = idx / kChunks;
    u32x4 w = {0, 0, 0, 0};
    if (j0 + token < there) w = load16(kp + (j0 + token) * p.k.token + chunk * F::kPer);
    *reinterpret_cast<u32x4*>(lds + F::key_at(chunk, token)) = w;
  }
  constexpr int kWide = F::kBytes == 4 ? 1 : 2;          // channels to a thread: a word
#pragma unroll
  for (int it = 0; it < 8 * (D / kWide) / 256 || it == 0; ++it) {
    const int idx = it * 256 + tid, at = idx % (D / kWide), eight = idx / (D / kWide);
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int token = j0 + eight * 8 + e;
      w[e] = token < there ? *as_global(reinterpret_cast<const uint32_t*>(vp + token * p.v.token + at * kWide)) : 0;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      bool odd = not_finite<T>(w[e]);
      if (kWide == 2) odd |= not_finite<T>(w[e] >> 16);
      if (odd) {
        atomicOr(&sh.bad, 1ull << (eight * 8 + e));
        w[e] = 0;
      }
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
// A wave's tile of values, 64 tokens: of each 16 channels lane 16 g + r has channel r of tokens 16 g .. + 15.
template <int D> struct ValueTile {
  u32x4 w[D / 16];
  __device__ __forceinline__ void load(const uint8_t* values, int lane) {
    const uint8_t* p = values + (lane >> 4) * 16 * D + (lane & 15) * 16;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) w[d] = load16(p + d * 256);
  }
  // Tokens from `there` on (of the lane's 16) hold no values: their bytes may be anything.
  __device__ __forceinline__ void cut(int there) {
    u32x4 keep;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n = there - 4 * e;
      keep[e] = n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
    }
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

// The call's own tokens, all of them that the wave's rows see, tile after tile; the waves of a workgroup that share rows take turns.
template <typename T, int D, int RT, int KS>
__device__ __forceinline__ void attend_fresh(const AttendParams& p, int64_t b, int h, int first_row, int last_row, int there, int wave_k,
                                             const Queries<T, D, RT>& q, RowState<D, RT>& st, uint8_t* lds, FreshShared& sh) {
  typedef Fresh<T, D> F;
  typedef Terms<T> W;
  const int lane = lane_id(), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  const uint32_t* mask = p.mask ? p.mask + b * p.mask_seq : nullptr;
  // (a token sees none behind itself where there is no mask: tiles behind the workgroup's last row's token are not looked at)
  const int reach = mask ? there : min(there, last_row / p.group + 1);
  for (int j0 = 0, turn = 0; j0 < reach; j0 += kPage, ++turn) {
    uint32_t seen[RT];
    bool any = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + rt * 16 + r, i = row / p.group, at = j0 + g * 16;
      uint32_t bits = 0;
      if (i < there && at < there) {
        if (mask) bits = as_global(mask)[int64_t(i) * p.mask_words + (at >> 5)] >> (at & 31) & 0xFFFFu;
        else bits = i - at >= 15 ? 0xFFFFu : i < at ? 0u : (2u << (i - at)) - 1;
        if (there - at < 16) bits &= (1u << (there - at)) - 1;
      }
      seen[rt] = bits;
      any |= bits != 0;
    }
    const bool wanted = ballot(any) != 0 && turn % KS == wave_k;
    if (ballot(any) != 0 && lane == 0) sh.wanted[turn & 1] = turn + 1;
    __syncthreads();                       // (also: what was staged before has been read)
    if (sh.wanted[turn & 1] != turn + 1) continue;
    if (tid == 0) sh.bad = 0;
    __syncthreads();
    stage_fresh<T, D>(p, b, h, j0, there, lds, sh);
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
        s[rt][i >> 2][i & 3] = x;
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
      }
    // Values that are not finite, token by token, to the rows that see them (a call without any comes past here at once).
    unsigned long long bad = sh.bad;
    bad = uint64_t(__builtin_amdgcn_readfirstlane(uint32_t(bad >> 32))) << 32 | uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(bad)));
    for (; bad; bad &= bad - 1) {
      const int j = __builtin_ctzll(bad);
      const T* vp = reinterpret_cast<const T*>(p.v.data) + b * p.v.seq + h * p.v.head + (j0 + j) * p.v.token;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float x = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) x = (j & 15) == i ? s[rt][i >> 2][i & 3] : x;
        x = __shfl(x, (j >> 4) * 16 + r);
        if (!(__shfl(int(seen[rt]), (j >> 4) * 16 + r) >> (j & 15) & 1)) continue;
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // (of a word of two channels both were left out if one was not finite)
            const float y = load_elem<T>(vp, d * 16 + g * 4 + i), z = load_elem<T>(vp, (d * 16 + g * 4 + i) ^ 1);
            if (!__builtin_isfinite(y) || (sizeof(T) == 2 && !__builtin_isfinite(z))) st.o[rt][d][i] = __builtin_fmaf(x, y, st.o[rt][d][i]);
          }
      }
    }
  }
}

template <typename T, int D, int RT, int KS> constexpr int attend_join_bytes() { return KS == 1 ? 0 : KS * 16 * RT * (4 / KS) * (D + 4) * 4; }
template <typename T, int D, int RT, int KS> constexpr int attend_lds_bytes(bool fresh) {
  return attend_join_bytes<T, D, RT, KS>() > (fresh ? Fresh<T, D>::kLds : 0) ? attend_join_bytes<T, D, RT, KS>() : fresh ? Fresh<T, D>::kLds : 0;
}

// KS of a workgroup's four waves share rows and take turns at the pages, 4 / KS have rows of their own.
template <typename T, int D, int RT, int KS>
__global__ __launch_bounds__(256, 2) void attend_kernel(const AttendParams p) {
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ FreshShared sh;
  __shared__ float2 join_ml[KS][4 / KS * 16 * RT];
  constexpr int RS = 4 / KS, kRows = RS * 16 * RT;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), r = lane & 15, g = lane >> 4, tid = int(threadIdx.x);
  const int wave_k = wave % KS, wave_r = wave / KS;
  // Workgroups go to the eight XCDs in turn.  Those that differ in their rows alone read the same pages: on one XCD, one after the other.
  const uint32_t block = blockIdx.x, slot = block >> 3;
  const uint64_t unit = uint64_t(slot / uint32_t(p.row_groups)) * 8 + (block & 7);
  const int rg = int(slot % uint32_t(p.row_groups));
  if (unit >= uint64_t(p.B) * p.c.heads * p.chunks) return;
  const int chunk = int(unit % uint32_t(p.chunks));
  const int h = int(unit / uint32_t(p.chunks) % uint32_t(p.c.heads));
  const int64_t b = int64_t(unit / (uint64_t(p.chunks) * p.c.heads));

  bool bad_length;
  const int len = cached_tokens(p.c, b, bad_length);
  const int n_pages = (len + kPage - 1) / kPage;
  const int active = max(1, (n_pages + p.chunk - 1) / p.chunk);
  if (chunk >= active) return;
  const int there = p.count ? min(max(as_global(p.count)[b], 0), p.n) : p.n;
  const int rows = p.n * p.group;
  const int first_row = rg * kRows + wave_r * 16 * RT;

  Queries<T, D, RT> q;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = min(first_row + rt * 16 + r, rows - 1);
    const int64_t at = b * p.q.seq + int64_t(row / p.group) * p.q.token + int64_t(h * p.group + row % p.group) * p.q.head;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) Operand<T>::load(p.q.data, at + step_channel(i, g), q.v[rt][i]);
  }
  RowState<D, RT> st;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    st.m[rt] = kNoMax;
    st.l[rt] = 0;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) st.o[rt][d] = f32x4{0, 0, 0, 0};
  }

  // The wave's pages: up to 64 entries of the table at a time, one a lane, with their scales.
  const int32_t* table = p.c.pages + b * p.c.width;
  const int from = chunk * p.chunk + wave_k, to = min((chunk + 1) * p.chunk, n_pages);
  const int turns = from < to ? (to - from + KS - 1) / KS : 0;
  bool bad = bad_length;
  for (int base = 0; base < turns; base += 64) {
    const int some = min(64, turns - base);
    int page = -1;
    float ks = 1.0f, vs = 1.0f;
    if (lane < some) page = as_global(table)[from + KS * (base + lane)];
    const bool in = page >= 0 && page < p.c.n_pages;
    if (lane < some) bad |= !in;
    if (!in) page = -1;
    else {
      const float* sc = p.c.scales + (int64_t(page) * p.c.heads + h) * 2;
      ks = as_global(sc)[0];
      vs = as_global(sc)[1];
    }
    KeyTile<D> kt;
    ValueTile<D> vt;
    const uint8_t* codes = page_codes(p.c, max(0, __builtin_amdgcn_readlane(page, 0)), h, D);
    kt.load(codes, lane);
    vt.load(codes + kPage * D, lane);
    for (int i = 0; i < some; ++i) {
      const int pg = __builtin_amdgcn_readlane(page, i);
      const float k_scale = as_f32(__builtin_amdgcn_readlane(as_u32(ks), i)), v_scale = as_f32(__builtin_amdgcn_readlane(as_u32(vs), i));
      const int t0 = (from + KS * (base + i)) * kPage;
      const int valid = pg < 0 ? 0 : min(kPage, len - t0);
      f32x4 s[RT][4];
      key_products<T, D, RT>(kt, q, s);
      const uint8_t* next = page_codes(p.c, max(0, __builtin_amdgcn_readlane(page, min(i + 1, some - 1))), h, D);
      if (i + 1 < some) kt.load(next, lane);
      bf16x8 w[RT][2][Terms<T>::kW];
      page_weights<T, D, RT>(s, st, p.scale2 * k_scale, valid, g, w);
      if (valid < kPage) vt.cut(valid - g * 16);
      page_values(vt, w, st, v_scale);
      if (i + 1 < some) vt.load(next + kPage * D, lane);
    }
  }
  if (chunk == active - 1 && p.k.data && there > 0) {
    if (tid == 0) sh.wanted[0] = sh.wanted[1] = 0;
    __syncthreads();
    attend_fresh<T, D, RT, KS>(p, b, h, first_row, min(rows, (rg + 1) * kRows) - 1, there, wave_k, q, st, lds, sh);
  }

  // The rows' sums: lane 16 g + r has its row's maximum, its groups' parts of the sum of weights, and its channels.
  const bool last = active == 1;
  const int64_t part = ((b * p.c.heads + h) * p.chunks + chunk) * int64_t(rows);
  if constexpr (KS == 1) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = first_row + rt * 16 + r;
      const float l = over_groups_sum(st.l[rt]);
      if (row >= rows) continue;
      if (!last) {
        if (g == 0) p.part_ml[part + row] = make_float2(st.m[rt], l);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) store4<float>(p.part_o, (part + row) * D + d * 16 + g * 4, st.o[rt][d]);
        continue;
      }
      const int i = row / p.group;
      const bool none = i >= there || l == 0;
      const float f = none ? 0.0f : 1.0f / l;
      const int64_t at = (b * p.n + i) * p.heads_q + h * p.group + row % p.group;
      if (g == 0) p.lse[at] = none ? -INFINITY : (st.m[rt] + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) store4<T>(p.out, at * D + d * 16 + g * 4, none ? f32x4{0, 0, 0, 0} : st.o[rt][d] * f);
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
    for (int at = tid; at < kRows * (D / 4); at += 256) {
      const int local = at / (D / 4), d = at % (D / 4) * 4, row = rg * kRows + local;
      if (row >= rows) break;
      float m = kNoMax, l = 0;
#pragma unroll
      for (int k = 0; k < KS; ++k) m = fmaxf(m, join_ml[k][local].x);
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        l += join_ml[k][local].y * exp2_fast(join_ml[k][local].x - m);
        o += *reinterpret_cast<const f32x4*>(sums + (k * kRows + local) * (D + 4) + d);
      }
      if (!last) {
        if (d == 0) p.part_ml[part + row] = make_float2(m, l);
        store4<float>(p.part_o, (part + row) * D + d, o);
        continue;
      }
      const int i = row / p.group;
      const bool none = i >= there || l == 0;
      const int64_t to_row = (b * p.n + i) * p.heads_q + h * p.group + row % p.group;
      if (d == 0) p.lse[to_row] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
      store4<T>(p.out, to_row * D + d, none ? f32x4{0, 0, 0, 0} : o * (1.0f / l));
    }
  }
  if (p.status && last && h == 0 && rg == 0) {
    if (__syncthreads_or(bad) != 0) { if (tid == 0) p.status[b] = kBadPage; }
    else if (tid == 0) p.status[b] = 0;
  }
}

// The chunks of a sequence joined: one workgroup to kJoinRows rows of a head.
constexpr int kJoinRows = 8;
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendParams p) {
  const int rows = p.n * p.group, groups = (rows + kJoinRows - 1) / kJoinRows, tid = int(threadIdx.x);
  const int rg = int(blockIdx.x % uint32_t(groups));
  const int h = int(blockIdx.x / uint32_t(groups) % uint32_t(p.c.heads));
  const int64_t b = blockIdx.x / (uint32_t(groups) * p.c.heads);
  bool bad;
  const int len = cached_tokens(p.c, b, bad);
  const int n_pages = (len + kPage - 1) / kPage;
  const int active = (n_pages + p.chunk - 1) / p.chunk;
  if (active <= 1) return;
  const int there = p.count ? min(max(as_global(p.count)[b], 0), p.n) : p.n;
  const int64_t part = (b * p.c.heads + h) * int64_t(p.chunks) * rows;
  for (int at = tid; at < kJoinRows * (D / 4); at += 256) {
    const int row = rg * kJoinRows + at / (D / 4), d = at % (D / 4) * 4;
    if (row >= rows) break;
    float m = kNoMax;
    for (int c = 0; c < active; ++c) m = fmaxf(m, p.part_ml[part + int64_t(c) * rows + row].x);
    float l = 0;
    f32x4 o = {0, 0, 0, 0};
    for (int c = 0; c < active; ++c) {
      const float2 ml = p.part_ml[part + int64_t(c) * rows + row];
      const float f = exp2_fast(ml.x - m);
      l += ml.y * f;
      o += *reinterpret_cast<const f32x4*>(p.part_o + (part + int64_t(c) * rows + row) * D + d) * f;
    }
    const int i = row / p.group;
    const bool none = i >= there || l == 0;
    const int64_t to_row = (b * p.n + i) * p.heads_q + h * p.group + row % p.group;
    if (d == 0) p.lse[to_row] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    store4<T>(p.out, to_row * D + d, none ? f32x4{0, 0, 0, 0} : o * (1.0f / l));
  }
  if (p.status && h == 0 && rg == 0) {
    for (int i = tid; i < n_pages; i += 256) {
      const int page = as_global(p.c.pages + b * p.c.width)[i];
      bad |= page < 0 || page >= p.c.n_pages;
    }
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) p.status[b] = bad ? kBadPage : 0;
  }
}

// The launches, for each type of the call in a source file of its own (attend_launch.h, attend_*.hip).
template <typename T> hipError_t launch_attend(const AttendParams& p, int D, hipStream_t s);
// Rows that a workgroup takes, of `rows` that share a head.
constexpr int attend_rows(int64_t rows) { return rows <= 16 ? 16 : 128; }

}  // namespace tslt
