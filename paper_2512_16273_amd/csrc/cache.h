// The 8-bit key/value cache of include/tslt.h: its layout, and what the kernels that read it share.
//
// A page holds 64 tokens.  For each head its keys lie [64 tokens][D] and its values [4][D][16 tokens], both e4m3, one byte a
// number, with one scale each.  Both orders are those in which the matrix instructions of the kernels take them, 16 bytes a lane
// straight from memory into the registers of an operand, no transpose and no LDS between; 16 tokens of values together, not
// 64, so that a token that is appended or moved touches 2 KB of a page's values (D = 128) and not all 8 KB.
//
// Scales are powers of two.  e4m3 is a floating-point format, so that a scale between two powers would not make a number's
// relative rounding smaller; and where a page's scale has to grow for a token that comes later, its codes are brought to
// the new scale exactly (but for those that become subnormal).
#pragma once
#include "rows.h"

namespace tslt {

constexpr int kPage = 64;                  // tokens of a page
constexpr int kMinScaleExp = -100;         // least exponent of a scale: a page of zeros has it

struct CacheView {
  uint8_t* codes;
  float* scales;
  int64_t n_pages;
  int heads;
  const int32_t* pages;                    // [B][width]
  int64_t width;
  const int32_t* length;                   // [B]
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// a / b of two powers of two; kept inside the normal numbers, where it is not exact any more.
__device__ __forceinline__ float power_ratio(float a, float b) {
  const int bits = int(as_u32(a)) - int(as_u32(b)) + 0x3F800000;
  return as_f32(uint32_t(min(max(bits, 0x00800000), 0x7F000000)));
}

// Cached tokens of a sequence: its length, kept inside its row of the page table.
__device__ __forceinline__ int cached_tokens(const CacheView& c, int64_t b, bool& bad) {
  const int64_t most = c.width * kPage;
  const int64_t len = as_global(c.length)[b];
  bad = len < 0 || len > most;
  return int(len < 0 ? 0 : len > most ? most : len);
}
__device__ __forceinline__ const uint8_t* page_codes(const CacheView& c, int64_t page, int head, int D) {
  return c.codes + (page * c.heads + head) * (2 * kPage * D);
}

// The same of what no other workgroup reads: it need not stay in a cache (4 x 131000 tokens 167 us so, 185 without).
__device__ __forceinline__ u32x4 load16_once(const void* p) { return __builtin_nontemporal_load(as_global(reinterpret_cast<const u32x4*>(p))); }

// Eight codes (two words) as an operand of a 16-bit matrix product: exact, as e4m3 has four significant bits and reaches from
// 2^-9 to 448; times a power of two in bfloat16, which reaches as far as fp32.
__device__ __forceinline__ f16x8 codes_as_f16(uint32_t lo, uint32_t hi) {
  constexpr float scale = 1.0f;
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ bf16x8 codes_as_bf16(uint32_t lo, uint32_t hi, float scale = 1.0f) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Three bfloat16 numbers whose sum is x: each takes the leading eight bits of what the ones before it leave.
__device__ __forceinline__ void split3(float x, __bf16& a, __bf16& b, __bf16& c) {
  const float x0 = as_f32(as_u32(x) & 0xFFFF0000u);
  const float r1 = x - x0, x1 = as_f32(as_u32(r1) & 0xFFFF0000u);
  a = __builtin_bit_cast(__bf16, uint16_t(as_u32(x0) >> 16));
  b = __builtin_bit_cast(__bf16, uint16_t(as_u32(x1) >> 16));
  c = __builtin_bit_cast(__bf16, uint16_t(as_u32(r1 - x1) >> 16));
}

// How a query's, or a new token's, row of type T enters the matrix products over the channels: as it is in 16 bits, and as
// the sum of three bfloat16 terms, which is exact, in 32.
template <typename T> struct Operand;
template <> struct Operand<Bf16> {
  static constexpr int kTerms = 1;
  typedef bf16x8 Vec;
  static __device__ __forceinline__ bf16x8 codes(uint32_t lo, uint32_t hi) { return codes_as_bf16(lo, hi); }
  static __device__ __forceinline__ void load(const void* p, int64_t at, bf16x8 (&v)[1]) {
    v[0] = __builtin_bit_cast(bf16x8, load16(reinterpret_cast<const uint16_t*>(p) + at));
  }
};
template <> struct Operand<F16> {
  static constexpr int kTerms = 1;
  typedef f16x8 Vec;
  static __device__ __forceinline__ f16x8 codes(uint32_t lo, uint32_t hi) { return codes_as_f16(lo, hi); }
  static __device__ __forceinline__ void load(const void* p, int64_t at, f16x8 (&v)[1]) {
    v[0] = __builtin_bit_cast(f16x8, load16(reinterpret_cast<const uint16_t*>(p) + at));
  }
};
template <> struct Operand<float> {
  static constexpr int kTerms = 3;
  typedef bf16x8 Vec;
  static __device__ __forceinline__ bf16x8 codes(uint32_t lo, uint32_t hi) { return codes_as_bf16(lo, hi); }
  static __device__ __forceinline__ void split(u32x4 x, u32x4 y, bf16x8 (&v)[3]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      __bf16 a, b, c;
      split3(as_f32(i < 4 ? x[i] : y[i - 4]), a, b, c);
      v[0][i] = a; v[1][i] = b; v[2][i] = c;
    }
  }
  static __device__ __forceinline__ void load(const void* p, int64_t at, bf16x8 (&v)[3]) {
    const float* f = reinterpret_cast<const float*>(p) + at;
    split(load16(f), load16(f + 4), v);
  }
};

// How the lanes of a wave share 64 tokens of one head and tiles of 16 of its rows (queries).  Lane l = 16 g + r has row r of each tile.  The
// first product is four matrix instructions of 16 tokens by 16 rows for each 32 channels, the second one of 16 channels by 16 rows for each 32 tokens.
// Tokens are dealt out to the first one's lines so that what a lane gets of its results, lines 4 g .. 4 g + 3 of each of the four, are tokens 16 g ..
// 16 g + 15: those whose values it reads as 16 bytes for the second, in the order in which it has their weights.  So nothing is exchanged between lanes.
// (Instructions of 32 by 32, half as many, leave more room for others beside them, and the same work takes a tenth fewer cycles; but the clock falls by
// more, and so few sums at a time leave each waiting for the one before it: 2048 tokens on 16000 875 us, 826 so, 32 rows on 4050 tokens 129 and 103.)
struct Tile {
  // Token of line `line` of instruction t, and the place of a token when tokens are put in the order instruction by instruction, line by line.
  static __device__ __forceinline__ int token(int t, int line) { return (line >> 2) * 16 + t * 4 + (line & 3); }
  static __device__ __forceinline__ int place(int token) { return (token >> 2 & 3) * 16 + (token >> 4) * 4 + (token & 3); }
  // The first of a lane's eight channels of step i, 32 channels.
  static __device__ __forceinline__ int channel(int i, int g) { return (i >> 1) * 64 + g * 16 + (i & 1) * 8; }
};

// 64 tokens' keys in a wave: the lane's 16 bytes j are channels 64 j + 16 g .. of its line's token.
template <int D> struct KeyTile {
  u32x4 w[4][D / 64];
  __device__ __forceinline__ void load(const uint8_t* keys, int lane) {
    const uint8_t* from = keys + Tile::token(0, lane & 15) * D + (lane >> 4) * 16;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < D / 64; ++j) w[t][j] = load16_once(from + t * 4 * D + j * 64);
  }
  // Operand of instruction t and step i.
  template <typename T> __device__ __forceinline__ typename Operand<T>::Vec operand(int t, int i) const {
    const u32x4 x = w[t][i >> 1];
    return (i & 1) ? Operand<T>::codes(x[2], x[3]) : Operand<T>::codes(x[0], x[1]);
  }
};
// A wave's rows, RT tiles of 16, as the other operand.
template <typename T, int D, int RT> struct Queries {
  typename Operand<T>::Vec v[RT][D / 32][Operand<T>::kTerms];
};
// Their scores: s[rt][t][i] is of row r of tile rt and token 16 g + 4 t + i.
template <typename T, int D, int RT> __device__ __forceinline__ void key_products(const KeyTile<D>& k, const Queries<T, D, RT>& q, f32x4 (&s)[RT][4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) s[rt][t] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const auto a = k.template operand<T>(t, i);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < Operand<T>::kTerms; ++e) s[rt][t] = mfma(a, q.v[rt][i][e], s[rt][t]);
    }
  }
}

}  // namespace tslt
