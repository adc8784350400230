// Rows of tokens as callers hold them (tslt_rows), and how many of a sequence's tokens there are: what the kernels that take them share.
#pragma once
#include "common.h"

namespace tslt {

struct RowsView { const void* data; int64_t seq, token, head; };       // strides in elements
constexpr int kBadPage = 16, kBadIndex = 32;           // TSLT_ROW_BAD_PAGE, TSLT_ROW_BAD_INDEX

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ u32x4 load16(const void* p) { return *as_global(reinterpret_cast<const u32x4*>(p)); }
// The same at any alignment of 16-bit elements.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
__device__ __forceinline__ u32x4 load16_any(const void* p) { return *(const u32x4_any __attribute__((address_space(1)))*)p; }
__device__ __forceinline__ void store16_any(void* p, u32x4 v) { *(u32x4_any __attribute__((address_space(1)))*)p = v; }

// New tokens of a sequence, of n: its count (null: all), kept inside 0 .. n; and a sequence's status, which says where that was needed.
__device__ __forceinline__ int counted(const int32_t* count, int64_t b, int n) { return count ? min(max(as_global(count)[b], 0), n) : n; }
__device__ __forceinline__ int sequence_status(const int32_t* count, int64_t b, int n, bool bad_page) {
  return (bad_page ? kBadPage : 0) | (count && as_global(count)[b] != counted(count, b, n) ? kBadIndex : 0);
}

// Eight numbers of a row, 16 bytes (32 of fp32), as fp32; and rounded to the row's type, to nearest-even.
template <typename T> struct Eight;
template <> struct Eight<float> {
  u32x4 w[2];
  __device__ __forceinline__ void load(const void* row, int64_t at) {
    const float* p = reinterpret_cast<const float*>(row) + at;
    w[0] = load16(p);
    w[1] = load16(p + 4);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = as_f32(w[i >> 2][i & 3]);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = as_u32(v[i]);
  }
  __device__ __forceinline__ void store(const void* row, int64_t at) const {
    u32x4* p = reinterpret_cast<u32x4*>(const_cast<float*>(reinterpret_cast<const float*>(row)) + at);
    p[0] = w[0];
    p[1] = w[1];
  }
};
template <typename T, typename E> struct Eight16 {
  typedef E E2 __attribute__((ext_vector_type(2)));
  u32x4 w;
  __device__ __forceinline__ void load(const void* row, int64_t at) { w = load16(reinterpret_cast<const uint16_t*>(row) + at); }
  __device__ __forceinline__ void get(float (&v)[8]) const { unpack<T>(make_uint4(w[0], w[1], w[2], w[3]), v); }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, E2{E(v[2 * i]), E(v[2 * i + 1])});
  }
  __device__ __forceinline__ void store(const void* row, int64_t at) const {
    *reinterpret_cast<u32x4*>(const_cast<uint16_t*>(reinterpret_cast<const uint16_t*>(row)) + at) = w;
  }
};
template <> struct Eight<Bf16> : Eight16<Bf16, __bf16> {};
template <> struct Eight<F16> : Eight16<F16, _Float16> {};

}  // namespace tslt
