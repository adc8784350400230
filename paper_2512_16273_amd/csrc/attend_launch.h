// Launches of attend.h's kernels for calls of one type; each type has a source file of its own (attend_*.hip).
#pragma once
#include "attend.h"

namespace tslt {

template <auto Kernel> hipError_t launch_attend_kernel(const AttendParams& p, int threads, int lds, hipStream_t s) {
  if (lds > 48 * 1024) {
    const hipError_t e = allow_dynamic_lds<Kernel>(160 * 1024 - 8192);
    if (e != hipSuccess) return e;
  }
  const int64_t units = p.B * p.c.heads * p.chunks;
  hipLaunchKernelGGL(Kernel, dim3(unsigned((units + 7) / 8 * 8 * p.row_groups)), dim3(threads), lds, s, p);
  return hipSuccess;
}
template <typename T, int D, int RT> hipError_t launch_attend_stream(const AttendParams& p, hipStream_t s) {
  return launch_attend_kernel<&attend_stream_kernel<T, D, RT>>(p, 256, stream_lds_bytes<T, D, RT>(p.k.data != nullptr), s);
}
template <typename T, int D> hipError_t launch_attend_rows(const AttendParams& p, hipStream_t s) {
  const AttendChoice choice = attend_choice_of<T, D>(int64_t(p.n) * p.group);
  if (choice.stream && choice.rows == 16) return launch_attend_stream<T, D, 1>(p, s);
  if constexpr (stream_most_tiles<T, D>() == 2) if (choice.stream) return launch_attend_stream<T, D, 2>(p, s);
  const int lds = rows_lds_bytes<T, D>(p.k.data != nullptr);
  if (choice.rows == 64) return launch_attend_kernel<&attend_rows_kernel<T, D, 1, 4, D == 256 ? 1 : 3, 2>>(p, 256, lds, s);
  if constexpr (rows_tiles<T, D>() == 2) return launch_attend_kernel<&attend_rows_kernel<T, D, 2, 4, 1, 1>>(p, 256, lds, s);
  else if constexpr (!(sizeof(T) == 4 && D == 256)) return launch_attend_kernel<&attend_rows_kernel<T, D, 1, 8, 1, 2>>(p, 512, lds, s);
  return hipErrorInvalidValue;
}
template <typename T> hipError_t launch_attend(const AttendParams& p, int D, hipStream_t s) {
  return D == 64 ? launch_attend_rows<T, 64>(p, s) : D == 128 ? launch_attend_rows<T, 128>(p, s) : launch_attend_rows<T, 256>(p, s);
}

}  // namespace tslt
