// Launches of attend.h's kernels for calls of one type; each type has a source file of its own (attend_*.hip).
#pragma once
#include "attend.h"

namespace tslt {

template <typename T, int D, int RT, int KS> hipError_t launch_attend_shape(const AttendParams& p, hipStream_t s) {
  constexpr auto fn = &attend_kernel<T, D, RT, KS>;
  const int lds = attend_lds_bytes<T, D, RT, KS>(p.k.data != nullptr);
  if (lds > 48 * 1024) {
    const hipError_t e = allow_dynamic_lds<fn>(160 * 1024 - 4096);
    if (e != hipSuccess) return e;
  }
  const int64_t units = p.B * p.c.heads * p.chunks;
  hipLaunchKernelGGL(fn, dim3(unsigned((units + 7) / 8 * 8 * p.row_groups)), dim3(256), lds, s, p);
  if (p.chunks > 1) {
    const int64_t groups = (int64_t(p.n) * p.group + kJoinRows - 1) / kJoinRows;
    hipLaunchKernelGGL((attend_join_kernel<T, D>), dim3(unsigned(p.B * p.c.heads * groups)), dim3(256), 0, s, p);
  }
  return hipSuccess;
}
template <typename T, int D> hipError_t launch_attend_rows(const AttendParams& p, hipStream_t s) {
  if (attend_rows(int64_t(p.n) * p.group) == 16) return launch_attend_shape<T, D, 1, 4>(p, s);
  return launch_attend_shape<T, D, 2, 1>(p, s);
}
template <typename T> hipError_t launch_attend(const AttendParams& p, int D, hipStream_t s) {
  return D == 64 ? launch_attend_rows<T, 64>(p, s) : D == 128 ? launch_attend_rows<T, 128>(p, s) : launch_attend_rows<T, 256>(p, s);
}

}  // namespace tslt
