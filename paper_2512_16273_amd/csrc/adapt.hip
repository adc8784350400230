// C ABI of the low-rank adapters (see include/tslt.h): argument checks, how the work is cut, launches.
#include "tslt.h"

#include <algorithm>

#include "adapt.h"
#include "checks.h"

namespace {

// Workgroups' tokens and how many cuts x's channels are in: twice as many workgroups as compute units, of 512 channels or more.
struct Plan { int token_tiles, rank_tiles, tiles, chunks, cuts; };
Plan plan_down(int64_t B, int32_t n, int32_t K, int32_t R) {
  Plan p;
  p.token_tiles = n > 16 ? 4 : 1;
  p.rank_tiles = R == 16 ? 1 : R == 32 ? 2 : 4;
  p.tiles = (n + 16 * p.token_tiles - 1) / (16 * p.token_tiles);
  p.chunks = (R / 16 + p.rank_tiles - 1) / p.rank_tiles;
  const int64_t blocks = std::min<int64_t>(B, 1 << 20) * p.tiles * p.chunks, most = std::min<int64_t>(8, K / 512);
  p.cuts = int(std::max<int64_t>(1, std::min<int64_t>(most, 2 * int64_t(tslt::compute_units()) / blocks)));
  return p;
}

template <typename T, int kTokenTiles> void launch_down(const tslt::AdaptParams& p, int rank_tiles, unsigned blocks, hipStream_t s) {
  if (rank_tiles == 1) hipLaunchKernelGGL((tslt::adapt_down_kernel<T, kTokenTiles, 1>), dim3(blocks), dim3(tslt::kBlock), 0, s, p);
  else if (rank_tiles == 2) hipLaunchKernelGGL((tslt::adapt_down_kernel<T, kTokenTiles, 2>), dim3(blocks), dim3(tslt::kBlock), 0, s, p);
  else hipLaunchKernelGGL((tslt::adapt_down_kernel<T, kTokenTiles, 4>), dim3(blocks), dim3(tslt::kBlock), 0, s, p);
}
template <typename T> void launch_adapt(tslt::AdaptParams p, const Plan& plan, hipStream_t s) {
  p.tiles = plan.tiles; p.chunks = plan.chunks; p.cuts = plan.cuts;
  const unsigned down = unsigned(p.B * p.tiles * p.chunks * p.cuts);
  if (plan.token_tiles == 1) launch_down<T, 1>(p, plan.rank_tiles, down, s);
  else launch_down<T, 4>(p, plan.rank_tiles, down, s);
  p.chunks = (p.N + 255) / 256;
  const unsigned up = unsigned(p.B * p.tiles * p.chunks);
  if (plan.token_tiles == 1) hipLaunchKernelGGL((tslt::adapt_up_kernel<T, 1>), dim3(up), dim3(tslt::kBlock), 0, s, p);
  else hipLaunchKernelGGL((tslt::adapt_up_kernel<T, 4>), dim3(up), dim3(tslt::kBlock), 0, s, p);
}
bool sizes_fit(int64_t B, int32_t n, int32_t K, int32_t N, int32_t R) {
  return B >= 1 && n >= 1 && K >= 1 && N >= 1 && R >= 16 && R <= TSLT_MAX_ADAPTER_RANK && R % 16 == 0 && B <= 0x7FFFFFFF / n;
}

}  // namespace

extern "C" {

size_t tslt_adapt_workspace_bytes(int64_t B, int32_t n, int32_t K, int32_t N, int32_t R) {
  if (!sizes_fit(B, n, K, N, R)) return 0;
  return (size_t(plan_down(B, n, K, R).cuts) * size_t(B) * n * R * 4 + 255) / 256 * 256;
}

int tslt_adapt(const tslt_rows* x, int32_t K, const tslt_rows* base, const tslt_rows* out, int32_t N, tslt_dtype dt, int64_t B, int32_t n,
               const void* a, const void* b, int64_t n_adapters, int32_t R, const int32_t* adapter, const float* scale, const int32_t* rank,
               const int32_t* count, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "tslt_adapt";
  if (!valid_dtype(dt)) return fail(TSLT_ERR_INVALID_ARG, "%s: unknown dtype %d", who, int(dt));
  if (B < 0 || n < 1 || K < 1 || N < 1 || n_adapters < 1)
    return fail(TSLT_ERR_INVALID_ARG, "%s: bad shape B=%lld n=%d K=%d N=%d n_adapters=%lld", who, (long long)B, int(n), int(K), int(N), (long long)n_adapters);
  if (R < 16 || R > TSLT_MAX_ADAPTER_RANK || R % 16)
    return fail(TSLT_ERR_UNSUPPORTED, "%s: R must be a multiple of 16 up to %d (got %d)", who, TSLT_MAX_ADAPTER_RANK, int(R));
  if (K % (16 / elem_bytes(dt))) return fail(TSLT_ERR_UNSUPPORTED, "%s: rows of K=%d elements are no multiple of 16 bytes", who, int(K));
  if (n_adapters > 0x7FFFFFFF || B > 0x7FFFFFFF / n) return fail(TSLT_ERR_UNSUPPORTED, "%s: adapters and tokens must fit 31 bits", who);
  if (B == 0) return TSLT_OK;
  tslt_rows rx = x ? *x : tslt_rows{}, rb = base ? *base : tslt_rows{}, ro = out ? *out : tslt_rows{};
  rx.head_stride = rb.head_stride = ro.head_stride = 0;
  if (int e = check_rows(who, "x", &rx, dt)) return e;
  if (!rb.data || !ro.data) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(rb.data, elem_bytes(dt)) || !aligned(ro.data, elem_bytes(dt))) return fail(TSLT_ERR_INVALID_ARG, "%s: rows not aligned to their type", who);
  if (rb.data == ro.data && (rb.seq_stride != ro.seq_stride || rb.token_stride != ro.token_stride))
    return fail(TSLT_ERR_INVALID_ARG, "%s: rows that are added to in place must have the same strides", who);
  if (!a || !b || !adapter) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(a, 16) || !aligned(b, 16)) return fail(TSLT_ERR_INVALID_ARG, "%s: adapters not aligned to 16 bytes", who);
  const Plan plan = plan_down(B, n, K, R);
  const size_t need = tslt_adapt_workspace_bytes(B, n, K, N, R);
  if (!ws || !aligned(ws, 256) || ws_bytes < need)
    return fail(TSLT_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed, 256-byte aligned", who, ws ? ws_bytes : size_t(0), need);
  int code;
  if (!grid_fits(who, B * plan.tiles * std::max<int64_t>(int64_t(plan.chunks) * plan.cuts, (int64_t(N) + 255) / 256), code)) return code;
  tslt::AdaptParams p{};
  p.x = view(&rx); p.base = view(&rb); p.out = view(&ro);
  p.K = K; p.N = N; p.R = R; p.n = n; p.B = B; p.n_adapters = n_adapters; p.a = a; p.b = b; p.adapter = adapter; p.rank = rank; p.count = count;
  p.scale = scale; p.status = status; p.h = reinterpret_cast<float*>(ws); p.copy = rb.data != ro.data;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dt == TSLT_F32) launch_adapt<float>(p, plan, s);
  else if (dt == TSLT_BF16) launch_adapt<tslt::Bf16>(p, plan, s);
  else launch_adapt<tslt::F16>(p, plan, s);
  return launched("tslt_adapt launch");
}

}  // extern "C"
