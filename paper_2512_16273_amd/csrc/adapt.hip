// C ABI of the low-rank adapters (see include/tslt.h): argument checks, how the work is cut, launches.
#include "tslt.h"

#include <algorithm>

#include "adapt.h"
#include "checks.h"

namespace {

// How a call is cut: tokens of a workgroup in both launches (in sixteens), ranks of one in the first (in sixteens), how many cuts x's channels are in, and how
// many workgroups share the channels of the result.
//   Cuts fill the GPU twice, but every workgroup of the second launch adds their sums up: 512 channels each at least, and fewer of high ranks (2 x 1000 tokens of rank 128, 4
//   / 8 cuts 35.6 / 37.0 us; 500 of rank 256, 1 / 2 / 8 cuts 53 / 39 / 43).
//   The second launch takes 64 tokens where that makes workgroups for half of the compute units at least (4 x 2001 tokens of rank 64, 32 / 64: 96 / 89 us; 16 x 85 of rank 16 19.8 /
//   25.6), and the channels in as many shares as there is room for at once (2 x 1000 fp32 tokens, two workgroups fit a compute unit, for 2 / 3 / 4 of them 38 / 46 / 44 us; 16 x 85
//   bfloat16 ones, three fit, 21.1 / 19.8 / 19.8; 256 x 9, five fit, for 4 / 5 / 8 25.5 / 24.6 / 25.7).
struct Plan { int token_tiles, rank_tiles, tiles, chunks, cuts, up_token_tiles, up_tiles, splits; };
Plan plan_adapt(tslt_dtype dt, int64_t B, int32_t n, int32_t K, int32_t N, int32_t R) {
  Plan p;
  const int64_t cus = tslt::compute_units(), sequences = std::min<int64_t>(B, 1 << 20);
  const auto between = [](int64_t least, int64_t x, int64_t most) { return int(std::max(least, std::min(x, most))); };
  p.token_tiles = n > 16 ? 4 : 1;
  p.rank_tiles = R == 16 ? 1 : R == 32 ? 2 : 4;
  p.tiles = int((int64_t(n) + 16 * p.token_tiles - 1) / (16 * p.token_tiles));
  p.chunks = (R / 16 + p.rank_tiles - 1) / p.rank_tiles;
  p.cuts = between(1, std::min<int64_t>(512 / R, K / 512), 8);
  p.cuts = between(1, 2 * cus / (sequences * p.tiles * p.chunks), p.cuts);
  p.up_token_tiles = n <= 16 ? 1 : dt == TSLT_F32 || sequences * ((int64_t(n) + 63) / 64) < cus / 2 ? 2 : 4;
  p.up_tiles = int((int64_t(n) + 16 * p.up_token_tiles - 1) / (16 * p.up_token_tiles));
  const int64_t fill = (n <= 16 ? 5 : p.up_token_tiles == 2 && dt != TSLT_F32 ? 3 : 2) * cus;
  p.splits = between(1, fill / (sequences * p.up_tiles), (int64_t(N) + 255) / 256);
  return p;
}
template <typename T, int kRankTiles> void launch_down(const tslt::AdaptParams& p, int token_tiles, hipStream_t s) {
  const dim3 blocks(unsigned(p.B * p.tiles * p.chunks * p.cuts)), threads(tslt::kBlock);
  if (token_tiles == 1) hipLaunchKernelGGL((tslt::adapt_down_few_kernel<T, kRankTiles>), blocks, threads, 0, s, p);
  else hipLaunchKernelGGL((tslt::adapt_down_many_kernel<T, kRankTiles>), blocks, threads, 0, s, p);
}
template <typename T, int kTokenTiles, bool kPacked> hipError_t launch_up(const tslt::AdaptParams& p, hipStream_t s) {
  const int lds = tslt::adapt_lds_bytes(p.R, kTokenTiles, kPacked);         // (64 KB of 64 tokens and 256 ranks)
  if (lds > 48 * 1024) {
    const hipError_t e = tslt::allow_dynamic_lds<&tslt::adapt_up_kernel<T, kTokenTiles, kPacked>>(64 * 1024);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((tslt::adapt_up_kernel<T, kTokenTiles, kPacked>), dim3(unsigned(p.B * p.up_tiles * p.splits)), dim3(tslt::kBlock), lds, s, p);
  return hipSuccess;
}
template <typename T> hipError_t launch_adapt(tslt::AdaptParams p, const Plan& plan, hipStream_t s) {
  p.tiles = plan.tiles; p.chunks = plan.chunks; p.cuts = plan.cuts; p.splits = plan.splits; p.up_tiles = plan.up_tiles;
  if (plan.rank_tiles == 1) launch_down<T, 1>(p, plan.token_tiles, s);
  else if (plan.rank_tiles == 2) launch_down<T, 2>(p, plan.token_tiles, s);
  else launch_down<T, 4>(p, plan.token_tiles, s);
  if (plan.up_token_tiles == 1) return p.R == 16 ? launch_up<T, 1, true>(p, s) : launch_up<T, 1, false>(p, s);
  if constexpr (sizeof(T) == 2)
    if (plan.up_token_tiles == 4) return p.R == 16 ? launch_up<T, 4, true>(p, s) : launch_up<T, 4, false>(p, s);
  return p.R == 16 ? launch_up<T, 2, true>(p, s) : launch_up<T, 2, false>(p, s);
}
constexpr int32_t kMostChannels = 1 << 28;                                 // (a row's bytes are counted in 32 bits)
bool sizes_fit(int64_t B, int32_t n, int32_t K, int32_t N, int32_t R) {
  return B >= 1 && n >= 1 && K >= 1 && N >= 1 && K <= kMostChannels && N <= kMostChannels && R >= 16 && R <= TSLT_MAX_ADAPTER_RANK && R % 16 == 0 && B <= 0x7FFFFFFF / n;
}

}  // namespace

extern "C" {

size_t tslt_adapt_workspace_bytes(int64_t B, int32_t n, int32_t K, int32_t N, int32_t R) {
  if (!sizes_fit(B, n, K, N, R)) return 0;
  return (size_t(plan_adapt(TSLT_F32, B, n, K, N, R).cuts) * size_t(B) * n * R * 4 + 255) / 256 * 256;
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
  if (K > kMostChannels || N > kMostChannels) return fail(TSLT_ERR_UNSUPPORTED, "%s: rows of K=%d, N=%d elements, %d at most", who, int(K), int(N), int(kMostChannels));
  if (n_adapters > 0x7FFFFFFF || B > 0x7FFFFFFF / n) return fail(TSLT_ERR_UNSUPPORTED, "%s: adapters and tokens must fit 31 bits", who);
  if (B == 0) return TSLT_OK;
  tslt_rows rx = x ? *x : tslt_rows{}, rb = base ? *base : tslt_rows{}, ro = out ? *out : tslt_rows{};
  rx.head_stride = rb.head_stride = ro.head_stride = 0;
  if (int e = check_rows(who, "x", &rx, dt)) return e;
  if (!rb.data || !ro.data) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(rb.data, elem_bytes(dt)) || !aligned(ro.data, elem_bytes(dt))) return fail(TSLT_ERR_INVALID_ARG, "%s: rows not aligned to their type", who);
  if (rb.data == ro.data && (rb.seq_stride != ro.seq_stride || rb.token_stride != ro.token_stride))
    return fail(TSLT_ERR_INVALID_ARG, "%s: rows that are added to in place must have the same strides", who);
  if (int e = check_distinct(who, "out", &ro, B, n, 1, N)) return e;
  if (!a || !b || !adapter) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(a, 16) || !aligned(b, 16)) return fail(TSLT_ERR_INVALID_ARG, "%s: adapters not aligned to 16 bytes", who);
  const Plan plan = plan_adapt(dt, B, n, K, N, R);
  const size_t need = tslt_adapt_workspace_bytes(B, n, K, N, R);
  if (!ws || !aligned(ws, 256) || ws_bytes < need)
    return fail(TSLT_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed, 256-byte aligned", who, ws ? ws_bytes : size_t(0), need);
  int code;
  if (!grid_fits(who, B * std::max<int64_t>(int64_t(plan.tiles) * plan.chunks * plan.cuts, int64_t(plan.up_tiles) * plan.splits), code, tslt::kBlock)) return code;
  tslt::AdaptParams p{};
  p.x = view(&rx); p.base = view(&rb); p.out = view(&ro);
  p.K = K; p.N = N; p.R = R; p.n = n; p.B = B; p.n_adapters = n_adapters; p.a = a; p.b = b; p.adapter = adapter; p.rank = rank; p.count = count;
  p.scale = scale; p.status = status; p.h = reinterpret_cast<float*>(ws); p.copy = rb.data != ro.data;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const hipError_t e = dt == TSLT_F32 ? launch_adapt<float>(p, plan, s) : dt == TSLT_BF16 ? launch_adapt<tslt::Bf16>(p, plan, s) : launch_adapt<tslt::F16>(p, plan, s);
  if (e != hipSuccess) return tslt::hip_fail(e, "hipFuncSetAttribute");
  return launched("tslt_adapt launch");
}

}  // extern "C"
