// C ABI of log probabilities and their gradient (see include/tslt.h): argument checks, how rows are shared, launches.
#include "tslt.h"

#include <algorithm>

#include "checks.h"
#include "logprob.h"

namespace {

// Workgroups of a row: where rows are fewer than fill the GPU, shares of 8 KB and more.  Twice as many where there are rows for half of the compute units (5 likeliest of
// 16 x 9 rows of 128256 for 2 / 4 / 8 workgroups a unit 28.2 / 22.9 / 28.6 us, of 4 x 9 rows, whose join they delay, 15.9 / 17.5 / 18.4).
int shares(int64_t entries, int64_t V, int bytes) {
  const int64_t cus = tslt::compute_units(), fill = (2 * entries >= cus ? 4 : 2) * cus, most = std::min<int64_t>(64, V * bytes / 8192);
  return int(std::max<int64_t>(1, std::min<int64_t>(most, fill / std::max<int64_t>(entries, 1))));
}
// Of the gradient, which leaves nothing to join, more: rows that do not count are only filled, so that shares take unequal times (8 x 256 rows of 128256, two thirds
// of which count, with 2 / 8 / 16 / 32 / 64 workgroups a compute unit 173 / 173 / 151 / 147 / 148 us, all counting 217 / 214 / 209 / 203 / 204).
int shares_back(int64_t entries, int64_t V, int bytes) {
  const int64_t fill = 32 * int64_t(tslt::compute_units()), most = std::min<int64_t>(64, V * bytes / 16384);
  return int(std::max<int64_t>(1, std::min<int64_t>(most, (fill + entries - 1) / std::max<int64_t>(entries, 1))));
}
size_t word_bytes(int64_t entries, int slices) { return (size_t(entries) * slices * 8 + 255) / 256 * 256; }
size_t shared_bytes(int64_t entries, int slices) { return slices == 1 ? 0 : word_bytes(entries, slices) + size_t(entries) * slices * tslt::kPartWords * 8; }

int check_logits(const char* who, tslt_dtype dt, int64_t B, int32_t n, int64_t V, float temperature, int32_t top) {
  if (!valid_dtype(dt)) return fail(TSLT_ERR_INVALID_ARG, "%s: unknown dtype %d", who, int(dt));
  if (B < 0 || n < 1 || V < 1) return fail(TSLT_ERR_INVALID_ARG, "%s: bad shape B=%lld n=%d V=%lld", who, (long long)B, int(n), (long long)V);
  if (V > 0x7FFFFFFF || V * elem_bytes(dt) >= (int64_t(1) << 32)) return fail(TSLT_ERR_UNSUPPORTED, "%s: a row must be shorter than 4 GiB", who);
  if (B > 0x7FFFFFFF / n) return fail(TSLT_ERR_UNSUPPORTED, "%s: the rows of a call must fit 31 bits", who);
  if (!(temperature > 0.0f) || !(1.0f / temperature > 0.0f) || !(1.0f / temperature < 1.0e38f))
    return fail(TSLT_ERR_INVALID_ARG, "%s: temperature must be > 0", who);
  if (top < 0 || top > TSLT_MAX_TOP) return fail(TSLT_ERR_UNSUPPORTED, "%s: top must be 0 to %d (got %d)", who, TSLT_MAX_TOP, int(top));
  return TSLT_OK;
}
// Many short rows: a wave to each, with nothing to wait for between waves (us with four waves / one, binary16 rows with 5 likeliest: 25000 rows of 2200 logits 144 / 60, 6000 of
// 8000 39 / 33, 6000 of 16000 66 / 54, of 32000 87 / 86; fewer rows leave too few waves: 1500 of 2200 13.1 / 9.7, of 8000 13.9 / 19.1, 2304 of 32000 41 / 52).
bool one_wave(int64_t entries, int64_t bytes) {
  const int64_t cus = tslt::compute_units();
  return (entries >= 8 * cus && bytes <= 32768) || (entries >= 4 * cus && bytes <= 8192);
}
template <typename T> void launch_logprob(const tslt::LogprobParams& p, bool one, unsigned blocks, hipStream_t s) {
  if (one) hipLaunchKernelGGL((tslt::logprob_kernel<T, 1>), dim3(blocks), dim3(64), 0, s, p);
  else hipLaunchKernelGGL((tslt::logprob_kernel<T, tslt::kLogprobWaves>), dim3(blocks), dim3(64 * tslt::kLogprobWaves), 0, s, p);
}
float exponent_scale(float rT) { return float(double(rT) * 1.4426950408889634074); }

}  // namespace

extern "C" {

size_t tslt_logprob_workspace_bytes(int64_t B, int32_t m, int64_t V, int32_t top) {
  if (B < 1 || m < 1 || V < 1 || top < 0 || top > TSLT_MAX_TOP || B > 0x7FFFFFFF / m) return 0;
  return std::max(shared_bytes(B * m, shares(B * m, V, 2)), shared_bytes(B * m, shares(B * m, V, 4)));
}

int tslt_logprob(const void* logits, tslt_dtype dt, int64_t B, int32_t n, int64_t V, int64_t seq_stride, int64_t row_stride, float temperature,
                 const int32_t* index, int32_t m, const int32_t* count, const int32_t* tokens, int32_t top, float* out_logp, float* out_entropy,
                 float* out_lse, int32_t* out_top_idx, float* out_top_logp, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "tslt_logprob";
  if (int e = check_logits(who, dt, B, n, V, temperature, top)) return e;
  if (m < 1 || (!index && m != n)) return fail(TSLT_ERR_INVALID_ARG, "%s: m must be at least 1, and n without index (got %d, %d)", who, int(m), int(n));
  if (B > 0x7FFFFFFF / m) return fail(TSLT_ERR_UNSUPPORTED, "%s: the entries of a call must fit 31 bits", who);
  if (B == 0) return TSLT_OK;
  if (!logits) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(logits, elem_bytes(dt))) return fail(TSLT_ERR_INVALID_ARG, "%s: logits not aligned to their type", who);
  if (top > 0 && (!out_top_idx || !out_top_logp)) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  tslt::LogprobParams p{};
  p.logits = logits; p.seq_stride = seq_stride; p.row_stride = row_stride; p.V = V;
  p.rT = 1.0f / temperature; p.k2 = exponent_scale(p.rT);
  p.B = B; p.n = n; p.m = m; p.top = top; p.index = index; p.count = count; p.tokens = tokens;
  p.logp = out_logp; p.entropy = out_entropy; p.lse = out_lse; p.top_idx = out_top_idx; p.top_logp = out_top_logp; p.status = status;
  const int64_t entries = B * m;
  p.slices = shares(entries, V, elem_bytes(dt));
  const size_t need = shared_bytes(entries, p.slices);
  if (need > 0) {
    if (!ws || !aligned(ws, 256) || ws_bytes < need)
      return fail(TSLT_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed, 256-byte aligned", who, ws ? ws_bytes : size_t(0), need);
    p.words = reinterpret_cast<uint64_t*>(ws);
    p.part = p.words + word_bytes(entries, p.slices) / 8;
    p.tag = tslt::next_tag();
  }
  int code;
  const bool one = one_wave(entries, V * elem_bytes(dt));
  if (!grid_fits(who, entries * p.slices, code, one ? 64 : 64 * tslt::kLogprobWaves)) return code;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const unsigned blocks = unsigned(entries * p.slices);
  dt == TSLT_F32 ? launch_logprob<float>(p, one, blocks, s) : dt == TSLT_BF16 ? launch_logprob<tslt::Bf16>(p, one, blocks, s) : launch_logprob<tslt::F16>(p, one, blocks, s);
  return launched("tslt_logprob launch");
}

int tslt_logprob_backward(const void* logits, tslt_dtype dt, int64_t B, int32_t n, int64_t V, int64_t seq_stride, int64_t row_stride, float temperature,
                          const int32_t* count, const int32_t* tokens, const float* lse, const float* entropy, const int32_t* top_idx, int32_t top,
                          const float* grad_logp, const float* grad_entropy, const float* grad_lse, const float* grad_top, void* out,
                          int64_t out_seq_stride, int64_t out_row_stride, void* stream) {
  const char* who = "tslt_logprob_backward";
  if (int e = check_logits(who, dt, B, n, V, temperature, top)) return e;
  if (B == 0) return TSLT_OK;
  if (!logits || !lse || !out) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(logits, elem_bytes(dt)) || !aligned(out, elem_bytes(dt))) return fail(TSLT_ERR_INVALID_ARG, "%s: logits not aligned to their type", who);
  if (grad_logp && !tokens) return fail(TSLT_ERR_INVALID_ARG, "%s: grad_logp needs tokens", who);
  if (grad_entropy && !entropy) return fail(TSLT_ERR_INVALID_ARG, "%s: grad_entropy needs entropy", who);
  if (grad_top && (!top_idx || top < 1)) return fail(TSLT_ERR_INVALID_ARG, "%s: grad_top needs top_idx", who);
  const tslt_rows made{out, out_seq_stride, out_row_stride, 0};
  if (int e = check_distinct(who, "out", &made, B, n, 1, V)) return e;
  if (out == logits && (seq_stride != out_seq_stride || row_stride != out_row_stride))
    return fail(TSLT_ERR_INVALID_ARG, "%s: logits that are written over must have the same strides", who);
  tslt::LogprobBackwardParams p{};
  p.logits = logits; p.out = out; p.seq_stride = seq_stride; p.row_stride = row_stride; p.out_seq_stride = out_seq_stride; p.out_row_stride = out_row_stride;
  p.V = V; p.rT = 1.0f / temperature; p.k2 = exponent_scale(p.rT); p.n = n; p.top = grad_top ? top : 0;
  p.count = count; p.tokens = tokens; p.top_idx = top_idx; p.lse = lse; p.entropy = entropy;
  p.grad_logp = grad_logp; p.grad_entropy = grad_entropy; p.grad_lse = grad_lse; p.grad_top = grad_top;
  p.slices = shares_back(B * n, V, elem_bytes(dt));
  int code;
  if (!grid_fits(who, B * n * p.slices, code, tslt::kBlock)) return code;
  const auto kernel = dt == TSLT_F32 ? tslt::logprob_backward_kernel<float> : dt == TSLT_BF16 ? tslt::logprob_backward_kernel<tslt::Bf16> : tslt::logprob_backward_kernel<tslt::F16>;
  hipLaunchKernelGGL(kernel, dim3(unsigned(B * n * p.slices)), dim3(tslt::kBlock), 0, reinterpret_cast<hipStream_t>(stream), p);
  return launched("tslt_logprob_backward launch");
}

}  // extern "C"
