// C ABI of the norms and rotation of queries and keys (see include/tslt.h): argument checks and launches.
#include "tslt.h"

#include <algorithm>
#include <cmath>

#include "checks.h"
#include "rotate.h"

namespace {

// Tokens of a workgroup: more of them have more angles to compute at once, fewer make more workgroups (64 x 21 tokens of 40 heads of 128, four / two 11.2 / 9.6 us).
int tokens_each(int64_t tokens) { return tokens <= int64_t(tslt::compute_units()) ? 1 : tokens <= 16 * int64_t(tslt::compute_units()) ? 2 : 4; }
// Backwards, where each goes on to others and keeps its share of the weights' gradients, three fit a compute unit (8 x 2048 tokens, 2 / 3 / 6 of them 130 / 108 / 115 us).
int tokens_back(int64_t tokens) { return tokens <= 4 * int64_t(tslt::compute_units()) ? 1 : 4; }
int64_t backward_blocks(int64_t tokens) {
  const int each = tokens_back(tokens);
  return std::min<int64_t>((tokens + each - 1) / each, 3 * int64_t(tslt::compute_units()));
}

template <typename T, int D, int kTokens> void launch_rotate_of(const tslt::RotateParams& p, hipStream_t s) {
  hipLaunchKernelGGL((tslt::rotate_kernel<T, D, kTokens>), dim3(unsigned((p.tokens + kTokens - 1) / kTokens)), dim3(tslt::kBlock), 0, s, p);
}
template <typename T, int D> void launch_rotate(const tslt::RotateParams& p, hipStream_t s) {
  const int each = tokens_each(p.tokens);
  each == 1 ? launch_rotate_of<T, D, 1>(p, s) : each == 2 ? launch_rotate_of<T, D, 2>(p, s) : launch_rotate_of<T, D, 4>(p, s);
}
template <int D> void launch_rotate_weights(const tslt::RotateParams& p, hipStream_t s) {
  hipLaunchKernelGGL((tslt::rotate_weights_kernel<D>), dim3(2 * D / 8), dim3(tslt::kBlock), 0, s, p);
}
template <typename T, int D> void launch_rotate_backward(const tslt::RotateParams& p, hipStream_t s) {
  if (tokens_back(p.tokens) == 1) hipLaunchKernelGGL((tslt::rotate_backward_kernel<T, D, 1>), dim3(unsigned(p.parts)), dim3(tslt::kBlock), 0, s, p);
  else hipLaunchKernelGGL((tslt::rotate_backward_kernel<T, D, 4>), dim3(unsigned(p.parts)), dim3(tslt::kBlock), 0, s, p);
  if (p.part) launch_rotate_weights<D>(p, s);
}

int check_rotation(const char* who, tslt_dtype dt, int64_t B, int32_t n, int32_t heads_q, int32_t heads, bool keys, int32_t D, const tslt_rotation* how) {
  if (!valid_dtype(dt)) return fail(TSLT_ERR_INVALID_ARG, "%s: unknown dtype %d", who, int(dt));
  if (D != 64 && D != 128 && D != 256) return fail(TSLT_ERR_UNSUPPORTED, "%s: head_dim must be 64, 128 or 256 (got %d)", who, int(D));
  if (B < 0 || n < 1 || heads_q < 1 || (keys && heads < 1))
    return fail(TSLT_ERR_INVALID_ARG, "%s: bad shape B=%lld n=%d heads_q=%d heads=%d", who, (long long)B, int(n), int(heads_q), int(heads));
  if (B > 0x7FFFFFFF / n) return fail(TSLT_ERR_UNSUPPORTED, "%s: the tokens of a call must fit 31 bits", who);
  if (heads_q > 0x3FFFFF || (keys && heads > 0x3FFFFF)) return fail(TSLT_ERR_UNSUPPORTED, "%s: too many heads", who);
  if (!how) return fail(TSLT_ERR_INVALID_ARG, "%s: null rotation", who);
  if (how->rotary < 0 || how->rotary > D || how->rotary % 16)
    return fail(TSLT_ERR_INVALID_ARG, "%s: rotary must be a multiple of 16 up to head_dim (got %d)", who, int(how->rotary));
  if (how->rotary > 0) {
    if (how->axes < 1 || how->axes > TSLT_MAX_AXES) return fail(TSLT_ERR_INVALID_ARG, "%s: axes must be 1 to %d (got %d)", who, TSLT_MAX_AXES, int(how->axes));
    if (!how->freq) return fail(TSLT_ERR_INVALID_ARG, "%s: null freq", who);
    if (how->position && how->position_seq_stride < 0) return fail(TSLT_ERR_INVALID_ARG, "%s: position_seq_stride must not be negative", who);
  }
  if (std::isnan(how->eps) || how->eps > 3.0e38f) return fail(TSLT_ERR_INVALID_ARG, "%s: eps must be a number, negative for no norm", who);
  if (how->eps < 0 && (how->q_weight || how->k_weight)) return fail(TSLT_ERR_INVALID_ARG, "%s: weights belong to a norm", who);
  return TSLT_OK;
}
bool same_rows(const tslt_rows* x, const tslt_rows* y) {
  return x->seq_stride == y->seq_stride && x->token_stride == y->token_stride && x->head_stride == y->head_stride;
}
tslt::RotateParams params(int64_t B, int32_t n, int32_t heads_q, int32_t heads, bool keys, const tslt_rotation* how, const int32_t* count, int32_t* status) {
  tslt::RotateParams p{};
  p.tokens = B * n; p.n = n; p.heads_q = heads_q; p.heads = keys ? heads : 0;
  p.position = how->position; p.position_seq = how->position_seq_stride; p.base = how->base; p.freq = how->freq; p.axis = how->axis;
  p.axes = how->axes; p.pairs = how->rotary / 2; p.adjacent = how->adjacent != 0; p.norm = how->eps >= 0; p.eps = how->eps;
  p.q_weight = how->q_weight; p.k_weight = how->k_weight; p.count = count; p.status = status;
  return p;
}
#define TSLT_BY_TYPE_AND_D(launch, dt, D, p, s)                                                                                                              \
  do {                                                                                                                                                       \
    if (dt == TSLT_F32) D == 64 ? launch<float, 64>(p, s) : D == 128 ? launch<float, 128>(p, s) : launch<float, 256>(p, s);                                  \
    else if (dt == TSLT_BF16) D == 64 ? launch<tslt::Bf16, 64>(p, s) : D == 128 ? launch<tslt::Bf16, 128>(p, s) : launch<tslt::Bf16, 256>(p, s);             \
    else D == 64 ? launch<tslt::F16, 64>(p, s) : D == 128 ? launch<tslt::F16, 128>(p, s) : launch<tslt::F16, 256>(p, s);                                     \
  } while (0)

}  // namespace

extern "C" {

int tslt_rotate(const tslt_rows* q, const tslt_rows* k, tslt_dtype dt, int64_t B, int32_t n, int32_t heads_q, int32_t heads, int32_t head_dim,
                const tslt_rotation* how, const int32_t* count, const tslt_rows* out_q, const tslt_rows* out_k, int32_t* status, void* stream) {
  const char* who = "tslt_rotate";
  if (int e = check_rotation(who, dt, B, n, heads_q, heads, k != nullptr, head_dim, how)) return e;
  if ((k == nullptr) != (out_k == nullptr)) return fail(TSLT_ERR_INVALID_ARG, "%s: k and out_k come together", who);
  if (B == 0) return TSLT_OK;
  if (int e = check_rows(who, "q", q, dt)) return e;
  if (int e = check_rows(who, "out_q", out_q, dt)) return e;
  if (int e = check_distinct(who, "out_q", out_q, B, n, heads_q, head_dim)) return e;
  if (k) {
    if (int e = check_rows(who, "k", k, dt)) return e;
    if (int e = check_rows(who, "out_k", out_k, dt)) return e;
    if (int e = check_distinct(who, "out_k", out_k, B, n, heads, head_dim)) return e;
  }
  if ((q->data == out_q->data && !same_rows(q, out_q)) || (k && k->data == out_k->data && !same_rows(k, out_k)))
    return fail(TSLT_ERR_INVALID_ARG, "%s: rows that are rotated in place must have the same strides", who);
  int code;
  if (!grid_fits(who, (B * n + tokens_each(B * n) - 1) / tokens_each(B * n), code, tslt::kBlock)) return code;
  tslt::RotateParams p = params(B, n, heads_q, heads, k != nullptr, how, count, status);
  p.q = view(q); p.k = view(k); p.out_q = view(out_q); p.out_k = view(out_k);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  TSLT_BY_TYPE_AND_D(launch_rotate, dt, head_dim, p, s);
  return launched("tslt_rotate launch");
}

size_t tslt_rotate_backward_workspace_bytes(int64_t B, int32_t n, int32_t heads_q, int32_t heads, int32_t head_dim) {
  (void)heads_q; (void)heads;
  if (B < 1 || n < 1 || B > 0x7FFFFFFF / n || (head_dim != 64 && head_dim != 128 && head_dim != 256)) return 0;
  return size_t(backward_blocks(B * n)) * 2 * head_dim * 4;
}

int tslt_rotate_backward(const tslt_rows* grad_q, const tslt_rows* grad_k, const tslt_rows* q, const tslt_rows* k, tslt_dtype dt, int64_t B, int32_t n,
                         int32_t heads_q, int32_t heads, int32_t head_dim, const tslt_rotation* how, const int32_t* count, const tslt_rows* out_q,
                         const tslt_rows* out_k, float* out_q_weight, float* out_k_weight, int32_t* status, void* ws, size_t ws_bytes, void* stream) {
  const char* who = "tslt_rotate_backward";
  if (int e = check_rotation(who, dt, B, n, heads_q, heads, grad_k != nullptr, head_dim, how)) return e;
  if ((grad_k == nullptr) != (out_k == nullptr)) return fail(TSLT_ERR_INVALID_ARG, "%s: grad_k and out_k come together", who);
  const bool norm = how->eps >= 0, weights = out_q_weight || out_k_weight;
  if (weights && !norm) return fail(TSLT_ERR_INVALID_ARG, "%s: weights belong to a norm", who);
  if (out_k_weight && !grad_k) return fail(TSLT_ERR_INVALID_ARG, "%s: out_k_weight without keys", who);
  if (B > 0) {
    if (int e = check_rows(who, "grad_q", grad_q, dt)) return e;
    if (int e = check_rows(who, "out_q", out_q, dt)) return e;
    if (int e = check_distinct(who, "out_q", out_q, B, n, heads_q, head_dim)) return e;
    if (norm)
      if (int e = check_rows(who, "q", q, dt)) return e;
    if (grad_k) {
      if (int e = check_rows(who, "grad_k", grad_k, dt)) return e;
      if (int e = check_rows(who, "out_k", out_k, dt)) return e;
      if (int e = check_distinct(who, "out_k", out_k, B, n, heads, head_dim)) return e;
      if (norm)
        if (int e = check_rows(who, "k", k, dt)) return e;
    }
    if ((grad_q->data == out_q->data && !same_rows(grad_q, out_q)) || (grad_k && grad_k->data == out_k->data && !same_rows(grad_k, out_k)))
      return fail(TSLT_ERR_INVALID_ARG, "%s: rows that are rotated in place must have the same strides", who);
  }
  tslt::RotateParams p = params(B, n, heads_q, heads, grad_k != nullptr, how, count, status);
  p.grad_q = view(grad_q); p.grad_k = view(grad_k); p.q = view(norm ? q : nullptr); p.k = view(norm ? k : nullptr); p.out_q = view(out_q); p.out_k = view(out_k);
  p.out_q_weight = out_q_weight; p.out_k_weight = out_k_weight;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (B > 0) {
    p.parts = int(backward_blocks(p.tokens));
    if (weights) {
      const size_t need = tslt_rotate_backward_workspace_bytes(B, n, heads_q, heads, head_dim);
      if (!ws || !aligned(ws, 256) || ws_bytes < need)
        return fail(TSLT_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed, 256-byte aligned", who, ws ? ws_bytes : size_t(0), need);
      p.part = reinterpret_cast<float*>(ws);
    }
    TSLT_BY_TYPE_AND_D(launch_rotate_backward, dt, head_dim, p, s);
  } else if (weights) {                    // no sequences: gradients of nothing
    head_dim == 64 ? launch_rotate_weights<64>(p, s) : head_dim == 128 ? launch_rotate_weights<128>(p, s) : launch_rotate_weights<256>(p, s);
  }
  return launched("tslt_rotate_backward launch");
}

}  // extern "C"
