// C ABI of the 8-bit key/value cache (see include/tslt.h): argument checks, launch plans, kernel launches.
#include "tslt.h"

#include <algorithm>
#include <cmath>

#include "append.h"
#include "attend.h"
#include "checks.h"
#include "evict.h"
#include "weigh.h"

namespace {

using tslt::fail;

// What every call says of its cache and its sequences; 0 if the kernels can take it.
int check_cache(const char* who, const tslt_cache* c, const int32_t* pages, int64_t width, const int32_t* length, int64_t B) {
  if (!c) return fail(TSLT_ERR_INVALID_ARG, "%s: null cache", who);
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return fail(TSLT_ERR_UNSUPPORTED, "%s: head_dim must be 64, 128 or 256 (got %d)", who, int(c->head_dim));
  if (c->heads < 1 || c->n_pages < 1 || c->n_pages > 0x7FFFFFFF || B < 0 || width < 1)
    return fail(TSLT_ERR_INVALID_ARG, "%s: bad shape heads=%d n_pages=%lld B=%lld width=%lld", who, int(c->heads), (long long)c->n_pages, (long long)B, (long long)width);
  if (width > 0x7FFFFFFF / TSLT_PAGE_TOKENS) return fail(TSLT_ERR_UNSUPPORTED, "%s: a sequence's tokens must fit 31 bits", who);
  if (B == 0) return TSLT_OK;
  if (!c->codes || !c->scales || !pages || !length) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(c->codes, 16)) return fail(TSLT_ERR_INVALID_ARG, "%s: codes not aligned to 16 bytes", who);
  return TSLT_OK;
}
tslt::CacheView view(const tslt_cache* c, const int32_t* pages, int64_t width, const int32_t* length) {
  return tslt::CacheView{c->codes, c->scales, c->n_pages, int(c->heads), pages, width, length};
}
template <template <typename, int> class Launch, typename P> void by_type(tslt_dtype dt, int D, const P& p, unsigned blocks, hipStream_t s) {
#define TSLT_BY_D(T) (D == 64 ? Launch<T, 64>::go(p, blocks, s) : D == 128 ? Launch<T, 128>::go(p, blocks, s) : Launch<T, 256>::go(p, blocks, s))
  dt == TSLT_F32 ? TSLT_BY_D(float) : dt == TSLT_BF16 ? TSLT_BY_D(tslt::Bf16) : TSLT_BY_D(tslt::F16);
#undef TSLT_BY_D
}
// Calls of up to 16 tokens: a wave to a page and head, four heads to a workgroup.
constexpr int kFewTokens = 16;
template <typename T, int D> struct Append {
  static void go(const tslt::AppendParams& p, unsigned blocks, hipStream_t s) {
    if (p.most <= kFewTokens) hipLaunchKernelGGL((tslt::append_kernel<T, D, 64, kFewTokens>), dim3(blocks), dim3(256), 0, s, p);
    else hipLaunchKernelGGL((tslt::append_kernel<T, D, 256, tslt::kPage>), dim3(blocks), dim3(256), 0, s, p);
  }
};
template <typename T, int D> struct Weigh {
  template <int RT> static void tiles(const tslt::WeighParams& p, unsigned blocks, hipStream_t s) {
    hipLaunchKernelGGL((tslt::weigh_kernel<T, D, RT, 1>), dim3(blocks), dim3(256), 0, s, p);
  }
  static void go(const tslt::WeighParams& p, unsigned blocks, hipStream_t s) {
    constexpr int kMost = tslt::weigh_tiles<T, D>();
    const int64_t rows = int64_t(p.n) * p.group;
    // Many rows on few pages: a workgroup to a page, its waves share the rows.  us with a wave to a page / so, 14 sequences of 21 to 122 tokens, 12 heads: 2368
    // bfloat16 rows of 128 86 / 47, of 256 154 / 93, fp32 of 128 277 / 92; 164 rows 15.8 / 13.6, 23.3 / 24.0, 25.2 / 16.7; 80 rows of 256 17.9 / 21.5.  More pages: 2
    // sequences of 1000 to 4000 tokens, 8 heads, 600 rows 29.2 / 32.8, 16 of 4000 to 16000 410 / 498.
    const int64_t pages = std::min<int64_t>(p.B * p.c.heads, 1 << 20) * p.c.width;
    if (rows > 128 && pages <= 2 * int64_t(tslt::compute_units())) {
      constexpr int kShare = kMost > 1 ? kMost / 2 : 1;
      hipLaunchKernelGGL((tslt::weigh_kernel<T, D, kShare, 4>), dim3(unsigned(pages)), dim3(256), 0, s, p);
      return;
    }
    if (kMost == 1 || rows <= 16) return tiles<1>(p, blocks, s);
    if constexpr (kMost >= 2) if (kMost == 2 || rows <= 32) return tiles<2>(p, blocks, s);
    if constexpr (kMost == 4) return rows <= 48 ? tiles<3>(p, blocks, s) : tiles<4>(p, blocks, s);
  }
};

// How an attention call is cut: row groups, and chunks of a sequence's pages (what the host knows of lengths is the width of the page table; where sequences are
// much shorter than it most chunks are empty and the others long).  `slots` counts two workgroups to a compute unit.  Of D = 256, and of eight waves (fp32, D = 128,
// and 16 bits, D = 256, of more than 64 rows), one fits: a round of those is two.
//   Few rows.  Where the rows make fewer workgroups than fit the GPU, chunks fill it: twice over with 16 rows, so that whoever has ended early finds
//   more, once with 32, whose parts cost more to join.  us by one round of workgroups / two: 4 sequences of 131000 tokens 167 / 172.  Where there are
//   enough without, 16 rows are still cut in four, as sequences differ in length: 64 sequences of 100 to 8000 tokens, 8 heads, in one / four: 4 rows
//   112.6 / 106.0, 32 rows 123 / 134; all of 4050 tokens 93.9 / 96.1, 106 / 124.
//   Up to 64 rows, the same in one / two / four: 36 rows 205 / 188 / 179, of 4050 tokens 150 / 155 / 168: three.  (Of neither more than eight rounds
//   in all: sequences even out by their number then.)
//   More rows: what takes least, in pages, of rounds of workgroups and what a chunk costs beside its pages (2048 tokens on 16000, 512 workgroups
//   in one / two / four chunks: 818 / 915 / 903).
void plan_attend(tslt::AttendParams& p, bool f32, int D) {
  const int64_t rows = int64_t(p.n) * p.group;
  const tslt::AttendChoice choice = tslt::attend_choice(f32, D, rows);
  p.row_groups = int((rows + choice.rows - 1) / choice.rows);
  const int64_t units = p.B * p.c.heads * p.row_groups, slots = 2 * int64_t(tslt::compute_units());
  int64_t chunks = 1;
  if (choice.stream) {
    chunks = choice.rows == 32 ? slots / units : 2 * units > slots ? std::min<int64_t>(4, 8 * slots / units) : 2 * slots / units;
    chunks = std::max<int64_t>(1, std::min<int64_t>({chunks, (p.c.width + 15) / 16, 256}));
  } else {
    int64_t least = 0;
    for (int64_t n = 1; n <= std::max<int64_t>(1, std::min<int64_t>({256, (p.c.width + 7) / 8, 2 * slots / units})); ++n) {
      const int64_t cost = (units * n + slots - 1) / slots * ((p.c.width + n - 1) / n + (n > 1 ? 20 : 8));
      if (n == 1 || cost < least) { least = cost; chunks = n; }
    }
    if (choice.rows == 64 && 2 * units > slots) chunks = std::max(chunks, std::min<int64_t>({3, 6 * slots / units, (p.c.width + 15) / 16}));
  }
  p.chunk = int((p.c.width + chunks - 1) / chunks);
  p.chunks = int((p.c.width + p.chunk - 1) / p.chunk);
}
// The workspace: a word for each chunk of each row group, then the chunks' parts.
size_t attend_word_bytes(const tslt::AttendParams& p) { return (size_t(p.B) * p.c.heads * p.row_groups * p.chunks * 8 + 255) / 256 * 256; }
size_t attend_part_bytes(const tslt::AttendParams& p, int D) {
  if (p.chunks == 1) return 0;
  const size_t rows = size_t(p.B) * p.c.heads * p.chunks * p.n * p.group;
  return attend_word_bytes(p) + (rows * (D * 4 + 8) + 255) / 256 * 256;
}

}  // namespace

extern "C" {

int tslt_cache_append(const tslt_cache* cache, const int32_t* pages, int64_t width, const int32_t* length, int64_t B, int32_t n,
                      const tslt_rows* k, const tslt_rows* v, tslt_dtype dt, const int32_t* index, int32_t index_width, const int32_t* count,
                      int32_t* out_length, int32_t* status, void* stream) {
  const char* who = "tslt_cache_append";
  if (int e = check_cache(who, cache, pages, width, length, B)) return e;
  if (!valid_dtype(dt)) return fail(TSLT_ERR_INVALID_ARG, "%s: unknown dtype %d", who, int(dt));
  if (n < 1) return fail(TSLT_ERR_INVALID_ARG, "%s: n must be at least 1", who);
  if (index && index_width < 1) return fail(TSLT_ERR_INVALID_ARG, "%s: index_width must be at least 1", who);
  if (B == 0) return TSLT_OK;
  if (int e = check_rows(who, "k", k, dt)) return e;
  if (int e = check_rows(who, "v", v, dt)) return e;
  if (!out_length) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (out_length == length) return fail(TSLT_ERR_INVALID_ARG, "%s: out_length must not be length", who);
  tslt::AppendParams p{};
  p.c = view(cache, pages, width, length);
  p.k = view(k); p.v = view(v);
  p.B = B; p.n = n; p.index = index; p.count = count; p.out_length = out_length; p.status = status;
  p.most = index ? index_width : n;
  p.most_pages = int((int64_t(p.most) + tslt::kPage - 2) / tslt::kPage + 1);
  const int64_t heads_each = p.most <= kFewTokens ? 4 : 1, blocks = B * ((cache->heads + heads_each - 1) / heads_each) * p.most_pages;
  int code;
  if (!grid_fits(who, blocks, code)) return code;
  by_type<Append>(dt, cache->head_dim, p, unsigned(blocks), reinterpret_cast<hipStream_t>(stream));
  return launched("tslt_cache_append launch");
}

size_t tslt_cache_attend_workspace_bytes(int64_t B, int32_t n, int32_t heads_q, int32_t heads, int32_t head_dim, int64_t width) {
  if (B < 1 || n < 1 || heads < 1 || heads_q < heads || heads_q % heads || width < 1 || width > 0x7FFFFFFF / TSLT_PAGE_TOKENS) return 0;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
  tslt::AttendParams p{};
  p.B = B; p.n = n; p.group = heads_q / heads; p.c.heads = heads; p.c.width = width;
  size_t most = 0;
  for (const bool f32 : {false, true}) {
    plan_attend(p, f32, head_dim);
    most = std::max(most, attend_part_bytes(p, head_dim));
  }
  return most;
}

int tslt_cache_attend(const tslt_cache* cache, const int32_t* pages, int64_t width, const int32_t* length, int64_t B, int32_t n,
                      int32_t heads_q, const tslt_rows* q, const tslt_rows* k, const tslt_rows* v, tslt_dtype dt, const uint32_t* mask,
                      int64_t mask_seq_stride, const int32_t* count, float scale, void* out, float* out_lse, int32_t* status, void* ws,
                      size_t ws_bytes, void* stream) {
  const char* who = "tslt_cache_attend";
  if (int e = check_cache(who, cache, pages, width, length, B)) return e;
  if (!valid_dtype(dt)) return fail(TSLT_ERR_INVALID_ARG, "%s: unknown dtype %d", who, int(dt));
  if (n < 1) return fail(TSLT_ERR_INVALID_ARG, "%s: n must be at least 1", who);
  if (heads_q < cache->heads || heads_q % cache->heads) return fail(TSLT_ERR_INVALID_ARG, "%s: heads_q must be a multiple of the cache's heads", who);
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(TSLT_ERR_INVALID_ARG, "%s: scale must be > 0", who);
  if (int64_t(n) * (heads_q / cache->heads) > 0x3FFFFFFF) return fail(TSLT_ERR_UNSUPPORTED, "%s: too many rows", who);
  if (B == 0) return TSLT_OK;
  if (int e = check_rows(who, "q", q, dt)) return e;
  if ((k == nullptr) != (v == nullptr)) return fail(TSLT_ERR_INVALID_ARG, "%s: k and v come together", who);
  if (k) {
    if (int e = check_rows(who, "k", k, dt)) return e;
    if (int e = check_rows(who, "v", v, dt)) return e;
  }
  if (!out || !out_lse) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!aligned(out, 16)) return fail(TSLT_ERR_INVALID_ARG, "%s: out not aligned to 16 bytes", who);
  if (mask && mask_seq_stride < 0) return fail(TSLT_ERR_INVALID_ARG, "%s: mask_seq_stride must not be negative", who);
  tslt::AttendParams p{};
  p.c = view(cache, pages, width, length);
  p.q = view(q); p.k = view(k); p.v = view(v);
  p.B = B; p.n = n; p.group = heads_q / cache->heads; p.heads_q = heads_q;
  p.mask = mask; p.mask_seq = mask_seq_stride; p.mask_words = (n + 31) / 32; p.count = count;
  p.scale2 = float(double(scale) * 1.4426950408889634074);
  p.out = out; p.lse = out_lse; p.status = status;
  plan_attend(p, dt == TSLT_F32, cache->head_dim);
  const size_t need = attend_part_bytes(p, cache->head_dim);
  if (need > 0) {
    if (!ws || !aligned(ws, 256) || ws_bytes < need)
      return fail(TSLT_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu are needed, 256-byte aligned", who, ws ? ws_bytes : size_t(0), need);
    p.words = reinterpret_cast<uint64_t*>(ws);
    p.part_ml = p.words + attend_word_bytes(p) / 8;
    p.part_o = p.part_ml + size_t(B) * cache->heads * p.chunks * n * p.group;
    p.tag = tslt::next_tag();
  }
  int code;
  if (!grid_fits(who, (B * cache->heads * p.chunks + 8) * p.row_groups, code)) return code;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const hipError_t e = dt == TSLT_F32 ? tslt::launch_attend<float>(p, cache->head_dim, s)
                       : dt == TSLT_BF16 ? tslt::launch_attend<tslt::Bf16>(p, cache->head_dim, s) : tslt::launch_attend<tslt::F16>(p, cache->head_dim, s);
  if (e != hipSuccess) return tslt::hip_fail(e, "hipFuncSetAttribute");
  return launched("tslt_cache_attend launch");
}

int tslt_cache_weigh(const tslt_cache* cache, const int32_t* pages, int64_t width, const int32_t* length, int64_t B, int32_t n,
                     int32_t heads_q, const tslt_rows* q, tslt_dtype dt, const float* lse, const int32_t* count, float scale,
                     const float* weight, float decay, float* out_weight, int32_t* status, void* stream) {
  const char* who = "tslt_cache_weigh";
  if (int e = check_cache(who, cache, pages, width, length, B)) return e;
  if (!valid_dtype(dt)) return fail(TSLT_ERR_INVALID_ARG, "%s: unknown dtype %d", who, int(dt));
  if (n < 1) return fail(TSLT_ERR_INVALID_ARG, "%s: n must be at least 1", who);
  if (heads_q < cache->heads || heads_q % cache->heads) return fail(TSLT_ERR_INVALID_ARG, "%s: heads_q must be a multiple of the cache's heads", who);
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(TSLT_ERR_INVALID_ARG, "%s: scale must be > 0", who);
  if (!std::isfinite(decay)) return fail(TSLT_ERR_INVALID_ARG, "%s: decay must be finite", who);
  if (int64_t(n) * (heads_q / cache->heads) > 0x3FFFFFFF) return fail(TSLT_ERR_UNSUPPORTED, "%s: too many rows", who);
  if (B == 0) return TSLT_OK;
  if (int e = check_rows(who, "q", q, dt)) return e;
  if (!lse || !weight || !out_weight) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  tslt::WeighParams p{};
  p.c = view(cache, pages, width, length);
  p.q = view(q);
  p.B = B; p.n = n; p.group = heads_q / cache->heads; p.heads_q = heads_q; p.count = count; p.lse = lse;
  p.scale2 = float(double(scale) * 1.4426950408889634074);
  p.decay = decay; p.weight = weight; p.out_weight = out_weight; p.status = status;
  // One round of workgroups, two to a compute unit (of D = 256 one fits: two rounds), or a page to each wave.
  const int64_t blocks = std::min<int64_t>(2 * int64_t(tslt::compute_units()), (std::min<int64_t>(B * cache->heads, 1 << 20) * width + 3) / 4);
  by_type<Weigh>(dt, cache->head_dim, p, unsigned(blocks), reinterpret_cast<hipStream_t>(stream));
  return launched("tslt_cache_weigh launch");
}

int tslt_cache_evict(const tslt_cache* cache, const int32_t* pages, int64_t width, const int32_t* length, int64_t B, const float* weight,
                     int32_t keep, int32_t recent, const int32_t* new_pages, int64_t new_width, int32_t* out_length, int32_t* out_kept,
                     float* out_weight, int32_t* status, void* stream) {
  const char* who = "tslt_cache_evict";
  if (int e = check_cache(who, cache, pages, width, length, B)) return e;
  if (keep < 1 || recent < 0) return fail(TSLT_ERR_INVALID_ARG, "%s: keep must be at least 1, recent at least 0", who);
  if (new_width < (int64_t(keep) + tslt::kPage - 1) / tslt::kPage) return fail(TSLT_ERR_INVALID_ARG, "%s: %lld new pages a sequence do not hold %d tokens", who, (long long)new_width, int(keep));
  if (new_width > 0x7FFFFFFF / TSLT_PAGE_TOKENS) return fail(TSLT_ERR_UNSUPPORTED, "%s: a sequence's tokens must fit 31 bits", who);
  if (B == 0) return TSLT_OK;
  if (!weight || !new_pages || !out_length || !out_kept || !out_weight) return fail(TSLT_ERR_INVALID_ARG, "%s: null pointer", who);
  if (out_length == length) return fail(TSLT_ERR_INVALID_ARG, "%s: out_length must not be length", who);
  if (out_weight == weight) return fail(TSLT_ERR_INVALID_ARG, "%s: out_weight must not be weight", who);
  tslt::EvictParams p{};
  p.c = view(cache, pages, width, length);
  p.B = B; p.weight = weight; p.keep = keep; p.recent = recent; p.new_pages = new_pages; p.new_width = new_width;
  p.out_length = out_length; p.out_kept = out_kept; p.out_weight = out_weight; p.status = status;
  const int64_t heads = B * cache->heads, moves = heads * ((keep + tslt::kPage - 1) / tslt::kPage);
  int code;
  if (!grid_fits(who, std::max(heads, moves), code)) return code;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // (weights in registers where as many fit as the table has room for: 16 waves of 64 lanes)
  const auto select = width <= 64 ? tslt::evict_select_kernel<4> : width <= 512 ? tslt::evict_select_kernel<32> : tslt::evict_select_kernel<0>;
  hipLaunchKernelGGL(select, dim3(unsigned(heads)), dim3(tslt::kEvictThreads), 0, s, p);
  const auto move = cache->head_dim == 64 ? tslt::evict_move_kernel<64> : cache->head_dim == 128 ? tslt::evict_move_kernel<128> : tslt::evict_move_kernel<256>;
  hipLaunchKernelGGL(move, dim3(unsigned(moves)), dim3(256), 0, s, p);
  return launched("tslt_cache_evict launch");
}

}  // extern "C"
