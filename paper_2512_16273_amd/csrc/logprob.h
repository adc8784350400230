// tslt_logprob: of rows of logits the normaliser, a token's log probability, the entropy and the likeliest tokens, in one pass; and the gradient of
// the logits.
//
// With k = log2(e) / T and a reference c of the row's logits (the largest that a wave has met), a term is e_j = 2^(k z_j - fl(k c)), one multiply-add and
// one exponential; S = sum e_j and E = sum e_j log2 e_j.  Then, with rho = k c - fl(k c) (taken back in fp64 where terms are added up), lse = c / T + ln S - rho ln 2
// and H = ln S - ln 2 E / S.  A wave whose logits pass its reference takes the larger one: S 2^d and 2^d (E + d S), d < 0 the difference of the two fl(k c).
//
// The `top` largest: each wave keeps a list in LDS of the logits above a threshold that `top` of the row's logits are known to reach.  At first that are the largest
// logits of the workgroup's lanes in the first loads: `top` of those 256 numbers are reached by as many logits, and by few more.  Whenever four times as much of the row has been
// met the waves put their lists together, cut what they have to `top`, and take the least of them as threshold, so that between two of these
// some three times `top` logits are listed (256 x 9 bfloat16 rows of 128256 with 20 of them 117 us, 122 twice as often).  A logit costs no more than its share of a comparison a load, which the reference needs as well.
//
// Few rows: several workgroups to a row, whose sums and lists the last of them to end joins (handover.h).  What it joins goes by a threshold from the waves' largest
// logits again.
//
// Bound by memory, of 16-bit rows with vector instructions close behind (11 a logit: unpacking, multiply-add, exponential, two sums, a share of the largest).  bfloat16, 256 x 9
// rows of 128256: 99 us (6.0 TB/s) with none of the likeliest, 104 with 5, 116 with 20; fp32, half as many rows 95.  9 rows 8.1 us with none, 13.8 with 5, 15 with 20: the launch, the row's way
// through memory, the hand-over, and two thresholds, lists and sorts one after the other.
#pragma once
#include "handover.h"
#include "rows.h"

namespace tslt {

constexpr int kMaxTop = 32;
constexpr int kListRoom = 128;           // records of a wave's list
constexpr int kLogprobWaves = 4;         // of a workgroup; short rows have one
constexpr int kPartHead = 4 + kLogprobWaves / 2, kPartWords = kPartHead + 64;

struct LogprobParams {
  const void* logits;
  int64_t seq_stride, row_stride, V;
  float rT, k2;                          // fl(1 / T), fl(log2(e) / T)
  int64_t B;
  int n, m, top;
  const int32_t *index, *count, *tokens;
  float *logp, *entropy, *lse, *top_logp;
  int32_t *top_idx, *status;
  int slices;                            // workgroups of a row, 64 at most
  uint64_t* words;                       // [entries][slices]
  uint64_t* part;                        // [entries][slices][kPartWords]: reference, S, E, length of the list, the waves' largest logits, the list
  Tag tag;
};

// A wave's list of candidate records (make_cand): value descending, index ascending; they lie in no order.
struct List {
  uint64_t* at;                          // kListRoom records of LDS
  int n;                                 // the same in all lanes, as are the thresholds
  float above;                           // nothing that is not greater than this can be among the `top`
  uint64_t least;                        // nor a record that is less than this
};

// The largest number that `top` of the records reach, a bit at a time (there are more than `top` of them; 0 stands for none).
template <int N> __device__ __forceinline__ uint64_t least_of_top(const uint64_t (&r)[N], int top) {
  // values' leading bits that all have in common
  uint32_t most = 0, low = 0xFFFFFFFFu;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    most = max(most, uint32_t(r[i] >> 32));
    low = min(low, r[i] != 0 ? uint32_t(r[i] >> 32) : 0xFFFFFFFFu);
  }
  most = wave_max_u32(most);
  low = ~wave_max_u32(~low);
  const int same = most == low ? 32 : __builtin_clz(most ^ low);
  uint64_t least = same == 0 ? 0 : uint64_t(most >> (32 - same)) << (64 - same);
  for (int bit = 63 - same; bit >= 0; --bit) {
    const uint64_t trial = least | uint64_t(1) << bit;
    int reach = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) reach += __popcll(ballot(r[i] >= trial));
    if (reach >= top) least = trial;
    if (reach == top) break;
  }
  return least;
}
// Those records that reach `least` to `to`, in no order; how many.
template <int N> __device__ __forceinline__ int keep_from(const uint64_t (&r)[N], uint64_t least, uint64_t* to) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool mine = r[i] != 0 && r[i] >= least;
    const uint64_t keep = ballot(mine);
    if (mine) to[n + lanes_below(keep)] = r[i];
    n += __popcll(keep);
  }
  return n;
}
// The least of `top` records as a number that all of them reach and nothing between it and the least one is.
template <int N> __device__ __forceinline__ uint64_t least_record(const uint64_t (&r)[N], uint64_t least) {
  uint32_t hi = 0xFFFFFFFFu;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (r[i] != 0 && r[i] >= least) hi = min(hi, uint32_t(r[i] >> 32));
  hi = ~wave_max_u32(~hi);
  return max(least, uint64_t(hi) << 32);
}

// The wave's list cut down to its `top` largest records.
__device__ __forceinline__ void cut(List& l, int top) {
  wave_sync();
  if (l.n <= top) return;
  const int lane = lane_id();
  uint64_t r[kListRoom / 64];
#pragma unroll
  for (int i = 0; i < kListRoom / 64; ++i) r[i] = lane + 64 * i < l.n ? l.at[lane + 64 * i] : 0;
  const uint64_t least = least_of_top(r, top);
  wave_sync();
  l.n = keep_from(r, least, l.at);
  l.least = least_record(r, least);
  l.above = fmaxf(l.above, cand_value(l.least));
  wave_sync();
}
// Records of those lanes that have one.
__device__ __forceinline__ void offer(List& l, bool mine, uint64_t record, int top) {
  const uint64_t who = ballot(mine);
  if (who == 0) return;
  if (l.n > kListRoom - 64) cut(l, top);
  if (mine) l.at[l.n + lanes_below(who)] = record;
  l.n += __popcll(who);
}
// A threshold from N numbers a lane: `top` of them are greater.  (-inf if there are not so many; 16 bits of it, so that it is some 1 % low.)
template <int N> __device__ __forceinline__ float reached_by(const float (&largest)[N], int top) {
  uint32_t key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) key[i] = mono_key(largest[i] + 0.0f) >> 16;
  uint32_t least = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t trial = least | 1u << bit;
    int reach = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) reach += __popcll(ballot(key[i] >= trial));
    if (reach >= top) least = trial;
  }
  least <<= 16;
  // the number before it (before both zeros, which are equal)
  return least > kKeyNegInf ? key_to_f32(least == 0x80000000u ? least - 2 : least - 1) : -INFINITY;
}

// Sums of a wave or of more: reference (raw logit), rho, S and E as above.
struct RowSums { float c; double rho, S, E; };
// Those of a wave's lanes, with one reference and no rho.  (What has nothing has S = 0.)
__device__ __forceinline__ RowSums join(const RowSums& x, double k2) {
  RowSums r{wave_max_f32(x.c), 0.0, 0.0, 0.0};
  const double d = (x.c == r.c ? 0.0 : k2 * (double(x.c) - double(r.c))) - x.rho;
  const double f = fast_exp2(float(d));
  double sum[2] = {x.S == 0.0 ? 0.0 : f * x.S, x.S == 0.0 || f == 0.0 ? 0.0 : f * (x.E + d * x.S)};
  wave_sums_f64<2>(sum);
  r.S = sum[0];
  r.E = sum[1];
  return r;
}

// What a wave has of a row.
struct RowWave {
  float c = -INFINITY, kc = 0.0f;        // reference, fl(k c)
  float S = 0.0f, E = 0.0f;
  bool far = false;                      // k c is too large for rho to be small: differences are taken first
  List list;
  // A vector's terms, added up by themselves first; nothing of what is -inf.
  template <int N> __device__ __forceinline__ void terms(const float (&z)[N], float k2) {
    if (same_in_wave(far)) add<N, true>(z, k2);
    else add<N, false>(z, k2);
  }
  template <int N, bool kFar> __device__ __forceinline__ void add(const float (&z)[N], float k2) {
    float s[N], t[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float d = kFar ? (z[e] - c) * k2 : fmaf(z[e], k2, -kc);
      s[e] = fast_exp2(d);
      const float u = fmaxf(d, -200.0f);                 // (2^-200 is 0, and 0 times a number is 0)
      t[e] = e < N / 2 || N == 1 ? s[e] * u : fmaf(s[e], u, t[e - N / 2]);
    }
#pragma unroll
    for (int w = N / 2; w > 0; w /= 2)
#pragma unroll
      for (int e = 0; e < w; ++e) {
        s[e] += s[e + w];
        if (w < N / 2) t[N / 2 + e] += t[N / 2 + e + w];
      }
    S += s[0];
    E += t[N / 2];
  }
  // A term is 2^(k z - k c + rho), rho = k c - fl(k c) of the reference that it met (0 where differences are taken first): what a new one changes is both.
  __device__ __forceinline__ void refer(float most, float k2) {
#pragma clang fp contract(off)           // (kc - now is of the rounded products)
    const float now = most * k2;
    const bool now_far = !(fabsf(now) < 4194304.0f);
    if (c != -INFINITY) {
      float d = kc - now;
      if (same_in_wave(far || now_far)) d = (c - most) * k2 + ((now_far ? 0.0f : fmaf(most, k2, -now)) - (far ? 0.0f : fmaf(c, k2, -kc)));
      const float f = fast_exp2(d);
      E = f > 0.0f ? f * fmaf(d, S, E) : 0.0f;
      S = f * S;
    }
    c = most;
    kc = now;
    far = now_far;
  }
};

template <int W> struct LogprobShared {
  uint64_t list[W][kListRoom];
  double rho[W], S[W], E[W];
  float c[W];
  float largest[64 * W];
  int n[W];
  uint64_t least;
  int told, mine;
};

// The waves' lists put together and cut down to `top` records, or to 64 at most if they need not be the least; the first wave's list then has them.  All threads.
template <bool kLast, int W> __device__ __forceinline__ void put_together(List& l, int top, LogprobShared<W>& sh) {
  const int wave = wave_id(), lane = lane_id();
  if (l.n > 64) cut(l, top);
  if (lane == 0) sh.n[wave] = l.n;
  __syncthreads();
  if (wave == 0) {
    uint64_t r[W];
    int total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int n = sh.n[w];
      r[w] = lane < n ? sh.list[w][lane] : 0;
      total += n;
    }
    uint64_t least = 0;
    if (total > (kLast ? 64 : top)) least = least_of_top(r, top);
    wave_sync();
    l.n = keep_from(r, least, l.at);
    if constexpr (kLast) return;
    if (total >= top) least = least_record(r, least);
    if (lane == 0) sh.least = least;
  } else {
    l.n = 0;
  }
  if constexpr (kLast) return;
  __syncthreads();
  l.least = sh.least;
  if (l.least != 0) l.above = fmaxf(l.above, cand_value(l.least));
}

// Values of a vector's elements that lie past the row's end: -inf, which adds nothing and is never chosen.
template <typename T> __device__ __forceinline__ uint4 row_vector(const uint4* body, int64_t v, int64_t end) {
  return v < end ? load_vec_stream(body + v) : neg_inf_vec<T>();
}

template <int E> __device__ __forceinline__ float largest_of(const float (&z)[E]) {
  const float most = max3f(z[0], z[1], z[2]);
  if constexpr (E == 4) return fmaxf(most, z[3]);
  else return max3f(max3f(most, z[3], z[4]), max3f(z[5], z[6], z[7]), most);
}

// Those of a vector's numbers that are greater than `above`.
template <int E> __device__ __forceinline__ void list_vector(List& l, const float (&z)[E], float above, uint32_t first, int top) {
  uint64_t who[E];
  int all = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    who[e] = ballot(z[e] > above);
    all += __popcll(who[e]);
  }
  if (l.n + all <= kListRoom) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (who[e] != 0) {
        if (z[e] > above) l.at[l.n + lanes_below(who[e])] = make_cand(z[e], first + e);
        l.n += __popcll(who[e]);
      }
    return;
  }
#pragma unroll 1
  for (int i = 0; i < E; ++i) {                          // (rare: one place in the code for all of them)
    float x = z[0];
#pragma unroll
    for (int e = 1; e < E; ++e) x = i == e ? z[e] : x;
    offer(l, x > above, make_cand(x, first + i), top);
  }
}

// All lanes of a wave: their vector's numbers, of indices first .. first + E - 1.  (A vector's numbers are not met in their order: what is offered
// goes by the threshold from before it, which all of those behind its numbers have reached with lower indices.)
template <typename T> __device__ __forceinline__ void take(RowWave& w, const uint4& x, int64_t first, float k2, int top) {
  constexpr int E = ElemTraits<T>::kPerVec;
  float z[E];
  unpack<T>(x, z);
  const float most = largest_of(z), above = w.list.above;
  if (ballot(most > fminf(above, w.c)) != 0) {
    if (ballot(most > w.c) != 0) w.refer(wave_max_f32(fmaxf(most, w.c)), k2);
    if (top == 0) w.list.above = w.c;
    else list_vector(w.list, z, above, uint32_t(first), top);
  }
  w.terms(z, k2);
}

constexpr int kAhead = 4;                // vectors of a lane that are asked for together

// A workgroup's share of a row: its waves' sums in LDS, and the likeliest in the first wave's list.
template <typename T, int W> __device__ void row_share(const void* row, const LogprobParams& p, int slice, LogprobShared<W>& sh, List& list) {
  constexpr int E = ElemTraits<T>::kPerVec, kThreads = 64 * W, kRound = kThreads * kAhead;
  const int wave = wave_id(), lane = lane_id(), top = p.top;
  const RowSplit rs = split_row<T>(row, p.V);
  const int64_t each = (rs.nvec + p.slices - 1) / p.slices, begin = min(each * slice, rs.nvec), end = min(begin + each, rs.nvec);
  RowWave w;
  w.list = List{sh.list[wave], 0, -INFINITY, 0};
  // numbers before the aligned ones are the row's first, those behind them its last: equal numbers are met in their order
  const auto edge = [&](int from, int to) {
    const bool mine = from + lane < to;
    const int64_t i = edge_index<T>(rs, mine ? from + lane : from);
    const float z = mine ? load_elem<T>(row, i) : -INFINITY, most = wave_max_f32(z);
    if (most > w.c) w.refer(most, p.k2);
    if (top > 0) offer(w.list, z > w.list.above, make_cand(z, uint32_t(i)), top);
    const float one[1] = {z};
    w.terms(one, p.k2);
  };
  if (slice == 0 && wave == 0 && rs.head > 0) edge(0, rs.head);
  uint4 x[kAhead];
  int64_t v = begin + wave * 64 + lane;
#pragma unroll
  for (int u = 0; u < kAhead; ++u) x[u] = row_vector<T>(rs.body, v + u * kThreads, end);
  {
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      float z[E];
      unpack<T>(x[u], z);
      most = fmaxf(most, largest_of(z));
    }
    const float all = wave_max_f32(fmaxf(most, w.c));
    if (all > w.c) w.refer(all, p.k2);
    if (top == 0) {
      w.list.above = w.c;
    } else {
      sh.largest[threadIdx.x] = most;
      __syncthreads();
      float largest[W];
#pragma unroll
      for (int i = 0; i < W; ++i) largest[i] = sh.largest[64 * i + lane];
      w.list.above = fmaxf(w.list.above, reached_by(largest, top));
    }
  }
  int round = 0, together = 4;
  for (int64_t v0 = begin; v0 < end; v0 += kRound, v += kRound) {
    uint4 next[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) next[u] = row_vector<T>(rs.body, v + kRound + u * kThreads, end);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) take<T>(w, x[u], rs.head + (v + u * kThreads) * E, p.k2, top);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) x[u] = next[u];
    if (top > 0 && ++round == together && v0 + 2 * kRound < end) {
      put_together<false, W>(w.list, top, sh);
      together = 4 * round;
    }
  }
  if (slice == p.slices - 1 && wave == 0 && rs.tail > 0) edge(rs.head, rs.head + rs.tail);
  double sum[2] = {double(w.S), double(w.E)};
  wave_sums_f64<2>(sum);
  if (lane == 0) {
    sh.rho[wave] = w.far || w.c == -INFINITY ? 0.0 : double(p.k2) * double(w.c) - double(w.kc);
    sh.S[wave] = sum[0];
    sh.E[wave] = sum[1];
    sh.c[wave] = w.c;
  }
  list = w.list;
  if (top > 0) put_together<true, W>(list, top, sh);
  else __syncthreads();
}

// The first wave: the sums of all.
template <int W> __device__ __forceinline__ RowSums all_waves(const LogprobShared<W>& sh, double k2) {
  const int w = min(lane_id(), W - 1);
  RowSums mine{sh.c[w], sh.rho[w], sh.S[w], sh.E[w]};
  if (lane_id() >= W) mine = RowSums{-INFINITY, 0.0, 0.0, 0.0};
  return join(mine, k2);
}

// The first wave: the results of an entry, from its row's sums and the list.
__device__ __forceinline__ void finish(const LogprobParams& p, int64_t entry, int32_t token, float z, const RowSums& sums, int status, const List& list) {
  const int lane = lane_id(), top = p.top;
  status |= sums.S != sums.S || sums.c == INFINITY ? 1 : sums.c == -INFINITY ? 2 : 0;
  const bool usable = (status & 3) == 0, there = token >= 0 && token < p.V;
  // (log probabilities from differences to the reference: of logits near fp32's largest the normaliser has no room for ln S)
  const double rT = p.rT, c = sums.c, ln_S = log(sums.S);
  if (!there && token != -1) status |= kBadIndex;
  if (lane == 0) {
    if (p.logp) p.logp[entry] = there && usable ? float((double(z) - c) * rT - ln_S) : NAN;
    if (p.entropy) p.entropy[entry] = usable ? float(fmax(ln_S - 0.69314718055994530942 * sums.E / sums.S, 0.0)) : NAN;
    if (p.lse) p.lse[entry] = usable ? float(c * rT + ln_S) : status & 1 ? NAN : -INFINITY;
    if (p.status) p.status[entry] = status;
  }
  if (top == 0) return;
  // a record's place is how many are larger
  const int n = usable ? list.n : 0;
  const uint64_t mine = lane < n ? list.at[lane] : 0;
  int place = 0;
  for (int i = 0; i < n; ++i) {
    const uint64_t other = uint64_t(uint32_t(__builtin_amdgcn_readlane(int(mine >> 32), i))) << 32 | uint32_t(__builtin_amdgcn_readlane(int(mine), i));
    place += other > mine ? 1 : 0;
  }
  if (lane < n && place < top) {
    p.top_idx[entry * top + place] = int32_t(cand_index(mine));
    p.top_logp[entry * top + place] = float((double(cand_value(mine)) - c) * rT - ln_S);
  }
  if (lane >= n && lane < top) {
    p.top_idx[entry * top + lane] = -1;
    p.top_logp[entry * top + lane] = -INFINITY;
  }
}

// An entry whose row cannot be used.
__device__ __forceinline__ void refuse(const LogprobParams& p, int64_t entry, int status) {
  const int tid = threadIdx.x;
  if (tid == 0) {
    if (p.logp) p.logp[entry] = NAN;
    if (p.entropy) p.entropy[entry] = NAN;
    if (p.lse) p.lse[entry] = NAN;
    if (p.status) p.status[entry] = status;
  }
  if (tid < p.top) {
    p.top_idx[entry * p.top + tid] = -1;
    p.top_logp[entry * p.top + tid] = -INFINITY;
  }
}

template <typename T, int W>
__global__ __launch_bounds__(64 * W) void logprob_kernel(const LogprobParams p) {
  __shared__ LogprobShared<W> sh;
  const int tid = threadIdx.x, wave = wave_id(), lane = lane_id();
  const uint32_t entry = blockIdx.x / uint32_t(p.slices);
  const int slice = int(blockIdx.x - entry * uint32_t(p.slices));
  const uint32_t b = entry / uint32_t(p.m);
  const int j = int(entry - b * uint32_t(p.m));
  // (asked for together)
  const int named = p.count ? as_global(p.count)[b] : p.m, at = p.index ? as_global(p.index)[entry] : j;
  const int32_t token = p.tokens ? as_global(p.tokens)[entry] : -1;
  const int count = min(max(named, 0), p.m);
  // (a count that does not fit is told in the status of the sequence's first entry, also where that one does not count)
  const int odd = j == 0 && named != count ? kBadIndex : 0;
  if (j >= count) {
    if (odd && slice == 0 && tid == 0 && p.status) p.status[entry] = odd;
    return;
  }
  if (at < 0 || at >= p.n) {
    if (slice == 0) refuse(p, entry, kBadIndex);
    return;
  }
  const void* row = reinterpret_cast<const char*>(p.logits) + (int64_t(b) * p.seq_stride + at * p.row_stride) * ElemTraits<T>::kBytes;
  const float z = token >= 0 && token < p.V ? load_elem<T>(row, token) : 0.0f;
  List list;
  row_share<T, W>(row, p, slice, sh, list);
  if (W == 1 || p.slices == 1) {
    if (wave == 0) finish(p, entry, token, z, all_waves(sh, p.k2), odd, list);
    return;
  }
  if constexpr (W == kLogprobWaves) {
    uint64_t* words = p.words + int64_t(entry) * p.slices;
    uint64_t* part = p.part + int64_t(entry) * p.slices * kPartWords;
    if (wave == 0) {
      const RowSums sums = all_waves(sh, p.k2);
      uint64_t* own = part + slice * kPartWords;
      if (p.top > 0 && lane < list.n) store_through(own + kPartHead + lane, list.at[lane]);
      if (lane < kLogprobWaves / 2) store_through(own + 4 + lane, uint64_t(as_u32(sh.c[2 * lane + 1])) << 32 | as_u32(sh.c[2 * lane]));
      if (lane == 0) {
        store_through(own, as_u32(sums.c));
        store_through(own + 1, __builtin_bit_cast(uint64_t, sums.S));
        store_through(own + 2, __builtin_bit_cast(uint64_t, sums.E));
        store_through(own + 3, uint64_t(list.n));
      }
    }
    if (!all_arrived(words, slice, p.slices, p.tag, sh.told)) return;
    if (wave == 0) {
      const bool mine = claimed(words, p.slices, p.tag);
      if (lane == 0) sh.mine = mine;
    }
    __syncthreads();
    if (!sh.mine) return;
    // a lane has a slice's sums
    const uint64_t* from = part + min(lane, p.slices - 1) * kPartWords;
    uint64_t head[kPartHead];
#pragma unroll
    for (int i = 0; i < kPartHead; ++i) head[i] = i < 3 || p.top > 0 ? load_through(from + i) : 0;
    RowSums got{as_f32(uint32_t(head[0])), 0.0, __builtin_bit_cast(double, head[1]), __builtin_bit_cast(double, head[2])};
    if (lane >= p.slices) got = RowSums{-INFINITY, 0.0, 0.0, 0.0};
    if (p.top > 0) {
      float largest[kLogprobWaves];
#pragma unroll
      for (int i = 0; i < kLogprobWaves; ++i) largest[i] = lane < p.slices ? as_f32(uint32_t(head[4 + i / 2] >> (32 * (i & 1)))) : -INFINITY;
      const float above = reached_by(largest, p.top);
      const int length = lane < p.slices ? int(head[3]) : 0;
      list = List{sh.list[wave], 0, -INFINITY, 0};
      constexpr int kTogether = 8;
      for (int s0 = wave; s0 < p.slices; s0 += kLogprobWaves * kTogether) {
        uint64_t r[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
          const int s = min(s0 + u * kLogprobWaves, 63);
          r[u] = lane < __builtin_amdgcn_readlane(length, s) ? load_through(part + s * kPartWords + kPartHead + lane) : 0;
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u)
          offer(list, s0 + u * kLogprobWaves < p.slices && r[u] != 0 && cand_value(r[u]) > above && r[u] >= list.least, r[u], p.top);
      }
      put_together<true, W>(list, p.top, sh);
    }
    if (wave == 0) finish(p, entry, token, z, join(got, p.k2), odd, list);
  }
}

// ---- the gradient of the logits ---------------------------------------------------------------------------------
//
// dz = (1 / T) (p (c0 + c1 log2 p) + what the token and the likeliest ones were given), p = 2^(k z - k T lse): elementwise, bound by
// reading a row and writing one (8 x 256 bfloat16 rows of 128256, all of which count, 203 us, 5.2 TB/s; 42 % of which count, the others filled with zeros, 147).  The few
// numbers of the second part are put in place by one wave at the end.  Stores go past the caches (173 us with them, then without 178).
// A row whose lse holds nothing of ln S any more (|lse| from 2^23 on) is added up again, p = 2^(k z - k c) / S with c the largest, by one workgroup, which reads it three times
// (865 such bfloat16 rows of 128256 187 us, of others 70; 9 of them 43 and 5).

struct LogprobBackwardParams {
  const void* logits;
  void* out;
  int64_t seq_stride, row_stride, out_seq_stride, out_row_stride, V;
  float rT, k2;
  int n, top;
  const int32_t *count, *tokens, *top_idx;
  const float *lse, *entropy, *grad_logp, *grad_entropy, *grad_lse, *grad_top;
  int slices;
};

template <typename T> __device__ __forceinline__ void store_elem(void* row, int64_t i, float v);
template <> __device__ __forceinline__ void store_elem<float>(void* row, int64_t i, float v) { reinterpret_cast<float*>(row)[i] = v; }
template <> __device__ __forceinline__ void store_elem<Bf16>(void* row, int64_t i, float v) { reinterpret_cast<__bf16*>(row)[i] = __bf16(v); }
template <> __device__ __forceinline__ void store_elem<F16>(void* row, int64_t i, float v) { reinterpret_cast<_Float16*>(row)[i] = _Float16(v); }
template <typename T> struct Vector16;
template <> struct Vector16<float> {
  static __device__ __forceinline__ u32x4 pack(const float (&v)[4]) { return u32x4{as_u32(v[0]), as_u32(v[1]), as_u32(v[2]), as_u32(v[3])}; }
};
template <typename T> struct Vector16 {
  static __device__ __forceinline__ u32x4 pack(const float (&v)[8]) {
    Eight<T> e;
    e.set(v);
    return e.w;
  }
};

template <typename T>
__global__ __launch_bounds__(kBlock) void logprob_backward_kernel(const LogprobBackwardParams p) {
  constexpr int E = ElemTraits<T>::kPerVec, kBytes = ElemTraits<T>::kBytes;
  const int tid = threadIdx.x, lane = lane_id();
  const uint32_t entry = blockIdx.x / uint32_t(p.slices);
  const int slice = int(blockIdx.x - entry * uint32_t(p.slices));
  const uint32_t b = entry / uint32_t(p.n);
  const int i = int(entry - b * uint32_t(p.n));
  const char* row = reinterpret_cast<const char*>(p.logits) + (int64_t(b) * p.seq_stride + i * p.row_stride) * kBytes;
  char* out = reinterpret_cast<char*>(p.out) + (int64_t(b) * p.out_seq_stride + i * p.out_row_stride) * kBytes;
  const bool there = i < counted(p.count, b, p.n);
  // Where fp32 has steps of 1 and more the lse says nothing of ln S (a row of nothing but the type's lowest number): one workgroup has the whole row then, and adds it up again.
  const float lse = there ? as_global(p.lse)[entry] : 0.0f;
  const bool again = fabsf(lse) >= 8388608.0f;
  if (again && slice > 0) return;
  // the split goes by where the results lie; the logits may lie otherwise
  const RowSplit rs = split_row<T>(out, p.V);
  const int64_t each = (rs.nvec + p.slices - 1) / p.slices, begin = again ? 0 : min(each * slice, rs.nvec), end = again ? rs.nvec : min(begin + each, rs.nvec);
  const bool first = slice == 0, last = again || slice == p.slices - 1;
  const int edges = (first ? rs.head : 0) + (last ? rs.tail : 0);
  const int64_t edge_at = tid < edges ? edge_index<T>(rs, first ? tid : rs.head + tid) : 0;
  u32x4* body = reinterpret_cast<u32x4*>(out + size_t(rs.head) * kBytes);
  const char* from = row + size_t(rs.head) * kBytes;

  // the row's constants, in every wave
  double c0 = 0.0, c1 = 0.0, rho = 0.0;
  float far_c = 0.0f, hi = 0.0f;
  bool known = true, far = false;
  int place = -1;                        // of lane 0 the token, of those behind it the likeliest ones; -1: none
  float given = 0.0f;
  if (again) {
    const auto all = [&](auto use) {
      if (tid < edges) use(load_elem<T>(row, edge_at));
#pragma unroll 1
      for (int64_t v = tid; v < rs.nvec; v += kBlock) {
        const u32x4 r = load16_any(from + v * 16);
        float z[E];
        unpack<T>(make_uint4(r[0], r[1], r[2], r[3]), z);
#pragma unroll
        for (int e = 0; e < E; ++e) use(z[e]);
      }
    };
    __shared__ float most[kBlock / 64];
    __shared__ double sums[kBlock / 64];
    float c = -INFINITY;
    all([&](float z) { c = fmaxf(c, z); });
    c = wave_max_f32(c);
    if (lane == 0) most[wave_id()] = c;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBlock / 64; ++w) c = fmaxf(c, most[w]);
    double S = 0.0;                      // NaN of a row that cannot be used
    all([&](float z) { S += double(fast_exp2((z - c) * p.k2)); });
    S = wave_sum_f64(S);
    if (lane == 0) sums[wave_id()] = S;
    __syncthreads();
    S = 0.0;
#pragma unroll
    for (int w = 0; w < kBlock / 64; ++w) S += sums[w];
    known = S == S;
    far = true;
    far_c = c;
    rho = log2(S);
  } else if (there) {
    known = lse == lse;
    const double reference = double(lse) / double(p.rT), scaled = double(p.k2) * reference;
    far = !(fabs(scaled) < 4194304.0);
    far_c = float(reference);
    hi = float(scaled);
    rho = far ? (reference - double(far_c)) * double(p.k2) : scaled - double(hi);
  }
  if (there) {
    if (p.grad_lse) c0 += as_global(p.grad_lse)[entry];
    if (p.grad_entropy) {
      const double g = as_global(p.grad_entropy)[entry];
      c0 -= g * as_global(p.entropy)[entry];
      c1 = -g * 0.69314718055994530942;
    }
    if (lane == 0 && p.grad_logp) {
      place = as_global(p.tokens)[entry];
      given = as_global(p.grad_logp)[entry];
    } else if (lane > 0 && lane <= p.top) {
      place = as_global(p.top_idx)[int64_t(entry) * p.top + lane - 1];
      given = as_global(p.grad_top)[int64_t(entry) * p.top + lane - 1];
    }
    if (place < 0 || place >= p.V) { place = -1; given = 0.0f; }
    c0 -= wave_sum_f64(double(given));
  }
  const float f = float(exp2(-rho) * double(p.rT)), a0 = f * float(c0 - c1 * rho), a1 = f * float(c1), k2 = p.k2, none = there ? NAN : 0.0f;
  const bool fill = !there || !known;
  // (a p of 0 gives 0, whatever its logarithm)
  const auto of = [&](float d) { return fast_exp2(d) * fmaf(a1, fmaxf(d, -200.0f), a0); };
  const auto gradient = [&](float z) { return fill ? none : of(far ? (z - far_c) * k2 : fmaf(z, k2, -hi)); };
  // the first wave: the numbers at the given places in this share, before they are written over where the results lie on the logits (by this share alone)
  const int64_t lo = first ? 0 : rs.head + begin * E, hi_at = last ? p.V : rs.head + end * E;
  const bool some = !fill && (p.grad_logp || p.top > 0), mine = some && tid <= p.top && place >= lo && place < hi_at;
  const float z_there = mine ? load_elem<T>(row, place) : 0.0f;
  if (p.out == p.logits && some) {
    stores_arrived();                                    // (and loads)
    __syncthreads();
  }
  if (tid < edges) store_elem<T>(out, edge_at, gradient(fill ? 0.0f : load_elem<T>(row, edge_at)));
  constexpr int kAheadBack = 4;
  for (int64_t v0 = begin + tid; v0 < end; v0 += kBlock * kAheadBack) {
    uint4 x[kAheadBack];
#pragma unroll
    for (int u = 0; u < kAheadBack; ++u)
      if (!fill && v0 + u * kBlock < end) {
        const u32x4 r = load16_any(from + (v0 + u * kBlock) * 16);
        x[u] = make_uint4(r[0], r[1], r[2], r[3]);
      }
#pragma unroll
    for (int u = 0; u < kAheadBack; ++u) {
      if (v0 + u * kBlock >= end) break;
      float z[E];
      if (fill) {
#pragma unroll
        for (int e = 0; e < E; ++e) z[e] = none;
      } else {
        unpack<T>(x[u], z);
        if (same_in_wave(far)) {
#pragma unroll
          for (int e = 0; e < E; ++e) z[e] = of((z[e] - far_c) * k2);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) z[e] = of(fmaf(z[e], k2, -hi));
        }
      }
      __builtin_nontemporal_store(Vector16<T>::pack(z), body + v0 + u * kBlock);
    }
  }
  if (!some) return;
  // the given places, behind everything that was written there
  stores_arrived();
  __syncthreads();
  if (wave_id() > 0) return;
  float sum = 0.0f;
  for (int k = 0; k <= p.top; ++k) {
    const int other = __builtin_amdgcn_readlane(place, k);
    sum += other == place ? as_f32(__builtin_amdgcn_readlane(as_u32(given), k)) : 0.0f;
  }
  if (mine) store_elem<T>(out, place, fmaf(p.rT, sum, gradient(z_there)));
}

}  // namespace tslt
