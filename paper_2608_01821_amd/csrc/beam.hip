// Beams: the best continuations over all beams of a request and the vocabulary, and
// the move of a paged cache along with them.
//
//   value(b, w) = score_b + x_bw - lse_b,  lse_b = m_b + ln S_b
//
// A beam's best continuations are its largest logits, so each row gives its `top` by
// (logit, id) and its (m, S) in one pass over the logits (the kernels of logprobs.h),
// and a second launch, a workgroup a request, joins them: its wavefronts turn the rows'
// lists into float64 values (two beams' candidates may be closer than float32
// roundings) and keep the best 64 in order, one a lane; then their lists are joined.
//
// Bound by latency: 64 rows of 126,464 bf16 logits, 4 of 16 requests, take 12.2 us (1.4
// TB/s), their join 4.5; 4 fp32 rows, 15 slices each, 7.3 and 6.4; 4 requests of 16 beams,
// 16 best each, 12.5 and 8.5 (9.8 with the wavefronts' lists joined two by two).  The move of 64 sequences' last pages, 8 heads of 55 rows
// of 128, takes 5.0 us (26 MB, 5.2 TB/s), of one row each 3.
//
// Order: value, then row, then (logit, id): within a row values only ever tie where
// logits do, or where the score is so large that they vanish beside it.

#include "logprobs.h"

namespace davet {
namespace {

// a candidate: ordered bits of its value (0: none), its row's key, its row
struct Cand {
  uint64_t v, key;
  uint32_t row;
};
__device__ __forceinline__ bool better(const Cand& a, const Cand& b) {
  if (a.v != b.v) return a.v > b.v;
  if (a.row != b.row) return a.row < b.row;
  return a.key > b.key;
}
// order of finite doubles (larger first), never 0
__device__ __forceinline__ uint64_t value_key(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x == 0.0 ? 0.0 : x);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double value_of(uint64_t k) {
  return __builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k);
}
// One step of a bitonic network: of each pair (l, l ^ O) the better one to the lower
// lane, or, where lane & S, or with `up`, to the upper one (both: the lower again).
template <int O, int S>
__device__ __forceinline__ void exchange(Cand& c, bool up) {
  const Cand o = {lane_xor<O>(c.v), lane_xor<O>(c.key), lane_xor<O>(c.row)};
  const bool lower = ((threadIdx.x & O) == 0) == (((threadIdx.x & S & 63) == 0) != up);
  if (lower != better(c, o)) c = o;
}
// steps O, O / 2, .. 1
template <int O, int S>
__device__ __forceinline__ void exchanges(Cand& c, bool up) {
  exchange<O, S>(c, up);
  if constexpr (O > 1) exchanges<O / 2, S>(c, up);
}
// the 64 best of two lists in order, the second one given in reverse
__device__ __forceinline__ void join(Cand& c, const Cand& reversed) {
  if (better(reversed, c)) c = reversed;
  exchanges<32, 64>(c, false);
}

// First every row's base, score - lse, four rows a wavefront, 16 lanes for the slices
// of each.  Then the lists, each in order: a wavefront takes 64 / P of them at a time, P
// the power of two that holds k, every other one in reverse, and merges them pair by
// pair (k = 4: 18 steps for 16 lists, where a join each is 96).
constexpr int kJoinWaves = 16;
static_assert(kMaxSlices <= 16 && DAVET_MAX_BEAMS <= 4 * kJoinWaves, "lanes of a row");
__global__ void __launch_bounds__(64 * kJoinWaves)
beam_join_kernel(int rows, int beams, int slices, int k, int P,
                 const char* __restrict__ part, const float* scores,
                 const int32_t* __restrict__ done, int pad, float* out_scores,
                 int32_t* __restrict__ out_rows, int32_t* __restrict__ out_tokens,
                 int wg0) {
  __shared__ uint64_t s_v[2][kJoinWaves * 64], s_key[2][kJoinWaves * 64];
  __shared__ uint32_t s_row[2][kJoinWaves * 64];
  __shared__ double s_base[DAVET_MAX_BEAMS];    // (NaN: nothing to offer)
  __shared__ double s_over[DAVET_MAX_BEAMS];    // the score of a row that is over, or NaN
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wg0 + (int)blockIdx.x;
  const int row0 = group * beams, lists = beams * slices;
  const uint64_t* keys = reinterpret_cast<const uint64_t*>(part);
  const Stat* stats = reinterpret_cast<const Stat*>(keys + (int64_t)rows * slices * k);
  keys += (int64_t)row0 * slices * k;

  const int per = 64 / P, chunks = (lists + per - 1) / per;
  auto key_of = [&](int chunk, bool up) {       // this lane's entry
    const int run = lane / P, l = chunk * per + run;
    const int j = ((run & 1) != 0) != up ? P - 1 - lane % P : lane % P;
    return l < lists && j < k ? keys[(int64_t)l * k + j] : 0;
  };
  // (what a row that is over left unwritten is not used)
  uint64_t next = wave < chunks ? key_of(wave, false) : 0;
  {
    const int b = wave * 4 + lane / 16, sl = lane % 16;
    const float score = b < beams ? scores[row0 + b] : 0.f;
    const int over = b < beams && done ? done[row0 + b] : 0;
    Stat s = stat_none();
    if (b < beams && sl < slices && !over) s = stats[((int64_t)row0 + b) * slices + sl];
    s = stat_step<1>(s);
    s = stat_step<2>(s);
    s = stat_step<4>(s);
    s = stat_step<8>(s);
    const double base = (double)score - ((double)s.m + log((double)s.S));
    if (b < beams && sl == 0) {
      s_base[b] = !over && fabs(base) < INFINITY ? base : __builtin_nan("");
      s_over[b] = over && fabsf(score) < INFINITY ? (double)score : __builtin_nan("");
    }
  }
  __syncthreads();
  const Cand none = {0, 0, 0xffffffffu};
  // 64 / P lists of P entries, every other one reversed, to one (with `up` reversed); the
  // first n of them, if the others are empty and it is not to be reversed
  auto merge = [&](Cand& c, int n, bool up) {
    const int end = up ? 64 : n * P;
    if (P < 2 && end > 1) exchanges<1, 2>(c, up);
    if (P < 4 && end > 2) exchanges<2, 4>(c, up);
    if (P < 8 && end > 4) exchanges<4, 8>(c, up);
    if (P < 16 && end > 8) exchanges<8, 16>(c, up);
    if (P < 32 && end > 16) exchanges<16, 32>(c, up);
    if (P < 64 && end > 32) exchanges<32, 64>(c, up);
  };
  Cand best = none;
  for (int chunk = wave; chunk < chunks; chunk += kJoinWaves) {
    const bool up = chunk != wave;              // (the first one as it is kept)
    const uint64_t key = next;
    if (chunk + kJoinWaves < chunks) next = key_of(chunk + kJoinWaves, true);
    const int run = lane / P, l = chunk * per + run, b = min(l / slices, beams - 1);
    const bool first = l < lists && l % slices == 0 &&
                       lane % P == (((run & 1) != 0) != up ? P - 1 : 0);
    const double base = s_base[b], over = s_over[b];
    Cand c = none;
    if (base == base && key)
      c = {value_key(base + (double)key_value(key)), key, (uint32_t)(row0 + b)};
    if (over == over && first) c = {value_key(over), top_key(0.f, pad), (uint32_t)(row0 + b)};
    merge(c, lists - chunk * per, up);
    if (up)
      join(best, c);
    else
      best = c;
  }
  // the wavefronts' lists, P entries of each, in the same way (of 64: two at a time)
  int active = min(kJoinWaves, chunks);
  for (int half = 0; active > 1; half ^= 1) {
    if (wave < active && lane < P) {
      s_v[half][wave * P + lane] = best.v;
      s_key[half][wave * P + lane] = best.key;
      s_row[half][wave * P + lane] = best.row;
    }
    __syncthreads();
    auto entry = [&](int l, int j) {
      const int i = min(l, active - 1) * P + j;
      const Cand c = {s_v[half][i], s_key[half][i], s_row[half][i]};
      return l < active ? c : none;
    };
    const int take = max(2, per), run = lane / P, l = wave * take + run;
    if (wave * take < active) {
      best = entry(l, run & 1 ? P - 1 - lane % P : lane % P);
      merge(best, active - wave * take, false);
      if (P == 64) join(best, entry(l + 1, 63 - lane));
    }
    active = (active + take - 1) / take;
  }
  if (wave != 0 || lane >= k) return;
  const int64_t at = (int64_t)group * k + lane;
  out_scores[at] = best.v ? (float)value_of(best.v) : -INFINITY;
  out_rows[at] = best.v ? (int)best.row : -1;
  out_tokens[at] = best.v ? key_id(best.key) : -1;
}

size_t beam_bytes(int64_t rows, int vocab, int k) {
  const int64_t n = rows * plan_slices((int)rows, vocab);
  return align_up((size_t)n * ((size_t)k * 8 + sizeof(Stat)), 256);
}

int check_beams(int32_t groups, int32_t beams, int32_t vocab, int32_t top,
                const std::string& who) {
  DAVET_CHECK_ARG(groups >= 0 && beams >= 1 && beams <= DAVET_MAX_BEAMS &&
                      (int64_t)groups * beams <= (1 << 22) && vocab >= 1 &&
                      vocab <= (1 << 30) && top >= 1 && top <= DAVET_MAX_TOP,
                  DAVET_ESHAPE,
                  who + ": beams and top in [1, 64], at most 2^22 rows, vocab in "
                        "[1, 2^30]");
  return DAVET_OK;
}

struct ReorderPack { int32_t kv[DAVET_MAX_SEQS]; };

// One workgroup a (sequence, key head): its share of the last page, keys and values;
// that of key head 0 also writes the sequence's table.
__global__ void __launch_bounds__(256)
cache_reorder_kernel(CacheView cv, ReorderPack rp, int n_seqs, int row_bytes,
                     const int32_t* __restrict__ parent,
                     const int32_t* __restrict__ fresh, int32_t* __restrict__ dst,
                     int dst_max_pages) {
  const int s = blockIdx.x / cv.n_kv, h = blockIdx.x % cv.n_kv;
  const int from = parent[s], kv = rp.kv[s];
  const int whole = kv >> cv.lg, rest = kv & ((1 << cv.lg) - 1);
  const bool known = (unsigned)from < (unsigned)n_seqs;
  const int32_t* src = cv.table + (int64_t)(known ? from : 0) * cv.max_pages;
  int32_t* to = dst + (int64_t)s * dst_max_pages;
  if (h == 0)
    for (int i = threadIdx.x; i < whole; i += 256) to[i] = known ? src[i] : -1;
  if (rest == 0) return;
  const int a = known ? src[whole] : -1, b = fresh[s];
  const bool move = (unsigned)a < (unsigned)cv.n_pages && (unsigned)b < (unsigned)cv.n_pages;
  if (h == 0 && threadIdx.x == 0) to[whole] = move ? b : -1;
  if (!move || a == b) return;
  const int n = rest * row_bytes / 16;
  const int64_t block = (int64_t)row_bytes << cv.lg;
  const int64_t ao = ((int64_t)a * cv.n_kv + h) * block;
  const int64_t bo = ((int64_t)b * cv.n_kv + h) * block;
  const u32x4* ka = reinterpret_cast<const u32x4*>(static_cast<const char*>(cv.k) + ao);
  const u32x4* va = reinterpret_cast<const u32x4*>(static_cast<const char*>(cv.v) + ao);
  u32x4* kb = reinterpret_cast<u32x4*>(static_cast<char*>(cv.k) + bo);
  u32x4* vb = reinterpret_cast<u32x4*>(static_cast<char*>(cv.v) + bo);
  constexpr int U = 4;
  for (int i0 = threadIdx.x; i0 < n; i0 += 256 * U) {
    u32x4 x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = ka[min(i0 + u * 256, n - 1)];
      y[u] = va[min(i0 + u * 256, n - 1)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * 256 < n) {
        kb[i0 + u * 256] = x[u];
        vb[i0 + u * 256] = y[u];
      }
  }
}

}  // namespace
}  // namespace davet

extern "C" int davet_beam_workspace_bytes(int32_t groups, int32_t beams, int32_t vocab,
                                          int32_t top, size_t* bytes) {
  using namespace davet;
  DAVET_CHECK_ARG(bytes, DAVET_EINVAL, "davet_beam_workspace_bytes: bytes is null");
  const int rc = check_beams(groups, beams, vocab, top, "davet_beam_workspace_bytes");
  if (rc) return rc;
  *bytes = groups ? beam_bytes((int64_t)groups * beams, vocab, top) : 0;
  return DAVET_OK;
}

extern "C" int davet_beam_select(int32_t groups, int32_t beams, int32_t vocab,
                                 const void* logits, int32_t dtype, int64_t ld,
                                 int32_t exclude, const float* scores,
                                 const int32_t* done, int32_t pad, int32_t top,
                                 float* out_scores, int32_t* out_rows,
                                 int32_t* out_tokens, void* workspace, size_t ws_bytes,
                                 hipStream_t stream) {
  using namespace davet;
  DAVET_CHECK_ARG(dtype == DAVET_F32 || is16(dtype), DAVET_EDTYPE,
                  "davet_beam_select: dtype must be DAVET_F32, DAVET_BF16 or DAVET_F16");
  int rc = check_beams(groups, beams, vocab, top, "davet_beam_select");
  if (rc) return rc;
  const int rows = groups * beams;
  DAVET_CHECK_ARG(ld >= vocab && ld < (1ll << 40), DAVET_ESHAPE,
                  "davet_beam_select: row stride below vocab, or 2^40 and more");
  if (groups == 0) return DAVET_OK;
  DAVET_CHECK_ARG(logits && scores && out_scores && out_rows && out_tokens, DAVET_EINVAL,
                  "davet_beam_select: null pointer");
  DAVET_CHECK_ARG(((uintptr_t)logits & (dtype_size(dtype) - 1)) == 0, DAVET_EINVAL,
                  "davet_beam_select: logits misaligned for their type");
  DAVET_CHECK_ARG(aligned4({scores, done, out_scores, out_rows, out_tokens}),
                  DAVET_EINVAL,
                  "davet_beam_select: scores, done and outputs must be 4-byte aligned");
  DAVET_CHECK_ARG((out_scores == scores && top == beams) ||
                      !overlap(out_scores, (size_t)groups * top * 4, scores,
                               (size_t)rows * 4),
                  DAVET_EINVAL,
                  "davet_beam_select: out_scores overlaps scores (the same address "
                  "needs top = beams)");
  const size_t need = beam_bytes(rows, vocab, top);
  DAVET_CHECK_ARG(workspace && ((uintptr_t)workspace & 255) == 0 && ws_bytes >= need,
                  DAVET_ENOMEM,
                  "davet_beam_select: workspace missing, misaligned or below " +
                      std::to_string(need) + " bytes");
  char* part = static_cast<char*>(workspace);
  const bool brief = vocab <= 64 * kWaves * kShort;
  const int slices = brief ? 1 : plan_slices(rows, vocab);
#define ROWS(F)                                                                \
  do {                                                                         \
    const auto* x = static_cast<const F::st*>(logits);                         \
    if (brief)                                                                 \
      hipLaunchKernelGGL((logprobs_short_kernel<F, true>), dim3(rows),         \
                         dim3(64 * kWaves), 0, stream, x, ld, vocab, exclude,  \
                         top, nullptr, Out{}, part, done);                     \
    else                                                                       \
      hipLaunchKernelGGL((logprobs_kernel<F, true>), dim3(rows * slices),      \
                         dim3(64 * kWaves), 0, stream, x, ld, vocab, exclude,  \
                         top, nullptr, Out{}, slices, part, done);             \
  } while (0)
  {
    ProfScope ps(KC_MISC, stream);
    if (dtype == DAVET_F16) ROWS(F16S);
    else if (dtype == DAVET_BF16) ROWS(BF16S);
    else ROWS(F32S);
    DAVET_HIP(hipGetLastError());
  }
#undef ROWS
  int P = 1;
  while (P < top) P *= 2;
  ProfScope ps(KC_MISC, stream);
  in_runs(groups, 64 * kJoinWaves, [&](int at, int64_t n) {
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)n), dim3(64 * kJoinWaves), 0,
                       stream, rows, beams, slices, top, P, part, scores, done, pad,
                       out_scores, out_rows, out_tokens, at);
  });
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}

extern "C" int davet_cache_reorder(const davet_kv_cache* cache, int32_t n_seqs,
                                   const int32_t* kv_len, const int32_t* parent,
                                   const int32_t* fresh, int32_t* dst_table,
                                   int32_t dst_max_pages, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_reorder";
  CacheView cv;
  const int rc = check_cache(cache, true, who, &cv);
  if (rc) return rc;
  DAVET_CHECK_ARG(n_seqs >= 1 && n_seqs <= DAVET_MAX_SEQS, DAVET_ESHAPE,
                  "davet_cache_reorder: n_seqs out of range [1, 64]");
  DAVET_CHECK_ARG(kv_len && parent && fresh && dst_table, DAVET_EINVAL,
                  "davet_cache_reorder: null pointer");
  DAVET_CHECK_ARG(aligned4({parent, fresh, dst_table}), DAVET_EINVAL,
                  "davet_cache_reorder: parent, fresh and dst_table must be 4-byte "
                  "aligned");
  ReorderPack rp{};
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t pages = ((int64_t)kv_len[s] + cache->page_size - 1) >> cv.lg;
    DAVET_CHECK_ARG(kv_len[s] >= 0 && kv_len[s] <= (1 << 30) &&
                        pages <= cv.max_pages && pages <= dst_max_pages,
                    DAVET_ESHAPE,
                    "davet_cache_reorder: kv_len out of range of max_pages or "
                    "dst_max_pages (or 2^30)");
    rp.kv[s] = kv_len[s];
  }
  DAVET_CHECK_ARG(dst_max_pages >= 0 &&
                      !overlap(dst_table, (size_t)n_seqs * dst_max_pages * 4,
                               cache->page_table, (size_t)n_seqs * cv.max_pages * 4),
                  DAVET_EINVAL, "davet_cache_reorder: dst_table overlaps page_table");
  ProfScope ps(KC_MISC, stream);
  hipLaunchKernelGGL(cache_reorder_kernel, dim3((unsigned)(n_seqs * cv.n_kv)), dim3(256),
                     0, stream, cv, rp, n_seqs,
                     cache->head_dim * (int)dtype_size(cache->dtype), parent, fresh,
                     dst_table, dst_max_pages);
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}
