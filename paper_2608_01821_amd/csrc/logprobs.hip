// Log probabilities of given tokens, entropy and the top alternatives of rows of
// logits, in one pass over them.
//
// With m = max x, S = sum exp(x - m), A = sum exp(x - m) (x - m):
//   log p(t) = x_t - m - ln S,      entropy = ln S - A / S
// and the k largest logits in (value descending, id ascending) order.
//
// A row is cut into slices of one workgroup; each of its four wavefronts walks
// its part in batches of 16-byte loads and keeps (m, S, A) per lane, rescaled
// when a batch moves the maximum.  The top k (at most 64) of a wavefront is a
// sorted list with one entry a lane, as 64-bit keys whose order is the wanted
// one.  A batch enters the list only where a lane's maximum beats the k-th
// entry; the first batch starts from the k-th largest of the 64 lane maxima, so
// that it enters about k values and not all.  Lists are joined in LDS at the end
// of a workgroup, and a second launch joins the slices of a row where there are
// several.  Bound by HBM (one read of the logits) for many rows, by two launches'
// latency for few.

#include <math.h>

#include <algorithm>

#include "cache.h"

namespace davet {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxSlices = 64;

struct Stat { float m, S, A; };

__device__ __forceinline__ Stat stat_none() { return {-INFINITY, 0.f, 0.f}; }
// exp(d) and exp(d) d for d = x - m <= 0 (0 and 0 for -inf)
__device__ __forceinline__ void term(float x, float ref, float& S, float& A) {
  const float d = x - ref;
  const float e = __builtin_amdgcn_exp2f(d * kLog2e);
  S += e;
  if (e != 0.f) A = fmaf(e, d, A);
}
__device__ __forceinline__ Stat stat_to(const Stat& a, float m) {
  // nothing yet: its sums are 0 (or NaN, which stays)
  const float d = a.m == -INFINITY ? 0.f : a.m - m;
  const float e = __builtin_amdgcn_exp2f(d * kLog2e);
  return {m, a.S * e, a.S != 0.f && e != 0.f ? e * fmaf(a.S, d, a.A) : 0.f * a.S};
}
__device__ __forceinline__ Stat stat_join(const Stat& a, const Stat& b) {
  const float m = fmaxf(a.m, b.m);
  const Stat x = stat_to(a, m), y = stat_to(b, m);
  return {m, x.S + y.S, x.A + y.A};
}
__device__ __forceinline__ Stat stat_wave(Stat s) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const Stat t = {__shfl_xor(s.m, o, 64), __shfl_xor(s.S, o, 64),
                    __shfl_xor(s.A, o, 64)};
    s = stat_join(s, t);
  }
  return s;
}

// 64-bit key of a (value, id): larger value first, then lower id; never 0 for
// a value above -inf
__device__ __forceinline__ uint64_t top_key(float x, int id) {
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return (uint64_t)o << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_id(uint64_t k) { return (int)~(uint32_t)k; }

__device__ __forceinline__ uint64_t lane64(uint64_t v, int l) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, l);
}
// puts `key` into the descending list held one entry a lane
__device__ __forceinline__ void list_insert(uint64_t& list, uint64_t key) {
  const int at = (int)__popcll(__ballot(list > key));
  const int lane = threadIdx.x & 63;
  const uint64_t up =
      (uint64_t)(uint32_t)__shfl_up((int)(list >> 32), 1, 64) << 32 |
      (uint32_t)__shfl_up((int)(uint32_t)list, 1, 64);
  list = lane < at ? list : lane == at ? key : up;
}
// k-th largest (k in 1..64) of the 64 lanes' values; NaN lanes hold -inf
__device__ __forceinline__ float kth_of_lanes(float x, int k) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
    for (int o = size >> 1; o > 0; o >>= 1) {
      const float y = __shfl_xor(x, o, 64);
      const bool desc = (lane & size) == 0;       // (size 64: always)
      const bool low = (lane & o) == 0;
      x = low == desc ? fmaxf(x, y) : fminf(x, y);
    }
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), k - 1));
}

// 16 bytes of logits as fp32
template <typename F> struct Vec;
template <> struct Vec<F32S> { static constexpr int N = 4; };
template <> struct Vec<F16S> { static constexpr int N = 8; };
template <> struct Vec<BF16S> { static constexpr int N = 8; };
template <typename F>
__device__ __forceinline__ void unpack(const u32x4& w, float* x) {
  if constexpr (F::dtype == DAVET_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = F::load((uint16_t)(w[i] & 0xffffu));
      x[2 * i + 1] = F::load((uint16_t)(w[i] >> 16));
    }
  }
}

struct Out {
  float* logp;
  float* entropy;
  float* top_logp;
  int32_t* top_ids;
};

// One wavefront writes a row's results.
template <typename F>
__device__ __forceinline__ void finish(const Stat& s, uint64_t list, int row,
                                       int vocab, int exclude, int k,
                                       const typename F::st* x,
                                       const int32_t* targets, const Out& out) {
  const int lane = threadIdx.x & 63;
  const float lnS = logf(s.S);
  if (lane == 0) {
    if (out.logp) {
      const int t = targets[row];
      float v = -INFINITY;                        // no such token
      if ((unsigned)t < (unsigned)vocab && t != exclude && s.S != 0.f)
        v = F::load(x[t]) - s.m - lnS;
      out.logp[row] = v;
    }
    if (out.entropy)
      // nothing to choose from: 0; one certain token: not below 0
      out.entropy[row] = s.S == 0.f ? 0.f : lnS - s.A / s.S;
  }
  if (lane < k) {
    out.top_ids[(int64_t)row * k + lane] = list ? key_id(list) : -1;
    out.top_logp[(int64_t)row * k + lane] =
        list ? key_value(list) - s.m - lnS : -INFINITY;
  }
}

constexpr int kBatch = 4;     // 16-byte loads a lane in flight

template <typename F>
__global__ void __launch_bounds__(256)
logprobs_kernel(const typename F::st* __restrict__ logits, int64_t ld, int vocab,
                int exclude, int k, const int32_t* __restrict__ targets, Out out,
                int slices, char* __restrict__ part) {
  using st = typename F::st;
  constexpr int N = Vec<F>::N;
  __shared__ uint64_t s_list[4][64];
  __shared__ Stat s_stat[4];
  const int row = blockIdx.x / slices, slice = blockIdx.x % slices;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const st* x = logits + (int64_t)row * ld;
  // [0, head) and [tail, vocab): elements outside whole 16-byte pieces
  const int head = min(vocab, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(st));
  const int nvec = (vocab - head) / N, tail = head + nvec * N;
  const u32x4* xv = reinterpret_cast<const u32x4*>(x + head);

  Stat s = stat_none();
  uint64_t list = 0;
  float thr = -INFINITY;        // value of the k-th entry
  bool full = false;            // thr is an entry of the list, not a bound

  // a batch of E values a lane; value e has id(e)
  constexpr int E = kBatch * N;
  auto take = [&](float (&v)[E], auto id) {
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) mx = fmaxf(mx, v[e]);
    if (mx > s.m) s = stat_to(s, mx);
    const float ref = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int e = 0; e < E; ++e) term(v[e], ref, s.S, s.A);
    if (k == 0) return;
    if (!full) {
      const float low = kth_of_lanes(mx, k);
      thr = fmaxf(thr, low);
    }
    if (!__any(full ? mx > thr : mx >= thr && mx > -INFINITY)) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      // a later equal value has a higher id and loses to a full list
      uint64_t who = __ballot(full ? v[e] > thr : v[e] >= thr && v[e] > -INFINITY);
      const uint64_t key = top_key(v[e], id(e));
      while (who) {
        const int l = __ffsll((unsigned long long)who) - 1;
        who &= who - 1;
        list_insert(list, lane64(key, l));
      }
    }
    const uint64_t kth = lane64(list, k - 1);
    full = kth != 0;
    if (full) thr = key_value(kth);
  };

  // this wavefront's 16-byte pieces
  const int parts = slices * 4, mine = slice * 4 + wave;
  const int per = ((nvec + parts - 1) / parts + 63) & ~63;
  const int v0 = min(nvec, mine * per), v1 = min(nvec, v0 + per);
  for (int b = v0; b < v1; b += 64 * kBatch) {
    u32x4 w[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      w[u] = xv[min(b + u * 64 + lane, v1 - 1)];
    float v[E];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      unpack<F>(w[u], v + u * N);
      if (b + u * 64 + lane >= v1)
#pragma unroll
        for (int e = 0; e < N; ++e) v[u * N + e] = -INFINITY;
    }
    const int first = head + b * N;
    if (exclude >= first && exclude < first + 64 * kBatch * N) {
#pragma unroll
      for (int e = 0; e < kBatch * N; ++e)
        if (head + (b + (e / N) * 64 + lane) * N + e % N == exclude)
          v[e] = -INFINITY;
    }
    take(v, [&](int e) { return head + (b + (e / N) * 64 + lane) * N + e % N; });
  }
  if (mine == parts - 1 && (head || tail < vocab)) {
    // the edges: fewer than 16 values.  Lanes in id order within each edge; a
    // head value has a lower id than any listed one and may equal the k-th.
    const int ne = head + vocab - tail;
    const int id = lane < head ? lane : tail + lane - head;
    float v[1] = {lane < ne && id != exclude ? F::load(x[id]) : -INFINITY};
    if (k > 0) {
      uint64_t who = __ballot(v[0] > -INFINITY);
      const uint64_t key = top_key(v[0], id);
      while (who) {
        const int l = __ffsll((unsigned long long)who) - 1;
        who &= who - 1;
        list_insert(list, lane64(key, l));
      }
    }
    if (v[0] > s.m) s = stat_to(s, v[0]);
    term(v[0], s.m == -INFINITY ? 0.f : s.m, s.S, s.A);
  }
  s = stat_wave(s);
  if (lane == 0) s_stat[wave] = s;
  if (lane < k) s_list[wave][lane] = list;
  __syncthreads();
  if (wave != 0) return;
  for (int o = 1; o < 4; ++o) {
    s = stat_join(s, s_stat[o]);
    for (int i = 0; i < k; ++i) {
      const uint64_t key = s_list[o][i];
      if (key <= lane64(list, k - 1)) break;      // sorted: the rest is below
      list_insert(list, key);
    }
  }
  if (slices == 1) {
    finish<F>(s, list, row, vocab, exclude, k, x, targets, out);
    return;
  }
  // partial results: [rows][slices] Stat, then [rows][slices][k] keys
  const int64_t at = (int64_t)row * slices + slice;
  const int64_t n_rows = gridDim.x / slices;
  uint64_t* pl = reinterpret_cast<uint64_t*>(part);
  if (lane < k) pl[at * k + lane] = list;
  if (lane == 0) reinterpret_cast<Stat*>(pl + n_rows * slices * k)[at] = s;
}

// Joins the slices of one row: one wavefront a row, one slice a lane.  Every
// round takes the largest of the slices' next keys.
template <typename F>
__global__ void __launch_bounds__(64)
logprobs_join_kernel(const typename F::st* __restrict__ logits, int64_t ld,
                     int vocab, int exclude, int k,
                     const int32_t* __restrict__ targets, Out out, int slices,
                     const char* __restrict__ part, int rows) {
  extern __shared__ uint64_t keys[];     // [slices][k]
  const int row = blockIdx.x, lane = threadIdx.x;
  const uint64_t* pl = reinterpret_cast<const uint64_t*>(part);
  const Stat* ps = reinterpret_cast<const Stat*>(pl + (int64_t)rows * slices * k);
  for (int i = lane; i < slices * k; i += 64)
    keys[i] = pl[(int64_t)row * slices * k + i];
  Stat s = stat_none();
  if (lane < slices) s = ps[(int64_t)row * slices + lane];
  s = stat_wave(s);
  __syncthreads();
  uint64_t list = 0;
  int next = 0;
  for (int i = 0; i < k; ++i) {
    const uint64_t mine =
        lane < slices && next < k ? keys[lane * k + next] : 0;
    uint64_t best = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t y = (uint64_t)(uint32_t)__shfl_xor((int)(best >> 32), o, 64) << 32 |
                         (uint32_t)__shfl_xor((int)(uint32_t)best, o, 64);
      best = best > y ? best : y;
    }
    if (best == 0) break;
    if (mine == best) ++next;            // keys are distinct: ids are
    if (lane == i) list = best;
  }
  finish<F>(s, list, row, vocab, exclude, k, logits + (int64_t)row * ld, targets, out);
}

// Slices a row: enough workgroups for the chip, at least 4096 logits each.
int plan_slices(int rows, int vocab) {
  const int want = (1024 + rows - 1) / rows;
  return std::max(1, std::min({want, kMaxSlices, vocab / 4096}));
}

size_t part_bytes(int rows, int vocab, int k) {
  const int sl = plan_slices(rows, vocab);
  if (sl == 1) return 0;
  return (size_t)rows * sl * ((size_t)k * 8 + sizeof(Stat));
}

}  // namespace
}  // namespace davet

extern "C" int davet_logprobs_workspace_bytes(int32_t rows, int32_t vocab,
                                              int32_t top, size_t* bytes) {
  using namespace davet;
  DAVET_CHECK_ARG(bytes, DAVET_EINVAL,
                  "davet_logprobs_workspace_bytes: bytes is null");
  DAVET_CHECK_ARG(rows >= 1 && rows <= (1 << 22) && vocab >= 1 &&
                      vocab <= (1 << 30) && top >= 0 && top <= DAVET_MAX_TOP,
                  DAVET_ESHAPE, "davet_logprobs_workspace_bytes: out of range");
  *bytes = part_bytes(rows, vocab, top);
  return DAVET_OK;
}

extern "C" int davet_token_logprobs(int32_t rows, int32_t vocab,
                                    const void* logits, int32_t dtype,
                                    int64_t ld, int32_t exclude,
                                    const int32_t* targets, float* logp,
                                    float* entropy, int32_t top, float* top_logp,
                                    int32_t* top_ids, void* workspace,
                                    size_t ws_bytes, hipStream_t stream) {
  using namespace davet;
  DAVET_CHECK_ARG(dtype == DAVET_F32 || is16(dtype), DAVET_EDTYPE,
                  "davet_token_logprobs: dtype must be DAVET_F32, DAVET_BF16 or "
                  "DAVET_F16");
  DAVET_CHECK_ARG(rows >= 0 && rows <= (1 << 22) && vocab >= 1 &&
                      vocab <= (1 << 30) && ld >= vocab,
                  DAVET_ESHAPE,
                  "davet_token_logprobs: rows, vocab or ld out of range");
  DAVET_CHECK_ARG(top >= 0 && top <= DAVET_MAX_TOP, DAVET_ESHAPE,
                  "davet_token_logprobs: top out of range [0, 64]");
  if (rows == 0) return DAVET_OK;
  DAVET_CHECK_ARG(logits && (!logp || targets) && (top == 0 || (top_logp && top_ids)),
                  DAVET_EINVAL, "davet_token_logprobs: null pointer");
  DAVET_CHECK_ARG(((uintptr_t)logits & (dtype_size(dtype) - 1)) == 0, DAVET_EINVAL,
                  "davet_token_logprobs: logits misaligned for their type");
  const int slices = plan_slices(rows, vocab);
  const size_t need = part_bytes(rows, vocab, top);
  DAVET_CHECK_ARG(need == 0 || (workspace && ((uintptr_t)workspace & 255) == 0 &&
                                ws_bytes >= need),
                  DAVET_ENOMEM,
                  "davet_token_logprobs: workspace missing, misaligned or below " +
                      std::to_string(need) + " bytes");
  const Out out{logp, entropy, top_logp, top_ids};
  char* part = static_cast<char*>(workspace);
#define LOGP(F)                                                                \
  do {                                                                         \
    const auto* x = static_cast<const F::st*>(logits);                         \
    {                                                                          \
      ProfScope ps(KC_MISC, stream);                                           \
      hipLaunchKernelGGL(logprobs_kernel<F>, dim3(rows * slices), dim3(256), 0, \
                         stream, x, ld, vocab, exclude, top, targets, out,     \
                         slices, part);                                        \
      DAVET_HIP(hipGetLastError());                                            \
    }                                                                          \
    if (slices > 1) {                                                          \
      ProfScope ps(KC_MISC, stream);                                           \
      hipLaunchKernelGGL(logprobs_join_kernel<F>, dim3(rows), dim3(64),        \
                         (size_t)slices * top * 8, stream, x, ld, vocab,       \
                         exclude, top, targets, out, slices, part, rows);      \
      DAVET_HIP(hipGetLastError());                                            \
    }                                                                          \
  } while (0)
  if (dtype == DAVET_F16) LOGP(F16S);
  else if (dtype == DAVET_BF16) LOGP(BF16S);
  else LOGP(F32S);
#undef LOGP
  return DAVET_OK;
}
