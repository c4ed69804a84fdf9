// Rows of logits in one pass: log-sum-exp, entropy and the top k of each, for the
// token log probabilities (logprobs.hip) and the beams (beam.hip).
//
// With m the largest logit, c = log2(e) and t = c (x - m):
//   S = sum 2^t,  B = sum 2^t t
//   log p(w) = x_w - m - ln S,   entropy = ln S - B / (c S)
//
// A row is cut into slices of one workgroup (one slice from 256 rows on); each of
// its eight wavefronts walks its part in batches of 8 KB held in registers as
// they came, the next batch on its way while one is worked on.  The top k (at
// most 64) of a wavefront is a sorted list with one entry a lane, as 64-bit keys
// whose order is the wanted one; values enter one by one.  So that few do, each of
// the A wavefronts finds the ceil(k / A)-th largest of its lanes' maxima over its
// first batch: the smallest of them bounds the row's k-th value from below.  Two
// sorted lists join by one compare against the reversed other and six exchange
// steps: in LDS between the wavefronts, and in a second launch between the slices
// of a row where there are several.  Rows of up to 1024 logits have a kernel of their
// own, below.
//
// Measured with 126,464 logits a row.  256 fp32 rows: 27 us without a list (4.7
// TB/s of logits), 32 with the top 20; bf16 18 and 27 us (3.5 and 2.4 TB/s): bound
// by HBM and, in 16 bits, by the eight instructions and one exponential a logit; what
// of the list's 9 us is finding candidates and what inserting them (about 100 cycles
// each) is not measured.  (Sorting the candidates of a wavefront at once instead took
// 64 kept ones from 19 to 17 us in two rows, but 20 of 256 rows from 27 to 31.)  Two
// rows, 15 slices each: 7.0 us and 4 to join them, the latency of two launches; one
// slice a row takes 22.

#pragma once

#include <math.h>

#include <algorithm>

#include "cache.h"

namespace davet {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxSlices = 16;
constexpr int kWaves = 8;

struct Stat { float m, S, B; };       // m = -inf: nothing yet

__device__ __forceinline__ Stat stat_none() { return {-INFINITY, 0.f, 0.f}; }
__device__ __forceinline__ Stat stat_to(const Stat& a, float m) {
  // nothing yet: its sums are 0 (or NaN, which stays)
  const float d = a.m == -INFINITY ? 0.f : (a.m - m) * kLog2e;
  const float e = __builtin_amdgcn_exp2f(d);
  return {m, a.S * e, a.S != 0.f && e != 0.f ? e * fmaf(a.S, d, a.B) : 0.f * a.S};
}
__device__ __forceinline__ Stat stat_join(const Stat& a, const Stat& b) {
  const float m = fmaxf(a.m, b.m);
  const Stat x = stat_to(a, m), y = stat_to(b, m);
  return {m, x.S + y.S, x.B + y.B};
}
template <int O>
__device__ __forceinline__ Stat stat_step(const Stat& s) {
  return stat_join(s, {lane_xor<O>(s.m), lane_xor<O>(s.S), lane_xor<O>(s.B)});
}
__device__ __forceinline__ Stat stat_wave(Stat s) {
  s = stat_step<1>(s);
  s = stat_step<2>(s);
  s = stat_step<4>(s);
  s = stat_step<8>(s);
  s = stat_step<16>(s);
  return stat_step<32>(s);
}
// one logit; ref: s.m, or 0 while that is -inf; without B where no entropy is asked for
template <bool B = true>
__device__ __forceinline__ void term(float x, float ref, Stat& s) {
  const float t = (x - ref) * kLog2e;
  const float e = __builtin_amdgcn_exp2f(t);
  s.S += e;
  if (B) s.B = fmaf(e, fmaxf(t, -200.f), s.B);     // -inf: 0 times a finite number
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
  // every lane's left neighbour (DPP wave_shr:1)
  const uint64_t up =
      (uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(0, (int)(list >> 32), 0x138,
                                                      0xf, 0xf, false) << 32 |
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)list, 0x138, 0xf, 0xf,
                                            false);
  list = lane < at ? list : lane == at ? key : up;
}
// One step of a bitonic network: of each pair (l, l ^ O) the larger to the lower
// lane, or, where lane & S, to the upper one.
template <int O, int S>
__device__ __forceinline__ uint64_t exchange(uint64_t v) {
  const uint64_t y = lane_xor<O>(v);
  const bool larger = ((threadIdx.x & O) == 0) == ((threadIdx.x & S & 63) == 0);
  return larger == (v > y) ? v : y;
}
// steps O, O / 2, .. 1
template <int O, int S>
__device__ __forceinline__ uint64_t exchanges(uint64_t v) {
  v = exchange<O, S>(v);
  if constexpr (O > 1) v = exchanges<O / 2, S>(v);
  return v;
}
// the 64 largest of two descending lists, the second one given in reverse
__device__ __forceinline__ uint64_t list_join(uint64_t list, uint64_t reversed) {
  return exchanges<32, 64>(list > reversed ? list : reversed);
}
// 64 keys into ascending order (descending order of the complements)
__device__ __forceinline__ uint64_t sort_up(uint64_t v) {
  v = exchanges<1, 2>(~v);
  v = exchanges<2, 4>(v);
  v = exchanges<4, 8>(v);
  v = exchanges<8, 16>(v);
  v = exchanges<16, 32>(v);
  return ~exchanges<32, 64>(v);
}
// lane l's value in lane 63 - l
__device__ __forceinline__ uint64_t lane_reverse(uint64_t v) {
  v = lane_xor<1>(v);
  v = lane_xor<2>(v);
  v = lane_xor<4>(v);
  v = lane_xor<8>(v);
  v = lane_xor<16>(v);
  return lane_xor<32>(v);
}
// The lists of W wavefronts (entries past k do not count) into wavefront 0's; called
// by all, once.  Short ones at once (two rows' top 5: 7.4 to 7.0 us), longer ones in
// log2 W steps.
template <int W>
__device__ __forceinline__ void join_waves(uint64_t& list, int k, int wave,
                                           uint64_t (*s_list)[64]) {
  static_assert(W == 4 || W == 8);
  const int lane = threadIdx.x & 63;
  constexpr int P = 64 / W;
  if (k <= P) {
    if (lane < P) s_list[0][wave * P + (wave & 1 ? P - 1 - lane : lane)] = lane < k ? list : 0;
    __syncthreads();
    if (wave != 0) return;
    list = s_list[0][lane];
    if (W == 8) list = exchanges<8, 16>(list);
    list = exchanges<32, 64>(exchanges<16, 32>(list));
    return;
  }
#pragma unroll
  for (int o = 1; o < W; o <<= 1) {
    if (lane >= k) list = 0;
    if ((wave & (2 * o - 1)) == o) s_list[wave / (2 * o)][lane] = list;
    __syncthreads();
    if (k > 0 && (wave & (2 * o - 1)) == 0)
      list = list_join(list, s_list[wave / (2 * o)][63 - lane]);
    __syncthreads();
  }
}
// largest of the 64 lanes' values, in every lane: DPP row shifts by 1, 2, 4, 8 and
// the two row broadcasts leave it in lane 63
__device__ __forceinline__ float max_of_lanes(float x) {
  const int none = __float_as_int(-INFINITY);
#define STEP(ctrl, rows)                                                       \
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(                     \
                   none, __float_as_int(x), ctrl, rows, 0xf, false)))
  STEP(0x111, 0xf);
  STEP(0x112, 0xf);
  STEP(0x114, 0xf);
  STEP(0x118, 0xf);
  STEP(0x142, 0xa);
  STEP(0x143, 0xc);
#undef STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
// j-th largest of the 64 lanes' values, or -inf once there are none
__device__ __forceinline__ float jth_of_lanes(float x, int j) {
  float m = max_of_lanes(x);
  for (; j > 1 && m > -INFINITY; --j) {
    const uint64_t who = __ballot(x == m);
    if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)who) - 1) x = -INFINITY;
    m = max_of_lanes(x);
  }
  return m;
}
// the smallest float above x (finite)
__device__ __forceinline__ float above(float x) {
  return key_value(top_key(x, 0) + (1ull << 32));
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

// and back, values that came from unpack (or -inf)
template <typename F>
__device__ __forceinline__ u32x4 pack(const float* x) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F::dtype == DAVET_F32)
      w[i] = __float_as_uint(x[i]);
    else
      w[i] = F::store2(x[2 * i], x[2 * i + 1]);
  }
  return w;
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
  const double z = (double)s.m + lnS;
  if (lane == 0) {
    if (out.logp) {
      const int t = targets[row];
      float v = -INFINITY;                        // no such token
      if ((unsigned)t < (unsigned)vocab && t != exclude && s.S != 0.f)
        v = (float)((double)F::load(x[t]) - z);
      out.logp[row] = v;
    }
    if (out.entropy)                              // nothing to choose from: 0
      out.entropy[row] = s.S == 0.f ? 0.f : lnS - s.B / s.S * (1.0f / kLog2e);
  }
  if (lane < k) {
    out.top_ids[(int64_t)row * k + lane] = list ? key_id(list) : -1;
    out.top_logp[(int64_t)row * k + lane] =
        list ? (float)((double)key_value(list) - z) : -INFINITY;
  }
}

// partial results: [rows][slices][k] keys, then [rows][slices] Stat; one wavefront
// leaves entry `at` of n
__device__ __forceinline__ void leave(char* part, int64_t n, int64_t at, int k,
                                      const Stat& s, uint64_t list) {
  const int lane = threadIdx.x & 63;
  uint64_t* pl = reinterpret_cast<uint64_t*>(part);
  if (lane < k) pl[at * k + lane] = list;
  if (lane == 0) reinterpret_cast<Stat*>(pl + n * k)[at] = s;
}

constexpr int kBatch = 8;     // 16-byte loads a lane and batch

// PART: leaves a row's list and Stat in `part` even where it has one slice; rows with
// a `skip` entry other than 0 (NULL: none) leave nothing.
template <typename F, bool PART>
__global__ void __launch_bounds__(64 * kWaves)
logprobs_kernel(const typename F::st* __restrict__ logits, int64_t ld, int vocab,
                int exclude, int k, const int32_t* __restrict__ targets, Out out,
                int slices, char* __restrict__ part, const int32_t* __restrict__ skip) {
  using st = typename F::st;
  constexpr int N = Vec<F>::N;
  __shared__ uint64_t s_list[kWaves / 2][64];
  __shared__ Stat s_stat[kWaves];
  __shared__ float s_bound[kWaves];
  const int row = blockIdx.x / slices, slice = blockIdx.x % slices;
  if (PART && skip && skip[row]) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const st* x = logits + (int64_t)row * ld;
  // [0, head) and [tail, vocab): elements outside whole 16-byte pieces
  const int head = min(vocab, (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(st));
  const int nvec = (vocab - head) / N, tail = head + nvec * N;
  const u32x4* xv = reinterpret_cast<const u32x4*>(x + head);

  Stat s = stat_none();
  uint64_t list = 0;
  float bound = -INFINITY;      // no value below it is among the row's top k
  uint64_t kth = 0;             // the list's k-th entry
  auto insert = [&](uint64_t who, uint64_t key) {
    while (who) {
      const int l = __ffsll((unsigned long long)who) - 1;
      who &= who - 1;
      list_insert(list, lane64(key, l));
    }
  };

  // this wavefront's 16-byte pieces; all have as many batches
  const int parts = slices * kWaves, mine = slice * kWaves + wave;
  const int per = ((nvec + parts - 1) / parts + 63) & ~63;
  const int v0 = min(nvec, mine * per), v1 = min(nvec, v0 + per);
  u32x4 w[kBatch], next[kBatch];
  auto load = [&](int b, u32x4 (&d)[kBatch]) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (b + u * 64 < v1) d[u] = xv[min(b + u * 64 + lane, v1 - 1)];
  };
  load(v0, next);
  for (int b = v0, i = 0; i < per; i += 64 * kBatch, b += 64 * kBatch) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) w[u] = next[u];
    load(b + 64 * kBatch, next);
    float mx = -INFINITY, vmax[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      vmax[u] = -INFINITY;
      if (b + u * 64 >= v1) continue;
      const int first = head + (b + u * 64) * N;
      // lanes past the end, and the excluded token, hold -inf
      if (b + u * 64 + 64 > v1 || (exclude >= first && exclude < first + 64 * N)) {
        float v[N];
        unpack<F>(w[u], v);
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (b + u * 64 + lane >= v1 || first + lane * N + e == exclude)
            v[e] = -INFINITY;
        w[u] = pack<F>(v);
      }
      float v[N];
      unpack<F>(w[u], v);
#pragma unroll
      for (int e = 0; e < N; ++e) vmax[u] = fmaxf(vmax[u], v[e]);
      mx = fmaxf(mx, vmax[u]);
    }
    if (mx > s.m) s = stat_to(s, mx);
    const float ref = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (b + u * 64 >= v1) continue;
      float v[N];
      unpack<F>(w[u], v);
#pragma unroll
      for (int e = 0; e < N; ++e) term<!PART>(v[e], ref, s);
    }
    if (k == 0) continue;
    if (i == 0) {
      // (by the wavefronts whose lanes all have values; by the first, if none)
      const int got = nvec - slice * kWaves * per;
      const int A = max(1, min(kWaves, got / per + (got % per >= 64)));
      const float j = wave < A ? jth_of_lanes(mx, (k + A - 1) / A) : INFINITY;
      if (lane == 0) s_bound[wave] = j;
      __syncthreads();
      bound = s_bound[0];
#pragma unroll
      for (int o = 1; o < kWaves; ++o) bound = fminf(bound, s_bound[o]);
    }
    // wanted: above -inf, not below the bound, and above the list's k-th entry
    // (a later equal value has a higher id)
    const float least = fmaxf(fmaxf(bound, -3.402823466e38f),
                              kth ? above(key_value(kth)) : -INFINITY);
    if (!__any(mx >= least)) continue;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (!__any(vmax[u] >= least)) continue;
      float v[N];
      unpack<F>(w[u], v);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint64_t who = __ballot(v[e] >= least);
        if (who)
          insert(who, top_key(v[e], head + (b + u * 64 + lane) * N + e));
      }
    }
    kth = lane64(list, k - 1);
  }
  if (mine == parts - 1 && (head || tail < vocab)) {
    // the edges, fewer than 16 values (whole keys decide: their ids may be
    // lower than those of equal values listed)
    const int ne = head + vocab - tail;
    const int id = lane < head ? lane : tail + lane - head;
    const float v = lane < ne && id != exclude ? F::load(x[id]) : -INFINITY;
    if (k > 0) insert(__ballot(v > -INFINITY), top_key(v, id));
    if (v > s.m) s = stat_to(s, v);
    term<!PART>(v, s.m == -INFINITY ? 0.f : s.m, s);
  }
  s = stat_wave(s);
  if (lane == 0) s_stat[wave] = s;
  join_waves<kWaves>(list, k, wave, s_list);
  if (wave != 0) return;
  s = stat_wave(lane < kWaves ? s_stat[lane] : stat_none());
  if (!PART && slices == 1) {
    finish<F>(s, list, row, vocab, exclude, k, x, targets, out);
    return;
  }
  leave(part, (int64_t)gridDim.x, blockIdx.x, k, s, list);
}

// A row of at most 64 kWaves kShort logits, one workgroup: a lane holds up to kShort
// of them, wavefront w the runs of 64 w, w + 8, ..; each run is sorted and joined to
// the wavefront's list.  Batches of 8 KB would give such a row to one wavefront, and
// a list of its inserts: 98 rows of 326, top 64, 28 us, 7.2 so; 4096 rows of 1000,
// top 20, 74 and 44 us.  From about 2000 logits on the sorts are the slower ones (98
// rows of 4096, top 20: 13.4 us, 8.0 by inserts).
constexpr int kShort = 2;
template <typename F, bool PART>
__global__ void __launch_bounds__(64 * kWaves)
logprobs_short_kernel(const typename F::st* __restrict__ logits, int64_t ld,
                      int vocab, int exclude, int k,
                      const int32_t* __restrict__ targets, Out out,
                      char* __restrict__ part, const int32_t* __restrict__ skip) {
  __shared__ uint64_t s_list[kWaves / 2][64];
  __shared__ Stat s_stat[kWaves];
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  if (PART && skip && skip[row]) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const typename F::st* x = logits + (int64_t)row * ld;
  float v[kShort];
#pragma unroll
  for (int i = 0; i < kShort; ++i) {
    const int id = (i * kWaves + wave) * 64 + lane;
    v[i] = id < vocab ? F::load(x[id]) : -INFINITY;
    if (id == exclude) v[i] = -INFINITY;
  }
  Stat s = stat_none();
#pragma unroll
  for (int i = 0; i < kShort; ++i) s.m = fmaxf(s.m, v[i]);
  const float ref = s.m == -INFINITY ? 0.f : s.m;
  uint64_t list = 0;
#pragma unroll
  for (int i = 0; i < kShort; ++i) {
    const int first = (i * kWaves + wave) * 64;
    if (first >= vocab) break;
    term<!PART>(v[i], ref, s);
    if (k == 0) continue;
    const uint64_t run = sort_up(v[i] > -INFINITY ? top_key(v[i], first + lane) : 0);
    list = i == 0 ? lane_reverse(run) : list_join(list, run);
  }
  s = stat_wave(s);
  if (lane == 0) s_stat[wave] = s;
  join_waves<kWaves>(list, k, wave, s_list);
  if (wave != 0) return;
  s = stat_wave(lane < kWaves ? s_stat[lane] : stat_none());
  if constexpr (PART)
    leave(part, gridDim.x, row, k, s, list);
  else
    finish<F>(s, list, row, vocab, exclude, k, x, targets, out);
}

// Slices a row: 256 workgroups fill the chip, at least 8192 logits each (two rows of
// 126,464 take 22 us in one slice each, 11.5 in 15; 256 rows 27 in one, 31 in two).
int plan_slices(int rows, int vocab) {
  const int want = (256 + rows - 1) / rows;
  return std::max(1, std::min({want, kMaxSlices, vocab / 8192}));
}

}  // namespace
}  // namespace davet
