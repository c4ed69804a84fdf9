// Pages that a cheap score selects: the elementwise bounds of each page's keys, and the
// choice of pages for each new token and key head.  (Their attention:
// cache_page_attention.hip.)
//
// For a page with keys k_j, lo = min_j k_j and hi = max_j k_j, element by element:
//   q.k_j = sum_e q_e k_je <= sum_e max(q_e lo_e, q_e hi_e) = q+.hi + q-.lo
// with q+ = max(q, 0), q- = min(q, 0).  The query heads that share a key head choose
// together, by the sum of their bounds; that is one product with Q+ = sum q+ and
// Q- = sum q-, whatever their number.
//
// That product is NaN where an infinite bound meets a half of Q that is 0 because of the
// signs (q = 1, lo = -inf: max(q lo, q hi) is q hi, but Q- lo is 0 times an infinity).  An
// infinity or NaN among bounds or queries always leaves a sum that is not finite, so
// such pages, and no others, are scored again term by term.
//
// Scores are float64 sums rounded to float32, and equal ones go to the lower page.  The
// forms below add in different orders: of 16-bit values products are exact, and sums too
// unless they span more than 2^20 or so; then, and in fp32, a score may seldom come out
// as the neighbouring float32.
//
// Three forms:
//   group  a workgroup each (token, key head)
//   waves  where they are many: a wavefront each, by vector ops, no LDS
//   tiles  many, and chunks of 8 tokens and more: 16 tokens x 16 pages by float64 matrix
//          ops, which read a page's bounds once for all 16
// In the last two a page's bounds are read 16 bytes a lane by 16 to 64 lanes, which keep
// their elements of Q in registers; the sums of several pages are added over the lanes
// and dealt out to them at once.
//
// Then the key of the last page taken is found from its highest bit down, by counting,
// and the pages are written in ascending order.
//
// Measured with 8 key heads of 128, 16 bits.  Bounds of a page 4 to 5 us (a chain of
// loads); of 49,408 tokens' pages, over and over, 72 us in pages of 16 (1.6 TB/s: 4 KB of
// work a workgroup, and of each lane's four loads three repeat the last row), 40 of 32,
// 22 of 64 (4.8 TB/s; fp32 40 and 32, 5.7 and 6.6 TB/s, part of it from the last-level
// cache).
// The choice of 64 of up to 1022 pages for eight tokens 21.4 us, of them 16 the scores:
// vector ops, three of each 16-bit element's five being its way to float64 and its
// product, 64 CUs at work (fp32 2 us more).  Of 32 among up to 234 for 512 tokens 20.4 us
// (fp32 the same): about 7 of launch, loads and Q's sums, 9 of products (6.8 at the
// float64 matrix rate, 64 cycles for 16 x 16 x 4) and 6 of ranking, each timed by leaving
// the others out; of 64 pages 13.7, of them 4, 4 and 6.

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "cache.h"

namespace davet {
namespace {

// ---- bounds

struct BoundsPack {
  int32_t n_seqs;
  int32_t item[DAVET_MAX_SEQS + 1];   // first (page) item of each sequence
  int32_t page[DAVET_MAX_SEQS];       // its first page
  int32_t kv[DAVET_MAX_SEQS];
};

// min and max that keep a NaN
__device__ __forceinline__ float min_nan(float a, float b) {
  return a != a || a < b ? a : b;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  return a != a || a > b ? a : b;
}

// One workgroup a (page, key head): each wavefront every fourth group of rows.  The
// values are the keys' own, so storing them rounds nothing.
template <typename F, int D>
__global__ void __launch_bounds__(256)
page_bounds_kernel(CacheView cv, BoundsPack bp, typename F::st* __restrict__ bounds,
                   int wg0) {
  using st = typename F::st;
  constexpr int N = 16 / (int)sizeof(st);       // elements a lane
  constexpr int C = D / N, R = 64 / C;          // lanes a row, rows a load
  constexpr int U = 4;
  __shared__ float s_lo[4][D], s_hi[4][D];
  const int wg = wg0 + (int)blockIdx.x, item = wg / cv.n_kv, h = wg % cv.n_kv;
  const Lanes items(bp.item);
  const int pages = bp.page[threadIdx.x & 63], kvs = bp.kv[threadIdx.x & 63];
  const int s = items.owner(bp.n_seqs, item), psz = 1 << cv.lg;
  const int page = __builtin_amdgcn_readlane(pages, s) + item - items.start(s);
  const int phys = cv.table[(int64_t)s * cv.max_pages + page];
  if ((unsigned)phys >= (unsigned)cv.n_pages) return;
  const int valid = min(psz, __builtin_amdgcn_readlane(kvs, s) - page * psz);
  const int lane = threadIdx.x & 63, c = lane % C;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t at = (int64_t)phys * cv.n_kv + h;
  const st* k = static_cast<const st*>(cv.k) + (at << cv.lg) * D + c * N;
  float lo[N], hi[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    lo[e] = INFINITY;
    hi[e] = -INFINITY;
  }
  for (int r0 = wave * R; r0 < valid; r0 += 4 * R * U) {
    u32x4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      w[u] = *reinterpret_cast<const u32x4*>(
          k + (int64_t)min(r0 + u * 4 * R + lane / C, valid - 1) * D);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float x;
        if constexpr (F::dtype == DAVET_F32)
          x = __uint_as_float(w[u][e]);
        else
          x = F::load((uint16_t)(w[u][e >> 1] >> (16 * (e & 1))));
        lo[e] = min_nan(lo[e], x);
        hi[e] = max_nan(hi[e], x);
      }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
#pragma unroll
    for (int o = C; o < 64; o <<= 1) {
      lo[e] = min_nan(lo[e], __shfl_xor(lo[e], o, 64));
      hi[e] = max_nan(hi[e], __shfl_xor(hi[e], o, 64));
    }
    if (lane < C) {
      s_lo[wave][c * N + e] = lo[e];
      s_hi[wave][c * N + e] = hi[e];
    }
  }
  __syncthreads();
  const int e = threadIdx.x;
  if (e < 2 * D) {
    const bool upper = e >= D;
    const float(*sv)[D] = upper ? s_hi : s_lo;
    float x = sv[0][e % D];
#pragma unroll
    for (int w = 1; w < 4; ++w)
      x = upper ? max_nan(x, sv[w][e % D]) : min_nan(x, sv[w][e % D]);
    bounds[at * 2 * D + e] = F::store(x);
  }
}

// ---- selection

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kMaxPages = 32768;        // of a sequence: their keys fill the LDS
constexpr int kFewPages = 4096;         // whose keys a wavefront's registers hold
constexpr int kManyItems = 1024;        // of them a wavefront each

// order of a score: larger first; NaN with -inf, -0 with +0; never 0
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) x = -INFINITY;
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kAgain = 1;  // no score's: one still to be worked out term by term

// a where this lane's bit O is clear, b where it is set, each plus that of lane ^ O
template <int O>
__device__ __forceinline__ double deal(double a, double b) {
  const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
  if constexpr (O >= 16) {
    uint32_t p[2], q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t xi = (uint32_t)(x >> (32 * i)), yi = (uint32_t)(y >> (32 * i));
      if constexpr (O == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(xi, yi, false, false);
        p[i] = r[0];
        q[i] = r[1];
      } else {
        const auto r = __builtin_amdgcn_permlane16_swap(xi, yi, false, false);
        p[i] = r[0];
        q[i] = r[1];
      }
    }
    return __builtin_bit_cast(double, (uint64_t)p[1] << 32 | p[0]) +
           __builtin_bit_cast(double, (uint64_t)q[1] << 32 | q[0]);
  } else {
    const bool set = threadIdx.x & O;
    const uint64_t keep = set ? y : x, send = set ? x : y;
    return __builtin_bit_cast(double, keep) +
           __builtin_bit_cast(double, lane_xor<O>(send));
  }
}

// Scores of one (token, key head).
template <typename F, int D>
struct Scorer {
  using st = typename F::st;
  static constexpr int N = 16 / (int)sizeof(st);    // elements a lane
  static constexpr int LP = 2 * D / N;              // lanes a page: lo, then hi
  static constexpr int H = LP / 2;
  double q[N];          // of this lane's elements: Q- in the lower half, Q+ above
  const char* bounds;   // of key head hk of page 0, at this lane's elements
  uint32_t page;        // bytes from page to page

  __device__ __forceinline__ static float elem(const u32x4& w, int e) {
    if constexpr (F::dtype == DAVET_F32)
      return __uint_as_float(w[e]);
    else
      return F::load((uint16_t)(w[e >> 1] >> (16 * (e & 1))));
  }
  // what a query's element adds to Q- or Q+ (a NaN to both)
  __device__ __forceinline__ static double part(float v, bool lower) {
    return (double)(lower ? (v > 0.f ? 0.f : v) : (v < 0.f ? 0.f : v));
  }
  __device__ __forceinline__ void prepare(const st* b, int n_kv, int hk) {
    bounds = reinterpret_cast<const char*>(b + (int64_t)hk * 2 * D +
                                           (threadIdx.x & (LP - 1)) * N);
    page = (uint32_t)(n_kv * 2 * D * (int)sizeof(st));
  }
  // heads: the g query heads' rows
  __device__ __forceinline__ void init(const st* heads, int g) {
    const int l = threadIdx.x & (LP - 1);
#pragma unroll
    for (int e = 0; e < N; ++e) q[e] = 0.0;
    for (int h = 0; h < g; ++h) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(heads + (int64_t)h * D +
                                                      (l & (H - 1)) * N);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        q[e] += part(elem(w, e), l < H);
      }
    }
  }
  // The score by its definition, term by term: of the g query heads' rows at `heads` for
  // the page whose bounds start at b.
  __device__ __forceinline__ static float defined(const st* heads, int g, const st* b) {
    double x = 0.0;
#pragma unroll 1
    for (int i = 0; i < g * H; ++i) {
      const int at = i % H * N;
      const u32x4 w = *reinterpret_cast<const u32x4*>(heads + (int64_t)(i / H) * D + at);
      const u32x4 lo = *reinterpret_cast<const u32x4*>(b + at);
      const u32x4 hi = *reinterpret_cast<const u32x4*>(b + D + at);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const double u = (double)elem(w, e) * (double)elem(lo, e);
        const double v = (double)elem(w, e) * (double)elem(hi, e);
        x += u != u || u > v ? u : v;           // (a NaN stays)
      }
    }
    return (float)x;
  }
  // of the 64 pages whose places the lanes hold (0 for none): lane l's score is its own
  // page's
  __device__ __forceinline__ float score64(int phys) const {
    const int lane = threadIdx.x & 63;
    // page u 4 + j + b H of each LP lanes' share: b the highest bit of a lane's number
    // in it, j the lowest two
    auto load = [&](int u, u32x4 (&w)[8]) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        w[i] = read(__shfl(phys, (lane & ~(LP - 1)) + u * 4 + (i & 3) + (i >> 2) * H, 64));
    };
    u32x4 w[2][8];
    load(0, w[0]);
    double sum[LP / 8];
#pragma unroll
    for (int u = 0; u < LP / 8; ++u) {
      if (u + 1 < LP / 8) load(u + 1, w[(u + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
      sum[u] = eight(w[u & 1]);
    }
    if constexpr (LP >= 64)
#pragma unroll
      for (int u = 0; u < LP / 16; ++u) sum[u] = deal<16>(sum[u], sum[u + LP / 16]);
    if constexpr (LP >= 32)
#pragma unroll
      for (int u = 0; u < 2; ++u) sum[u] = deal<8>(sum[u], sum[u + 2]);
    return (float)deal<4>(sum[0], sum[1]);
  }
  // of 8 pages for each LP lanes: theirs is page (lane & 3) + (lane & H ? 4 : 0)
  static constexpr int PAGES = 8 * 64 / LP;         // of a wavefront
  __device__ __forceinline__ float score8(const u32x4 (&w)[8]) const {
    double x = eight(w);
    x += swapped<4>(x);
    if constexpr (LP >= 32) x += swapped<8>(x);
    if constexpr (LP >= 64) x += swapped<16>(x);
    return (float)x;
  }
  __device__ __forceinline__ u32x4 read(int phys) const {
    // (one multiply-add of 32 x 32 bits: of 64 x 64 they were an eighth of the loop)
    return *reinterpret_cast<const u32x4*>(bounds + (uint64_t)(uint32_t)phys * page);
  }

 private:
  template <int O>
  __device__ __forceinline__ static double swapped(double x) {
    return __builtin_bit_cast(double, lane_xor<O>(__builtin_bit_cast(uint64_t, x)));
  }
  __device__ __forceinline__ double eight(const u32x4 (&w)[8]) const {
    double x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = 0.0;
#pragma unroll
      for (int e = 0; e < N; ++e) x[i] = fma((double)elem(w[i], e), q[e], x[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = deal<H>(x[i], x[i + 4]);
    return deal<2>(deal<1>(x[0], x[1]), deal<1>(x[2], x[3]));
  }
};

// What a selection is about: pages 0 .. np of sequence s, for one token and key head.
struct Choice {
  int s, np, hk;
  const int32_t* table;
  int32_t* out;
};
__device__ __forceinline__ Choice choice_of(const CacheView& cv, const ChunkPack& cp,
                                            int64_t item, int block, int top,
                                            int32_t* out, int* row) {
  Choice c;
  *row = (int)(item / cv.n_kv);
  c.hk = (int)(item - (int64_t)*row * cv.n_kv);
  const Lanes rows(cp.row0);
  const int kvs = cp.kv[threadIdx.x & 63];
  c.s = rows.owner(cp.n_seqs, *row);
  const int row0 = rows.start(c.s), n = rows.end(c.s) - row0;
  const int kv = __builtin_amdgcn_readlane(kvs, c.s);
  c.np = (visible_end(*row - row0, n, kv, block) + (1 << cv.lg) - 1) >> cv.lg;
  c.table = cv.table + (int64_t)c.s * cv.max_pages;
  c.out = out + item * top;
  return c;
}
__device__ __forceinline__ uint32_t lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
}

// the largest of the lanes' values
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  x = max(x, lane_xor<1>(x));
  x = max(x, lane_xor<2>(x));
  x = max(x, lane_xor<4>(x));
  x = max(x, lane_xor<8>(x));
  x = max(x, lane_xor<16>(x));
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)max(x, lane_xor<32>(x)));
}

// The pages of one item by one wavefront: lane l's kr[i] is the key of page 64 i + l, 0
// past the last one.  (No loop over them stops early: 16 branches a round took 7 us of
// a selection's 12.)
template <int R>
__device__ __forceinline__ void choose(const uint32_t (&kr)[R], int top, bool all,
                                       int32_t* out) {
  const int lane = threadIdx.x & 63;
  auto at_least = [&](uint32_t x) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) n += (uint32_t)__popcll(__ballot(kr[i] >= x));
    return n;
  };
  const uint32_t keep = min((uint32_t)top, at_least(1u));
  uint32_t T = 1;                       // key of the last page taken, or one below it
  if (!all && keep > 0) {
    T = 0xffffffffu;
    if (at_least(T) < keep) {           // (that many are sure)
      // the rest from what their keys begin with
      uint32_t least = 0xfffffffeu, most = 1;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const bool ranked = kr[i] - 1u < 0xfffffffeu;
        least = ranked ? min(least, kr[i]) : least;
        most = ranked ? max(most, kr[i]) : most;
      }
      least = ~lanes_max(~least);
      most = lanes_max(most);
      const int bits = 32 - __builtin_clz((least ^ most) | 1);
      T = most >> (bits - 1) >> 1 << (bits - 1) << 1;
      for (int b = bits - 1; b >= 0; --b) {
        const uint32_t x = T | 1u << b, n = at_least(x);
        if (n == keep) {                // (a border between keys: half the rounds)
          T = x - 1;
          break;
        }
        if (n > keep) T = x;
      }
    }
  }
  uint32_t gts = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) gts += (uint32_t)__popcll(__ballot(kr[i] > T));
  const uint32_t need = keep - gts;     // of those equal to T, the first ones
  uint32_t gt0 = 0, eq0 = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const uint64_t mg = __ballot(kr[i] > T), me = __ballot(kr[i] == T);
    const uint32_t rg = gt0 + lanes_below(mg), re = eq0 + lanes_below(me);
    if (kr[i] > T || (kr[i] == T && re < need)) out[rg + min(re, need)] = i * 64 + lane;
    gt0 += (uint32_t)__popcll(mg);
    eq0 += (uint32_t)__popcll(me);
  }
  for (int i = (int)keep + lane; i < top; i += 64) out[i] = -1;
}

// One workgroup an item.  CAP: pages that the LDS holds keys of.
template <typename F, int D, int CAP>
__global__ void __launch_bounds__(kSelThreads)
page_select_kernel(CacheView cv, ChunkPack cp, const typename F::st* __restrict__ q,
                   int64_t ld_q, int n_heads, int block,
                   const typename F::st* __restrict__ bounds, int first, int last,
                   int top, int32_t* __restrict__ out, int wg0) {
  using S = Scorer<F, D>;
  constexpr int P = S::PAGES;                   // a wavefront's pages at a time
  __shared__ uint32_t s_keys[CAP];
  __shared__ __attribute__((aligned(16))) uint32_t s_cnt[2][3][kSelWaves];
  int row;
  const Choice c = choice_of(cv, cp, wg0 + (int)blockIdx.x, block, top, out, &row);
  const int np = c.np, g = n_heads / cv.n_kv;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool all = np <= top;                   // nothing to choose

  if (all) {
    for (int p = threadIdx.x; p < ((np + 63) & ~63); p += kSelThreads)
      s_keys[p] = p < np && (unsigned)c.table[p] < (unsigned)cv.n_pages ? 0xffffffffu : 0u;
  } else if (wave * P < np) {
    auto place = [&](int p0) {                  // of page p0 + lane % P
      const int p = p0 + lane % P;
      return c.table[min(p, np - 1)];
    };
    auto known = [&](int id) { return (unsigned)id < (unsigned)cv.n_pages; };
    S sc;
    sc.prepare(bounds, cv.n_kv, c.hk);
    constexpr int STEP = kSelWaves * P;
    const int base = lane / S::LP * 8;          // this lane's pages in the step
    const int mine = base + (lane & 3) + (lane & S::H ? 4 : 0);
    u32x4 w[8];
    int id = place(wave * P), next = place(wave * P + STEP);
    auto load = [&](int ids) {
      const int safe = known(ids) ? ids : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = sc.read(__shfl(safe, base + i, 64));
    };
    load(id);
    const typename F::st* heads = q + (int64_t)row * ld_q + (int64_t)c.hk * g * D;
    sc.init(heads, g);
#pragma unroll 1
    for (int p0 = wave * P; p0 < np; p0 += STEP) {
      float x = sc.score8(w);
      const int now = __shfl(id, mine, 64), p = p0 + mine;
      // (the other lanes of a page have the same)
      const bool own = (lane & (S::H - 4)) == 0;
      if (own && !(fabsf(x) < INFINITY) && known(now) && p >= first && p < np - last)
        x = S::defined(heads, g, bounds + ((int64_t)now * cv.n_kv + c.hk) * 2 * D);
      id = next;
      if (p0 + STEP < np) load(id);
      next = place(p0 + 2 * STEP);
      if (own)
        s_keys[p] = p >= np || !known(now)             ? 0u
                    : p < first || p >= np - last ? 0xffffffffu
                                                  : score_key(x);
    }
  }
  // keys behind the last step's, up to whole 64s
  {
    const int from = all ? (np + 63) & ~63 : (np + P - 1) / P * P;
    if (from + (int)threadIdx.x < ((np + 63) & ~63)) s_keys[from + threadIdx.x] = 0;
  }
  __syncthreads();

  if constexpr (CAP <= kFewPages) {
    // One wavefront ranks them, and the next workgroup's may begin (eight lists of 1024
    // pages 21.8 us, by all 16 wavefronts 31.3; of 4096 66.6 and 71.6, 64 of them 113 and
    // 144).
    if (wave != 0) return;
    auto few = [&](auto r) {
      constexpr int R = decltype(r)::value;
      uint32_t kr[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const uint32_t k = s_keys[i * 64 + lane];
        kr[i] = i * 64 < np ? k : 0u;
      }
      choose(kr, top, all, c.out);
    };
    if (np <= 256) few(std::integral_constant<int, 4>());
    else if (np <= 512) few(std::integral_constant<int, 8>());
    else if (np <= 1024) few(std::integral_constant<int, 16>());
    else if (np <= 2048) few(std::integral_constant<int, 32>());
    else few(std::integral_constant<int, CAP / 64>());
    return;
  }
  // Each wavefront counts and writes a run of whole 64s.
  const int per = ((np + kSelWaves - 1) / kSelWaves + 63) & ~63;
  const int lo = min(np, wave * per), hi = min(np, lo + per);
  // f(64 pages' first one, their keys) of this wavefront
  auto each = [&](auto f) {
    for (int i = lo; i < hi; i += 64) f(i, s_keys[i + lane]);
  };
  // keys of this wavefront that are at least each of x, y, z (above 0)
  auto count = [&](uint32_t x, uint32_t y, uint32_t z, uint32_t (&cnt)[3]) {
    cnt[0] = cnt[1] = cnt[2] = 0;
    each([&](int, uint32_t k) {
      cnt[0] += (uint32_t)__popcll(__ballot(k >= x));
      cnt[1] += (uint32_t)__popcll(__ballot(k >= y));
      cnt[2] += (uint32_t)__popcll(__ballot(k >= z));
    });
  };
  int flip = 0;
  // Of all wavefronts; one barrier: the next call writes the other half.  (Each lane
  // reads one count: all of them in every lane, 16 wavefronts of reads, took 10 us of
  // a selection's 17.)
  static_assert(kSelWaves == 16, "a row of lanes");
  auto total = [&](uint32_t (&cnt)[3]) {
    if (lane < 3) s_cnt[flip][lane][wave] = lane == 0 ? cnt[0] : lane == 1 ? cnt[1] : cnt[2];
    __syncthreads();
    uint32_t x = s_cnt[flip][min(lane >> 4, 2)][lane & 15];
    x += lane_xor<1>(x);
    x += lane_xor<2>(x);
    x += lane_xor<4>(x);
    x += lane_xor<8>(x);
#pragma unroll
    for (int i = 0; i < 3; ++i) cnt[i] = (uint32_t)__builtin_amdgcn_readlane((int)x, 16 * i);
    flip ^= 1;
  };
  uint32_t cnt[3];
  count(1u, 1u, 1u, cnt);
  total(cnt);
  const uint32_t keep = min((uint32_t)top, cnt[0]);
  uint32_t T = 1;                       // key of the last page taken
  if (!all && keep > 0) {
    T = 0;
    for (int b = 30; b >= 0; b -= 2) {
      count(T | 1u << b, T | 2u << b, T | 3u << b, cnt);
      total(cnt);
      const uint32_t d = cnt[2] >= keep ? 3u : cnt[1] >= keep ? 2u : cnt[0] >= keep ? 1u : 0u;
      const uint32_t n = d == 3 ? cnt[2] : d == 2 ? cnt[1] : cnt[0];
      T |= d << b;
      if (d > 0 && n == keep) {                 // a border between keys
        --T;
        break;
      }
    }
  }
  // above T, and equal to it, in each wavefront
  count(T, T, T == 0xffffffffu ? T : T + 1, cnt);
  const uint32_t gt = T == 0xffffffffu ? 0u : cnt[2], eq = cnt[0] - gt;
  if (lane == 0) {
    s_cnt[flip][0][wave] = gt;
    s_cnt[flip][1][wave] = eq;
  }
  __syncthreads();
  // sums over the wavefronts before this one, and over all
  uint32_t gt0 = 0, eq0 = 0, gts = 0;
  {
    const uint32_t x = lane < 2 * kSelWaves ? s_cnt[flip][lane >> 4][lane & 15] : 0u;
    uint32_t before = (lane & 15) < wave ? x : 0u, sum = x;
    before += lane_xor<1>(before);
    before += lane_xor<2>(before);
    before += lane_xor<4>(before);
    before += lane_xor<8>(before);
    sum += lane_xor<1>(sum);
    sum += lane_xor<2>(sum);
    sum += lane_xor<4>(sum);
    sum += lane_xor<8>(sum);
    gt0 = (uint32_t)__builtin_amdgcn_readlane((int)before, 0);
    eq0 = (uint32_t)__builtin_amdgcn_readlane((int)before, 16);
    gts = (uint32_t)__builtin_amdgcn_readlane((int)sum, 0);
  }
  const uint32_t need = keep - gts;     // of those equal to T, the first ones
  if (keep > 0)
    each([&](int i, uint32_t k) {
      const uint64_t mg = __ballot(k > T), me = __ballot(k == T);
      const uint32_t rg = gt0 + lanes_below(mg), re = eq0 + lanes_below(me);
      if (k > T || (k == T && re < need)) c.out[rg + min(re, need)] = i + lane;
      gt0 += (uint32_t)__popcll(mg);
      eq0 += (uint32_t)__popcll(me);
    });
  for (int i = (int)keep + (int)threadIdx.x; i < top; i += kSelThreads) c.out[i] = -1;
}

// One wavefront an item of at most 64 kWaveSteps pages, whose keys are in registers.
constexpr int kWaveSteps = 8;
template <typename F, int D>
__global__ void __launch_bounds__(256)
page_select_wave_kernel(CacheView cv, ChunkPack cp, const typename F::st* __restrict__ q,
                        int64_t ld_q, int n_heads, int block,
                        const typename F::st* __restrict__ bounds, int first, int last,
                        int top, int32_t* __restrict__ out, int64_t items) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // neighbours in a workgroup: the tokens of one key head
  const int64_t at = (int64_t)blockIdx.x * 4 + wave;
  const int64_t rows = items / cv.n_kv;
  if (at >= items) return;
  const int64_t item = at % rows * cv.n_kv + at / rows;
  int row;
  const Choice c = choice_of(cv, cp, item, block, top, out, &row);
  const int np = c.np, g = n_heads / cv.n_kv, lane = threadIdx.x & 63;
  const bool all = np <= top;
  Scorer<F, D> sc;
  int next = c.table[min(lane, np - 1)];
  sc.prepare(bounds, cv.n_kv, c.hk);
  const typename F::st* heads = q + (int64_t)row * ld_q + (int64_t)c.hk * g * D;
  if (!all) sc.init(heads, g);
  uint32_t kr[kWaveSteps] = {};
  const int steps = (np + 63) / 64;
#pragma unroll 1
  for (int i = 0; i < steps; ++i) {
    const int p = i * 64 + lane;
    const bool there = p < np && (unsigned)next < (unsigned)cv.n_pages;
    const int phys = there ? next : 0;
    if (i + 1 < steps) next = c.table[min(p + 64, np - 1)];
    uint32_t key = 0xffffffffu;
    if (!all) {
      float x = sc.score64(phys);
      if (there && p >= first && p < np - last) {
        if (!(fabsf(x) < INFINITY))
          x = sc.defined(heads, g, bounds + ((int64_t)phys * cv.n_kv + c.hk) * 2 * D);
        key = score_key(x);
      }
    }
    if (!there) key = 0;
#pragma unroll
    for (int r = 0; r < kWaveSteps; ++r) kr[r] = r == i ? key : kr[r];
  }
  choose(kr, top, all, c.out);
}

// 16 tokens of a sequence against pages of one key head.  Matrix op (c, e) takes element
// e of chunk c of the lanes' pages, 16 of them by four lanes each, and the same element
// of Q of 16 tokens, which are in LDS; lane l then holds the scores of token l % 16 and
// pages 4 i + l / 16.
struct TilePack {
  int32_t first[DAVET_MAX_SEQS + 1];    // first tile of each sequence
};
constexpr int kTileTokens = 16, kTileThreads = 1024, kTileWaves = kTileThreads / 64;
// (16 bits: two workgroups a CU where their LDS allows it)
template <typename F, int D, int CAP>
__global__ void __launch_bounds__(kTileThreads, CAP <= 512 && F::dtype != DAVET_F32 ? 8 : 4)
page_select_tile_kernel(CacheView cv, ChunkPack cp, TilePack tp,
                        const typename F::st* __restrict__ q, int64_t ld_q, int n_heads,
                        int block, const typename F::st* __restrict__ bounds, int first,
                        int last, int top, int32_t* __restrict__ out, int wg0) {
  using st = typename F::st;
  using S = Scorer<F, D>;
  typedef double d4 __attribute__((ext_vector_type(4)));
  constexpr int N = S::N, LP = S::LP, NC = LP / 4;
  constexpr int KS = CAP + 1;                   // (tokens' keys in different banks)
  __shared__ double s_q[2 * D][kTileTokens];
  __shared__ uint32_t s_keys[kTileTokens * KS];
  const int wg = wg0 + (int)blockIdx.x, tile = wg / cv.n_kv, hk = wg % cv.n_kv;
  const Lanes tiles(tp.first), rows(cp.row0);
  const int kvs = cp.kv[threadIdx.x & 63];
  const int s = tiles.owner(cp.n_seqs, tile);
  const int tok0 = (tile - tiles.start(s)) * kTileTokens;
  const int row0 = rows.start(s), n = rows.end(s) - row0, lg = cv.lg;
  const int kv = __builtin_amdgcn_readlane(kvs, s);
  const int nt = min(kTileTokens, n - tok0), g = n_heads / cv.n_kv;
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t* table = cv.table + (int64_t)s * cv.max_pages;
  auto pages_of = [&](int tok) {
    return (visible_end(tok, n, kv, block) + (1 << lg) - 1) >> lg;
  };
  // (a later token sees no fewer)
  const int np = pages_of(tok0 + nt - 1), mine = pages_of(tok0 + min(l16, nt - 1));

  if (np > top) {
    for (int i = threadIdx.x; i < kTileTokens * LP; i += kTileThreads) {
      const int tok = i % kTileTokens, l = i / kTileTokens;     // (in LDS side by side)
      double x[N] = {};
      const st* qp = q + (int64_t)(row0 + tok0 + min(tok, nt - 1)) * ld_q +
                     (int64_t)hk * g * D + l % S::H * N;
      for (int h = 0; h < g; ++h) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(qp + (int64_t)h * D);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] += S::part(S::elem(w, e), l < S::H);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) s_q[l * N + e][tok] = x[e];
    }
    __syncthreads();
  }
  for (int p0 = wave * 16; p0 < np; p0 += kTileWaves * 16) {
    const int id = table[min(p0 + l16, np - 1)];
    const bool there = p0 + l16 < np && (unsigned)id < (unsigned)cv.n_pages;
    const uint32_t known = (uint32_t)__ballot(there);       // (16 bits, four times)
    d4 acc[2] = {};
    if (np > top) {
      const st* b = bounds + ((int64_t)(there ? id : 0) * cv.n_kv + hk) * 2 * D + quad * N;
      u32x4 w[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) w[c] = *reinterpret_cast<const u32x4*>(b + c * 4 * N);
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < N; ++e)
          acc[e & 1] = __builtin_amdgcn_mfma_f64_16x16x4f64(
              (double)S::elem(w[c], e), s_q[(c * 4 + quad) * N + e][l16], acc[e & 1], 0, 0,
              0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 4 * i + quad, p = p0 + at;
      uint32_t key = 0;
      if (p < mine && (known >> at & 1)) {
        key = 0xffffffffu;
        if (mine > top && p >= first && p < mine - last) {
          const float x = (float)(acc[0][i] + acc[1][i]);
          key = fabsf(x) < INFINITY ? score_key(x) : kAgain;
        }
      }
      s_keys[l16 * KS + p] = key;
    }
  }
  __syncthreads();
  for (int tok = wave; tok < nt; tok += kTileWaves) {
    const int mp = pages_of(tok0 + tok);
    uint32_t kr[CAP / 64];
    bool again = false;
    auto read = [&]() {
#pragma unroll
      for (int i = 0; i < CAP / 64; ++i) {
        const int p = i * 64 + lane;
        kr[i] = p < mp ? s_keys[tok * KS + p] : 0u;
        again |= kr[i] == kAgain;
      }
    };
    read();
    if (__any(again)) {
      const st* heads = q + (int64_t)(row0 + tok0 + tok) * ld_q + (int64_t)hk * g * D;
#pragma unroll 1
      for (int p = lane; p < mp; p += 64)
        if (s_keys[tok * KS + p] == kAgain)
          s_keys[tok * KS + p] = score_key(
              S::defined(heads, g, bounds + ((int64_t)table[p] * cv.n_kv + hk) * 2 * D));
      read();
    }
    choose(kr, top, mp <= top,
           out + ((int64_t)(row0 + tok0 + tok) * cv.n_kv + hk) * top);
  }
}

}  // namespace
}  // namespace davet

extern "C" int davet_cache_page_bounds(const davet_kv_cache* cache, int32_t n_seqs,
                                       const int32_t* cu_q, const int32_t* kv_len,
                                       void* bounds, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_page_bounds";
  CacheView cv;
  ChunkPack cp;
  int rc = check_cache(cache, false, who, &cv);
  if (!rc) rc = check_chunk(cache, n_seqs, cu_q, kv_len, who, &cp);
  if (rc) return rc;
  DAVET_CHECK_ARG(bounds && ((uintptr_t)bounds & 15) == 0, DAVET_EINVAL,
                  "davet_cache_page_bounds: bounds null or not 16-byte aligned");
  BoundsPack bp{};
  bp.n_seqs = n_seqs;
  int64_t at = 0;
  for (int s = 0; s < n_seqs; ++s) {
    const int n = cu_q[s + 1] - cu_q[s];
    bp.kv[s] = kv_len[s];
    bp.page[s] = (kv_len[s] - n) >> cv.lg;
    at += n > 0 ? ((kv_len[s] - 1) >> cv.lg) - bp.page[s] + 1 : 0;
    DAVET_CHECK_ARG(at * cv.n_kv < (1ll << 31), DAVET_ESHAPE,
                    "davet_cache_page_bounds: too many pages");
    bp.item[s + 1] = (int)at;
  }
  if (at == 0) return DAVET_OK;
  ProfScope ps(KC_MISC, stream);
#define BOUNDS(F, DIM)                                                            \
  in_runs(at * cv.n_kv, 256, [&](int wg, int64_t n) {                             \
    hipLaunchKernelGGL((page_bounds_kernel<F, DIM>), dim3((unsigned)n), dim3(256), \
                       0, stream, cv, bp, (F::st*)bounds, wg);                    \
  })
#define BOUNDS_D(F) \
  do { if (cache->head_dim == 128) BOUNDS(F, 128); else BOUNDS(F, 64); } while (0)
  if (cache->dtype == DAVET_F16) BOUNDS_D(F16S);
  else if (cache->dtype == DAVET_BF16) BOUNDS_D(BF16S);
  else BOUNDS_D(F32S);
#undef BOUNDS_D
#undef BOUNDS
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}

extern "C" int davet_cache_page_select(const davet_kv_cache* cache, int32_t n_seqs,
                                       const int32_t* cu_q, const int32_t* kv_len,
                                       const void* q, int64_t ld_q, int32_t n_heads,
                                       int32_t block, const void* bounds,
                                       int32_t first, int32_t last, int32_t top,
                                       int32_t* pages, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_page_select";
  CacheView cv;
  ChunkPack cp;
  int rc = check_cache(cache, false, who, &cv);
  if (!rc) rc = check_heads(cache, n_heads, who);
  if (!rc) rc = check_chunk(cache, n_seqs, cu_q, kv_len, who, &cp);
  const int64_t total = rc ? 0 : cp.row0[n_seqs];
  if (!rc && total > 0)
    rc = check_rows(q, ld_q, (int64_t)n_heads * cache->head_dim, cache->dtype, who,
                    "q");
  if (rc) return rc;
  DAVET_CHECK_ARG(block >= 0 && first >= 0 && last >= 0, DAVET_EINVAL,
                  "davet_cache_page_select: block, first and last must not be negative");
  DAVET_CHECK_ARG(top >= 1 && top <= kMaxPages && (int64_t)first + last <= top,
                  DAVET_ESHAPE,
                  "davet_cache_page_select: top in [1, 32768], first + last at most top");
  int64_t most = 0;
  for (int s = 0; s < n_seqs; ++s)
    if (cu_q[s + 1] > cu_q[s])
      most = std::max<int64_t>(most, ((int64_t)kv_len[s] + cache->page_size - 1) >> cv.lg);
  DAVET_CHECK_ARG(most <= kMaxPages, DAVET_ESHAPE,
                  "davet_cache_page_select: a sequence of more than 32768 pages");
  DAVET_CHECK_ARG(total * cv.n_kv < (1ll << 31), DAVET_ESHAPE,
                  "davet_cache_page_select: too many tokens");
  if (total == 0) return DAVET_OK;
  DAVET_CHECK_ARG(bounds && ((uintptr_t)bounds & 15) == 0, DAVET_EINVAL,
                  "davet_cache_page_select: bounds null or not 16-byte aligned");
  DAVET_CHECK_ARG(pages && aligned4({pages}), DAVET_EINVAL,
                  "davet_cache_page_select: pages null or not 4-byte aligned");
  ProfScope ps(KC_MISC, stream);
  const int64_t items = total * cv.n_kv;
  int longest = 0;
  TilePack tp{};
  for (int s = 0; s < n_seqs; ++s) {
    const int n = cu_q[s + 1] - cu_q[s];
    longest = std::max(longest, n);
    tp.first[s + 1] = tp.first[s] + (n + kTileTokens - 1) / kTileTokens;
  }
  // fp16, 8 heads of 128, pages x (sequences x tokens), us of tiles, waves and group:
  //    64 x (16 x  8)  11.1   9.5  15.2      512 x (16 x  1)  28.8  28.8  14.4
  //    64 x (16 x 16)  13.5  12.0  26.7      512 x (16 x  6)  29.4  30.3  32.5
  //   512 x ( 1 x 16)  29.3  26.8  13.1      512 x (16 x  8)  29.3  30.9  40.8
  //   512 x (64 x  1)  48.4  31.4  30.0      512 x (16 x 16)  31.7  46.1  74.3
  //   512 x (64 x  2)  47.5  32.2  44.6     1024 x ( 1 x 16)  53.1     -  21.2
  //   512 x (64 x  4)  48.1  46.4  75.8     1024 x (16 x  8)  52.9     -  63.1
  // (Of few pages waves are faster by 1.5 us than the tiles that the rule takes; and one
  // chunk of 8 tokens takes shorter ones beside it into tiles that are mostly empty.)
  const bool tiles = items >= kManyItems && longest >= 8 && most <= 1024;
  const bool waves = items >= kManyItems && most <= 64 * kWaveSteps;
  const int64_t tile_wgs = (int64_t)tp.first[n_seqs] * cv.n_kv;
#define TILES(F, DIM, CAP)                                                        \
  in_runs(tile_wgs, kTileThreads, [&](int at, int64_t n) {                        \
    hipLaunchKernelGGL((page_select_tile_kernel<F, DIM, CAP>), dim3((unsigned)n), \
                       dim3(kTileThreads), 0, stream, cv, cp, tp,                 \
                       (const F::st*)q, ld_q, n_heads, block,                     \
                       (const F::st*)bounds, first, last, top, pages, at);        \
  })
#define SELECT(F, DIM, CAP)                                                       \
  in_runs(items, kSelThreads, [&](int at, int64_t n) {                            \
    hipLaunchKernelGGL((page_select_kernel<F, DIM, CAP>), dim3((unsigned)n),      \
                       dim3(kSelThreads), 0, stream, cv, cp, (const F::st*)q,     \
                       ld_q, n_heads, block, (const F::st*)bounds, first, last,   \
                       top, pages, at);                                           \
  })
// (at most 64 sequences of 7 tokens, or they would be tiles)
#define WAVES(F, DIM)                                                             \
  hipLaunchKernelGGL((page_select_wave_kernel<F, DIM>),                           \
                     dim3((unsigned)((items + 3) / 4)), dim3(256), 0, stream, cv, \
                     cp, (const F::st*)q, ld_q, n_heads, block,                   \
                     (const F::st*)bounds, first, last, top, pages, items)
#define SELECT_N(F, DIM)                                                          \
  do {                                                                            \
    if (tiles && most <= 512) TILES(F, DIM, 512);                                 \
    else if (tiles) TILES(F, DIM, 1024);                                          \
    else if (waves) WAVES(F, DIM);                                                \
    else if (most <= kFewPages) SELECT(F, DIM, kFewPages);                                  \
    else SELECT(F, DIM, kMaxPages);                                               \
  } while (0)
#define SELECT_D(F) \
  do { if (cache->head_dim == 128) SELECT_N(F, 128); else SELECT_N(F, 64); } while (0)
  if (cache->dtype == DAVET_F16) SELECT_D(F16S);
  else if (cache->dtype == DAVET_BF16) SELECT_D(BF16S);
  else SELECT_D(F32S);
#undef SELECT_D
#undef SELECT_N
#undef WAVES
#undef SELECT
#undef TILES
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}
