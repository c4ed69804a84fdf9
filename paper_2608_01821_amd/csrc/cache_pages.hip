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
// Scores are float64 sums rounded to float32: the products of 16-bit values are exact
// and their sum almost, so the order of summation does not decide which of two close
// pages is taken, and equal scores go to the lower page.
//
// A page's bounds are 256 to 1024 bytes, read 16 a lane by 16 to 64 lanes; a lane keeps
// its elements of Q in registers and multiplies as many pages as there are such lanes,
// whose sums are then added and dealt out at once, a page a lane (31 additions for 32
// pages of 32 lanes).  So a wavefront's step is 64 pages, one a lane.
//
// Selection: the key of the last page taken is found two bits at a time by counting,
// and the pages are written in ascending order.  Either a workgroup takes one (token,
// key head), or, where there are many, a wavefront does, by itself and without LDS.

#include <math.h>

#include <algorithm>

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
page_bounds_kernel(CacheView cv, BoundsPack bp, typename F::st* __restrict__ bounds) {
  using st = typename F::st;
  constexpr int N = 16 / (int)sizeof(st);       // elements a lane
  constexpr int C = D / N, R = 64 / C;          // lanes a row, rows a load
  constexpr int U = 4;
  __shared__ float s_lo[4][D], s_hi[4][D];
  const int item = blockIdx.x / cv.n_kv, h = blockIdx.x % cv.n_kv;
  const int s = owner(bp.item, bp.n_seqs, item);
  const int page = bp.page[s] + item - bp.item[s], psz = 1 << cv.lg;
  const int phys = cv.table[(int64_t)s * cv.max_pages + page];
  if ((unsigned)phys >= (unsigned)cv.n_pages) return;
  const int valid = min(psz, bp.kv[s] - page * psz);
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

constexpr int kSelThreads = 512, kSelWaves = kSelThreads / 64;
constexpr int kMaxPages = 32768;        // of a sequence: their keys fill the LDS
constexpr int kManyItems = 1024;

// order of a score: larger first; NaN with -inf, -0 with +0; never 0
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) x = -INFINITY;
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

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
  const st* bounds;     // of key head hk of page 0, at this lane's elements
  int64_t page;         // elements from page to page

  __device__ __forceinline__ static float elem(const u32x4& w, int e) {
    if constexpr (F::dtype == DAVET_F32)
      return __uint_as_float(w[e]);
    else
      return F::load((uint16_t)(w[e >> 1] >> (16 * (e & 1))));
  }
  // heads: the g query heads' rows
  __device__ __forceinline__ void init(const st* heads, int g, const st* b, int n_kv,
                                       int hk) {
    const int l = threadIdx.x & (LP - 1);
    bounds = b + (int64_t)hk * 2 * D + l * N;
    page = (int64_t)n_kv * 2 * D;
#pragma unroll
    for (int e = 0; e < N; ++e) q[e] = 0.0;
    for (int h = 0; h < g; ++h) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(heads + (int64_t)h * D +
                                                      (l & (H - 1)) * N);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = elem(w, e);             // (a NaN makes both sums NaN)
        q[e] += (double)(l < H ? (v > 0.f ? 0.f : v) : (v < 0.f ? 0.f : v));
      }
    }
  }
  // of the 64 pages whose places the lanes hold (0 for none): lane l's score is its own
  // page's
  __device__ __forceinline__ float score(int phys) const {
    const int lane = threadIdx.x & 63;
    // page u 4 + j + b H of each LP lanes' share: b the highest bit of a lane's number
    // in it, j the lowest two
    auto load = [&](int u, u32x4 (&w)[8]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int ph = __shfl(phys, (lane & ~(LP - 1)) + u * 4 + (i & 3) + (i >> 2) * H, 64);
        w[i] = *reinterpret_cast<const u32x4*>(bounds + (int64_t)ph * page);
      }
    };
    u32x4 w[2][8];
    load(0, w[0]);
    double sum[LP / 8];
#pragma unroll
    for (int u = 0; u < LP / 8; ++u) {
      if (u + 1 < LP / 8) load(u + 1, w[(u + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
      double x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = 0.0;
#pragma unroll
        for (int e = 0; e < N; ++e) x[i] = fma((double)elem(w[u & 1][i], e), q[e], x[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = deal<H>(x[i], x[i + 4]);
      sum[u] = deal<2>(deal<1>(x[0], x[1]), deal<1>(x[2], x[3]));
    }
    if constexpr (LP >= 64)
#pragma unroll
      for (int u = 0; u < LP / 16; ++u) sum[u] = deal<16>(sum[u], sum[u + LP / 16]);
    if constexpr (LP >= 32)
#pragma unroll
      for (int u = 0; u < 2; ++u) sum[u] = deal<8>(sum[u], sum[u + 2]);
    return (float)deal<4>(sum[0], sum[1]);
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
  c.s = owner(cp.row0, cp.n_seqs, *row);
  const int n = cp.row0[c.s + 1] - cp.row0[c.s];
  c.np = (visible_end(*row - cp.row0[c.s], n, cp.kv[c.s], block) + (1 << cv.lg) - 1) >> cv.lg;
  c.table = cv.table + (int64_t)c.s * cv.max_pages;
  c.out = out + item * top;
  return c;
}
__device__ __forceinline__ uint32_t lanes_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
}

// One workgroup an item.  Wavefront w takes a run of whole 64s: their keys stay in
// registers (LDS false: up to 4096 pages) or in LDS.
template <typename F, int D, bool LDS>
__global__ void __launch_bounds__(kSelThreads)
page_select_kernel(CacheView cv, ChunkPack cp, const typename F::st* __restrict__ q,
                   int64_t ld_q, int n_heads, int block,
                   const typename F::st* __restrict__ bounds, int first, int last,
                   int top, int32_t* __restrict__ out) {
  constexpr int REGS = 8;
  __shared__ uint32_t s_keys[LDS ? kMaxPages : 1];
  __shared__ __attribute__((aligned(16))) uint32_t s_cnt[2][3][kSelWaves];
  int row;
  const Choice c = choice_of(cv, cp, blockIdx.x, block, top, out, &row);
  const int np = c.np, g = n_heads / cv.n_kv;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = ((np + kSelWaves - 1) / kSelWaves + 63) & ~63;
  const int lo = min(np, wave * per), hi = min(np, lo + per);
  const bool all = np <= top;                   // nothing to choose

  uint32_t kr[REGS] = {};
  // f(64 pages' first one, their keys) of this wavefront
  auto each = [&](auto f) {
    if constexpr (LDS) {
      for (int i = lo; i < hi; i += 64) f(i, s_keys[i + lane]);
    } else {
#pragma unroll
      for (int i = 0; i < REGS; ++i)
        if (lo + i * 64 < hi) f(lo + i * 64, kr[i]);
    }
  };
  if (lo < hi) {
    Scorer<F, D> sc;
    int next = c.table[min(lo + lane, np - 1)];
    if (!all)
      sc.init(q + (int64_t)row * ld_q + (int64_t)c.hk * g * D, g, bounds, cv.n_kv, c.hk);
#pragma unroll 1
    for (int i = 0; lo + i * 64 < hi; ++i) {
      const int p = lo + i * 64 + lane;
      const bool there = p < np && (unsigned)next < (unsigned)cv.n_pages;
      const int phys = there ? next : 0;
      if (p + 64 - lane < hi) next = c.table[min(p + 64, np - 1)];
      uint32_t key = 0xffffffffu;
      if (!all) {
        const float x = sc.score(phys);
        if (p >= first && p < np - last) key = score_key(x);
      }
      if (!there) key = 0;
      if constexpr (LDS) {
        s_keys[p] = key;
      } else {
#pragma unroll
        for (int r = 0; r < REGS; ++r) kr[r] = r == i ? key : kr[r];
      }
    }
  }
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
  // of all wavefronts; one barrier: the next call writes the other half
  auto total = [&](uint32_t (&cnt)[3]) {
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < 3; ++i) s_cnt[flip][i][wave] = cnt[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      uint32_t x = 0;
#pragma unroll
      for (int w = 0; w < kSelWaves; ++w) x += s_cnt[flip][i][w];
      cnt[i] = x;
    }
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
      T |= (cnt[2] >= keep ? 3u : cnt[1] >= keep ? 2u : cnt[0] >= keep ? 1u : 0u) << b;
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
  uint32_t gt0 = 0, eq0 = 0, gts = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    const uint32_t x = s_cnt[flip][0][w], y = s_cnt[flip][1][w];
    gt0 += w < wave ? x : 0u;
    eq0 += w < wave ? y : 0u;
    gts += x;
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
  if (!all)
    sc.init(q + (int64_t)row * ld_q + (int64_t)c.hk * g * D, g, bounds, cv.n_kv, c.hk);
  uint32_t kr[kWaveSteps] = {};
  const int steps = (np + 63) / 64;
  uint32_t there_n = 0;
#pragma unroll 1
  for (int i = 0; i < steps; ++i) {
    const int p = i * 64 + lane;
    const bool there = p < np && (unsigned)next < (unsigned)cv.n_pages;
    const int phys = there ? next : 0;
    if (i + 1 < steps) next = c.table[min(p + 64, np - 1)];
    uint32_t key = 0xffffffffu;
    if (!all) {
      const float x = sc.score(phys);
      if (p >= first && p < np - last) key = score_key(x);
    }
    if (!there) key = 0;
    there_n += (uint32_t)__popcll(__ballot(key != 0));
#pragma unroll
    for (int r = 0; r < kWaveSteps; ++r) kr[r] = r == i ? key : kr[r];
  }
  const uint32_t keep = min((uint32_t)top, there_n);
  uint32_t T = 1;
  if (!all && keep > 0) {
    T = 0;
    for (int b = 31; b >= 0; --b) {
      const uint32_t x = T | 1u << b;
      uint32_t n = 0;
#pragma unroll
      for (int i = 0; i < kWaveSteps; ++i)
        if (i < steps) n += (uint32_t)__popcll(__ballot(kr[i] >= x));
      if (n >= keep) T = x;
    }
  }
  uint32_t gts = 0;
#pragma unroll
  for (int i = 0; i < kWaveSteps; ++i)
    if (i < steps) gts += (uint32_t)__popcll(__ballot(kr[i] > T));
  const uint32_t need = keep - gts;
  uint32_t gt0 = 0, eq0 = 0;
  if (keep > 0)
#pragma unroll
    for (int i = 0; i < kWaveSteps; ++i) {
      if (i >= steps) break;
      const uint64_t mg = __ballot(kr[i] > T), me = __ballot(kr[i] == T);
      const uint32_t rg = gt0 + lanes_below(mg), re = eq0 + lanes_below(me);
      if (kr[i] > T || (kr[i] == T && re < need))
        c.out[rg + min(re, need)] = i * 64 + lane;
      gt0 += (uint32_t)__popcll(mg);
      eq0 += (uint32_t)__popcll(me);
    }
  for (int i = (int)keep + lane; i < top; i += 64) c.out[i] = -1;
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
  const dim3 grid((unsigned)(at * cv.n_kv));
#define BOUNDS(F, DIM)                                                            \
  hipLaunchKernelGGL((page_bounds_kernel<F, DIM>), grid, dim3(256), 0, stream, cv, \
                     bp, (F::st*)bounds)
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
  // a wavefront each where they fill the chip
  const bool waves = items >= kManyItems && most <= 64 * kWaveSteps;
#define SELECT(F, DIM, LDS)                                                       \
  hipLaunchKernelGGL((page_select_kernel<F, DIM, LDS>), dim3((unsigned)items),    \
                     dim3(kSelThreads), 0, stream, cv, cp, (const F::st*)q, ld_q, \
                     n_heads, block, (const F::st*)bounds, first, last, top, pages)
#define WAVES(F, DIM)                                                             \
  hipLaunchKernelGGL((page_select_wave_kernel<F, DIM>),                           \
                     dim3((unsigned)((items + 3) / 4)), dim3(256), 0, stream, cv, \
                     cp, (const F::st*)q, ld_q, n_heads, block,                   \
                     (const F::st*)bounds, first, last, top, pages, items)
#define SELECT_N(F, DIM)                                                          \
  do {                                                                            \
    if (waves) WAVES(F, DIM);                                                     \
    else if (most <= 64 * 8 * kSelWaves) SELECT(F, DIM, false);                   \
    else SELECT(F, DIM, true);                                                    \
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
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}
