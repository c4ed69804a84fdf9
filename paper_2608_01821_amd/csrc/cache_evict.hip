// Eviction from a paged cache: which entries stay, by the attention weight they
// received, and their move to new pages.
//
// Selection, one workgroup a sequence: the first and last entries asked for
// stay, the rest are taken by (weight descending, index ascending).  Weights are
// mapped to 32-bit keys whose unsigned order is theirs (NaN as -inf, -0 as +0,
// protected entries above everything); three passes of 11, 11 and 10 bits over
// an LDS histogram find the key T of the last entry kept and how many of the
// entries equal to it stay, and a last pass writes the indices in ascending
// order.  Each wavefront owns one contiguous sixteenth of the entries, so the
// order needs one scan over 16 counts and no barrier inside the passes.
//
// Move: entry kept[j] of the source pages becomes entry j of the destination
// pages, in the same pools; 16 KB of one head's keys and of its values a
// workgroup, 16 bytes a thread and load.  Bound by HBM.
//
// Measured: 2964 entries cut to half, 7.9 us to select (the latency of five passes
// in one workgroup) and 10.9 to move them, 49 MB read and written (4.5 TB/s); eight
// sequences of up to 32,700, 26 us and 157 for 750 MB (4.8 TB/s; a copy of that
// size reaches 5.1).

#include <algorithm>

#include "cache.h"

namespace davet {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = 16, kBins = 2048;

struct SelectPack {
  int32_t n[DAVET_MAX_SEQS], keep[DAVET_MAX_SEQS];
};

__device__ __forceinline__ uint32_t weight_key(float w, int i, int first,
                                               int tail) {
  if (i < first || i >= tail) return 0xffffffffu;
  if (w != w) w = -INFINITY;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The entries of one wavefront: [lo, hi), lo a multiple of 256.  Counting takes
// 256 a step, four neighbours a lane, so that LDS reads and ballots overlap; what
// goes to or comes from memory goes 64 neighbours an instruction.  Up to kLdsKeys
// entries of a sequence are read once and stay in LDS as keys; more are read from
// L2 in every pass.  (Held in registers, 32 or 64 a lane, the five unrolled
// passes are 40 KB of code, and its fetch took twice the work's time.)  Places
// past hi have key 0, below that of any entry, so no pass asks.
constexpr int kStep = 256;
constexpr int kLdsKeys = 36 * 1024;

template <bool LDS>
struct Entries {
  const float* w;
  uint32_t* keys;       // LDS: of the sequence
  int lo, hi, first, tail;
  // f(index, key, weight) of 64 places a step, in index order, U steps of loads
  // in flight; with `weigh` false the weight is not read where keys are in LDS
  template <int U, typename Fn>
  __device__ __forceinline__ void each64(bool fresh, bool weigh, Fn f) const {
    const int lane = threadIdx.x & 63;
    for (int i0 = lo; i0 < hi; i0 += U * 64) {
      float x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        x[u] = fresh || weigh ? w[min(i0 + u * 64 + lane, hi - 1)] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u * 64 >= hi) break;
        const int i = i0 + u * 64 + lane;
        if (fresh)
          f(i, i < hi ? weight_key(x[u], i, first, tail) : 0u, x[u]);
        else
          f(i, keys[i], x[u]);
      }
    }
  }
  __device__ __forceinline__ void load() {
    if constexpr (LDS) {
      each64<16>(true, true, [&](int i, uint32_t key, float) { keys[i] = key; });
      // the rest of the last step
      for (int i = (hi + 63) / 64 * 64 + (int)(threadIdx.x & 63);
           i < (hi + kStep - 1) / kStep * kStep; i += 64)
        if (hi > lo) keys[i] = 0;
    }
  }
  // f(four keys), any order
  template <typename Fn>
  __device__ __forceinline__ void count(Fn f) const {
    const int lane = threadIdx.x & 63;
    if constexpr (LDS) {
#pragma unroll 2
      for (int i0 = lo; i0 < hi; i0 += kStep)
        f(*reinterpret_cast<const u32x4*>(keys + i0 + lane * 4));
    } else {
      for (int i0 = lo; i0 < hi; i0 += 4 * kStep) {
        float x[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[u][e] = w[min(i0 + u * kStep + e * 64 + lane, hi - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          u32x4 k;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = i0 + u * kStep + e * 64 + lane;
            k[e] = i < hi ? weight_key(x[u][e], i, first, tail) : 0u;
          }
          f(k);
        }
      }
    }
  }
};

// sum of the first n of 16 counts
__device__ __forceinline__ uint32_t sum_before(const uint32_t (&c)[kSelWaves], int n) {
  uint32_t s = 0;
#pragma unroll
  for (int i = 0; i < kSelWaves; ++i) s += i < n ? c[i] : 0u;
  return s;
}

// sum over the lanes up to each: DPP row shifts by 1, 2, 4, 8 and the two row
// broadcasts
__device__ __forceinline__ uint32_t scan_lanes(uint32_t x) {
#define STEP(ctrl, rows) \
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false)
  STEP(0x111, 0xf);
  STEP(0x112, 0xf);
  STEP(0x114, 0xf);
  STEP(0x118, 0xf);
  STEP(0x142, 0xa);
  STEP(0x143, 0xc);
#undef STEP
  return x;
}

template <bool LDS>
__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(SelectPack sp, const float* __restrict__ weights,
                    int64_t ld_w, int first, int last, int32_t* __restrict__ kept,
                    int64_t ld_kept, float* __restrict__ weights_out,
                    int64_t ld_wo) {
  __shared__ __attribute__((aligned(16))) uint32_t s_keys[LDS ? kLdsKeys : 4];
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t wsum[kSelWaves], weq[kSelWaves];
  __shared__ uint32_t s_bin, s_need;
  const int s = blockIdx.x;
  const int n = sp.n[s], keep = sp.keep[s];
  if (keep == 0) return;
  const float* w = weights + (int64_t)s * ld_w;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = ((n + kSelWaves - 1) / kSelWaves + kStep - 1) / kStep * kStep;
  Entries<LDS> en;
  en.w = w;
  en.keys = s_keys;
  en.lo = min(n, wave * per);
  en.hi = min(n, en.lo + per);
  en.first = first;
  en.tail = n - last;
  en.load();

  uint32_t prefix = 0, mask = 0;
  uint32_t need = keep;          // entries still to find among those matching
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digit = pass == 2 ? 1023u : 2047u;
    for (int b = threadIdx.x; b < kBins; b += kSelThreads) hist[b] = 0;
    __syncthreads();
    en.count([&](u32x4 key) {
      bool on[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) on[e] = (key[e] & mask) == prefix;
      if (!__any(on[0] || on[1] || on[2] || on[3])) return;
      uint32_t bin[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) bin[e] = (key[e] >> shift) & digit;
      // One counter for all would be added to 256 times in turn (equal weights
      // do that in every pass).
      const uint32_t one = __builtin_amdgcn_readfirstlane(bin[0]);
      if (__all(on[0] && on[1] && on[2] && on[3] && bin[0] == one &&
                bin[1] == one && bin[2] == one && bin[3] == one)) {
        if (lane == 0) atomicAdd(&hist[one], (uint32_t)kStep);
        return;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (on[e]) atomicAdd(&hist[bin[e]], 1u);
    });
    __syncthreads();
    // from the top: thread t holds bins 2047 - 2t and 2046 - 2t
    const int b1 = kBins - 1 - 2 * (int)threadIdx.x;
    const uint32_t c1 = hist[b1], c0 = hist[b1 - 1];
    const uint32_t sum = scan_lanes(c1 + c0);
    if (lane == 63) wsum[wave] = sum;
    __syncthreads();
    const uint32_t before = sum - c1 - c0 + sum_before(wsum, wave);
    if (before < need && need <= before + c1) {
      s_bin = b1;
      s_need = need - before;
    } else if (before + c1 < need && need <= before + c1 + c0) {
      s_bin = b1 - 1;
      s_need = need - before - c1;
    }
    __syncthreads();
    prefix |= s_bin << shift;
    mask |= digit << shift;
    need = s_need;
  }
  const uint32_t T = prefix;     // key of the last entry kept; `need` of them
  uint32_t gt = 0, eq = 0;
  en.count([&](u32x4 key) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      gt += (uint32_t)__popcll(__ballot(key[e] > T));
      eq += (uint32_t)__popcll(__ballot(key[e] == T));
    }
  });
  if (lane == 0) {
    wsum[wave] = gt;
    weq[wave] = eq;
  }
  __syncthreads();
  uint32_t gt0 = sum_before(wsum, wave), eq0 = sum_before(weq, wave);
  // bits of m below this lane
  auto below = [](uint64_t m) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                     __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
  };
  int32_t* ko = kept + (int64_t)s * ld_kept;
  float* wo = weights_out ? weights_out + (int64_t)s * ld_wo : nullptr;
  en.template each64<8>(!LDS, wo, [&](int i, uint32_t key, float x) {
    const uint64_t mg = __ballot(key > T), me = __ballot(key == T);
    // entries above T, and equal to it, before this one; of the latter the first
    // `need` of the sequence stay
    const uint32_t rg = gt0 + below(mg), re = eq0 + below(me);
    if (key > T || (key == T && re < need)) {
      const uint32_t at = rg + min(re, need);
      ko[at] = i;
      if (wo) wo[at] = x;
    }
    gt0 += (uint32_t)__popcll(mg);
    eq0 += (uint32_t)__popcll(me);
  });
}

struct GatherPack {
  int32_t n_seqs;
  int32_t blk[DAVET_MAX_SEQS + 1];    // first block of entries of each sequence
  int32_t keep[DAVET_MAX_SEQS];
};

// 16 KB of K and of V a workgroup: four loads of each a thread
constexpr int gather_rows(int row_bytes) { return 16384 / row_bytes; }

template <int RB>     // bytes of a row
__global__ void __launch_bounds__(256)
cache_gather_kernel(CacheView cv, GatherPack gp, const int32_t* __restrict__ kept,
                    int64_t ld_kept, const int32_t* __restrict__ dst_table,
                    int32_t dst_max_pages, int wg0) {
  constexpr int kRows = gather_rows(RB);
  constexpr int C = RB / 16, PER = kRows * C / 256;   // loads a thread, of K or V
  __shared__ int64_t src[kRows], dst[kRows];
  const int nblk = gp.blk[gp.n_seqs];
  const int wg = wg0 + (int)blockIdx.x, blk = wg % nblk, h = wg / nblk;
  const int s = owner(gp.blk, gp.n_seqs, blk);
  const int j0 = (blk - gp.blk[s]) * kRows, lg = cv.lg, psz = 1 << lg;
  if (threadIdx.x < kRows) {
    const int j = j0 + threadIdx.x;
    int64_t a = -1, b = -1;               // rows of the pool; -1: none
    if (j < gp.keep[s]) {
      const int i = kept[(int64_t)s * ld_kept + j];
      if (i >= 0 && (i >> lg) < cv.max_pages) {
        const int p = cv.table[(int64_t)s * cv.max_pages + (i >> lg)];
        if ((unsigned)p < (unsigned)cv.n_pages)
          a = ((((int64_t)p * cv.n_kv + h) << lg) + (i & (psz - 1))) * RB;
      }
      const int p = dst_table[(int64_t)s * dst_max_pages + (j >> lg)];
      if ((unsigned)p < (unsigned)cv.n_pages)
        b = ((((int64_t)p * cv.n_kv + h) << lg) + (j & (psz - 1))) * RB;
    }
    src[threadIdx.x] = a;
    dst[threadIdx.x] = b;
  }
  __syncthreads();
  u32x4 k[PER], v[PER];
  const int c = (threadIdx.x % C) * 16;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int64_t a = src[(threadIdx.x + i * 256) / C];
    k[i] = v[i] = u32x4{0, 0, 0, 0};
    if (a >= 0) {
      k[i] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(cv.k) + a + c);
      v[i] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(cv.v) + a + c);
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int64_t b = dst[(threadIdx.x + i * 256) / C];
    if (b >= 0) {
      *reinterpret_cast<u32x4*>(static_cast<char*>(cv.k) + b + c) = k[i];
      *reinterpret_cast<u32x4*>(static_cast<char*>(cv.v) + b + c) = v[i];
    }
  }
}

}  // namespace
}  // namespace davet

extern "C" int davet_evict_select(int32_t n_seqs, const int32_t* n,
                                  const int32_t* keep, const float* weights,
                                  int64_t ld_weights, int32_t first, int32_t last,
                                  int32_t* kept, int64_t ld_kept,
                                  float* weights_out, int64_t ld_weights_out,
                                  hipStream_t stream) {
  using namespace davet;
  DAVET_CHECK_ARG(n_seqs >= 1 && n_seqs <= DAVET_MAX_SEQS, DAVET_ESHAPE,
                  "davet_evict_select: n_seqs out of range [1, 64]");
  DAVET_CHECK_ARG(n && keep && weights && kept, DAVET_EINVAL,
                  "davet_evict_select: null pointer");
  DAVET_CHECK_ARG(aligned4({weights, kept, weights_out}), DAVET_EINVAL,
                  "davet_evict_select: weights, kept and weights_out must be 4-byte "
                  "aligned");
  DAVET_CHECK_ARG(first >= 0 && last >= 0, DAVET_EINVAL,
                  "davet_evict_select: first and last must not be negative");
  SelectPack sp{};
  int64_t most_n = 0, most_keep = 0;
  for (int s = 0; s < n_seqs; ++s) {
    DAVET_CHECK_ARG(n[s] >= 0 && n[s] <= (1 << 30) && keep[s] >= 0 &&
                        keep[s] <= n[s],
                    DAVET_ESHAPE, "davet_evict_select: 0 <= keep <= n required");
    DAVET_CHECK_ARG(keep[s] == 0 || (int64_t)first + last <= keep[s], DAVET_ESHAPE,
                    "davet_evict_select: first + last beyond keep");
    sp.n[s] = n[s];
    sp.keep[s] = keep[s];
    most_n = std::max<int64_t>(most_n, n[s]);
    most_keep = std::max<int64_t>(most_keep, keep[s]);
  }
  DAVET_CHECK_ARG(most_n <= ld_weights && most_keep <= ld_kept &&
                      (!weights_out || most_keep <= ld_weights_out),
                  DAVET_ESHAPE, "davet_evict_select: row stride below a length");
  DAVET_CHECK_ARG(std::max({ld_weights, ld_kept, weights_out ? ld_weights_out : 0}) <
                      (1ll << 40),
                  DAVET_ESHAPE, "davet_evict_select: row stride of 2^40 or more");
  DAVET_CHECK_ARG(
      !weights_out ||
          !rows_overlap(weights_out, ld_weights_out, most_keep, weights, ld_weights,
                        most_n, n_seqs, 4),
      DAVET_EINVAL, "davet_evict_select: weights_out overlaps weights");
  if (most_keep == 0) return DAVET_OK;
  ProfScope ps(KC_MISC, stream);
#define SELECT(LDS)                                                            \
  hipLaunchKernelGGL((evict_select_kernel<LDS>), dim3(n_seqs),                 \
                     dim3(kSelThreads), 0, stream, sp, weights, ld_weights,    \
                     first, last, kept, ld_kept, weights_out, ld_weights_out)
  // keys in LDS where they fit: 36,000 entries 33 us with the move of one head,
  // 50 read from L2 in every pass; 2964 the same within 1 us
  if ((most_n + kStep - 1) / kStep * kStep <= kLdsKeys) SELECT(true);
  else SELECT(false);
#undef SELECT
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}

extern "C" int davet_cache_gather(const davet_kv_cache* cache, int32_t n_seqs,
                                  const int32_t* keep, const int32_t* kept,
                                  int64_t ld_kept, const int32_t* dst_table,
                                  int32_t dst_max_pages, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_gather";
  CacheView cv;
  int rc = check_cache(cache, true, who, &cv);
  if (rc) return rc;
  DAVET_CHECK_ARG(n_seqs >= 1 && n_seqs <= DAVET_MAX_SEQS, DAVET_ESHAPE,
                  "davet_cache_gather: n_seqs out of range [1, 64]");
  DAVET_CHECK_ARG(keep && kept && dst_table, DAVET_EINVAL,
                  "davet_cache_gather: null pointer");
  DAVET_CHECK_ARG(aligned4({kept, dst_table}), DAVET_EINVAL,
                  "davet_cache_gather: kept and dst_table must be 4-byte aligned");
  GatherPack gp{};
  gp.n_seqs = n_seqs;
  const int rb = cache->head_dim * (int)dtype_size(cache->dtype);
  const int rows = gather_rows(rb);
  int64_t at = 0;
  for (int s = 0; s < n_seqs; ++s) {
    DAVET_CHECK_ARG(keep[s] >= 0 && keep[s] <= ld_kept &&
                        keep[s] <= (int64_t)dst_max_pages * cache->page_size,
                    DAVET_ESHAPE,
                    "davet_cache_gather: keep out of range of ld_kept or of "
                    "dst_max_pages * page_size");
    gp.keep[s] = keep[s];
    at += (keep[s] + rows - 1) / rows;
    DAVET_CHECK_ARG(at * cv.n_kv < (1ll << 31), DAVET_ESHAPE,
                    "davet_cache_gather: too many entries");
    gp.blk[s + 1] = (int)at;
  }
  if (at == 0) return DAVET_OK;
  ProfScope ps(KC_MISC, stream);
#define GATHER(RB)                                                             \
  in_runs(at * cv.n_kv, 256, [&](int wg, int64_t n) {                          \
    hipLaunchKernelGGL((cache_gather_kernel<RB>), dim3((unsigned)n), dim3(256), \
                       0, stream, cv, gp, kept, ld_kept, dst_table,            \
                       dst_max_pages, wg);                                     \
  })
  if (rb == 128) GATHER(128);
  else if (rb == 256) GATHER(256);
  else GATHER(512);
#undef GATHER
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}
