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
// order needs one scan over 16 counts and no barrier inside the passes.  Up to
// 65536 entries are read once and stay in registers; more are read from L2 in
// each of the five passes.
//
// Move: entry kept[j] of the source pages becomes entry j of the destination
// pages, in the same pools; 64 entries of one head a workgroup, 16 bytes a
// thread and load.  Bound by HBM.

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

// The entries of one wavefront: [lo, hi), entry lo + 64 u + lane in slot u.  With
// R slots or fewer they are read once and held in registers as keys; R = 0 reads
// them again in every pass, 8 loads in flight.
template <int R>
struct Entries {
  const float* w;
  int lo, hi, first, tail;
  uint32_t key[R ? R : 1];
  __device__ __forceinline__ uint32_t key_of(float x, int i) const {
    return i < hi ? weight_key(x, i, first, tail) : 0u;
  }
  __device__ __forceinline__ void load() {
    if constexpr (R > 0) {
      const int lane = threadIdx.x & 63;
#pragma unroll
      for (int u = 0; u < R; ++u)       // (clamped: every slot's load is valid)
        key[u] = hi > lo ? __float_as_uint(w[min(lo + u * 64 + lane, hi - 1)]) : 0u;
#pragma unroll
      for (int u = 0; u < R; ++u)
        key[u] = key_of(__uint_as_float(key[u]), lo + u * 64 + lane);
    }
  }
  // f(index, inside, key) of 64 entries a step, in index order, all lanes at once
  template <typename Fn>
  __device__ __forceinline__ void each(Fn f) const {
    const int lane = threadIdx.x & 63;
    if constexpr (R > 0) {
#pragma unroll
      for (int u = 0; u < R; ++u) {
        const int i = lo + u * 64 + lane;
        if (lo + u * 64 < hi) f(i, i < hi, key[u]);
      }
    } else {
      for (int i0 = lo; i0 < hi; i0 += 512) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int i = i0 + u * 64 + lane;
          x[u] = i < hi ? w[i] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int i = i0 + u * 64 + lane;
          if (i0 + u * 64 < hi) f(i, i < hi, key_of(x[u], i));
        }
      }
    }
  }
};

template <int R>
__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(SelectPack sp, const float* __restrict__ weights,
                    int64_t ld_w, int first, int last, int32_t* __restrict__ kept,
                    int64_t ld_kept, float* __restrict__ weights_out,
                    int64_t ld_wo) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t wsum[kSelWaves], weq[kSelWaves];
  __shared__ uint32_t s_bin, s_need;
  const int s = blockIdx.x;
  const int n = sp.n[s], keep = sp.keep[s];
  if (keep == 0) return;
  const float* w = weights + (int64_t)s * ld_w;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = ((n + kSelWaves - 1) / kSelWaves + 63) & ~63;
  Entries<R> en;
  en.w = w;
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
    en.each([&](int, bool in, uint32_t key) {
      if (in && (key & mask) == prefix) {
        const uint32_t bin = (key >> shift) & digit;
        // one counter for all lanes would be added to 64 times in turn (equal
        // weights do that in every pass)
        const uint32_t lead = __builtin_amdgcn_readfirstlane(bin);
        const uint64_t on = __ballot(1), same = __ballot(bin == lead);
        if (same != on)
          atomicAdd(&hist[bin], 1u);
        else if (lane == __ffsll((unsigned long long)on) - 1)
          atomicAdd(&hist[lead], (uint32_t)__popcll(on));
      }
    });
    __syncthreads();
    // from the top: thread t holds bins 2047 - 2t and 2046 - 2t
    const int b1 = kBins - 1 - 2 * (int)threadIdx.x;
    const uint32_t c1 = hist[b1], c0 = hist[b1 - 1];
    uint32_t sum = c1 + c0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t y = __shfl_up(sum, o, 64);
      if (lane >= o) sum += y;
    }
    if (lane == 63) wsum[wave] = sum;
    __syncthreads();
    uint32_t before = sum - c1 - c0;
    for (int i = 0; i < wave; ++i) before += wsum[i];
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
  en.each([&](int, bool in, uint32_t key) {
    gt += (uint32_t)__popcll(__ballot(in && key > T));
    eq += (uint32_t)__popcll(__ballot(in && key == T));
  });
  if (lane == 0) {
    wsum[wave] = gt;
    weq[wave] = eq;
  }
  __syncthreads();
  uint32_t gt0 = 0, eq0 = 0;
  for (int i = 0; i < wave; ++i) {
    gt0 += wsum[i];
    eq0 += weq[i];
  }
  // bits of m below this lane
  auto below = [](uint64_t m) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                     __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
  };
  int32_t* ko = kept + (int64_t)s * ld_kept;
  float* wo = weights_out ? weights_out + (int64_t)s * ld_wo : nullptr;
  en.each([&](int i, bool in, uint32_t key) {
    const uint64_t mg = __ballot(in && key > T), me = __ballot(in && key == T);
    const uint32_t rg = gt0 + below(mg), re = eq0 + below(me);
    if (in && (key > T || (key == T && re < need))) {
      const uint32_t at = rg + min(re, need);
      ko[at] = i;
      if (wo) wo[at] = w[i];
    }
    gt0 += (uint32_t)__popcll(mg);
    eq0 += (uint32_t)__popcll(me);
  });
}

struct GatherPack {
  int32_t n_seqs;
  int32_t blk[DAVET_MAX_SEQS + 1];    // first 64-entry block of each sequence
  int32_t keep[DAVET_MAX_SEQS];
};

constexpr int kRows = 64;

template <int RB>     // bytes of a row
__global__ void __launch_bounds__(256)
cache_gather_kernel(CacheView cv, GatherPack gp, const int32_t* __restrict__ kept,
                    int64_t ld_kept, const int32_t* __restrict__ dst_table,
                    int32_t dst_max_pages) {
  constexpr int C = RB / 16, PER = kRows * C / 256;   // loads a thread, of K or V
  __shared__ int64_t src[kRows], dst[kRows];
  const int nblk = gp.blk[gp.n_seqs];
  const int blk = blockIdx.x % nblk, h = blockIdx.x / nblk;
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
  DAVET_CHECK_ARG(
      !weights_out ||
          !overlap(weights_out, ((n_seqs - 1) * ld_weights_out + most_keep) * 4,
                   weights, ((n_seqs - 1) * ld_weights + most_n) * 4),
      DAVET_EINVAL, "davet_evict_select: weights_out overlaps weights");
  if (most_keep == 0) return DAVET_OK;
  ProfScope ps(KC_MISC, stream);
#define SELECT(R)                                                              \
  hipLaunchKernelGGL((evict_select_kernel<R>), dim3(n_seqs), dim3(kSelThreads), \
                     0, stream, sp, weights, ld_weights, first, last, kept,    \
                     ld_kept, weights_out, ld_weights_out)
  // slots a lane: the largest wavefront's sixteenth, in steps of 64 entries
  const int64_t slots = (most_n + 1023) / 1024;
  if (slots <= 8) SELECT(8);
  else if (slots <= 32) SELECT(32);
  else if (slots <= 64) SELECT(64);
  else SELECT(0);
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
  GatherPack gp{};
  gp.n_seqs = n_seqs;
  int64_t at = 0;
  for (int s = 0; s < n_seqs; ++s) {
    DAVET_CHECK_ARG(keep[s] >= 0 && keep[s] <= ld_kept &&
                        keep[s] <= (int64_t)dst_max_pages * cache->page_size,
                    DAVET_ESHAPE,
                    "davet_cache_gather: keep out of range of ld_kept or of "
                    "dst_max_pages * page_size");
    gp.keep[s] = keep[s];
    at += (keep[s] + kRows - 1) / kRows;
    DAVET_CHECK_ARG(at * cv.n_kv < (1ll << 31), DAVET_ESHAPE,
                    "davet_cache_gather: too many entries");
    gp.blk[s + 1] = (int)at;
  }
  if (at == 0) return DAVET_OK;
  ProfScope ps(KC_MISC, stream);
  const dim3 grid((unsigned)(at * cv.n_kv));
  const int rb = cache->head_dim * (int)dtype_size(cache->dtype);
#define GATHER(RB)                                                             \
  hipLaunchKernelGGL((cache_gather_kernel<RB>), grid, dim3(256), 0, stream, cv, \
                     gp, kept, ld_kept, dst_table, dst_max_pages)
  if (rb == 128) GATHER(128);
  else if (rb == 256) GATHER(256);
  else GATHER(512);
#undef GATHER
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}
