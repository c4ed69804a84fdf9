// The cache's host checks, and the entry of a chunk into it: per-head RMSNorm
// and rotary embedding of queries and keys, and the copy of the values, in one
// pass over the projected rows.
//
// For head row x (D elements, h = D / 2) of a token at position p:
//   y = x * rsqrt(mean(x^2) + eps) * gain          (norm optional)
//   out[i]     = y[i] cos a_i - y[i + h] sin a_i
//   out[i + h] = y[i + h] cos a_i + y[i] sin a_i,   a_i = p theta^(-2 i / D)
//
// A thread owns elements 8j .. 8j+7 of both halves of one head, so that the
// pairs that turn together, and one of the two 16-byte (fp32: 32-byte) pieces
// of each half, are in its registers: D / 16 threads a head, the sum of squares
// is a butterfly over them.  A workgroup takes whole rows: the D / 2 angles of
// a row are computed once, into LDS, and serve all its heads.  The angle is
// reduced in float64 turns (p * theta^(-2i/D) / 2 pi minus its nearest whole
// number), which keeps far positions exact; what is left, at most half a turn,
// goes through the fp32 sine and cosine.  A rotary table would be read instead,
// but bounds the positions and is one more buffer to own.
//
// Bound by HBM: a row is read once and written once.  Measured: 3092 bf16 rows of
// (32 + 8 + 8) x 128, 76 MB in all, 15.3 us (5.0 TB/s; a copy of 76 MB takes 15.0),
// in fp32, 152 MB, 32.1 (4.7 TB/s); one row 3.3 us, a launch's latency.

#include <math.h>

#include "cache.h"

namespace davet {

int check_cache(const davet_kv_cache* c, bool need_v, const char* who,
                CacheView* out) {
  const std::string w = std::string(who) + ": ";
  DAVET_CHECK_ARG(c, DAVET_EINVAL, w + "cache is null");
  DAVET_CHECK_ARG(c->dtype == DAVET_F32 || is16(c->dtype), DAVET_EDTYPE,
                  w + "cache.dtype must be DAVET_F32, DAVET_BF16 or DAVET_F16");
  DAVET_CHECK_ARG(c->k && c->page_table && (c->v || !need_v), DAVET_EINVAL,
                  w + "null cache pointer");
  DAVET_CHECK_ARG((((uintptr_t)c->k | (uintptr_t)c->v) & 15) == 0 &&
                      ((uintptr_t)c->page_table & 3) == 0,
                  DAVET_EINVAL,
                  w + "cache.k and cache.v must be 16-byte aligned");
  DAVET_CHECK_ARG(c->head_dim == 64 || c->head_dim == 128, DAVET_ESHAPE,
                  w + "cache.head_dim must be 64 or 128");
  DAVET_CHECK_ARG(c->page_size >= kCacheGroup &&
                      c->page_size <= DAVET_MAX_PAGE_SIZE &&
                      (c->page_size & (c->page_size - 1)) == 0,
                  DAVET_ESHAPE,
                  w + "cache.page_size must be a power of two in [16, 256]");
  DAVET_CHECK_ARG(c->n_kv_heads >= 1 && c->n_kv_heads <= 1024 &&
                      c->n_pages >= 1 && c->max_pages >= 1,
                  DAVET_ESHAPE,
                  w + "cache: n_kv_heads in [1, 1024], n_pages and max_pages >= 1");
  if (out)
    *out = CacheView{c->k,         c->v,          c->page_table,
                     c->max_pages, c->n_pages,    __builtin_ctz(c->page_size),
                     c->n_kv_heads};
  return DAVET_OK;
}

int check_chunk(const davet_kv_cache* c, int32_t n_seqs, const int32_t* cu_q,
                const int32_t* kv_len, const char* who, ChunkPack* out) {
  const std::string w = std::string(who) + ": ";
  DAVET_CHECK_ARG(n_seqs >= 1 && n_seqs <= DAVET_MAX_SEQS, DAVET_ESHAPE,
                  w + "n_seqs out of range [1, 64]");
  DAVET_CHECK_ARG(cu_q && kv_len, DAVET_EINVAL, w + "null pointer");
  DAVET_CHECK_ARG(cu_q[0] == 0, DAVET_ESHAPE, w + "cu_q[0] must be 0");
  out->n_seqs = n_seqs;
  out->row0[0] = 0;
  for (int s = 0; s < n_seqs; ++s) {
    DAVET_CHECK_ARG(cu_q[s + 1] >= cu_q[s], DAVET_ESHAPE,
                    w + "cu_q must be non-decreasing");
    DAVET_CHECK_ARG(kv_len[s] >= cu_q[s + 1] - cu_q[s], DAVET_ESHAPE,
                    w + "kv_len counts the chunk: it must not be below its length");
    DAVET_CHECK_ARG(kv_len[s] <= (int64_t)c->max_pages * c->page_size &&
                        kv_len[s] <= (1 << 30),
                    DAVET_ESHAPE,
                    w + "kv_len beyond max_pages * page_size (or 2^30)");
    out->row0[s + 1] = cu_q[s + 1];
    out->kv[s] = kv_len[s];
  }
  DAVET_CHECK_ARG(cu_q[n_seqs] <= (1 << 24), DAVET_ESHAPE,
                  w + "more than 2^24 new tokens");
  return DAVET_OK;
}

int check_rows(const void* p, int64_t ld, int64_t width, int dtype,
               const char* who, const char* what) {
  const std::string w = std::string(who) + ": " + what;
  DAVET_CHECK_ARG(p, DAVET_EINVAL, w + " is null");
  DAVET_CHECK_ARG(((uintptr_t)p & 15) == 0 &&
                      (ld * (int64_t)dtype_size(dtype)) % 16 == 0,
                  DAVET_EINVAL, w + ": rows must start at 16-byte boundaries");
  DAVET_CHECK_ARG(ld >= width && ld < (1ll << 31), DAVET_ESHAPE,
                  w + ": row stride below the row's width");
  return DAVET_OK;
}

int check_heads(const davet_kv_cache* c, int32_t n_heads, const char* who) {
  DAVET_CHECK_ARG(n_heads >= 1 && n_heads <= 1024 &&
                      n_heads % c->n_kv_heads == 0,
                  DAVET_ESHAPE,
                  std::string(who) +
                      ": n_heads must be a multiple of n_kv_heads, at most 1024");
  return DAVET_OK;
}

namespace {

constexpr int kMaxThreads = 512;
// Threads of all workgroups, which then take runs of rows.  32,000 rows of 9 x 64:
// 85 us with 512 workgroups of their 128 threads, 25 with 1536; rows of 48 x 128
// (384 threads) gain nothing from more than 512 (3092 of them 15.3 us, 16-18 with
// 768 to 2048).
constexpr int kMaxInFlight = 512 * 384;

// 8 elements as memory holds them
template <typename F>
struct Piece {
  static constexpr int N = sizeof(typename F::st) / 2;    // 16-byte words
  u32x4 w[N];
  __device__ __forceinline__ void load(const typename F::st* p) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void store(typename F::st* p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<u32x4*>(p)[i] = w[i];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (F::dtype == DAVET_F32)
        v[i] = __uint_as_float(w[i >> 2][i & 3]);
      else
        v[i] = F::load((uint16_t)(w[0][i >> 1] >> (16 * (i & 1))));
    }
  }
  __device__ __forceinline__ void put(const float (&v)[8]) {
    if constexpr (F::dtype == DAVET_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[0][i] = round2<F>(v[2 * i], v[2 * i + 1]);
    }
  }
};

template <typename F, int D>
__global__ void __launch_bounds__(kMaxThreads)
cache_append_kernel(CacheView cv, ChunkPack cp, double log2_theta,
                    const typename F::st* qkv, int64_t ld_qkv,
                    int n_heads, const int32_t* __restrict__ pos, int norm,
                    const float* __restrict__ q_gain,
                    const float* __restrict__ k_gain, float eps,
                    typename F::st* q_out, int64_t ld_q, int rows_per_wg) {
  using st = typename F::st;
  constexpr int H = D / 2, TH = D / 16;       // threads a head
  __shared__ float cs[2][2][H];               // of even and odd rows
  __shared__ int64_t slot[2];                 // cache row of key head 0; -1: hole
  const int r0 = blockIdx.x * rows_per_wg;
  const int r1 = min(r0 + rows_per_wg, cp.row0[cp.n_seqs]);
  const int heads = n_heads + 2 * cv.n_kv;
  const int per = blockDim.x / TH, passes = (heads + per - 1) / per;
  const int j = threadIdx.x % TH, h0 = threadIdx.x / TH;

  // This thread's share of the angles: pair i turns theta^(-2 i / D) / (2 pi)
  // times round per position.  (A table of them in the kernel's arguments would
  // be read from host memory by every workgroup: 3092 rows took 42 us with it, 23
  // without, before the loads ahead.)
  const int i = threadIdx.x % H;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const double freq = exp2(log2_theta * (-2.0 / D) * i) * 0.15915494309189533577;
  auto angles = [&](int r) {
    // one wavefront a row, in turn, so that no other waits for the same one
    if (wave == r % (int)(blockDim.x >> 6) && (int)(threadIdx.x & 63) < H) {
      const int s = owner(cp.row0, cp.n_seqs, r);
      const int at = cp.kv[s] - cp.row0[s + 1] + r;
      const double turns = (double)(pos ? pos[r] : at) * freq;
      const float part = (float)(turns - rint(turns));
      cs[r & 1][0][i] = cospif(2.f * part);
      cs[r & 1][1][i] = sinpif(2.f * part);
      if (i == 0) {
        const int page = cv.table[(int64_t)s * cv.max_pages + (at >> cv.lg)];
        slot[r & 1] = (unsigned)page < (unsigned)cv.n_pages
                          ? (((int64_t)page * cv.n_kv) << cv.lg) +
                                (at & ((1 << cv.lg) - 1))
                          : -1;
      }
    }
  };
  // item: one pass over the heads of one row; the next one's loads are out while
  // one is worked on
  Piece<F> a, b, na, nb;
  auto load = [&](int r, int pass) {
    const int h = pass * per + h0;
    if (r < r1 && h < heads) {
      const st* x = qkv + (int64_t)r * ld_qkv + (int64_t)h * D + 8 * j;
      na.load(x);
      nb.load(x + H);
    }
  };
  load(r0, 0);
  // the gains of this thread's elements
  float gq[16], gk[16];
  auto gains = [&](const float* g, float (&v)[16]) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      f32x4 x = {1.f, 1.f, 1.f, 1.f};
      if (norm && g)
        x = *reinterpret_cast<const f32x4*>(g + 8 * j + (e & 7) + (e < 8 ? 0 : H));
#pragma unroll
      for (int u = 0; u < 4; ++u) v[e + u] = x[u];
    }
  };
  gains(q_gain, gq);
  gains(k_gain, gk);
  angles(r0);
  for (int r = r0; r < r1; ++r) {
    __syncthreads();
    if (r + 1 < r1) angles(r + 1);
    for (int pass = 0; pass < passes; ++pass) {
      a = na;
      b = nb;
      load(pass + 1 < passes ? r : r + 1, pass + 1 < passes ? pass + 1 : 0);
      const int h = pass * per + h0;
      if (h >= heads) continue;
      st* out;
      if (h < n_heads) {
        out = q_out + (int64_t)r * ld_q + (int64_t)h * D + 8 * j;
      } else {
        const bool key = h - n_heads < cv.n_kv;
        const int kh = key ? h - n_heads : h - n_heads - cv.n_kv;
        st* base = static_cast<st*>(key ? cv.k : cv.v);
        // a hole in the page table takes nothing
        const int64_t at = slot[r & 1];
        if (at < 0) continue;
        out = base + (at + ((int64_t)kh << cv.lg)) * D + 8 * j;
        if (!key) {                     // values, as they are
          a.store(out);
          b.store(out + H);
          continue;
        }
      }
      float x[8], y[8];
      a.get(x);
      b.get(y);
      if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[e] * x[e] + y[e] * y[e];
#pragma unroll
        for (int o = 1; o < TH; o <<= 1) ss += __shfl_xor(ss, o, 64);
        const float inv = 1.0f / sqrtf(ss * (1.0f / D) + eps);
        const bool query = h < n_heads;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] *= inv * (query ? gq[e] : gk[e]);
          y[e] *= inv * (query ? gq[8 + e] : gk[8 + e]);
        }
      }
      float c[8], d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float co = cs[r & 1][0][8 * j + e], si = cs[r & 1][1][8 * j + e];
        c[e] = x[e] * co - y[e] * si;
        d[e] = y[e] * co + x[e] * si;
      }
      a.put(c);
      b.put(d);
      a.store(out);
      b.store(out + H);
    }
  }
}

}  // namespace
}  // namespace davet

extern "C" int davet_cache_append(const davet_kv_cache* cache, int32_t n_seqs,
                                  const int32_t* cu_q, const int32_t* kv_len,
                                  const void* qkv, int64_t ld_qkv,
                                  int32_t n_heads, const int32_t* pos,
                                  int32_t norm, const float* q_gain,
                                  const float* k_gain, float eps, float theta,
                                  void* q_out, int64_t ld_q,
                                  hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_append";
  CacheView cv;
  ChunkPack cp;
  int rc = check_cache(cache, true, who, &cv);
  if (!rc) rc = check_heads(cache, n_heads, who);
  if (!rc) rc = check_chunk(cache, n_seqs, cu_q, kv_len, who, &cp);
  const int D = cache ? cache->head_dim : 0;
  const int64_t width = (int64_t)(n_heads + 2 * (cache ? cache->n_kv_heads : 0)) * D;
  const int total = rc ? 0 : cp.row0[n_seqs];
  if (!rc && total > 0)
    rc = check_rows(qkv, ld_qkv, width, cache->dtype, who, "qkv");
  if (!rc && total > 0)
    rc = check_rows(q_out, ld_q, (int64_t)n_heads * D, cache->dtype, who, "q_out");
  if (rc) return rc;
  DAVET_CHECK_ARG(norm == 0 || norm == 1, DAVET_EINVAL,
                  "davet_cache_append: norm must be 0 or 1");
  DAVET_CHECK_ARG(theta > 0.f && std::isfinite(theta) &&
                      (!norm || (eps >= 0.f && std::isfinite(eps))),
                  DAVET_EINVAL,
                  "davet_cache_append: theta > 0 and eps >= 0 required, finite");
  DAVET_CHECK_ARG((((uintptr_t)q_gain | (uintptr_t)k_gain) & 15) == 0 &&
                      ((uintptr_t)pos & 3) == 0,
                  DAVET_EINVAL,
                  "davet_cache_append: q_gain and k_gain must be 16-byte aligned");
  if (total == 0) return DAVET_OK;
  const size_t es = dtype_size(cache->dtype);
  // (a single row has no stride)
  DAVET_CHECK_ARG((q_out == qkv && (ld_q == ld_qkv || total == 1)) ||
                      !rows_overlap(q_out, ld_q, (int64_t)n_heads * D, qkv, ld_qkv,
                                    width, total, es),
                  DAVET_EINVAL,
                  "davet_cache_append: q_out overlaps qkv (in place needs the "
                  "same address and, of several rows, stride)");
  // threads for all heads of a row, or for equal passes over them; one row a
  // workgroup while there are few, then runs of rows
  const int units = (n_heads + 2 * cv.n_kv) * (D / 16);
  const int passes = (units + kMaxThreads - 1) / kMaxThreads;
  const int threads = (int)align_up((units + passes - 1) / passes, 64);  // >= D / 2
  const int groups = kMaxInFlight / threads;
  const int rpw = (total + groups - 1) / groups;
  const int grid = (total + rpw - 1) / rpw;
  ProfScope ps(KC_MISC, stream);
#define APPEND(F, DIM)                                                         \
  hipLaunchKernelGGL((cache_append_kernel<F, DIM>), dim3(grid), dim3(threads), \
                     0, stream, cv, cp, log2((double)theta), (const F::st*)qkv, ld_qkv, n_heads,\
                     pos, norm, q_gain, k_gain, eps, (F::st*)q_out, ld_q, rpw)
#define APPEND_D(F) do { if (D == 128) APPEND(F, 128); else APPEND(F, 64); } while (0)
  if (cache->dtype == DAVET_F16) APPEND_D(F16S);
  else if (cache->dtype == DAVET_BF16) APPEND_D(BF16S);
  else APPEND_D(F32S);
#undef APPEND_D
#undef APPEND
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}
