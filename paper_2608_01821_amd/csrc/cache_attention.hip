// Attention of a chunk over the paged cache (its kernels: cache_attn.h), and the
// attention weight each cached key received.

#include "cache_attn.h"

namespace davet {
namespace {

// Weights: w_j = prev_j + sum over the rows r that see key j of
// exp(scale q_r.k_j - lse_r).  S = Q K^T this time: a lane holds 16 rows' scores
// of ONE key and adds them in registers.  A workgroup takes 128 keys (32 a wave, or
// 64, held as fragments) and walks the rows of its key heads in tiles of 32 that the
// four waves share through LDS.  Chunks of (key head, row range) leave partial
// sums that a second kernel adds in order.
//
// Measured, 128 dims, 16 bits.  One token of eight histories of up to 32,700, 8 key
// heads: 74.5 us for 376 MB of keys (5.0 TB/s), bound by HBM.  128 queries, 32 heads,
// 3092 keys: 14.4 us and 4 to add the partial sums, where 26 MB take 5: bound by the
// chain of page, keys, rows and four tiles, gone through once with the whole chip's
// workgroups at it (loading the keys ahead of the rows: 16.1 us).  Four prompts of up
// to 3092 in full, 163 GFLOP: 231 to 256 us (0.64 to 0.71 PFLOP/s), bound by the
// vector ops and waits of four waves at one tile of rows.  fp32, the 128 queries: 50
// us (65 TFLOP/s).
struct WeightPlan {
  int32_t blk[DAVET_MAX_SEQS + 1];    // first block of keys of each sequence
  int32_t heads;                      // key heads a chunk
  int32_t qsplit;                     // row ranges a key head (heads = 1)
  int32_t chunks;
};

// KW: tiles of 32 keys a wave.  prev may be weights: neither is __restrict__.
template <typename F, int D, int KW>
__global__ void __launch_bounds__(256, 2)
cache_weights_kernel(CacheView cv, ChunkPack cp, WeightPlan wp,
                     const typename F::st* __restrict__ q, int64_t ld_q,
                     const float* __restrict__ lse, int n_heads, int block,
                     Scale sc_, const float* prev, float* weights, int64_t ld_w,
                     float* __restrict__ part, int wg0) {
  using st = typename F::st;
  using T = Tile<F, D>;
  using v8 = typename Frag<F>::v8;
  constexpr int QB = 32 * T::RB;
  constexpr int NI = 32 / T::RPI / 4;             // loads of rows a wave
  constexpr int NBUF = 4;                         // tiles of rows under way
  __shared__ __attribute__((aligned(1024))) char qs[NBUF][QB];
  // each wave's: lse of the 32 rows (and again), the keys each row sees
  __shared__ __attribute__((aligned(16))) float ls[NBUF][4][64];
  __shared__ __attribute__((aligned(16))) int lim[NBUF][4][32];
  const int nblk = wp.blk[cp.n_seqs];
  const int wg = wg0 + (int)blockIdx.x, blk = wg % nblk, chunk = wg / nblk;
  const int s = owner(wp.blk, cp.n_seqs, blk);
  const int g = n_heads / cv.n_kv;
  const int row0 = cp.row0[s], n = cp.row0[s + 1] - row0, kv = cp.kv[s];
  const int rows = n * g, nqb = (rows + 31) / 32;
  const int lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int KEYS = kWeightKeys * KW;          // of the workgroup
  int key[KW];
  bool hole[KW];
  int64_t kbase[KW];
#pragma unroll
  for (int t = 0; t < KW; ++t) {
    key[t] = (blk - wp.blk[s]) * KEYS + (wave * KW + t) * 32 + l32;
    const int kc = min(key[t], kv - 1);
    const int page = cv.table[(int64_t)s * cv.max_pages + (kc >> cv.lg)];
    hole[t] = (unsigned)page >= (unsigned)cv.n_pages;
    kbase[t] = hole[t] ? 0
                       : (((int64_t)page * cv.n_kv) << cv.lg) +
                             (kc & ((1 << cv.lg) - 1));
  }
  // the row tiles from the first one that sees any of the keys; rows from `all` on
  // see them all
  int h0, h1, b0 = 0, b1 = nqb, all = 0;
  if (block > 0) {
    const int own = (blk - wp.blk[s]) * KEYS - (kv - n), end = min(own + KEYS, n);
    if (own > 0) b0 = min(nqb, (int)((int64_t)(own / block) * block * g / 32));
    if (end > 0) all = (end - 1) / block * block * g;
  }
  auto masked = [&](int qb) { return qb * 32 < all || qb * 32 + 32 > rows; };
  if (wp.qsplit > 1) {
    h0 = chunk / wp.qsplit;
    h1 = h0 + 1;
    const int per = (nqb - b0 + wp.qsplit - 1) / wp.qsplit;
    b0 = min(nqb, b0 + (chunk % wp.qsplit) * per);
    b1 = min(nqb, b0 + per);
  } else {
    h0 = chunk * wp.heads;
    h1 = min(h0 + wp.heads, cv.n_kv);
  }
  const int nb = b1 - b0, steps = (h1 - h0) * nb;
  // Token and head of the group of this lane's NI rows, and of the row whose lse
  // it moves, kept as the rows advance (a division each would cost more than the
  // products): row r is token r / g, head r % g.
  int tok[NI + 1], hd[NI + 1];
  auto lane_row = [&](int i) {
    return i < NI ? (wave * NI + i) * T::RPI + lane / T::C : l32;
  };
  auto start = [&]() {
#pragma unroll
    for (int i = 0; i <= NI; ++i) {
      const int r = b0 * 32 + lane_row(i);
      tok[i] = r / g;
      hd[i] = r - tok[i] * g;
    }
  };
  const int t32 = 32 / g, h32 = 32 - t32 * g;
  int ih = h0, iqb = b0, ib = 0;        // the step to issue next, its buffer
  // its rows and their lse: NI + 1 loads a wave; rows past the last repeat it
  auto issue = [&]() {
    if (iqb == b0) start();
#pragma unroll
    for (int i = 0; i <= NI; ++i) {
      const bool past = iqb * 32 + lane_row(i) >= rows;
      const int64_t tk = row0 + (past ? n - 1 : tok[i]);
      const int hq = ih * g + (past ? g - 1 : hd[i]);
      if (i < NI) {
        const int lr = lane_row(i);
        dma16_at(reinterpret_cast<const char*>(q + tk * ld_q + (int64_t)hq * D) +
                     T::k_slot(lr, lane % T::C) * 16,
                 qs[ib] + (wave * NI + i) * 1024);
      } else {
        dma4_at(lse + tk * n_heads + hq, ls[ib][wave]);
        if (masked(iqb) && hh == 0)
          lim[ib][wave][l32] = past ? 0 : visible_end(tok[i], n, kv, block);
      }
      tok[i] += t32;
      hd[i] += h32;
      if (hd[i] >= g) { hd[i] -= g; ++tok[i]; }
    }
    ib = (ib + 1) % NBUF;
    if (++iqb == b1) { iqb = b0; ++ih; }
  };
  v8 kf[KW][D / 16];
  float acc[KW] = {};
  for (int i = 0; i < min(NBUF - 1, steps); ++i) issue();
  int h = h0, qb = b0;
  for (int step = 0; step < steps; ++step) {
    if (qb == b0) {
#pragma unroll
      for (int t = 0; t < KW; ++t) {
        const st* kp = static_cast<const st*>(cv.k) +
                       (kbase[t] + ((int64_t)h << cv.lg)) * D + hh * 8;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) kf[t][ks] = load_frag<F>(kp + ks * 16);
      }
    }
    // the loads of up to two later steps may stay out
    static_assert(NBUF == 4, "the waits below");
    if (steps - step > 2)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * (NI + 1)) : "memory");
    else if (steps - step == 2)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NI + 1) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    sync_lds();
    // into the buffer that every wave has done with
    if (step + NBUF - 1 < steps) issue();
    // lse in units of log2; a row that saw nothing gives 0: exp(x - inf)
    float* lw = ls[step % NBUF][wave];
    const float le = lw[lane];
    lw[lane] = le == -INFINITY ? INFINITY : le * kLog2e;
    const bool large = __any(fabsf(le) > kLargeLse && le != -INFINITY);
    const char* Qb = qs[step % NBUF];
    f32x16 sc[KW];
#pragma unroll
    for (int t = 0; t < KW; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[t][e] = 0.f;
    if constexpr (F::dtype == DAVET_F32) {
#pragma unroll
      for (int t = 0; t < KW; ++t) {
        f32x16 half = sc[t];            // two sums of half the length
#pragma unroll
        for (int ks = 0; ks < D / 16; ks += 2) {
          sc[t] = mm<F>(T::k_frag(Qb, l32, ks, hh), kf[t][ks], sc[t]);
          half = mm<F>(T::k_frag(Qb, l32, ks + 1, hh), kf[t][ks + 1], half);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[t][e] += half[e];
      }
    } else {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const v8 qf = T::k_frag(Qb, l32, ks, hh);
#pragma unroll
        for (int t = 0; t < KW; ++t) sc[t] = mm<F>(qf, kf[t][ks], sc[t]);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const f32x4 lv = *reinterpret_cast<const f32x4*>(lw + u * 8 + hh * 4);
#pragma unroll
      for (int t = 0; t < KW; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // (fp32: c_lo > 0, so that a score of -inf gives 0)
          const float x = sc[t][u * 4 + e];
          sc[t][u * 4 + e] = __builtin_amdgcn_exp2f(
              F::dtype == DAVET_F32 ? fmaf(x, sc_.c, fmaf(x, sc_.c_lo, -lv[e]))
                                    : fmaf(x, sc_.c, -lv[e]));
        }
    }
    // no term is above 1 but for the roundings of its score and lse, which are past
    // any bound once those are (a branch: as a minimum in every term 4 % slower)
    if (large) {
#pragma unroll
      for (int t = 0; t < KW; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[t][e] = sc[t][e] > 1.f ? 1.f : sc[t][e];
    }
    if (masked(qb)) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const i32x4 end = *reinterpret_cast<const i32x4*>(
            &lim[step % NBUF][wave][u * 8 + hh * 4]);
#pragma unroll
        for (int t = 0; t < KW; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sc[t][u * 4 + e] = key[t] < end[e] ? sc[t][u * 4 + e] : 0.f;
      }
    }
    float sum[KW] = {};
#pragma unroll
    for (int t = 0; t < KW; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[t] += sc[t][e];
#pragma unroll
    for (int t = 0; t < KW; ++t) acc[t] += sum[t];
    if (++qb == b1) { qb = b0; ++h; }
  }
#pragma unroll
  for (int t = 0; t < KW; ++t) {
    float w = pair_sum32(acc[t]);
    if (hole[t]) w = 0.f;
    if (hh != 0) continue;
    if (wp.chunks > 1) {
      part[((int64_t)chunk * nblk + blk) * KEYS + (wave * KW + t) * 32 + l32] = w;
    } else if (key[t] < kv) {
      const int64_t at = (int64_t)s * ld_w + key[t];
      weights[at] = (prev ? prev[at] : 0.f) + w;
    }
  }
}

// one thread a key; blockDim.x: keys of a block
__global__ void __launch_bounds__(2 * kWeightKeys)
cache_weights_join_kernel(ChunkPack cp, WeightPlan wp,
                          const float* __restrict__ part,
                          const float* prev, float* weights, int64_t ld_w) {
  const int nblk = wp.blk[cp.n_seqs], blk = blockIdx.x;
  const int s = owner(wp.blk, cp.n_seqs, blk);
  const int keys = blockDim.x, key = (blk - wp.blk[s]) * keys + threadIdx.x;
  if (key >= cp.kv[s]) return;
  float acc = 0.f;
#pragma unroll 8
  for (int c = 0; c < wp.chunks; ++c)
    acc += part[((int64_t)c * nblk + blk) * keys + threadIdx.x];
  const int64_t at = (int64_t)s * ld_w + key;
  weights[at] = (prev ? prev[at] : 0.f) + acc;
}

// The same with a positive second float: a score of -inf times both is -inf (plus an
// infinity of the other sign it would be NaN).  For arguments that use both.
Scale lower_scale(Scale r) {
  if (r.c_lo <= 0.f) {
    const float below = nextafterf(r.c, 0.f);
    r.c_lo += r.c - below;
    r.c = below;
  }
  return r;
}

template <typename F, int D, int KW>
int launch_weights(const CacheView& cv, const ChunkPack& cp, const void* q,
                int64_t ld_q, const float* lse, int n_heads, int block,
                Scale scale, const float* prev, float* weights, int64_t ld_w,
                float* part, hipStream_t stream) {
  constexpr int KEYS = kWeightKeys * KW;
  WeightPlan wp{};
  int most = 0;
  for (int s = 0; s < cp.n_seqs; ++s) {
    const int n = cp.row0[s + 1] - cp.row0[s];
    most = std::max(most, n);
    wp.blk[s + 1] = wp.blk[s] + (cp.kv[s] + KEYS - 1) / KEYS;
  }
  const int nblk = wp.blk[cp.n_seqs];
  if (nblk == 0) return DAVET_OK;
  const int g = n_heads / cv.n_kv;
  const int64_t nqb = ((int64_t)most * g + 31) / 32;
  int64_t steps = 0;
  for (int s = 0; s < cp.n_seqs; ++s)
    steps += (int64_t)(wp.blk[s + 1] - wp.blk[s]) * cv.n_kv *
             (((int64_t)(cp.row0[s + 1] - cp.row0[s]) * g + 31) / 32);
  // Workgroups: the chip twice over (1024), or with more work up to kWeightGroups of
  // at least 16 tiles of rows each (four prompts of up to 3092 in full, unequal:
  // 390 us with 1024, 270 so, both before later steps).
  const int groups = (int)std::max<int64_t>(
      1024, std::min<int64_t>(kWeightGroups, steps / 16));
  const int want = std::max(1, groups / nblk);
  wp.qsplit = 1;
  if (want >= cv.n_kv) {
    wp.heads = 1;
    wp.qsplit = (int)std::max<int64_t>(1, std::min<int64_t>(want / cv.n_kv, nqb / 2));
    wp.chunks = cv.n_kv * wp.qsplit;
  } else {
    wp.heads = (cv.n_kv + want - 1) / want;
    wp.chunks = (cv.n_kv + wp.heads - 1) / wp.heads;
  }
  const int64_t grid = (int64_t)nblk * wp.chunks;
  DAVET_CHECK_ARG(grid < (1ll << 31), DAVET_ESHAPE,
                  "davet_cache_weights: too many key blocks");
  {
    ProfScope ps(KC_MISC, stream);
    in_runs(grid, 256, [&](int at, int64_t wgs) {
      hipLaunchKernelGGL((cache_weights_kernel<F, D, KW>), dim3((unsigned)wgs),
                         dim3(256), 0, stream, cv, cp, wp, (const typename F::st*)q,
                         ld_q, lse, n_heads, block, scale, prev, weights, ld_w, part, at);
    });
    DAVET_HIP(hipGetLastError());
  }
  if (wp.chunks > 1) {
    ProfScope ps(KC_MISC, stream);
    hipLaunchKernelGGL(cache_weights_join_kernel, dim3(nblk), dim3(KEYS),
                       0, stream, cp, wp, part, prev, weights, ld_w);
    DAVET_HIP(hipGetLastError());
  }
  return DAVET_OK;
}

template <typename F, int D>
int run_weights(const CacheView& cv, const ChunkPack& cp, const void* q,
                int64_t ld_q, const float* lse, int n_heads, int block,
                Scale scale, const float* prev, float* weights, int64_t ld_w,
                float* part, hipStream_t stream) {
  int64_t tiles = 0;                    // 32 rows x 128 keys, of all key heads
  for (int s = 0; s < cp.n_seqs; ++s)
    tiles += ((int64_t)(cp.row0[s + 1] - cp.row0[s]) * n_heads + 31) / 32 *
             ((cp.kv[s] + kWeightKeys - 1) / kWeightKeys);
  // Two tiles of keys a wave (half the LDS reads and waits) from enough work on:
  // 30,000 tiles 62 us, 66 with one; 14,000 tiles 42.5 and 38; fp32 has no room.
  if constexpr (F::dtype != DAVET_F32)
    if (tiles > 20000)
      return launch_weights<F, D, 2>(cv, cp, q, ld_q, lse, n_heads, block, scale,
                                     prev, weights, ld_w, part, stream);
  return launch_weights<F, D, 1>(cv, cp, q, ld_q, lse, n_heads, block, scale, prev,
                                 weights, ld_w, part, stream);
}

}  // namespace
}  // namespace davet

extern "C" int davet_cache_workspace_bytes(int32_t n_heads, int32_t head_dim,
                                           int32_t max_q, size_t* bytes) {
  using namespace davet;
  DAVET_CHECK_ARG(bytes, DAVET_EINVAL, "davet_cache_workspace_bytes: bytes is null");
  DAVET_CHECK_ARG(n_heads >= 1 && n_heads <= 1024 &&
                      (head_dim == 64 || head_dim == 128) && max_q >= 1 &&
                      max_q <= (1 << 24),
                  DAVET_ESHAPE, "davet_cache_workspace_bytes: sizes out of range");
  // the need of a chunk is not monotonic in its rows (fewer rows may be cut
  // into more pieces): the bound is that of the worst chunk up to max_q
  const int64_t rows = (int64_t)max_q * n_heads;
  size_t b = workspace_bytes(max_q, n_heads, head_dim);
  const int64_t most = std::min<int64_t>(rows * kMaxPieces, kMaxPartRows);
  b = std::max(b, align_up((size_t)most * (head_dim + 2) * sizeof(float), 256));
  *bytes = b;
  return DAVET_OK;
}

extern "C" int davet_cache_attention(const davet_kv_cache* cache, int32_t n_seqs,
                                     const int32_t* cu_q, const int32_t* kv_len,
                                     const void* q, int64_t ld_q, int32_t n_heads,
                                     float scale, int32_t block, void* out,
                                     int64_t ld_out, float* lse, void* workspace,
                                     size_t ws_bytes, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_attention";
  CacheView cv;
  ChunkPack cp;
  int64_t total = 0;
  const int rc = check_attention(cache, n_seqs, cu_q, kv_len, q, ld_q, n_heads, scale,
                                 block, out, ld_out, lse, workspace, ws_bytes, who, &cv,
                                 &cp, &total);
  if (rc || total == 0) return rc;
  const int D = cache->head_dim;
  const Scale sc = make_scale(scale, D);
  float* part = static_cast<float*>(workspace);
#define ATT(F, DIM)                                                            \
  run_attention<F, DIM, kChunk>(cv, cp, q, ld_q, out, ld_out, lse, n_heads, block, \
                                sc, part, nullptr, who, stream)
  if (cache->dtype == DAVET_F16) return D == 128 ? ATT(F16S, 128) : ATT(F16S, 64);
  if (cache->dtype == DAVET_BF16) return D == 128 ? ATT(BF16S, 128) : ATT(BF16S, 64);
  return D == 128 ? ATT(F32S, 128) : ATT(F32S, 64);
#undef ATT
}

extern "C" int davet_cache_weights(const davet_kv_cache* cache, int32_t n_seqs,
                                   const int32_t* cu_q, const int32_t* kv_len,
                                   const void* q, int64_t ld_q, int32_t n_heads,
                                   float scale, int32_t block, const float* lse,
                                   const float* prev, float* weights,
                                   int64_t ld_weights, void* workspace,
                                   size_t ws_bytes, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_weights";
  CacheView cv;
  ChunkPack cp;
  int rc = check_cache(cache, false, who, &cv);
  if (!rc) rc = check_heads(cache, n_heads, who);
  if (!rc) rc = check_chunk(cache, n_seqs, cu_q, kv_len, who, &cp);
  const int D = cache ? cache->head_dim : 0;
  const int total = rc ? 0 : cp.row0[n_seqs];
  if (!rc && total > 0)
    rc = check_rows(q, ld_q, (int64_t)n_heads * D, cache->dtype, who, "q");
  if (rc) return rc;
  DAVET_CHECK_ARG((lse || total == 0) && weights, DAVET_EINVAL,
                  "davet_cache_weights: null pointer");
  DAVET_CHECK_ARG(aligned4({lse, prev, weights}), DAVET_EINVAL,
                  "davet_cache_weights: lse, prev and weights must be 4-byte aligned");
  DAVET_CHECK_ARG(good_scale(scale) && block >= 0, DAVET_EINVAL,
                  "davet_cache_weights: scale must be 0 or in [1e-30, 1e30], "
                  "block not negative");
  for (int s = 0; s < n_seqs; ++s)
    DAVET_CHECK_ARG(kv_len[s] <= ld_weights, DAVET_ESHAPE,
                    "davet_cache_weights: kv_len beyond ld_weights");
  DAVET_CHECK_ARG((int64_t)total * n_heads <= (1ll << 30), DAVET_ESHAPE,
                  "davet_cache_weights: too many query rows");
  rc = check_workspace(workspace, ws_bytes, total, n_heads, D, who);
  if (rc) return rc;
  Scale sc = make_scale(scale, D);
  if (cache->dtype == DAVET_F32) sc = lower_scale(sc);
  float* part = static_cast<float*>(workspace);
#define WGT(F, DIM) run_weights<F, DIM>(cv, cp, q, ld_q, lse, n_heads, block, sc, \
                                        prev, weights, ld_weights, part, stream)
  if (cache->dtype == DAVET_F16) return D == 128 ? WGT(F16S, 128) : WGT(F16S, 64);
  if (cache->dtype == DAVET_BF16) return D == 128 ? WGT(BF16S, 128) : WGT(BF16S, 64);
  return D == 128 ? WGT(F32S, 128) : WGT(F32S, 64);
#undef WGT
}
