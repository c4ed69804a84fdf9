// Attention of new tokens over listed pages of the cache: every (token, key head) has
// its own list, so its g query heads are all that shares a key.
//
//   o_i = sum_j p_ij v_j over the keys j of the token's listed pages that it sees
//
// The keys of a list are its pages' one after the other ("listed keys"); 16 aligned
// ones share a page.  A wavefront takes 32 of them (fp32: 16) against up to 16 query
// heads:
//
//   S^T = K Q^T    16 x 16 matrix ops: lane l holds the scores of query head l % 16 and
//                  keys 4 (l / 16) + 0 .. 3 of each 16.  K goes through LDS by DMA, a
//                  row's bytes side by side: as operands straight from memory, a
//                  quarter of a load's lanes would touch 16 rows, and the sixteen
//                  ragged blocks below took 86 us, bound by that.
//   O^T = V^T P^T  which takes those probabilities where they are as its B operand;
//                  for its A operand lane l loads 8 (fp32: 4) neighbouring dims,
//                  8 (l % 16) on, of the same keys, so that matrix op d, which takes
//                  element d of each, gives dims 8 m + d.  16 bits: the lane's 8 x 8
//                  block is transposed by 32 byte permutes.  No LDS.
//
// Every wavefront goes its own way, with the next keys on their way while it adds up
// values, and the next values while it multiplies keys.  Rows of Q past the last head
// repeat it.
//
// Eight wavefronts share a list's keys and are joined in LDS; four, a piece of a long
// list, and a second launch joins the pieces in order (cache_attn.h); or, where there
// are lists enough to fill the chip, each has its own.
//
// Measured, 32 heads over 8 of 128: eight tokens with 64 pages of 64 each, fp16, 25.3 us
// (136 MB, 5.4 TB/s: HBM) and 4.8 to join the pieces; 512 tokens with 32 pages of 16,
// bf16, 63 us.  Those read 1.07 GB (17 TB/s), the most of it from L2, and every 512 tokens
// more cost 52 us (21 TB/s).  The difference is the last round: 768 of the 1024 workgroups
// run at once, three a CU, and 256 after them.  No unit is busy throughout: the load path
// of a CU for 58 % of the time, vector ALUs for 30, matrix pipes for 16, and a wavefront
// waits for data for 37 % and for its turn for 39.  Registers hold three wavefronts a SIMD;
// four, with tiles of 16 keys, gain 4 % at 512 keys a list and nothing at 1024.  fp32, over
// and over: 155 us for the 512 tokens where fp16 takes 50, 35 for the eight where it
// takes 20.

#include "cache_attn.h"

namespace davet {
namespace {

// keys of a token's list in a sequence of kv cached tokens
__host__ __device__ inline int listed_keys(int kv, int top, int lg) {
  const int np = (kv + (1 << lg) - 1) >> lg;
  return (top < np ? top : np) << lg;
}

// 64 consecutive entries of a token's list, one a lane: where each page starts (a byte of
// the pools; 0 for none) and how many of its first keys the token sees (0 for none).
// Worked out for all at once; a tile then only picks its own.
struct ListIds {
  uint32_t lo, hi;
  int vis, base;
  __device__ __forceinline__ int64_t at(int entry) const {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, entry - base) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)lo, entry - base));
  }
  __device__ __forceinline__ int sees(int entry) const {
    return __builtin_amdgcn_readlane(vis, entry - base);
  }
};

// The largest (the sum) of the four lanes that hold one query head's keys.
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, lane_xor<16>(x));
  return fmaxf(x, lane_xor<32>(x));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += lane_xor<16>(x);
  return x + lane_xor<32>(x);
}

template <typename F>
__device__ __forceinline__ f32x4 mm16(typename Frag<F>::v8 a, typename Frag<F>::v8 b,
                                      f32x4 c) {
  return F::mfma16(a, b, c);
}

// W: wavefronts that share a list (4, 8; 1: each of four has its own).
template <typename F, int D, int W>
__global__ void __launch_bounds__(W == 8 ? 512 : 256,
                                  W == 8 ? 1 : F::dtype == DAVET_F32 && D == 128 ? 2 : 3)
page_attn_kernel(CacheView cv, ChunkPack cp, AttnPlan ap,
                 const typename F::st* __restrict__ q, int64_t ld_q,
                 typename F::st* __restrict__ out, int64_t ld_o,
                 float* __restrict__ lse, int n_heads, int block, Scale sc_,
                 float* __restrict__ part, int part_rows,
                 const int32_t* __restrict__ lists, int top, int wg0) {
  using st = typename F::st;
  constexpr bool F32 = F::dtype == DAVET_F32;
  constexpr int RB = D * (int)sizeof(st);       // bytes of a row
  constexpr int GR = F32 ? 1 : 2, KT = 16 * GR; // groups of 16 keys a tile
  constexpr int KC = RB / 64;                   // 16-byte loads of K a group
  constexpr int VC = F32 ? D / 64 : 1;          // loads of V a key
  constexpr int VD = F32 ? 4 : D / 16;          // dims each gives
  constexpr int NO = D / 16;                    // 16 x 16 tiles of O
  constexpr float BIAS = Frag<F>::kBias;
  using T = Tile<F, D>;
  constexpr int KB = KT * RB;                   // a tile of keys, 4 or 8 KB
  // each wavefront's keys; then O of its rows, as large
  constexpr int WAVES = W == 8 ? 8 : 4;
  __shared__ __attribute__((aligned(1024))) char smem[WAVES * KB];
  static_assert(KB == 16 * D * 4, "O takes the keys' place");
  __shared__ float s_m[WAVES][16], s_l[WAVES][16];

  const int g = n_heads / cv.n_kv, rt = (g + 15) / 16, lg = cv.lg, psz = 1 << lg;
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // workgroups of a sequence: [key head][piece][tile, or four of them], tiles fastest
  const int wg = wg0 + (int)blockIdx.x, b = ap.xcd ? wg >> 3 : wg;
  const Lanes blks(ap.blk), rows(cp.row0);
  const int orders = ap.order[lane], kvs = cp.kv[lane];
  const int si = blks.owner(cp.n_seqs, b), s = __builtin_amdgcn_readlane(orders, si);
  const int row_s = rows.start(s), n = rows.end(s) - row_s;
  const int kv_all = __builtin_amdgcn_readlane(kvs, s);
  const int tiles = n * rt, units = W > 1 ? tiles : (tiles + 3) / 4;
  const int kv = listed_keys(kv_all, top, lg);
  const int np = (kv + ap.piece - 1) / ap.piece;
  int rem = b - blks.start(si);
  const int h_ = rem / (units * np);
  rem -= h_ * units * np;
  const int hk = ap.xcd ? (wg & 7) + 8 * h_ : h_;
  const int piece = rem / units;
  const int tile = W > 1 ? rem - piece * units : (rem - piece * units) * 4 + wave;
  if (tile >= tiles) return;                    // (W = 1: no barrier follows)
  const int tok = tile / rt, r0 = (tile - tok * rt) * 16, nr = min(16, g - r0);
  const int row = row_s + tok;
  // cache indices below it are visible
  const int lim = visible_end(tok, n, kv_all, block);
  const int begin = piece * ap.piece, end = min(begin + ap.piece, kv);

  const int32_t* list = lists + ((int64_t)row * cv.n_kv + hk) * top;
  const int32_t* table = cv.table + (int64_t)s * cv.max_pages;
  ListIds ids;
  ids.base = -64;
  auto need = [&](int entry) {
    if (entry - ids.base < 64) return;
    ids.base = entry;
    const int e = entry + lane;
    const int page = e < kv >> lg ? list[e] : -1;
    const bool listed = (unsigned)page < (unsigned)((kv_all + psz - 1) >> lg);
    const int phys = listed ? table[page] : -1;
    const bool there = (unsigned)phys < (unsigned)cv.n_pages;
    const uint64_t at =
        there ? (uint64_t)((((int64_t)phys * cv.n_kv + hk) << lg) * RB) : 0;
    ids.lo = (uint32_t)at;
    ids.hi = (uint32_t)(at >> 32);
    ids.vis = there ? min(psz, max(0, lim - (page << lg))) : 0;
  };
  // Where 16 listed keys are, and how many of them nobody sees: the last ones.  All 16
  // are read: what lies behind the cached ones is still their page's, or, for a hole and
  // behind the list's end, the first page's.
  struct Group { int64_t at; int hidden; };
  struct Tile16 { Group g[GR]; };
  auto tile_at = [&](int k0) {
    // (a tile's pages are in one window: windows start at a tile, and hold whole ones)
    need(k0 >> lg);
    Tile16 t;
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const int key = k0 + i * 16, off = key & (psz - 1);
      t.g[i].at = ids.at(key >> lg) + off * RB;
      t.g[i].hidden = 16 - min(16, max(0, ids.sees(key >> lg) - off));
    }
    return t;
  };
  char* const kbuf = smem + wave * KB;
  typedef uint32_t vreg __attribute__((ext_vector_type(F32 ? 4 : VD / 2)));
  vreg vr[GR][4][VC];
  // Row r = j RPI + lane / C of a group, chunk lane % C of its place in LDS, holds
  // chunk k_slot(r, lane % C) of memory.
  auto load_k = [&](const Tile16& t) {
    constexpr int N = 16 / T::RPI, RUN = N < 4 ? N : 4;
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const char* p = static_cast<const char*>(cv.k) + t.g[i].at;
#pragma unroll
      for (int j = 0; j < N; j += RUN) {
        uint32_t at[RUN];
#pragma unroll
        for (int u = 0; u < RUN; ++u)
          at[u] = (uint32_t)(lane * 16) ^
                  (T::k_slot((j + u) * T::RPI + lane / T::C, 0) * 16);
        dma16_run(p + j * 1024, at, kbuf + i * 16 * RB + j * 1024);
      }
    }
  };
  const uint32_t v_at = quad * 4 * RB + l16 * (int)sizeof(vreg);
  auto load_v = [&](const Tile16& t) {
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const char* p = static_cast<const char*>(cv.v) + t.g[i].at;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VC; ++c)
          vr[i][e][c] = *reinterpret_cast<const vreg*>(p + (v_at + e * RB + c * 256));
    }
  };

  u32x4 qr[KC];
  {
    const st* qp = q + (int64_t)row * ld_q + (int64_t)(hk * g + r0 + min(l16, nr - 1)) * D;
#pragma unroll
    for (int c = 0; c < KC; ++c)
      qr[c] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(qp) +
                                              quad * 16 + c * 64);
  }
  f32x4 o[NO];
#pragma unroll
  for (int i = 0; i < NO; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  // scores are kept as differences from `ref`, near the row's largest
  float ref = 0.f, l_run = 0.f;
  bool seen = false;                // some score above -inf so far

  constexpr int NV = GR * 4 * VC;       // loads of V a tile
  constexpr int STEP = W * KT;
  int k0 = begin + (W > 1 ? wave * KT : 0);
  Tile16 cur = {};
  if (k0 < end) {
    cur = tile_at(k0);
    load_k(cur);
    load_v(cur);
  }
  for (; k0 < end; k0 += STEP) {
    const bool more = k0 + STEP < end;
    // the tile's keys are there; its values, loaded after them, may not be
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NV) : "memory");
    u32x4 kr[GR][KC];
#pragma unroll
    for (int i = 0; i < GR; ++i)
#pragma unroll
      for (int c = 0; c < KC; ++c)
        kr[i][c] = *reinterpret_cast<const u32x4*>(
            kbuf + (i * 16 + l16) * RB + T::k_slot(l16, c * 4 + quad) * 16);
    f32x4 sc[GR];
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      sc[i] = f32x4{-ref, -ref, -ref, -ref};
      if constexpr (F32) {
        // two sums of half the length: a chain of D roundings would show in lse
        f32x4 half = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f32x4& to = c & 1 ? half : sc[i];
            to = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr[i][c][j]),
                                                      __uint_as_float(qr[c][j]), to, 0,
                                                      0, 0);
          }
        sc[i] += half;
      } else {
        using v8 = typename Frag<F>::v8;
#pragma unroll
        for (int c = 0; c < KC; ++c)
          sc[i] = mm16<F>(__builtin_bit_cast(v8, kr[i][c]), __builtin_bit_cast(v8, qr[c]),
                          sc[i]);
      }
    }
    Tile16 next = {};
    if (more) next = tile_at(k0 + STEP);
    // hidden keys: score -inf, and values of 0 (0 times an infinity would be NaN)
    bool some = false;
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const int hid = cur.g[i].hidden;
      some |= hid < 16;
      if (hid == 0) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (quad * 4 + e >= 16 - hid) {
          sc[i][e] = -INFINITY;
#pragma unroll
          for (int c = 0; c < VC; ++c) vr[i][e][c] = vreg{};
        }
    }
    // The next keys, once this tile's are read and its values there (the compiler does
    // not count the DMA: a wait for values behind it would be for both).
    auto next_k = [&]() {
#pragma unroll
      for (int i = 0; i < GR; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < VC; ++c) asm volatile("" : "+v"(vr[i][e][c]));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) load_k(next);
    };
    if (some) {
      float tmax = -INFINITY;
#pragma unroll
      for (int i = 0; i < GR; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) tmax = fmaxf(tmax, sc[i][e]);
      tmax = quad_max(tmax);
      // ref moves only when it is 2^8 behind the largest score (or with the first one)
      const bool move = seen ? tmax * sc_.c > 8.0f : tmax > -INFINITY;
      if (__any(move)) {
        const float to = move ? ref + tmax : ref;
        const float by = move ? to - ref : 0.f;
        const float alpha = seen ? __builtin_amdgcn_exp2f(-by * sc_.c) : 0.f;
        ref = to;
        seen = seen || move;
        l_run *= alpha;
#pragma unroll
        for (int i = 0; i < GR; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[i][e] -= by;
#pragma unroll
        for (int i = 0; i < NO; ++i) o[i] *= alpha;
      }
      float p[GR * 4];
#pragma unroll
      for (int i = 0; i < GR * 4; ++i) {
        const float x = sc[i >> 2][i & 3];
        p[i] = __builtin_amdgcn_exp2f(F32 ? exact_arg(x, sc_) : fmaf(x, sc_.c, BIAS));
        l_run += p[i];
      }
      next_k();
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < VC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              o[c * 4 + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  __uint_as_float(vr[0][e][c][j]), p[e], o[c * 4 + j], 0, 0, 0);
      } else {
        // probabilities rounded to 16 bits, and what that took off them
        using v8 = typename Frag<F>::v8;
        u32x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t h = round2<F>(p[2 * e], p[2 * e + 1]);
          hi[e] = h;
          lo[e] = round2<F>(p[2 * e] - F::load((uint16_t)(h & 0xffffu)),
                            p[2 * e + 1] - F::load((uint16_t)(h >> 16)));
        }
#pragma unroll
        for (int d = 0; d < VD; ++d) {
          // element d of the eight keys
          u32x4 a;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            a[e] = __builtin_amdgcn_perm(vr[e >> 1][(e & 1) * 2 + 1][0][d / 2],
                                         vr[e >> 1][(e & 1) * 2][0][d / 2],
                                         d & 1 ? 0x07060302u : 0x05040100u);
          o[d] = mm16<F>(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, hi), o[d]);
          o[d] = mm16<F>(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, lo), o[d]);
        }
      }
    } else {
      next_k();
    }
    if (more) load_v(next);
    __builtin_amdgcn_sched_barrier(0);
    cur = next;
  }

  // this lane: query head l16, and of its dims those below (tile t, element i)
  auto dim_of = [&](int t, int i) {
    return F32 ? (t >> 2) * 64 + 16 * quad + 4 * i + (t & 3) : VD * (4 * quad + i) + t;
  };
  l_run = quad_sum(l_run);
  float m_run = l_run == 0.f ? -INFINITY : ref;
  const float bias_ln = BIAS * kLn2;
  const int64_t head = (int64_t)row * n_heads + hk * g + r0;
  if constexpr (W == 1) {
    if (l16 >= nr) return;
    // a row that sees nothing (or only scores of -inf): zeros, lse -inf
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
    st* op = out + (int64_t)row * ld_o + (int64_t)(hk * g + r0 + l16) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int t = 0; t < NO; t += F32 ? 4 : VD) {
        const int d0 = dim_of(t, i);
        if constexpr (F32) {
          f32x4 x;
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = l_run == 0.f ? 0.f : o[t + j][i] * inv;
          *reinterpret_cast<f32x4*>(op + d0) = x;
        } else {
          vreg x;
#pragma unroll
          for (int j = 0; j < VD; j += 2)
            x[j / 2] = l_run == 0.f ? 0u
                                    : round2<F>(o[t + j][i] * inv, o[t + j + 1][i] * inv);
          *reinterpret_cast<vreg*>(op + d0) = x;
        }
      }
    }
    if (lse && quad == 0)
      lse[head + l16] = l_run == 0.f ? -INFINITY
                                     : m_run * sc_.scale + (logf(l_run) - bias_ln);
  } else {
    float* const s_o = reinterpret_cast<float*>(smem);
    auto o_at = [&](int w, int r, int d) -> float& {
      // (rows' 16-byte pieces in turn: 16 rows at a time are written at one dim)
      return s_o[(w * 16 + r) * D + (d ^ ((r & 15) * 4))];
    };
#pragma unroll
    for (int t = 0; t < NO; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) o_at(wave, l16, dim_of(t, i)) = o[t][i];
    if (quad == 0) {
      s_m[wave][l16] = m_run;
      s_l[wave][l16] = l_run;
    }
    __syncthreads();
    // a row's dims over 16 threads, or 32
    constexpr int DT = W * 4, DP = D / DT;
    const int r = threadIdx.x / DT, d0 = threadIdx.x % DT * DP;
    if (r >= nr) return;
    float m = -INFINITY, l = 0.f, wt[W];
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, s_m[w][r]);
    bool use[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      use[w] = s_l[w][r] != 0.f;        // (NaN scores: sum NaN, maximum -inf)
      wt[w] = use[w] ? __builtin_amdgcn_exp2f((s_m[w][r] - m) * sc_.c) : 0.f;
      if (use[w]) l += wt[w] * s_l[w][r];
    }
    float acc[DP];
#pragma unroll
    for (int i = 0; i < DP; ++i) {
      acc[i] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w)
        if (use[w]) acc[i] += wt[w] * o_at(w, r, d0 + i);
    }
    if (ap.pieces > 1) {
      const int64_t at = (int64_t)piece * part_rows + head + r;
      float* po = part + at * D + d0;
#pragma unroll
      for (int i = 0; i < DP; ++i) po[i] = acc[i];
      if (d0 == 0) {
        float* pm = part + (int64_t)ap.pieces * part_rows * D + at * 2;
        pm[0] = m;
        pm[1] = l;
      }
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      st* op = out + (int64_t)row * ld_o + (int64_t)(hk * g + r0 + r) * D + d0;
      if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < DP; ++i) op[i] = acc[i] * inv;
      } else {
        typedef uint32_t words __attribute__((ext_vector_type(DP / 2)));
        words x;
#pragma unroll
        for (int i = 0; i < DP; i += 2) x[i / 2] = round2<F>(acc[i] * inv, acc[i + 1] * inv);
        *reinterpret_cast<words*>(op) = x;
      }
      if (lse && d0 == 0)
        lse[head + r] = l == 0.f ? -INFINITY : m * sc_.scale + (logf(l) - bias_ln);
    }
  }
}

template <typename F, int D>
int run_page_attention(const CacheView& cv, const ChunkPack& cp, const void* q,
                       int64_t ld_q, void* out, int64_t ld_o, float* lse, int n_heads,
                       int block, Scale sc, float* part, const int32_t* lists, int top,
                       hipStream_t stream) {
  using st = typename F::st;
  const int g = n_heads / cv.n_kv, rt = (g + 15) / 16;
  const int64_t rows = (int64_t)cp.row0[cp.n_seqs] * n_heads;
  ChunkPack keys = cp;                  // with the keys of the lists
  for (int s = 0; s < cp.n_seqs; ++s)
    keys.kv[s] = listed_keys(cp.kv[s], top, cv.lg);
  const int64_t items = (int64_t)cp.row0[cp.n_seqs] * rt * cv.n_kv;
  int longest = 0;
  for (int s = 0; s < cp.n_seqs; ++s)
    if (cp.row0[s + 1] > cp.row0[s]) longest = std::max(longest, keys.kv[s]);
  // fp16, 32 heads of 128 over 8, us of four wavefronts a list (in pieces that a second
  // launch joins, where there are few), of eight and of one:
  //     8 lists of  512 keys   8.7   7.8          512 of  512  14.1  16.7  21.1
  //     8       of 1024        8.6   9.8         1024 of  512  23.6  29.4  23.3
  //     8       of 2048        9.3  14.5         1024 of 4096   101         127
  //   128       of 1024       11.5  10.5         2048 of  512  37.4        31.9
  //   256       of  512       12.5   9.3         2048 of 1024  58.2        54.3
  //   256       of 1024       18.4  14.1         4096 of  512  65.8        57.0
  // (8 of 1024: called one by one, not from a graph, the second launch costs 3 more.)
  const int W = items >= 2048 ? 1 : longest <= 1024 && items <= 256 ? 8 : 4;
  auto units = [&](int s) {
    const int64_t t = (int64_t)(cp.row0[s + 1] - cp.row0[s]) * rt;
    return W > 1 ? t : (t + 3) / 4;
  };
  const AttnPlan ap =
      W == 4 ? plan_attn(keys, cv.n_kv, units, 256 * 3, 128, 128, 384, max_pieces(rows))
             : plan_attn(keys, cv.n_kv, units, 1, 128, 128, 1 << 30, 1);
  const int64_t grid = (int64_t)ap.blk[cp.n_seqs] * (ap.xcd ? 8 : 1);
  DAVET_CHECK_ARG(grid < (1ll << 31), DAVET_ESHAPE,
                  "davet_cache_page_attention: too many tokens");
  {
    ProfScope ps(KC_MISC, stream);
#define LAUNCH(WW, THREADS)                                                        \
  in_runs(grid, THREADS, [&](int at, int64_t wgs) {                                \
    hipLaunchKernelGGL((page_attn_kernel<F, D, WW>), dim3((unsigned)wgs),          \
                       dim3(THREADS), 0, stream, cv, cp, ap, (const st*)q, ld_q,   \
                       (st*)out, ld_o, lse, n_heads, block, sc, part, (int)rows,   \
                       lists, top, at);                                            \
  })
    if (W == 1) LAUNCH(1, 256);
    else if (W == 8) LAUNCH(8, 512);
    else LAUNCH(4, 256);
#undef LAUNCH
    DAVET_HIP(hipGetLastError());
  }
  return ap.pieces > 1 ? join_pieces<F, D>(keys, part, ap, out, ld_o, lse, n_heads, sc,
                                           stream)
                       : DAVET_OK;
}

}  // namespace
}  // namespace davet

extern "C" int davet_cache_page_attention(
    const davet_kv_cache* cache, int32_t n_seqs, const int32_t* cu_q,
    const int32_t* kv_len, const void* q, int64_t ld_q, int32_t n_heads, float scale,
    int32_t block, const int32_t* pages, int32_t top, void* out, int64_t ld_out,
    float* lse, void* workspace, size_t ws_bytes, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_page_attention";
  CacheView cv;
  ChunkPack cp;
  int64_t total = 0;
  const int rc = check_attention(cache, n_seqs, cu_q, kv_len, q, ld_q, n_heads, scale,
                                 block, out, ld_out, lse, workspace, ws_bytes, who, &cv,
                                 &cp, &total);
  if (rc) return rc;
  DAVET_CHECK_ARG(top >= 1 && top <= (1 << 26), DAVET_ESHAPE,
                  "davet_cache_page_attention: top out of range [1, 2^26]");
  if (total == 0) return DAVET_OK;
  DAVET_CHECK_ARG(pages && aligned4({pages}), DAVET_EINVAL,
                  "davet_cache_page_attention: pages null or not 4-byte aligned");
  const int D = cache->head_dim;
  const Scale sc = make_scale(scale, D);
  float* part = static_cast<float*>(workspace);
#define ATT(F, DIM)                                                               \
  run_page_attention<F, DIM>(cv, cp, q, ld_q, out, ld_out, lse, n_heads, block, sc, \
                             part, pages, top, stream)
  if (cache->dtype == DAVET_F16) return D == 128 ? ATT(F16S, 128) : ATT(F16S, 64);
  if (cache->dtype == DAVET_BF16) return D == 128 ? ATT(BF16S, 128) : ATT(BF16S, 64);
  return D == 128 ? ATT(F32S, 128) : ATT(F32S, 64);
#undef ATT
}
