// Attention of a chunk of new tokens over a paged key/value cache, and the
// attention weight each cached key received.
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i.k_j - lse_i),
//   lse_i = ln sum_j exp(scale q_i.k_j)
//
// over the keys j visible to query i.  The g = n_heads / n_kv_heads query heads
// that share a key head are rows of one tile: row r of (sequence, key head) is
// query r / g, head r % g of the group, so a decode step's few queries fill the
// matrix tile and every key is fetched once for all of them.
//
// A wavefront owns 32 rows and computes S^T = K Q^T with 32 x 32 matrix ops: a
// lane holds the scores of ONE row, the softmax statistics are per lane, and the
// probabilities are already laid out as the B operand of O^T += V^T P^T.  fp32
// runs the same code on v_mfma_f32_32x32x2: eight of them consume the eight
// elements that one 16-bit op takes, in the same lane layout.
//
// Keys move global -> LDS by DMA.  A page holds at least 16 aligned keys, so the
// 4 (8, 2) rows that one load instruction moves share a page and its address is
// scalar; the page ids of 64 pages at a time sit in one register per lane.
//
// Two forms, by the rows of a (sequence, key head), narrow up to 32 (fp32: 64):
//   wide    128 rows a workgroup: four wavefronts of 32 rows share 64-key tiles
//   narrow  32 rows a workgroup: each of four wavefronts streams its own 32-key
//           tiles through its own two buffers, with no barrier, and the four are
//           joined in LDS at the end
// Either way the keys of a tile may be cut into pieces, one workgroup each, that
// leave (max, sum, O) in fp32 in the workspace; a second kernel joins them in
// piece order, so no result depends on timing.
//
// Measured, 128 dims.  narrow, bound by HBM (one read of K and V): one token of
// eight histories of up to 32,700, 8 key heads, 16 bits, 748 MB, 135 us with the
// join's 5 (5.5 TB/s); 16 sequences of 32 queries over up to 3773, 32 key heads, 638
// MB, 121 us (5.3 TB/s).  wide, bound by the matrix ops and exponentials of two
// waves a SIMD: four prompts of up to 3092 in full, 325 GFLOP, 363 to 402 us in fp16
// (0.81 to 0.89 PFLOP/s with the clock, 0.77 when it runs for long; a large product
// reaches 1.34).  fp32: 92 TFLOP/s (a large product 154).  A call of 192 keys takes
// 12 us in fp32: the chain of its loads, and two tiles of 64 matrix ops in series a
// wavefront.

#include <math.h>

#include <algorithm>

#include "cache.h"

namespace davet {
namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s* lds_v4s_ptr;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxPieces = 64;
constexpr int kMaxPartRows = 1 << 17;     // rows x pieces in the workspace
constexpr int kWeightKeys = 128;          // keys a workgroup of the weights (or twice)
constexpr int kWeightGroups = 4096;       // most workgroups that leave partial sums
constexpr float kLargeLse = 65536.f;      // terms are off by 1 % and more
constexpr int kAhead = 4;                 // fragments read ahead of the matrix ops

// Fragments of 8 elements along the contracted axis and the op that takes them.
template <typename S> struct Frag;
template <> struct Frag<F16S> {
  using v8 = f16x8;
  // Probabilities are stored as 2^kBias times themselves: fp16 has few bits
  // below 2^-14, and a running maximum 2^8 behind still stays below 65504.
  static constexpr int kBias = 6;
};
template <> struct Frag<BF16S> { using v8 = bf16x8; static constexpr int kBias = 0; };
template <> struct Frag<F32S> { using v8 = f32x8; static constexpr int kBias = 0; };

template <typename F>
__device__ __forceinline__ f32x16 mm(typename Frag<F>::v8 a,
                                     typename Frag<F>::v8 b, f32x16 c) {
  if constexpr (F::dtype == DAVET_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  } else {
    return F::mfma32(a, b, c);
  }
}

// Global -> LDS DMA: lane l's 16 (or 4) bytes at base + offset go to lds + 16 l
// (4 l); base and lds are the wavefront's.  In asm, so that the compiler does not
// count it: it cannot tell the buffer that a load fills from the one an LDS read
// takes, and would wait for every load before each read.  Every use waits for
// its own loads (s_waitcnt vmcnt) and then for the other wavefronts'.  No register
// is written; what the compiler counts itself it only waits for longer.
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
__device__ __forceinline__ void dma16(const void* base, uint32_t offset, void* lds) {
  asm volatile("s_mov_b32 m0, %0\n\t"
               "s_nop 0\n\t"
               "global_load_lds_dwordx4 %1, %2"
               :: "s"(__builtin_amdgcn_readfirstlane(lds_at(lds))), "v"(offset),
                  "s"(base)
               : "memory", "m0");
}
// 2 or 4 of them in a row, 1024 bytes apart (the instruction's offset counts for
// both addresses)
__device__ __forceinline__ void dma16_run(const void* base, const uint32_t (&o)[2],
                                          void* lds) {
  asm volatile("s_mov_b32 m0, %0\n\t"
               "s_nop 0\n\t"
               "global_load_lds_dwordx4 %1, %3\n\t"
               "global_load_lds_dwordx4 %2, %3 offset:%4"
               :: "s"(__builtin_amdgcn_readfirstlane(lds_at(lds))), "v"(o[0]),
                  "v"(o[1]), "s"(base), "n"(1024)
               : "memory", "m0");
}
__device__ __forceinline__ void dma16_run(const void* base, const uint32_t (&o)[4],
                                          void* lds) {
  asm volatile("s_mov_b32 m0, %0\n\t"
               "s_nop 0\n\t"
               "global_load_lds_dwordx4 %1, %5\n\t"
               "global_load_lds_dwordx4 %2, %5 offset:%6\n\t"
               "global_load_lds_dwordx4 %3, %5 offset:%7\n\t"
               "global_load_lds_dwordx4 %4, %5 offset:%8"
               :: "s"(__builtin_amdgcn_readfirstlane(lds_at(lds))), "v"(o[0]),
                  "v"(o[1]), "v"(o[2]), "v"(o[3]), "s"(base), "n"(1 * 1024),
                  "n"(2 * 1024), "n"(3 * 1024)
               : "memory", "m0");
}
__device__ __forceinline__ void dma16_at(const void* g, void* lds) {
  asm volatile("s_mov_b32 m0, %0\n\t"
               "s_nop 0\n\t"
               "global_load_lds_dwordx4 %1, off"
               :: "s"(__builtin_amdgcn_readfirstlane(lds_at(lds))), "v"(g)
               : "memory", "m0");
}
__device__ __forceinline__ void dma4_at(const void* g, void* lds) {
  asm volatile("s_mov_b32 m0, %0\n\t"
               "s_nop 0\n\t"
               "global_load_lds_dword %1, off"
               :: "s"(__builtin_amdgcn_readfirstlane(lds_at(lds))), "v"(g)
               : "memory", "m0");
}
__device__ __forceinline__ void sync_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// x combined with the value of lane l ^ 32
__device__ __forceinline__ float pair_max32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x),
                                                  __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x),
                                                  __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// LDS layout of a tile row of D elements: 16-byte chunks, chunk c of row r in
// slot c ^ f(r).  K: the 16 rows that a fragment read takes at one chunk cover
// all 64 banks.  V, 16-bit: the 64-byte pieces of four consecutive keys that a
// transposing read takes do; fp32: those of the two half-waves' keys.
template <typename F, int D>
struct Tile {
  using st = typename F::st;
  static constexpr int RB = D * (int)sizeof(st);   // bytes a row
  static constexpr int C = RB / 16;                // chunks a row
  static constexpr int RPI = 1024 / RB;            // rows a load instruction
  __device__ static __forceinline__ int k_slot(int r, int c) {
    return C == 8 ? c ^ ((r >> 1) & 7) : c ^ (r & 15);
  }
  __device__ static __forceinline__ int v_slot(int r, int c) {
    if constexpr (F::dtype == DAVET_F32) return c ^ (((r >> 2) & 1) << 3);
    return C == 8 ? c ^ (((r >> 1) & 1) << 2) : c ^ ((r & 3) << 2);
  }
  // elements 16 ks + 8 hh .. +7 of K row r
  __device__ static __forceinline__ typename Frag<F>::v8 k_frag(const char* b,
                                                                int r, int ks,
                                                                int hh) {
    if constexpr (F::dtype == DAVET_F32) {
      const int c = ks * 4 + hh * 2;
      const f32x4 x = *reinterpret_cast<const f32x4*>(b + r * RB + (k_slot(r, c) << 4));
      const f32x4 y = *reinterpret_cast<const f32x4*>(b + r * RB + (k_slot(r, c + 1) << 4));
      return f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    } else {
      return *reinterpret_cast<const typename Frag<F>::v8*>(
          b + r * RB + (k_slot(r, ks * 2 + hh) << 4));
    }
  }
  __device__ static __forceinline__ const char* v_at(const char* b, int r, int d) {
    const int byte = d * (int)sizeof(st);
    return b + r * RB + (v_slot(r, byte >> 4) << 4) + (byte & 15);
  }
  // V^T: dim 32 dt + lane % 32 of keys 16 ps + 8 (e / 4) + 4 hh + e % 4, e < 8
  __device__ static __forceinline__ typename Frag<F>::v8 v_frag(const char* b,
                                                                int ps, int dt,
                                                                int lane) {
    const int hh = lane >> 5;
    if constexpr (F::dtype == DAVET_F32) {
      f32x8 f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f[e] = *reinterpret_cast<const float*>(
            v_at(b, ps * 16 + (e >> 2) * 8 + hh * 4 + (e & 3),
                 dt * 32 + (lane & 31)));
      return f;
    } else {
      // transposing reads: in each group of 16 lanes, lane j addresses key
      // 4 hh + j / 4 and four dims from 4 (j % 4); lane i then holds element
      // i % 4 of the piece of lane 4 r + i / 4, for r = 0 .. 3
      const int j = lane & 15;
      const int r = ps * 16 + hh * 4 + (j >> 2);
      const int d = dt * 32 + 16 * ((lane >> 4) & 1) + 4 * (j & 3);
      const v4s t0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)v_at(b, r, d));
      const v4s t1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_ptr)v_at(b, r + 8, d));
      const u32x2 v0 = __builtin_bit_cast(u32x2, t0);
      const u32x2 v1 = __builtin_bit_cast(u32x2, t1);
      return __builtin_bit_cast(typename Frag<F>::v8, u32x4{v0[0], v0[1], v1[0], v1[1]});
    }
  }
};

// 8 consecutive elements of global memory as a fragment
template <typename F>
__device__ __forceinline__ typename Frag<F>::v8 load_frag(const typename F::st* p) {
  if constexpr (F::dtype == DAVET_F32) {
    const f32x4 x = reinterpret_cast<const f32x4*>(p)[0];
    const f32x4 y = reinterpret_cast<const f32x4*>(p)[1];
    return f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  } else {
    return *reinterpret_cast<const typename Frag<F>::v8*>(p);
  }
}

// 64 consecutive entries of a sequence's page table row, one a lane; moves on
// as the keys do (page numbers must not fall behind `base`).
struct PageIds {
  const int32_t* row;
  int max_pages, base, ids;
  __device__ __forceinline__ void init(const int32_t* r, int mp) {
    row = r;
    max_pages = mp;
    base = -64;
    ids = -1;
  }
  __device__ __forceinline__ int at(int page) {
    if (page - base >= 64) {
      base = page;
      const int e = page + (int)(threadIdx.x & 63);
      ids = e < max_pages ? row[e] : -1;
    }
    return __builtin_amdgcn_readlane(ids, page - base);
  }
};

// Launch plan, by value: workgroups of sequence order[i] start at blk[i] (of
// one eighth of the grid when the key heads divide by 8).
struct AttnPlan {
  int32_t blk[DAVET_MAX_SEQS + 1];
  int32_t order[DAVET_MAX_SEQS];   // (bytes would be vector loads)
  int32_t piece;        // keys a piece
  int32_t pieces;       // most pieces of a sequence; 1: no partials
  int32_t xcd;          // key heads dealt out to the 8 XCDs
};

// One sequence's workgroups: [key head][piece][row tile], row tile fastest.
// With `xcd`, workgroup b runs on XCD b % 8 and takes key heads = b mod 8 only,
// so the tiles and pieces of a key head share one L2 and every XCD has the same
// work.
struct Place { int s, hk, piece, tile; };
// The last tile comes first under a causal mask: it sees the most keys.
__device__ __forceinline__ Place place(const AttnPlan& ap, const ChunkPack& cp,
                                       int n_kv, int g, int rows, bool causal) {
  const int b = ap.xcd ? (int)blockIdx.x >> 3 : (int)blockIdx.x;
  const int i = owner(ap.blk, cp.n_seqs, b);
  Place p;
  p.s = ap.order[i];
  const int n = cp.row0[p.s + 1] - cp.row0[p.s];
  const int nt = (n * g + rows - 1) / rows;
  const int np = (cp.kv[p.s] + ap.piece - 1) / ap.piece;
  int rem = b - ap.blk[i];
  const int h = rem / (nt * np);
  rem -= h * nt * np;
  p.hk = ap.xcd ? ((int)blockIdx.x & 7) + 8 * h : h;
  p.piece = rem / nt;
  p.tile = rem - p.piece * nt;
  if (causal) p.tile = nt - 1 - p.tile;
  return p;
}

struct Scale {
  float c, c_lo;        // scale * log2(e) as a sum of two floats
  float scale;
};

// (x - m) scale log2(e) for fp32 operands, where the rounding of the constant
// would show (-inf apart: times the constant's rest it might be +inf)
__device__ __forceinline__ float exact_arg(float d, const Scale& s) {
  return d == -INFINITY ? d : fmaf(d, s.c, d * s.c_lo);
}

// G wavefronts share a tile (4: wide, 1: narrow); BUFS buffers a tile stream.
template <typename F, int D, int G, int BUFS, int MINB>
__global__ void __launch_bounds__(256, MINB)
cache_attn_kernel(CacheView cv, ChunkPack cp, AttnPlan ap,
                  const typename F::st* __restrict__ q, int64_t ld_q,
                  typename F::st* __restrict__ out, int64_t ld_o,
                  float* __restrict__ lse, int n_heads, int block, Scale sc_,
                  float* __restrict__ part, int part_rows) {
  using st = typename F::st;
  using T = Tile<F, D>;
  using v8 = typename Frag<F>::v8;
  constexpr int KT = G == 4 ? 64 : 32;            // keys a tile
  constexpr int MT = KT / 32;
  constexpr int KG = 4 / G;                       // tile streams
  constexpr int TILE = KT * T::RB;                // bytes of K (or V)
  constexpr int GROUP = BUFS * 2 * TILE;
  constexpr int MERGE = G == 1 ? 4 * (32 * D + 64) * 4 : 0;
  constexpr int LDS = KG * GROUP > MERGE ? KG * GROUP : MERGE;
  constexpr int OWN = KT / G;                     // tile rows a wave moves
  constexpr int NI = OWN / T::RPI;                // its loads, of K and of V
  constexpr float BIAS = Frag<F>::kBias;
  __shared__ __attribute__((aligned(1024))) char smem[LDS];
  __shared__ int s_bad;         // some value of a masked tile is not finite
  __shared__ uint32_t s_dead[G];          // rows without a score above -inf, a bit each

  const int g = n_heads / cv.n_kv;
  const Place pl = place(ap, cp, cv.n_kv, g, 32 * G, block > 0);
  const int s = pl.s, hk = pl.hk;
  const int row0 = cp.row0[s], n = cp.row0[s + 1] - row0, kv = cp.kv[s];
  const int rows = n * g;
  const int lane = threadIdx.x & 63, l32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wrow = pl.tile * 32 * G + (G == 4 ? wave * 32 : 0);
  // keys up to the last one that any row of the wave sees (the rest of the tiles
  // that the workgroup moves are nothing to it)
  const int wave_end = wrow < rows
                           ? visible_end(min(wrow + 31, rows - 1) / g, n, kv, block)
                           : 0;
  // keys of this piece, up to the last one that any row of the tile sees
  const int tile_last = min(pl.tile * 32 * G + 32 * G, rows) - 1;
  const int end = min((pl.piece + 1) * ap.piece,
                      visible_end(tile_last / g, n, kv, block));
  const int begin = pl.piece * ap.piece;
  const int lim = visible_end(min(wrow + l32, rows - 1) / g, n, kv, block);
  // keys before this are visible to every row of the wave
  const int lim_all = visible_end(min(wrow, rows - 1) / g, n, kv, block);
  const int lim_tile = visible_end(pl.tile * 32 * G / g, n, kv, block);

  v8 qf[D / 16];
  {
    const int r = min(wrow + l32, rows - 1);
    const st* qp = q + (int64_t)(row0 + r / g) * ld_q +
                   (int64_t)(hk * g + r % g) * D + hh * 8;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = load_frag<F>(qp + ks * 16);
    // waited for here: in the key loop the compiler's waits for them would be
    // for tiles on their way as well
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+v"(qf[ks]));
  }
  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  // Scores are kept as differences from `ref`, near the row's largest: the matrix
  // ops start from -ref, so the subtraction costs neither an op nor a rounding of
  // its own (the sums' error still grows with the scores' size).
  float ref = 0.f, l_run = 0.f;
  bool seen = false;                // some score above -inf so far
  f32x16 start;
#pragma unroll
  for (int e = 0; e < 16; ++e) start[e] = 0.f;

  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  const int grp = G == 4 ? 0 : wave;
  char* gbuf = smem + grp * GROUP;
  PageIds pages;
  pages.init(cv.table + (int64_t)s * cv.max_pages, cv.max_pages);
  const int lg = cv.lg, psz = 1 << lg;

  // A 16-key group on its way to LDS.  A page holds whole groups.
  struct Group {
    int64_t at;         // byte of its first row in the pools; -1: in a hole
    int last;           // its last valid row
  };
  auto group = [&](int k0, int gi, int page) {
    const int key = min(k0 + gi * 16, (kv - 1) & ~15);
    Group r;
    r.at = (unsigned)page < (unsigned)cv.n_pages
               ? ((((int64_t)page * cv.n_kv + hk) << lg) + (key & (psz - 1))) * T::RB
               : -1;
    r.last = kv - 1 - key;
    return r;
  };
  // Moves its rows of K or V.  Rows past the last valid one repeat it; rows of
  // holes are zeroed (their scores are masked, but a NaN left in LDS would meet a
  // weight of 0).  Row r = j RPI + lane / C of chunk lane % C comes from slot
  // lane % C ^ f(r), and f(r) = f(j RPI) ^ f(lane / C).
  auto move16 = [&](bool of_k, char* to, const Group& r) {
    constexpr int N = 16 / T::RPI, RUN = N < 4 ? N : 4;
    auto slot = [&](int row, int c) {
      return of_k ? T::k_slot(row, c) : T::v_slot(row, c);
    };
    if (r.at < 0) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        *reinterpret_cast<u32x4*>(to + j * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
      return;
    }
    const char* from = static_cast<const char*>(of_k ? cv.k : cv.v) + r.at;  // scalar
    if (r.last >= 15) {
      const uint32_t first = (uint32_t)(lane * 16) ^ (slot(lane / T::C, 0) * 16);
#pragma unroll
      for (int j = 0; j < N; j += RUN) {
        uint32_t at[RUN];
#pragma unroll
        for (int i = 0; i < RUN; ++i) at[i] = first ^ (slot((j + i) * T::RPI, 0) * 16);
        dma16_run(from + j * 1024, at, to + j * 1024);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int lr = j * T::RPI + lane / T::C, c = lane % T::C;
        dma16(from, (uint32_t)min(lr, r.last) * T::RB + slot(lr, c) * 16, to + j * 1024);
      }
    }
  };
  // G = 4: the 16-key groups of the tile at k0 that lie in holes, and the one
  // that this wave moves
  struct Tag { int holes; Group mine; };
  auto tag = [&](int k0) {
    Tag r = {};
    int page;
    if (lg >= 6) {                      // the tile is in one page
      page = pages.at(k0 >> lg);
      r.holes = (unsigned)page >= (unsigned)cv.n_pages ? (1 << KT / 16) - 1 : 0;
    } else {
      page = 0;
#pragma unroll
      for (int gi = 0; gi < KT / 16; ++gi) {
        const int p = pages.at(min(k0 + gi * 16, kv - 1) >> lg);
        r.holes |= ((unsigned)p >= (unsigned)cv.n_pages) << gi;
        if (gi == wave) page = p;
      }
    }
    r.mine = group(k0, wave, page);
    return r;
  };
  auto move_k = [&](const Tag& r, int b) {
    move16(true, gbuf + b * 2 * TILE + wave * 16 * T::RB, r.mine);
  };
  auto move_v = [&](const Tag& r, int b) {
    move16(false, gbuf + b * 2 * TILE + TILE + wave * 16 * T::RB, r.mine);
  };
  // G = 1: the whole tile; returns its holes
  auto issue = [&](int k0, int b) -> int {
    char* kd = gbuf + b * 2 * TILE;
    int holes = 0;
#pragma unroll
    for (int gi = 0; gi < KT / 16; ++gi) {
      const Group r = group(k0, gi, pages.at(min(k0 + gi * 16, kv - 1) >> lg));
      holes |= (r.at < 0) << gi;
      move16(true, kd + gi * 16 * T::RB, r);
      move16(false, kd + TILE + gi * 16 * T::RB, r);
    }
    return holes;
  };

  // S^T - ref of a tile's keys
  auto scores = [&](const char* Kb, f32x16 (&sc)[MT]) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sc[mt] = start;
    if constexpr (F::dtype == DAVET_F32) {
      // two sums of half the length: a chain of D roundings would show in lse
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        f32x16 half;
#pragma unroll
        for (int e = 0; e < 16; ++e) half[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ks += 2) {
          sc[mt] = mm<F>(T::k_frag(Kb, mt * 32 + l32, ks, hh), qf[ks], sc[mt]);
          half = mm<F>(T::k_frag(Kb, mt * 32 + l32, ks + 1, hh), qf[ks + 1], half);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[mt][e] += half[e];
      }
    } else {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          sc[mt] = mm<F>(T::k_frag(Kb, mt * 32 + l32, ks, hh), qf[ks], sc[mt]);
    }
  };
  auto largest = [&](const f32x16 (&sc)[MT]) {
    float m = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, sc[mt][e]);
    return m;
  };
  // Masks a tile's scores and moves ref if need be; tmax: the largest unmasked
  auto settle = [&](int k0, int holes, f32x16 (&sc)[MT], float tmax) {
    // keys past a row's limit, or in a hole, score -inf
    const bool masked = k0 + KT > lim_all || holes;
    if (masked) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = mt * 32 + (e >> 2) * 8 + hh * 4 + (e & 3);
          if (k0 + at >= lim || ((holes >> (at >> 4)) & 1)) sc[mt][e] = -INFINITY;
        }
      tmax = largest(sc);
    }
    tmax = pair_max32(tmax);
    // ref moves only when it is 2^8 behind the largest score (or with the first
    // one): O is rescaled rarely
    const bool move = seen ? tmax * sc_.c > 8.0f : tmax > -INFINITY;
    if (__any(move)) {
      const float to = move ? ref + tmax : ref;
      const float by = move ? to - ref : 0.f;
      const float alpha = seen ? __builtin_amdgcn_exp2f(-by * sc_.c) : 0.f;
      ref = to;
      seen = seen || move;
      l_run *= alpha;
#pragma unroll
      for (int e = 0; e < 16; ++e) start[e] = -ref;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[mt][e] -= by;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
    }
  };
  // Probabilities as operands of 16 keys each; lo: what rounding to 16 bits
  // took off them (few rows wait for memory, not for the matrix cores).
  auto weigh = [&](const f32x16 (&sc)[MT], v8 (&hi)[KT / 16], v8 (&lo)[KT / 16]) {
    float psum = 0.f;
#pragma unroll
    for (int ps = 0; ps < KT / 16; ++ps) {
      u32x4 w, w2;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float p[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float x = sc[ps >> 1][(ps & 1) * 8 + e + u];
          p[u] = __builtin_amdgcn_exp2f(F::dtype == DAVET_F32
                                            ? exact_arg(x, sc_)
                                            : fmaf(x, sc_.c, BIAS));
          psum += p[u];
        }
        if constexpr (F::dtype == DAVET_F32) {
          hi[ps][e] = p[0];
          hi[ps][e + 1] = p[1];
        } else {
          const uint32_t h = round2<F>(p[0], p[1]);
          w[e / 2] = h;
          if constexpr (G == 1)
            w2[e / 2] = round2<F>(p[0] - F::load((uint16_t)(h & 0xffffu)),
                                  p[1] - F::load((uint16_t)(h >> 16)));
        }
      }
      if constexpr (F::dtype != DAVET_F32) {
        hi[ps] = __builtin_bit_cast(v8, w);
        if constexpr (G == 1) lo[ps] = __builtin_bit_cast(v8, w2);
      }
    }
    l_run += psum;
  };
  auto values = [&](const char* Vb, const v8 (&hi)[KT / 16], const v8 (&lo)[KT / 16]) {
#pragma unroll
    for (int ps = 0; ps < KT / 16; ++ps)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        const v8 vf = T::v_frag(Vb, ps, dt, lane);
        o[dt] = mm<F>(vf, hi[ps], o[dt]);
        if constexpr (G == 1 && F::dtype != DAVET_F32)
          o[dt] = mm<F>(vf, lo[ps], o[dt]);
      }
  };
  auto compute = [&](int k0, const char* Kb, int holes) {
    f32x16 sc[MT];
    scores(Kb, sc);
    settle(k0, holes, sc, largest(sc));
    v8 hi[KT / 16], lo[KT / 16];
    weigh(sc, hi, lo);
    values(Kb + TILE, hi, lo);
  };

  // A masked weight of 0 times an infinite (or NaN) value would be NaN.  Where
  // a tile has masked places its values are looked over first (each wave its
  // rows) and those that are not finite become 0; the rows that do see them
  // get them added at the end.
  auto tile_masked = [&](int k0, int holes) {
    return k0 + KT > lim_tile || holes != 0;
  };
  auto clean = [&](char* Vb) {
    char* at = Vb + (G == 4 ? wave * (TILE / 4) : 0);
    bool found = false;
#pragma unroll 1
    for (int i = lane; i < TILE / G / 16; i += 64) {
      u32x4 w = *reinterpret_cast<const u32x4*>(at + i * 16);
      bool bad = false;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if constexpr (F::dtype == DAVET_F32) {
          const bool b = (w[u] & 0x7f800000u) == 0x7f800000u;
          bad |= b;
          w[u] = b ? 0u : w[u];
        } else {
          const bool b0 = F::nonfinite((uint16_t)(w[u] & 0xffffu));
          const bool b1 = F::nonfinite((uint16_t)(w[u] >> 16));
          bad |= b0 || b1;
          w[u] = (b0 ? 0u : w[u] & 0xffffu) | (b1 ? 0u : w[u] & 0xffff0000u);
        }
      }
      if (bad) *reinterpret_cast<u32x4*>(at + i * 16) = w;
      found |= bad;
    }
    if (__any(found) && lane == 0) s_bad = 1;
  };

  if constexpr (G == 4) {
    const int nt = max(0, (end - begin + KT - 1) / KT);
    if constexpr (BUFS == 1) {
      // one buffer, refilled once every wave is done with it; the other
      // workgroups of the CU hide the load
      auto load = [&](int it) {
        const Tag r = tag(begin + it * KT);
        move_k(r, 0);
        move_v(r, 0);
        return r.holes;
      };
      int holes = nt > 0 ? load(0) : 0;
      for (int it = 0; it < nt; ++it) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        sync_lds();
        if (tile_masked(begin + it * KT, holes)) {
          clean(gbuf + TILE);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          sync_lds();
        }
        if (begin + it * KT < wave_end) compute(begin + it * KT, gbuf, holes);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        sync_lds();
        if (it + 1 < nt) holes = load(it + 1);
      }
    } else {
      // Two waves a SIMD do not fill each other's gaps by themselves: the matrix
      // ops of a tile and its exponentials took turns.  So the scores of tile
      // it + 1 are multiplied between the exponentials of tile it (K is loaded a
      // tile further ahead than V), in an order fixed by hand.  Four ragged
      // prompts, 32 x 128 heads, fp16: 0.77 PFLOP/s (before: 0.72), 0.87 in bf16.
      static_assert(F::dtype != DAVET_F32, "16-bit probabilities");
      f32x16 even[MT], odd[MT];
      float tmax = -INFINITY;
      Tag cur = {}, nxt = {};
      if (nt > 0) {
        cur = tag(begin);
        move_k(cur, 0);
        move_v(cur, 0);
        if (nt > 1) {
          nxt = tag(begin + KT);
          move_k(nxt, 1);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        sync_lds();
        if (begin < wave_end) {
          scores(gbuf, even);
          tmax = largest(even);
        }
      }
      // tile `it`, whose K and V are in buffer b, with the scores `sc`
      auto step = [&](int it, int b, f32x16 (&sc)[MT], f32x16 (&ahead)[MT]) {
        const int k0 = begin + it * KT;
        char* Vb = gbuf + b * 2 * TILE + TILE;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        sync_lds();
        Tag far = {};
        if (it + 2 < nt) {
          far = tag(k0 + 2 * KT);
          move_k(far, b);
        }
        if (it + 1 < nt) move_v(nxt, b ^ 1);
        if (tile_masked(k0, cur.holes)) {
          clean(Vb);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          sync_lds();
        }
        if (k0 < wave_end) {
          settle(k0, cur.holes, sc, tmax);
          // NK products S^T of the next tile (behind the last one: of what the
          // buffer holds, for nothing), then NV products O^T of this one, each
          // with kAhead fragments read ahead; pairs of probabilities between
          // the first NK + NV / 2 of them, just before their products.
          const char* Kn = gbuf + (b ^ 1) * 2 * TILE;
          constexpr int NK = MT * D / 16, DT = D / 32, NV = KT / 16 * DT;
          constexpr int PAIRS = KT / 4, SLOTS = NK + NV / 2;
          v8 f[kAhead], hi[KT / 16];
          auto read = [&](int i) {
            f[i % kAhead] =
                i < NK ? T::k_frag(Kn, (i % MT) * 32 + l32, i / MT, hh)
                       : T::v_frag(Vb, (i - NK) / DT, (i - NK) % DT, lane);
          };
#pragma unroll
          for (int i = 0; i < kAhead; ++i) read(i);
          float sum[2] = {0.f, 0.f};
          u32x4 w = {};
          auto pairs = [&](int slot) {
#pragma unroll
            for (int pr = 0; pr < PAIRS; ++pr) {
              if (pr * SLOTS / PAIRS != slot) continue;
              const int ps = pr / 4, e = pr % 4 * 2;
              float p[2];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                p[u] = __builtin_amdgcn_exp2f(
                    fmaf(sc[ps >> 1][(ps & 1) * 8 + e + u], sc_.c, BIAS));
                sum[u] += p[u];
              }
              w[pr % 4] = round2<F>(p[0], p[1]);
              if (pr % 4 == 3) hi[ps] = __builtin_bit_cast(v8, w);
            }
          };
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int i = 0; i < NK; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            ahead[i % MT] = mm<F>(f[i % kAhead], qf[i / MT],
                                  i < MT ? start : ahead[i % MT]);
            read(i + kAhead);
            pairs(i);
          }
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            o[i % DT] = mm<F>(f[(NK + i) % kAhead], hi[i / DT], o[i % DT]);
            if (i + kAhead < NV) read(NK + i + kAhead);
            pairs(NK + i);
          }
          __builtin_amdgcn_s_setprio(0);
          l_run += sum[0] + sum[1];
          tmax = largest(ahead);
        }
        cur = nxt;
        nxt = far;
      };
      for (int it = 0; it < nt; it += 2) {
        step(it, 0, even, odd);
        if (it + 1 < nt) step(it + 1, 1, odd, even);
      }
    }
  } else {
    // tiles wave, wave + 4, ... of the piece
    int k0 = begin + wave * KT;
    int holes = k0 < end ? issue(k0, 0) : 0;
    for (int it = 0; k0 < end; ++it, k0 += 4 * KT) {
      const int cur = holes;
      if constexpr (BUFS == 2) {
        if (k0 + 4 * KT < end) {
          holes = issue(k0 + 4 * KT, (it + 1) & 1);
          // the loads of the next tile may stay out; holes issue fewer
          if (holes)
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
          else
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * NI) : "memory");
        } else {
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        }
        if (tile_masked(k0, cur)) {
          clean(gbuf + (it & 1) * 2 * TILE + TILE);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        compute(k0, gbuf + (it & 1) * 2 * TILE, cur);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      } else {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if (tile_masked(k0, cur)) {
          clean(gbuf + TILE);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        compute(k0, gbuf, cur);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (k0 + 4 * KT < end) holes = issue(k0 + 4 * KT, 0);
      }
    }
  }

  // The lane's coordinates again, from the lane number, so that none of them
  // is held in a register across the key loop.
  int lane_e;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\t"
               "v_mbcnt_hi_u32_b32 %0, -1, %0"
               : "=v"(lane_e));
  const int l32e = lane_e & 31, hhe = lane_e >> 5;
  const int re = min(wrow + l32e, rows - 1);
  const int qi = re / g, qh = hk * g + re % g;
  const float bias_ln = BIAS * kLn2;
  l_run = pair_sum32(l_run);
  const float m_run = l_run == 0.f ? -INFINITY : ref;
  if constexpr (G == 1) {
    // join the four streams: O as [wave][dim][32 rows], then max and sum
    __syncthreads();
    float* mo = reinterpret_cast<float*>(smem);
    float* ml = mo + 4 * D * 32;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        mo[(wave * D + dt * 32 + (e >> 2) * 8 + hhe * 4 + (e & 3)) * 32 + l32e] =
            o[dt][e];
    if (hhe == 0) {
      ml[wave * 64 + l32e] = m_run;
      ml[wave * 64 + 32 + l32e] = l_run;
    }
    __syncthreads();
    // thread: row l32e, dims (D / 8) (t / 32) ..
    constexpr int DP = D / 8;
    const int d0 = (wave * 2 + hhe) * DP;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w * 64 + l32e]);
    float wt[4], l = 0.f;
    bool use[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = ml[w * 64 + l32e], lw = ml[w * 64 + 32 + l32e];
      use[w] = lw != 0.f;                 // (NaN scores: sum NaN, maximum -inf)
      wt[w] = use[w] ? __builtin_amdgcn_exp2f((mw - m) * sc_.c) : 0.f;
      if (use[w]) l += wt[w] * lw;
    }
    const uint32_t dead = (uint32_t)__ballot(l == 0.f);
    if (wave == 0 && lane_e == 0) s_dead[0] = dead;
    float acc[DP];
#pragma unroll
    for (int i = 0; i < DP; ++i) {
      acc[i] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        if (use[w]) acc[i] += wt[w] * mo[(w * D + d0 + i) * 32 + l32e];
    }
    if (wrow + l32e < rows) {
      if (ap.pieces > 1) {
        const int64_t at = (int64_t)pl.piece * part_rows +
                           (int64_t)(row0 + qi) * n_heads + qh;
        float* po = part + at * D + d0;
#pragma unroll
        for (int i = 0; i < DP; i += 4)
          *reinterpret_cast<f32x4*>(po + i) =
              f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
        if (d0 == 0) {
          float* pm = part + (int64_t)ap.pieces * part_rows * D + at * 2;
          pm[0] = m;
          pm[1] = l;
        }
      } else {
        // a row that sees nothing (or only scores of -inf): zeros, lse -inf
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        st* op = out + (int64_t)(row0 + qi) * ld_o + (int64_t)qh * D + d0;
#pragma unroll
        for (int i = 0; i < DP; i += 2) {
          if constexpr (F::dtype == DAVET_F32) {
            op[i] = acc[i] * inv;
            op[i + 1] = acc[i + 1] * inv;
          } else {
            *reinterpret_cast<uint32_t*>(op + i) =
                round2<F>(acc[i] * inv, acc[i + 1] * inv);
          }
        }
        if (lse && d0 == 0)
          lse[(int64_t)(row0 + qi) * n_heads + qh] =
              l == 0.f ? -INFINITY : m * sc_.scale + (logf(l) - bias_ln);
      }
    }
  } else {
    const uint32_t dead = (uint32_t)__ballot(l_run == 0.f);
    if (lane_e == 0) s_dead[wave] = dead;
    if (l_run == 0.f) {         // (their O may be 0 times an infinity)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
    }
    if (wrow + l32e >= rows) {
      // nothing to write
    } else if (ap.pieces > 1) {
      const int64_t at = (int64_t)pl.piece * part_rows +
                         (int64_t)(row0 + qi) * n_heads + qh;
      float* po = part + at * D + hhe * 4;
      // (the join does not use the O of a piece that saw nothing)
      if (l_run != 0.f)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int u = 0; u < 4; ++u)
            *reinterpret_cast<f32x4*>(po + dt * 32 + u * 8) =
                f32x4{o[dt][u * 4], o[dt][u * 4 + 1], o[dt][u * 4 + 2], o[dt][u * 4 + 3]};
      if (hhe == 0) {
        float* pm = part + (int64_t)ap.pieces * part_rows * D + at * 2;
        pm[0] = m_run;
        pm[1] = l_run;
      }
    } else {
      const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
      st* op = out + (int64_t)(row0 + qi) * ld_o + (int64_t)qh * D + hhe * 4;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[dt][u * 4 + e] * inv;
          if constexpr (F::dtype == DAVET_F32)
            *reinterpret_cast<f32x4*>(op + dt * 32 + u * 8) =
                f32x4{x[0], x[1], x[2], x[3]};
          else
            *reinterpret_cast<u32x2*>(op + dt * 32 + u * 8) =
                u32x2{round2<F>(x[0], x[1]), round2<F>(x[2], x[3])};
        }
      if (lse && hhe == 0)
        lse[(int64_t)(row0 + qi) * n_heads + qh] =
            l_run == 0.f ? -INFINITY
                         : m_run * sc_.scale + (logf(l_run) - bias_ln);
    }
  }

  // Values that `clean` took out, for the rows that see them and have a score: a
  // positive weight times an infinity (or NaN) is that.  (The join may multiply a
  // piece by a weight that underflowed: NaN for an infinity.)  One thread a dim;
  // speed does not matter here.
  __syncthreads();
  if (s_bad && wave * 64 + lane_e < D) {
    const int d = wave * 64 + lane_e;
    for (int k0 = begin; k0 < end; k0 += KT) {
      int holes = 0;
      for (int gi = 0; gi < KT / 16; ++gi) {
        const int key = min(k0 + gi * 16, (kv - 1) & ~15);
        const int page = cv.table[(int64_t)s * cv.max_pages + (key >> lg)];
        holes |= ((unsigned)page >= (unsigned)cv.n_pages) << gi;
      }
      if (!tile_masked(k0, holes)) continue;
      for (int key = k0; key < min(k0 + KT, end); ++key) {
        const int page = cv.table[(int64_t)s * cv.max_pages + (key >> lg)];
        if ((unsigned)page >= (unsigned)cv.n_pages) continue;
        const float x = F::load(static_cast<const st*>(
            cv.v)[((((int64_t)page * cv.n_kv + hk) << lg) + (key & (psz - 1))) * D + d]);
        if (fabsf(x) < INFINITY) continue;
        for (int rr = pl.tile * 32 * G; rr <= tile_last; ++rr) {
          if (key >= visible_end(rr / g, n, kv, block)) continue;
          const int own = rr - pl.tile * 32 * G;
          if (s_dead[own >> 5] >> (own & 31) & 1) continue;
          const int tok = row0 + rr / g, hd = hk * g + rr % g;
          if (ap.pieces > 1) {
            part[((int64_t)pl.piece * part_rows + (int64_t)tok * n_heads + hd) * D + d] += x;
          } else {
            st* at = out + (int64_t)tok * ld_o + (int64_t)hd * D + d;
            *at = F::store(F::load(*at) + x);
          }
        }
      }
    }
  }
}

// Joins the pieces of every row: with m the largest piece maximum and
// w_p = 2^((m_p - m) c), o = sum w_p O_p / sum w_p l_p.  One wavefront a row: the
// row, and so its sequence's entries in the kernel's arguments, are scalar; piece p's
// maximum and sum are lane p's (there are at most 64), a lane adds D / 64 dims in
// piece order.  Nothing is loaded twice or one after the other: it is all latency.
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, lane_xor<1>(x));
  x = fmaxf(x, lane_xor<2>(x));
  x = fmaxf(x, lane_xor<4>(x));
  x = fmaxf(x, lane_xor<8>(x));
  x = fmaxf(x, lane_xor<16>(x));
  return fmaxf(x, lane_xor<32>(x));
}
__device__ __forceinline__ float wave_sum(float x) {
  x += lane_xor<1>(x);
  x += lane_xor<2>(x);
  x += lane_xor<4>(x);
  x += lane_xor<8>(x);
  x += lane_xor<16>(x);
  return x + lane_xor<32>(x);
}
template <typename F, int D>
__global__ void __launch_bounds__(256)
cache_merge_kernel(ChunkPack cp, const float* __restrict__ part, int part_rows,
                   int piece, int pieces, typename F::st* __restrict__ out,
                   int64_t ld_o, float* __restrict__ lse, int n_heads, Scale sc_) {
  constexpr int E = D / 64;
  constexpr int U = 8;                  // pieces' loads at a time
  typedef float vec __attribute__((ext_vector_type(E)));
  const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (row >= part_rows) return;
  const int lane = threadIdx.x & 63, d0 = lane * E;
  const int tok = row / n_heads, h = row % n_heads;
  const int s = owner(cp.row0, cp.n_seqs, tok);
  const int np = (cp.kv[s] + piece - 1) / piece;
  const float* pm = part + (int64_t)pieces * part_rows * D +
                    ((int64_t)min(lane, np - 1) * part_rows + row) * 2;
  const float mp = pm[0], lp = lane < np ? pm[1] : 0.f;
  vec o[U];
  auto load = [&](int p0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      o[u] = *reinterpret_cast<const vec*>(
          part + ((int64_t)min(p0 + u, np - 1) * part_rows + row) * D + d0);
  };
  load(0);
  // a piece that saw nothing: sum 0, maximum -inf (NaN scores: sum NaN)
  const bool use = lp != 0.f;
  const float m = wave_max(use ? mp : -INFINITY);
  const float w = use ? __builtin_amdgcn_exp2f((mp - m) * sc_.c) : 0.f;
  const float l = wave_sum(use ? w * lp : 0.f);
  const uint64_t used = __ballot(use);
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  for (int p0 = 0; p0 < np; p0 += U) {
    if (p0 > 0) load(p0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + u;
      if (p >= np || !(used >> p & 1)) continue;
      const float wp = __uint_as_float(
          (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(w), p));
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += wp * o[u][e];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  typename F::st* op = out + (int64_t)tok * ld_o + (int64_t)h * D + d0;
  if constexpr (F::dtype != DAVET_F32 && E == 2)
    *reinterpret_cast<uint32_t*>(op) = round2<F>(acc[0] * inv, acc[1] * inv);
  else
#pragma unroll
    for (int e = 0; e < E; ++e) op[e] = F::store(acc[e] * inv);
  if (lse && lane == 0)
    lse[row] = l == 0.f
                   ? -INFINITY
                   : m * sc_.scale + (logf(l) - Frag<F>::kBias * kLn2);
}

// The same for many rows, where throughput counts: four dims a lane, so D / 4 lanes a
// row and R rows of one token a wavefront (its sequence is scalar), and the sums in
// one pass over the pieces, U at a time.
template <typename F, int D>
__global__ void __launch_bounds__(256)
cache_merge_rows_kernel(ChunkPack cp, const float* __restrict__ part, int part_rows,
                        int piece, int pieces, typename F::st* __restrict__ out,
                        int64_t ld_o, float* __restrict__ lse, int n_heads,
                        Scale sc_) {
  constexpr int L = D / 4, R = 64 / L, U = 4;
  const int w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int per = (n_heads + R - 1) / R, tok = w / per;
  if (tok >= cp.row0[cp.n_seqs]) return;
  const int lane = threadIdx.x & 63;
  const int h = (w - tok * per) * R + lane / L, d0 = lane % L * 4;
  const int s = owner(cp.row0, cp.n_seqs, tok);
  const int np = (cp.kv[s] + piece - 1) / piece;
  const int64_t row = (int64_t)tok * n_heads + min(h, n_heads - 1);
  const float* pm = part + (int64_t)pieces * part_rows * D;
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < np; p0 += U) {
    float mp[U], lp[U];
    f32x4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = (int64_t)min(p0 + u, np - 1) * part_rows + row;
      mp[u] = pm[at * 2];
      lp[u] = pm[at * 2 + 1];
      o[u] = *reinterpret_cast<const f32x4*>(part + at * D + d0);
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p0 + u >= np) lp[u] = 0.f;
      if (lp[u] != 0.f) top = fmaxf(top, mp[u]);
    }
    const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * sc_.c);
    m = top;
    l *= alpha;
    acc *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (lp[u] == 0.f) continue;       // (its O is not written)
      const float wp = __builtin_amdgcn_exp2f((mp[u] - m) * sc_.c);
      l += wp * lp[u];
      acc += wp * o[u];
    }
  }
  if (h >= n_heads) return;
  acc *= l == 0.f ? 0.f : 1.0f / l;
  typename F::st* op = out + (int64_t)tok * ld_o + (int64_t)h * D + d0;
  if constexpr (F::dtype == DAVET_F32)
    *reinterpret_cast<f32x4*>(op) = acc;
  else
    *reinterpret_cast<u32x2*>(op) = u32x2{round2<F>(acc[0], acc[1]),
                                          round2<F>(acc[2], acc[3])};
  if (lse && d0 == 0)
    lse[row] = l == 0.f
                   ? -INFINITY
                   : m * sc_.scale + (logf(l) - Frag<F>::kBias * kLn2);
}

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
                     float* __restrict__ part) {
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
  const int blk = blockIdx.x % nblk, chunk = blockIdx.x / nblk;
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

// (its product with log2(e) and the rest of that stay normal numbers)
bool good_scale(float s) { return s == 0.f || (s >= 1e-30f && s <= 1e30f); }

Scale make_scale(float scale, int D) {
  const double s = scale == 0.f ? 1.0 / sqrt((double)D) : (double)scale;
  const double c = s * 1.4426950408889634074;
  Scale r;
  r.c = (float)c;
  r.c_lo = (float)(c - (double)r.c);
  r.scale = (float)s;
  return r;
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

size_t attn_part_floats(int64_t rows, int pieces, int D) {
  return (size_t)rows * pieces * (D + 2);
}

int max_pieces(int64_t rows) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMaxPieces, kMaxPartRows / rows));
}

// Cuts the keys into pieces, multiples of `unit`, so that the workgroups fill the
// chip once: `want` of them run at a time.  No piece is shorter than `least`, and
// up to `whole` keys stay in one (no second launch).
AttnPlan plan_attn(const ChunkPack& cp, int n_kv, int g, int rows, int want,
                   int unit, int least, int whole, int cap) {
  AttnPlan ap{};
  ap.xcd = n_kv % 8 == 0;
  int64_t work = 0;
  int longest = 1;
  for (int s = 0; s < cp.n_seqs; ++s) {
    const int64_t nt = ((int64_t)(cp.row0[s + 1] - cp.row0[s]) * g + rows - 1) / rows;
    work += nt * n_kv * cp.kv[s];
    if (nt) longest = std::max(longest, cp.kv[s]);
    ap.order[s] = s;
  }
  // longest first: what is left for the last round is short
  std::sort(ap.order, ap.order + cp.n_seqs, [&](int32_t a, int32_t b) {
    return cp.kv[a] != cp.kv[b] ? cp.kv[a] > cp.kv[b] : a < b;
  });
  int64_t piece = std::max<int64_t>((work + want - 1) / want,
                                    ((int64_t)longest + cap - 1) / cap);
  piece = std::max<int64_t>(align_up(piece, unit), longest <= whole ? whole : least);
  auto blocks = [&](int64_t p, int s) {
    const int64_t nt = ((int64_t)(cp.row0[s + 1] - cp.row0[s]) * g + rows - 1) / rows;
    return nt * n_kv * ((cp.kv[s] + p - 1) / p);
  };
  for (; piece < longest; piece = align_up(piece + piece / 16, unit)) {
    int64_t t = 0;
    for (int s = 0; s < cp.n_seqs; ++s) t += blocks(piece, s);
    if (t <= want) break;
  }
  piece = std::min<int64_t>(piece, align_up(longest, unit));
  ap.piece = (int)piece;
  ap.pieces = (int)((longest + piece - 1) / piece);
  int64_t at = 0;
  for (int i = 0; i < cp.n_seqs; ++i) {
    ap.blk[i] = (int)at;
    at += blocks(piece, ap.order[i]) / (ap.xcd ? 8 : 1);
  }
  ap.blk[cp.n_seqs] = (int)at;
  return ap;
}

template <typename F, int D>
int run_attention(const CacheView& cv, const ChunkPack& cp, const void* q,
                  int64_t ld_q, void* out, int64_t ld_o, float* lse,
                  int n_heads, int block, Scale sc, float* part,
                  hipStream_t stream) {
  using st = typename F::st;
  const int g = n_heads / cv.n_kv;
  const int64_t rows = (int64_t)cp.row0[cp.n_seqs] * n_heads;
  int most = 0;
  for (int s = 0; s < cp.n_seqs; ++s)
    most = std::max(most, cp.row0[s + 1] - cp.row0[s]);
  // Rows from which the wide form is taken, by the longest chunk of the batch (one
  // launch): a short one beside it has its probabilities rounded once too.  Error of
  // the output against 64 bits, its own rounding included: 2.1e-4 narrow, 2.8e-4 wide
  // in fp16; 1.7e-3 and 2.2e-3 in bf16.  16 bits: sixteen sequences over up to
  // 3000 keys, 32 heads of 128, take 109 us with 48 rows where narrow takes 161, and
  // 100 both with 32, where narrow keeps more of the probabilities.  fp32 (one
  // buffer): four sequences, 8 heads, 58 us with 64 rows where narrow takes 43, and
  // 62 with 96 where it takes 63.
  constexpr bool f32 = F::dtype == DAVET_F32;
  const bool wide = (int64_t)most * g > (f32 ? 64 : 32);
  constexpr int WB = f32 ? 1 : 2;                       // wide: buffers
  constexpr int WM = 2;                                 // workgroups a CU
  constexpr int NB = f32 && D == 128 ? 1 : 2;           // narrow
  constexpr int NM = !f32 && D == 64 ? 2 : 1;
  // Shortest pieces.  narrow, one tile a wave: one token, 8 key heads of 128 dims,
  // 2964 keys 15.1 us in pieces of 128, 16.1 of 256, 19.1 of 512; 640 keys 13.1, and
  // 18 in one piece; 250 keys 13.9, and 12.3 in one.  fp32, 64 dims: 250 keys 13.0
  // and 16.3 in one, 200 the same.  wide: 128 queries, 8 heads, 2964 keys 24.6 us in
  // pieces of 64, 20.2 of 128, 19.3 of 256; fp32, whose tile of 64 keys takes 4 to 8
  // us, 194 queries over 272 keys 23 us in pieces of 64, 32 of 128, 48 of 256.
  constexpr int NH = f32 ? 256 : 384;
  constexpr int WL = f32 ? 64 : 256, WH = f32 ? 128 : 256;
  const AttnPlan ap = plan_attn(cp, cv.n_kv, g, wide ? 128 : 32,
                                256 * (wide ? WM : NM), wide ? 64 : 128,
                                wide ? WL : 128, wide ? WH : NH,
                                max_pieces(rows));
  const int64_t grid = (int64_t)ap.blk[cp.n_seqs] * (ap.xcd ? 8 : 1);
  DAVET_CHECK_ARG(grid < (1ll << 31), DAVET_ESHAPE,
                  "davet_cache_attention: too many row tiles");
  {
    ProfScope ps(KC_MISC, stream);
    if (wide)
      hipLaunchKernelGGL((cache_attn_kernel<F, D, 4, WB, WM>), dim3((unsigned)grid),
                         dim3(256), 0, stream, cv, cp, ap, (const st*)q, ld_q,
                         (st*)out, ld_o, lse, n_heads, block, sc, part, (int)rows);
    else
      hipLaunchKernelGGL((cache_attn_kernel<F, D, 1, NB, NM>), dim3((unsigned)grid),
                         dim3(256), 0, stream, cv, cp, ap, (const st*)q, ld_q,
                         (st*)out, ld_o, lse, n_heads, block, sc, part, (int)rows);
    DAVET_HIP(hipGetLastError());
  }
  if (ap.pieces > 1) {
    ProfScope ps(KC_MISC, stream);
    // 27,000 rows of 64 dims in two pieces 13 us a wavefront each, 5 packed (of 128
    // dims 14 and 8); 4096 rows the same; 32 rows in 24 pieces 2.5 us more packed
    if (rows < 8192) {
      hipLaunchKernelGGL((cache_merge_kernel<F, D>),
                         dim3((unsigned)((rows + 3) / 4)), dim3(256), 0,
                         stream, cp, part, (int)rows, ap.piece, ap.pieces, (st*)out,
                         ld_o, lse, n_heads, sc);
    } else {
      constexpr int R = 256 / D;                // rows a wavefront
      const int64_t waves = (int64_t)cp.row0[cp.n_seqs] * ((n_heads + R - 1) / R);
      hipLaunchKernelGGL((cache_merge_rows_kernel<F, D>),
                         dim3((unsigned)((waves + 3) / 4)), dim3(256), 0,
                         stream, cp, part, (int)rows, ap.piece, ap.pieces, (st*)out,
                         ld_o, lse, n_heads, sc);
    }
    DAVET_HIP(hipGetLastError());
  }
  return DAVET_OK;
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
    hipLaunchKernelGGL((cache_weights_kernel<F, D, KW>), dim3((unsigned)grid), dim3(256),
                       0, stream, cv, cp, wp, (const typename F::st*)q, ld_q, lse,
                       n_heads, block, scale, prev, weights, ld_w, part);
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

size_t workspace_bytes(int64_t total_q, int n_heads, int D) {
  const int64_t rows = total_q * n_heads;
  size_t b = 0;
  if (rows > 0 && max_pieces(rows) > 1)
    b = attn_part_floats(rows, max_pieces(rows), D) * sizeof(float);
  const size_t w = (size_t)kWeightGroups * 2 * kWeightKeys * sizeof(float);
  return align_up(std::max(b, w), 256);
}

int check_workspace(const void* ws, size_t have, int64_t total_q, int n_heads,
                    int D, const char* who) {
  const size_t need = workspace_bytes(total_q, n_heads, D);
  DAVET_CHECK_ARG(ws && ((uintptr_t)ws & 255) == 0 && have >= need, DAVET_ENOMEM,
                  std::string(who) + ": workspace missing, misaligned or below " +
                      std::to_string(need) + " bytes");
  return DAVET_OK;
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
  int rc = check_cache(cache, true, who, &cv);
  if (!rc) rc = check_heads(cache, n_heads, who);
  if (!rc) rc = check_chunk(cache, n_seqs, cu_q, kv_len, who, &cp);
  const int D = cache ? cache->head_dim : 0;
  const int64_t total = rc ? 0 : cp.row0[n_seqs];
  if (!rc && total > 0)
    rc = check_rows(q, ld_q, (int64_t)n_heads * D, cache->dtype, who, "q");
  if (!rc && total > 0)
    rc = check_rows(out, ld_out, (int64_t)n_heads * D, cache->dtype, who, "out");
  if (rc) return rc;
  DAVET_CHECK_ARG(good_scale(scale), DAVET_EINVAL,
                  "davet_cache_attention: scale must be 0 or in [1e-30, 1e30]");
  DAVET_CHECK_ARG(block >= 0, DAVET_EINVAL,
                  "davet_cache_attention: block must not be negative");
  DAVET_CHECK_ARG(aligned4({lse}), DAVET_EINVAL,
                  "davet_cache_attention: lse must be 4-byte aligned");
  if (total == 0) return DAVET_OK;
  DAVET_CHECK_ARG(total * n_heads <= (1ll << 30), DAVET_ESHAPE,
                  "davet_cache_attention: too many query rows");
  rc = check_workspace(workspace, ws_bytes, total, n_heads, D, who);
  if (rc) return rc;
  const size_t es = dtype_size(cache->dtype);
  DAVET_CHECK_ARG(!rows_overlap(out, ld_out, n_heads * D, q, ld_q, n_heads * D, total,
                                es),
                  DAVET_EINVAL, "davet_cache_attention: out overlaps q");
  const Scale sc = make_scale(scale, D);
  float* part = static_cast<float*>(workspace);
#define ATT(F, DIM) run_attention<F, DIM>(cv, cp, q, ld_q, out, ld_out, lse,   \
                                          n_heads, block, sc, part, stream)
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
