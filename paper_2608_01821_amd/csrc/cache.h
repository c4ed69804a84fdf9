// Shared by the kernels over a paged key/value cache: its description as the
// kernels see it, the packed chunk of new tokens, and the host's checks.
#pragma once

#include <initializer_list>

#include "common.h"

namespace davet {

// The cache as kernels see it.  Keys (and values) of page p, head h, slot o
// start at element (((p * n_kv + h) << lg) + o) * head_dim, 64-bit arithmetic.
struct CacheView {
  void* k;
  void* v;
  const int32_t* table;     // [n_seqs, max_pages]
  int32_t max_pages, n_pages, lg, n_kv;
};

// The chunk: sequence s owns rows row0[s] .. row0[s+1], the last tokens of its
// kv[s] cached ones.
struct ChunkPack {
  int32_t n_seqs;
  int32_t row0[DAVET_MAX_SEQS + 1];
  int32_t kv[DAVET_MAX_SEQS];
};

// Two values rounded (nearest even) into one word, a in the low half, in one
// instruction of either 16-bit format.
template <typename F>
__device__ __forceinline__ uint32_t round2(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 v = {a, b};
  if constexpr (F::dtype == DAVET_BF16) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  } else {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
  }
}

// The value of lane ^ O without a trip through LDS: half-wave and row swaps (which
// leave the lower and the upper ones), a rotation by 8 in rows of 16, mirrored
// halves of 8, permuted fours.  Two rows of 126,464 logits, top 5: 12.6 us by
// way of LDS, 11.5 so.
template <int O>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
#define DPP(v, ctrl) \
  (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v), ctrl, 0xf, 0xf, false)
  if constexpr (O == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  } else if constexpr (O == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  } else if constexpr (O == 8) {
    return DPP(x, 0x128);
  } else if constexpr (O == 4) {
    return DPP(DPP(x, 0x141), 0x1b);
  } else {
    return DPP(x, O == 2 ? 0x4e : 0xb1);
  }
#undef DPP
}
template <int O>
__device__ __forceinline__ float lane_xor(float x) {
  return __uint_as_float(lane_xor<O>(__float_as_uint(x)));
}
template <int O>
__device__ __forceinline__ uint64_t lane_xor(uint64_t x) {
  return (uint64_t)lane_xor<O>((uint32_t)(x >> 32)) << 32 | lane_xor<O>((uint32_t)x);
}

constexpr int kCacheGroup = 16;   // smallest page: 16 aligned keys share one

// Keys visible to query i of a chunk of n among kv cached tokens: all of them
// (block 0), or those up to the end of the query's block.
__host__ __device__ inline int visible_end(int i, int n, int kv, int block) {
  if (block == 0) return kv;
  const int64_t e = ((int64_t)(i / block) + 1) * block;
  return kv - n + (int)(e < n ? e : n);
}

// The last entry of an ascending offset list (first[0] = 0, n + 1 entries)
// that is not above `at`: the sequence that owns a row, or a workgroup.
__device__ __forceinline__ int owner(const int32_t* first, int n, int at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}

// Checks of a cache and, below, of a chunk on it; both fill what kernels take.
int check_cache(const davet_kv_cache* c, bool need_v, const char* who,
                CacheView* out);
int check_chunk(const davet_kv_cache* c, int32_t n_seqs, const int32_t* cu_q,
                const int32_t* kv_len, const char* who, ChunkPack* out);
int check_rows(const void* p, int64_t ld, int64_t width, int dtype,
               const char* who, const char* what);
// n_heads a multiple of the cache's heads, at most 1024
int check_heads(const davet_kv_cache* c, int32_t n_heads, const char* who);
// whether all start at 4-byte boundaries (NULL does)
inline bool aligned4(std::initializer_list<const void*> ps) {
  uintptr_t x = 0;
  for (const void* p : ps) x |= (uintptr_t)p;
  return (x & 3) == 0;
}
// whether [a, a + an) and [b, b + bn) bytes overlap
inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return an && bn && x < y + bn && y < x + an;
}
// whether n rows of aw elements from a, every lda, share one with n rows of bw from
// b, every ldb: rows of one stride may lie side by side, others are taken as whole
// ranges (widths at most the strides)
inline bool rows_overlap(const void* a, int64_t lda, int64_t aw, const void* b,
                         int64_t ldb, int64_t bw, int64_t n, size_t es) {
  if (n == 0 || aw == 0 || bw == 0) return false;
  if (!overlap(a, ((n - 1) * lda + aw) * es, b, ((n - 1) * ldb + bw) * es)) return false;
  if (n == 1 || lda != ldb) return true;
  const uintptr_t row = lda * es;
  const uintptr_t d = ((uintptr_t)b % row + row - (uintptr_t)a % row) % row;
  return d < aw * es || d + bw * es > row;
}

}  // namespace davet
