// A tree of drafted tokens: its positions and ancestors, and its attention over the
// paged cache (the kernels of cache_attn.h with a mask for the chunk's own keys).
//
// Ancestors by doubling: with A_k(i) the first 2^k tokens on the way up from i (i
// itself the first) and J_k(i) the one that comes after them,
//   A_{k+1}(i) = A_k(i) + A_k(J_k(i)),  J_{k+1}(i) = J_k(J_k(i)),
// so a tree of depth d takes log2 d steps, not d.  A thread a token: drafts of up to 64
// tokens by a wavefront a sequence, the sets as two words a lane (16 of 64 tokens: 2.4
// us), larger ones by a workgroup, the sets in LDS (those 16: 4.4 us; of 256 tokens 5.5).
//
// The attention walks the cache once for all tokens of the tree, as for a chunk; only
// tiles that reach into the chunk read the rows' masks (LDS, a shift a lane and tile).
// Bound by HBM: eight trees of 26 tokens on 32,700 cached ones, 32 heads over 8 of 128,
// fp16, 151 us (779 MB, 5.1 TB/s) and 10 to join the pieces; sixteen of up to 64 on up to
// 3741, 32 heads, bf16, 127 us (607 MB, 4.8 TB/s).  fp32, eight of 64 to 256 on up to
// 3000, 32 heads over 8: 88 to 104 TFLOP/s of 154, with one buffer as the chunk's.

#include "cache_attn.h"

namespace davet {
namespace {

struct TreePack {
  int32_t n_seqs;
  int32_t row0[DAVET_MAX_SEQS + 1];
  int32_t first[DAVET_MAX_SEQS];      // position of a token without a parent
};

__global__ void __launch_bounds__(DAVET_MAX_TREE)
tree_plan_kernel(TreePack tp, const int32_t* __restrict__ parent,
                 int32_t* __restrict__ pos, uint32_t* __restrict__ mask) {
  constexpr int W = kTreeWords, S = W + 1;    // (rows' words in different banks)
  __shared__ uint32_t up[DAVET_MAX_TREE * S];
  __shared__ int jump[DAVET_MAX_TREE], above[DAVET_MAX_TREE];
  const int s = blockIdx.x, i = threadIdx.x;
  const int row0 = tp.row0[s], n = tp.row0[s + 1] - row0;
  int j = -1;
  if (i < n) {
    j = parent[row0 + i];
    if (j >= i) j = -1;                       // no parent comes later
    if (j < 0) j = -1;
  }
  uint32_t a[W];
#pragma unroll
  for (int w = 0; w < W; ++w) a[w] = w == i >> 5 ? 1u << (i & 31) : 0u;
  int d = j >= 0 ? 1 : 0;
  // (steps halve the way to the top: at most 8)
  while (__syncthreads_or(j >= 0)) {
#pragma unroll
    for (int w = 0; w < W; ++w) up[i * S + w] = a[w];
    jump[i] = j;
    above[i] = d;
    __syncthreads();
    if (j >= 0) {
#pragma unroll
      for (int w = 0; w < W; ++w) a[w] |= up[j * S + w];
      d += above[j];
      j = jump[j];
    }
  }
  if (i >= n) return;
  if (pos) pos[row0 + i] = tp.first[s] + d;
  if (mask) {
    uint32_t* m = mask + (int64_t)(row0 + i) * W;
#pragma unroll
    for (int w = 0; w < W; ++w) m[w] = a[w];
  }
}

// Sequences of at most 64 tokens.
__global__ void __launch_bounds__(64)
tree_plan_small_kernel(TreePack tp, const int32_t* __restrict__ parent,
                       int32_t* __restrict__ pos, uint32_t* __restrict__ mask) {
  constexpr int W = kTreeWords;
  const int s = blockIdx.x, i = threadIdx.x;
  const int row0 = tp.row0[s], n = tp.row0[s + 1] - row0, first = tp.first[s];
  int j = -1;
  if (i < n) {
    j = parent[row0 + i];
    if (j >= i || j < 0) j = -1;              // no parent comes later
  }
  uint32_t lo = i < 32 ? 1u << i : 0u, hi = i < 32 ? 0u : 1u << (i - 32);
  int d = j >= 0 ? 1 : 0;
  while (__any(j >= 0)) {
    const int at = max(j, 0);
    const uint32_t l = __shfl(lo, at, 64), h = __shfl(hi, at, 64);
    const int a = __shfl(d, at, 64), k = __shfl(j, at, 64);
    if (j >= 0) {
      lo |= l;
      hi |= h;
      d += a;
      j = k;
    }
  }
  if (i >= n) return;
  if (pos) pos[row0 + i] = first + d;
  if (mask) {
    uint32_t* m = mask + (int64_t)(row0 + i) * W;
#pragma unroll
    for (int w = 0; w < W; ++w) m[w] = w == 0 ? lo : w == 1 ? hi : 0u;
  }
}

}  // namespace
}  // namespace davet

extern "C" int davet_tree_plan(int32_t n_seqs, const int32_t* cu_q,
                               const int32_t* kv_len, const int32_t* first_pos,
                               const int32_t* parent, int32_t* pos, uint32_t* mask,
                               hipStream_t stream) {
  using namespace davet;
  DAVET_CHECK_ARG(n_seqs >= 1 && n_seqs <= DAVET_MAX_SEQS, DAVET_ESHAPE,
                  "davet_tree_plan: n_seqs out of range [1, 64]");
  DAVET_CHECK_ARG(cu_q && (kv_len || first_pos), DAVET_EINVAL,
                  "davet_tree_plan: null pointer");
  DAVET_CHECK_ARG(cu_q[0] == 0, DAVET_ESHAPE, "davet_tree_plan: cu_q[0] must be 0");
  TreePack tp{};
  tp.n_seqs = n_seqs;
  int64_t longest = 0;
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t n = (int64_t)cu_q[s + 1] - cu_q[s];
    DAVET_CHECK_ARG(n >= 0 && n <= DAVET_MAX_TREE, DAVET_ESHAPE,
                    "davet_tree_plan: a sequence has 0 to 256 drafted tokens");
    DAVET_CHECK_ARG(!kv_len || kv_len[s] >= n, DAVET_ESHAPE,
                    "davet_tree_plan: kv_len counts the drafted tokens: it must not be "
                    "below their number");
    DAVET_CHECK_ARG(!first_pos || first_pos[s] <= INT32_MAX - DAVET_MAX_TREE,
                    DAVET_ESHAPE, "davet_tree_plan: first_pos beyond int32");
    longest = std::max(longest, n);
    tp.row0[s + 1] = cu_q[s + 1];
    tp.first[s] = first_pos ? first_pos[s] : (int32_t)(kv_len[s] - n);
  }
  if (cu_q[n_seqs] == 0) return DAVET_OK;
  DAVET_CHECK_ARG(parent && (pos || mask), DAVET_EINVAL,
                  "davet_tree_plan: null pointer");
  DAVET_CHECK_ARG(aligned4({parent, pos, mask}), DAVET_EINVAL,
                  "davet_tree_plan: parent, pos and mask must be 4-byte aligned");
  ProfScope ps(KC_MISC, stream);
  if (longest <= 64)
    hipLaunchKernelGGL(tree_plan_small_kernel, dim3(n_seqs), dim3(64), 0, stream, tp,
                       parent, pos, mask);
  else
    hipLaunchKernelGGL(tree_plan_kernel, dim3(n_seqs), dim3(DAVET_MAX_TREE), 0, stream,
                       tp, parent, pos, mask);
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}

extern "C" int davet_cache_tree_attention(
    const davet_kv_cache* cache, int32_t n_seqs, const int32_t* cu_q,
    const int32_t* kv_len, const void* q, int64_t ld_q, int32_t n_heads, float scale,
    const uint32_t* mask, void* out, int64_t ld_out, float* lse, void* workspace,
    size_t ws_bytes, hipStream_t stream) {
  using namespace davet;
  static const char who[] = "davet_cache_tree_attention";
  CacheView cv;
  ChunkPack cp;
  int64_t total = 0;
  int rc = check_attention(cache, n_seqs, cu_q, kv_len, q, ld_q, n_heads, scale, 0, out,
                           ld_out, lse, workspace, ws_bytes, who, &cv, &cp, &total);
  if (rc) return rc;
  for (int s = 0; s < n_seqs; ++s)
    DAVET_CHECK_ARG(cu_q[s + 1] - cu_q[s] <= DAVET_MAX_TREE, DAVET_ESHAPE,
                    "davet_cache_tree_attention: more than 256 drafted tokens in a "
                    "sequence");
  if (total == 0) return DAVET_OK;
  DAVET_CHECK_ARG(mask, DAVET_EINVAL, "davet_cache_tree_attention: mask is null");
  DAVET_CHECK_ARG(aligned4({mask}), DAVET_EINVAL,
                  "davet_cache_tree_attention: mask must be 4-byte aligned");
  const int D = cache->head_dim;
  const Scale sc = make_scale(scale, D);
  float* part = static_cast<float*>(workspace);
#define ATT(F, DIM)                                                               \
  run_attention<F, DIM, kTree>(cv, cp, q, ld_q, out, ld_out, lse, n_heads, 0, sc, \
                               part, mask, who, stream)
  if (cache->dtype == DAVET_F16) return D == 128 ? ATT(F16S, 128) : ATT(F16S, 64);
  if (cache->dtype == DAVET_BF16) return D == 128 ? ATT(BF16S, 128) : ATT(BF16S, 64);
  return D == 128 ? ATT(F32S, 128) : ATT(F32S, 64);
#undef ATT
}
