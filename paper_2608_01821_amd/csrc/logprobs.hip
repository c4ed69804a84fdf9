// Log probabilities of given tokens, entropy and the top alternatives of rows of
// logits (the kernels of logprobs.h, and the join of a row's slices).

#include "logprobs.h"

namespace davet {
namespace {

// Joins the slices of one row: four wavefronts take every fourth list each.
template <typename F>
__global__ void __launch_bounds__(256)
logprobs_join_kernel(const typename F::st* __restrict__ logits, int64_t ld,
                     int vocab, int exclude, int k,
                     const int32_t* __restrict__ targets, Out out, int slices,
                     const char* __restrict__ part, int rows) {
  __shared__ uint64_t s_list[2][64];
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t* pl = reinterpret_cast<const uint64_t*>(part) +
                       (int64_t)row * slices * k;
  const Stat* ps = reinterpret_cast<const Stat*>(
                       reinterpret_cast<const uint64_t*>(part) +
                       (int64_t)rows * slices * k) + (int64_t)row * slices;
  Stat s = stat_none();
  if (wave == 0 && lane < slices) s = ps[lane];
  uint64_t list = 0;
  if (k > 0) {
    uint64_t other[kMaxSlices / 4];
#pragma unroll
    for (int i = 0; i < kMaxSlices / 4; ++i) {
      const int j = i == 0 ? lane : 63 - lane, sl = wave + 4 * i;
      other[i] = j < k && sl < slices ? pl[(int64_t)sl * k + j] : 0;
    }
    list = other[0];
#pragma unroll
    for (int i = 1; i < kMaxSlices / 4; ++i)
      if (wave + 4 * i < slices) list = list_join(list, other[i]);
  }
  join_waves<4>(list, k, wave, s_list);
  if (wave != 0) return;
  s = stat_wave(s);
  finish<F>(s, list, row, vocab, exclude, k, logits + (int64_t)row * ld, targets, out);
}

// Not monotonic in the rows: r rows of ceil(256 / r) slices each are at most r + 255
// slices, and from 256 rows on there are none.
size_t part_bytes(int rows, int vocab, int k) {
  const int sl = plan_slices(rows, vocab);
  if (sl == 1) return 0;
  return (size_t)rows * sl * ((size_t)k * 8 + sizeof(Stat));
}

}  // namespace
}  // namespace davet

extern "C" int davet_logprobs_workspace_bytes(int32_t rows, int32_t vocab,
                                              int32_t top, size_t* bytes) {
  using namespace davet;
  DAVET_CHECK_ARG(bytes, DAVET_EINVAL,
                  "davet_logprobs_workspace_bytes: bytes is null");
  DAVET_CHECK_ARG(rows >= 1 && rows <= (1 << 22) && vocab >= 1 &&
                      vocab <= (1 << 30) && top >= 0 && top <= DAVET_MAX_TOP,
                  DAVET_ESHAPE, "davet_logprobs_workspace_bytes: out of range");
  *bytes = part_bytes(rows, vocab, top);
  return DAVET_OK;
}

extern "C" int davet_token_logprobs(int32_t rows, int32_t vocab,
                                    const void* logits, int32_t dtype,
                                    int64_t ld, int32_t exclude,
                                    const int32_t* targets, float* logp,
                                    float* entropy, int32_t top, float* top_logp,
                                    int32_t* top_ids, void* workspace,
                                    size_t ws_bytes, hipStream_t stream) {
  using namespace davet;
  DAVET_CHECK_ARG(dtype == DAVET_F32 || is16(dtype), DAVET_EDTYPE,
                  "davet_token_logprobs: dtype must be DAVET_F32, DAVET_BF16 or "
                  "DAVET_F16");
  DAVET_CHECK_ARG(rows >= 0 && rows <= (1 << 22) && vocab >= 1 &&
                      vocab <= (1 << 30) && ld >= vocab,
                  DAVET_ESHAPE,
                  "davet_token_logprobs: rows, vocab or ld out of range");
  DAVET_CHECK_ARG(top >= 0 && top <= DAVET_MAX_TOP, DAVET_ESHAPE,
                  "davet_token_logprobs: top out of range [0, 64]");
  if (rows == 0) return DAVET_OK;
  DAVET_CHECK_ARG(logits && (!logp || targets) && (top == 0 || (top_logp && top_ids)),
                  DAVET_EINVAL, "davet_token_logprobs: null pointer");
  DAVET_CHECK_ARG(((uintptr_t)logits & (dtype_size(dtype) - 1)) == 0, DAVET_EINVAL,
                  "davet_token_logprobs: logits misaligned for their type");
  DAVET_CHECK_ARG(aligned4({targets, logp, entropy, top_logp, top_ids}), DAVET_EINVAL,
                  "davet_token_logprobs: targets and outputs must be 4-byte aligned");
  const int slices = plan_slices(rows, vocab);
  const size_t need = part_bytes(rows, vocab, top);
  DAVET_CHECK_ARG(need == 0 || (workspace && ((uintptr_t)workspace & 255) == 0 &&
                                ws_bytes >= need),
                  DAVET_ENOMEM,
                  "davet_token_logprobs: workspace missing, misaligned or below " +
                      std::to_string(need) + " bytes");
  const Out out{logp, entropy, top_logp, top_ids};
  char* part = static_cast<char*>(workspace);
#define LOGP(F)                                                                \
  do {                                                                         \
    const auto* x = static_cast<const F::st*>(logits);                         \
    if (vocab <= 64 * kWaves * kShort) {                                       \
      ProfScope ps(KC_MISC, stream);                                           \
      hipLaunchKernelGGL((logprobs_short_kernel<F, false>), dim3(rows),        \
                         dim3(64 * kWaves), 0, stream, x, ld, vocab, exclude, top, \
                         targets, out, nullptr, nullptr);                      \
      DAVET_HIP(hipGetLastError());                                            \
      break;                                                                   \
    }                                                                          \
    {                                                                          \
      ProfScope ps(KC_MISC, stream);                                           \
      hipLaunchKernelGGL((logprobs_kernel<F, false>), dim3(rows * slices),     \
                         dim3(64 * kWaves), 0, stream, x, ld, vocab, exclude, top, \
                         targets, out, slices, part, nullptr);                 \
      DAVET_HIP(hipGetLastError());                                            \
    }                                                                          \
    if (slices > 1) {                                                          \
      ProfScope ps(KC_MISC, stream);                                           \
      hipLaunchKernelGGL(logprobs_join_kernel<F>, dim3(rows), dim3(256), 0,    \
                         stream, x, ld, vocab,                                 \
                         exclude, top, targets, out, slices, part, rows);      \
      DAVET_HIP(hipGetLastError());                                            \
    }                                                                          \
  } while (0)
  if (dtype == DAVET_F16) LOGP(F16S);
  else if (dtype == DAVET_BF16) LOGP(BF16S);
  else LOGP(F32S);
#undef LOGP
  return DAVET_OK;
}
