// Rotary positions of rows of heads, by themselves: either pairing, part of the
// head, scaled frequencies, both directions.
//
// Pair i of a head, elements (a, b) = (i, i + dim/2) or (2 i, 2 i + 1), turns by
// t = 2 pi p turns[i] at position p:
//   a' = gain (a cos t - b sin t),  b' = gain (b cos t + a sin t)
// and by -t the other way, which is the transposed map: the gradient.
//
// The whole turns are taken off in float64 by a fused multiply-add, p turns[i] minus its
// nearest whole number, so a far position adds only what the rate itself is off by, up
// to |p| turns[i] 2^-53 turns.  What is left, at most half a turn, goes through the fp32
// sine and cosine, and what its rounding to float took off is added to first order
// (fp32: error 2.5e-8 in the 2-norm, 3.2e-8 without it, in the same time).
//
// A workgroup takes a run of rows: one wavefront computes the dim/2 angles of the next
// row into LDS while the others work on this one's heads, and the next pieces of x are
// on their way meanwhile.
//
// A thread moves vectors of V elements: V is the largest of 8, 4, 2, 1 that divides
// every offset (half the turned part, the rest of the head, the head, the strides,
// the addresses), so any even size works and the usual ones take 16-byte accesses.
//
// Bound by HBM: read once, written once.  Measured: those 3092 rows 13.5 us (4.7 TB/s),
// 4099 fp32 rows of 32 x 80, 32 of each head turned, 16.0 (5.2 TB/s; a large copy
// reaches 5.1); one row 2.4, a launch's latency.  An odd half, stride or address leaves
// one element an access: those 3092 rows in fp16, over and over, take 24 to 26 us in halves
// and 19 in pairs where 16 bytes an access take 11.3 (fp32 24 to 26, 22 and 20.8).

#include <math.h>

#include <algorithm>

#include "cache.h"

namespace davet {
namespace {

constexpr int kMaxWidth = 512, kMaxHalf = kMaxWidth / 2;
constexpr int kMaxThreads = 512;
// Threads of all workgroups, which then take runs of rows.  3092 bf16 rows of 40 x 128,
// half of each head in pairs: 17.7 us with 196,000, 14.5 with twice as many, 13.9 with
// four times, and 13.5 of those in workgroups of 256; one row takes 2.4 in one of 320,
// 2.8 in 192.
constexpr int kMaxInFlight = 2048 * 384, kManyRows = 512;

struct RotaryArgs {
  int rows, rows_per_wg, n_heads, width, half;
  int items;          // of a head: V-vectors (of pairs), then those of its rest
  int64_t ld_x, ld_o;
  float gain;
  int inverse, copy_rest;
};

// V elements as memory holds them
template <typename F, int V>
struct Elems {
  typename F::st e[V];
  __device__ __forceinline__ void load(const typename F::st* p) {
    __builtin_memcpy(e, __builtin_assume_aligned(p, sizeof(e) < 16 ? sizeof(e) : 16),
                     sizeof(e));
  }
  __device__ __forceinline__ void store(typename F::st* p) const {
    __builtin_memcpy(__builtin_assume_aligned(p, sizeof(e) < 16 ? sizeof(e) : 16), e,
                     sizeof(e));
  }
};

// PAIRS: neighbours turn together (V >= 2 of them in a vector, or V = 1: two single
// elements); else elements half apart.
template <typename F, bool PAIRS, int V>
__global__ void __launch_bounds__(kMaxThreads)
rotary_kernel(RotaryArgs ra, const typename F::st* x, typename F::st* out,
              const int32_t* __restrict__ pos, const double* __restrict__ turns) {
  using st = typename F::st;
  using E = Elems<F, V>;
  // a pairs item: two vectors, next to each other only for V = 1
  constexpr bool TWO = !PAIRS || V == 1;
  __shared__ float cs[2][2][kMaxHalf];          // cosines and sines of two rows
  const int r0 = blockIdx.x * ra.rows_per_wg;
  const int r1 = min(r0 + ra.rows_per_wg, ra.rows);
  const int half = ra.half, nt = (int)blockDim.x, total = ra.n_heads * ra.items;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double freq[kMaxHalf / 64];
#pragma unroll
  for (int i = 0; i < kMaxHalf / 64; ++i) {
    const int e = i * 64 + lane;
    freq[i] = i * 64 < half ? turns[min(e, half - 1)] : 0.0;
  }
  auto angles = [&](int r) {
    // one wavefront a row, in turn, so that no other waits for the same one
    if (wave != (r - r0) % (nt >> 6)) return;
    const double p = (double)(pos ? pos[r] : r);
#pragma unroll
    for (int i = 0; i < kMaxHalf / 64; ++i) {
      const int e = i * 64 + lane;
      if (i * 64 >= half) break;
      const double left = fma(p, freq[i], -rint(p * freq[i]));
      const float part = (float)left;
      const float rest = 6.2831853f * (float)(left - (double)part);
      const float s0 = sinpif(2.f * part), c0 = cospif(2.f * part);
      const float si = fmaf(c0, rest, s0);
      if (e < half) {
        cs[(r - r0) & 1][0][e] = ra.gain * fmaf(-s0, rest, c0);
        cs[(r - r0) & 1][1][e] = ra.gain * (ra.inverse ? -si : si);
      }
    }
  };
  // item t of a row: vector j of head h.  HALVES: j < half / V takes elements j V ..
  // and half + j V ..; the others one vector behind the turned part each.  PAIRS: the
  // head's vectors in order.
  const int turned = PAIRS ? ra.items : half / V;
  auto first = [&](int h, int j) {
    if (PAIRS) return h * ra.width + j * (TWO ? 2 : V);
    return h * ra.width + (j < turned ? j * V : half + j * V);
  };
  const int dh = nt / ra.items, dj = nt - dh * ra.items;
  const int h0 = (int)threadIdx.x / ra.items, j0 = (int)threadIdx.x - h0 * ra.items;
  E na, nb;
  // loads of the next item; (nr, nh, nj) is it
  int nr = r0, nh = h0, nj = j0, n_at = threadIdx.x;
  const int second = PAIRS ? 1 : half;
  auto load = [&]() {
    if (nr >= r1 || n_at >= total) return;
    const st* p = x + (int64_t)nr * ra.ld_x + first(nh, nj);
    na.load(p);
    if (TWO && nj < turned) nb.load(p + second);
  };
  auto advance = [&]() {
    n_at += nt;
    nh += dh;
    nj += dj;
    if (nj >= ra.items) { nj -= ra.items; ++nh; }
    if (n_at >= total) { n_at = threadIdx.x; nh = h0; nj = j0; ++nr; }
  };
  load();
  angles(r0);
  for (int r = r0; r < r1; ++r) {
    __syncthreads();
    if (r + 1 < r1) angles(r + 1);
    const float* co = cs[(r - r0) & 1][0];
    const float* si = cs[(r - r0) & 1][1];
    if ((int)threadIdx.x >= total) continue;    // (has no item in any row)
    while (nr == r) {
      E a = na, b = nb;
      const int h = nh, j = nj;
      advance();
      load();
      st* o = out + (int64_t)r * ra.ld_o + first(h, j);
      if constexpr (PAIRS) {
        const int e0 = j * (TWO ? 2 : V);       // element of the head
        if (e0 >= 2 * half && !ra.copy_rest) continue;
        if constexpr (TWO) {
          if (e0 < 2 * half) {
            const float u = F::load(a.e[0]), v = F::load(b.e[0]);
            const float c = co[e0 / 2], s = si[e0 / 2];
            a.e[0] = F::store(u * c - v * s);
            b.e[0] = F::store(v * c + u * s);
          }
          a.store(o);
          b.store(o + 1);
        } else {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const int i = e0 / 2 + e / 2;
            if (i >= half) break;
            const float u = F::load(a.e[e]), v = F::load(a.e[e + 1]);
            const float c = co[i], s = si[i];
            a.e[e] = F::store(u * c - v * s);
            a.e[e + 1] = F::store(v * c + u * s);
          }
          a.store(o);
        }
      } else if (j < turned) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float u = F::load(a.e[e]), v = F::load(b.e[e]);
          const float c = co[j * V + e], s = si[j * V + e];
          a.e[e] = F::store(u * c - v * s);
          b.e[e] = F::store(v * c + u * s);
        }
        a.store(o);
        b.store(o + half);
      } else if (ra.copy_rest) {
        a.store(o);
      }
    }
  }
}

// Elements a vector: the largest power of two up to 8 that divides all of these.
int vector_of(std::initializer_list<int64_t> ns) {
  int64_t x = 8;
  for (int64_t n : ns) x |= n;
  return (int)(x & -x);
}

template <typename F>
int launch_rotary(RotaryArgs ra, bool pairs, const void* x_, void* out_,
                  const int32_t* pos, const double* turns, hipStream_t stream) {
  using st = typename F::st;
  const st* x = (const st*)x_;
  st* out = (st*)out_;
  const int64_t ax = (int64_t)((uintptr_t)x / sizeof(st)),
                ao = (int64_t)((uintptr_t)out / sizeof(st));
  // (strides of one row mean nothing)
  const int64_t lx = ra.rows > 1 ? ra.ld_x : 0, lo = ra.rows > 1 ? ra.ld_o : 0;
  const int V = pairs ? vector_of({ra.width, lx, lo, ax, ao})
                      : vector_of({ra.half, ra.width, lx, lo, ax, ao});
  ra.items = pairs ? ra.width / std::max(V, 2)
                   : ra.half / V + (ra.width - 2 * ra.half) / V;
  const int total = ra.n_heads * ra.items;
  const int most = ra.rows < kManyRows ? kMaxThreads : kMaxThreads / 2;
  const int passes = (total + most - 1) / most;
  const int threads = (int)align_up((total + passes - 1) / passes, 64);
  const int groups = kMaxInFlight / threads;
  ra.rows_per_wg = (int)(((int64_t)ra.rows + groups - 1) / groups);
  const int grid = (int)(((int64_t)ra.rows + ra.rows_per_wg - 1) / ra.rows_per_wg);
  ProfScope ps(KC_MISC, stream);
#define ROTARY(P, VV)                                                          \
  hipLaunchKernelGGL((rotary_kernel<F, P, VV>), dim3(grid), dim3(threads), 0,  \
                     stream, ra, x, out, pos, turns)
#define ROTARY_V(P)                                                            \
  do {                                                                         \
    if (V == 8) ROTARY(P, 8);                                                  \
    else if (V == 4) ROTARY(P, 4);                                             \
    else if (V == 2) ROTARY(P, 2);                                             \
    else ROTARY(P, 1);                                                         \
  } while (0)
  if (pairs) ROTARY_V(true);
  else ROTARY_V(false);
#undef ROTARY_V
#undef ROTARY
  DAVET_HIP(hipGetLastError());
  return DAVET_OK;
}

}  // namespace
}  // namespace davet

extern "C" int davet_rotary_turns(int32_t dim, double theta, int32_t scaling,
                                  double factor, double trained, double fast,
                                  double slow, double* turns) {
  using namespace davet;
  DAVET_CHECK_ARG(turns, DAVET_EINVAL, "davet_rotary_turns: turns is null");
  DAVET_CHECK_ARG(dim >= 2 && dim <= kMaxWidth && dim % 2 == 0, DAVET_ESHAPE,
                  "davet_rotary_turns: dim must be even, 2 .. 512");
  DAVET_CHECK_ARG(scaling >= DAVET_ROTARY_PLAIN && scaling <= DAVET_ROTARY_RAMP,
                  DAVET_EINVAL, "davet_rotary_turns: no such scaling");
  DAVET_CHECK_ARG(theta >= 1.0 && std::isfinite(theta) &&
                      (scaling == DAVET_ROTARY_PLAIN ||
                       (factor >= 1.0 && std::isfinite(factor))),
                  DAVET_EINVAL,
                  "davet_rotary_turns: theta >= 1 and factor >= 1 required, finite");
  DAVET_CHECK_ARG(scaling != DAVET_ROTARY_RAMP ||
                      (trained > 0.0 && std::isfinite(trained) && slow >= 0.0 &&
                       fast > slow && std::isfinite(fast)),
                  DAVET_EINVAL,
                  "davet_rotary_turns: the ramp needs trained > 0 and "
                  "fast > slow >= 0, finite");
  const double two_pi = 6.283185307179586476925;
  for (int i = 0; i < dim / 2; ++i) {
    double f = pow(theta, -2.0 * i / dim);
    if (scaling == DAVET_ROTARY_LINEAR) {
      f /= factor;
    } else if (scaling == DAVET_ROTARY_BASE && dim > 2) {
      f *= pow(factor, -2.0 * i / (dim - 2));
    } else if (scaling == DAVET_ROTARY_RAMP) {
      const double r = (trained * f / two_pi - slow) / (fast - slow);
      const double keep = std::min(1.0, std::max(0.0, r));
      f = keep * f + (1.0 - keep) * (f / factor);
    }
    turns[i] = f / two_pi;
  }
  return DAVET_OK;
}

extern "C" int davet_rotary(int32_t rows, int32_t n_heads, int32_t head_dim,
                            int32_t dim, int32_t layout, const void* x,
                            int64_t ld_x, void* out, int64_t ld_out, int32_t dtype,
                            const int32_t* pos, const double* turns, float gain,
                            int32_t inverse, hipStream_t stream) {
  using namespace davet;
  DAVET_CHECK_ARG(dtype == DAVET_F32 || is16(dtype), DAVET_EDTYPE,
                  "davet_rotary: dtype must be DAVET_F32, DAVET_BF16 or DAVET_F16");
  DAVET_CHECK_ARG(layout == DAVET_ROTARY_HALVES || layout == DAVET_ROTARY_PAIRS,
                  DAVET_EINVAL, "davet_rotary: no such layout");
  DAVET_CHECK_ARG(inverse == 0 || inverse == 1, DAVET_EINVAL,
                  "davet_rotary: inverse must be 0 or 1");
  DAVET_CHECK_ARG(std::isfinite(gain), DAVET_EINVAL,
                  "davet_rotary: gain must be finite");
  DAVET_CHECK_ARG(rows >= 0 && rows <= (1 << 24) && n_heads >= 1 && n_heads <= 4096 &&
                      head_dim >= 2 && head_dim <= kMaxWidth && head_dim % 2 == 0 &&
                      dim >= 2 && dim <= head_dim && dim % 2 == 0,
                  DAVET_ESHAPE,
                  "davet_rotary: rows up to 2^24, n_heads in [1, 4096], head_dim "
                  "even in [2, 512], dim even in [2, head_dim]");
  const int64_t width = (int64_t)n_heads * head_dim;
  DAVET_CHECK_ARG(rows <= 1 || (ld_x >= width && ld_x < (1ll << 31) &&
                                ld_out >= width && ld_out < (1ll << 31)),
                  DAVET_ESHAPE, "davet_rotary: row stride below the row's width");
  if (rows == 0) return DAVET_OK;
  const size_t es = dtype_size(dtype);
  DAVET_CHECK_ARG(x && out && turns, DAVET_EINVAL, "davet_rotary: null pointer");
  DAVET_CHECK_ARG((((uintptr_t)x | (uintptr_t)out) & (es - 1)) == 0 &&
                      ((uintptr_t)turns & 7) == 0 && aligned4({pos}),
                  DAVET_EINVAL,
                  "davet_rotary: x, out, turns and pos must be aligned to their "
                  "elements");
  if (rows == 1) ld_x = ld_out = width;
  const bool in_place = out == x && ld_out == ld_x;
  DAVET_CHECK_ARG(in_place ||
                      !rows_overlap(out, ld_out, width, x, ld_x, width, rows, es),
                  DAVET_EINVAL,
                  "davet_rotary: out overlaps x (in place needs the same address and, "
                  "of several rows, stride)");
  RotaryArgs ra{};
  ra.rows = rows;
  ra.n_heads = n_heads;
  ra.width = head_dim;
  ra.half = dim / 2;
  ra.ld_x = ld_x;
  ra.ld_o = ld_out;
  ra.gain = gain;
  ra.inverse = inverse;
  ra.copy_rest = !in_place;
  const bool pairs = layout == DAVET_ROTARY_PAIRS;
  if (dtype == DAVET_F16)
    return launch_rotary<F16S>(ra, pairs, x, out, pos, turns, stream);
  if (dtype == DAVET_BF16)
    return launch_rotary<BF16S>(ra, pairs, x, out, pos, turns, stream);
  return launch_rotary<F32S>(ra, pairs, x, out, pos, turns, stream);
}
