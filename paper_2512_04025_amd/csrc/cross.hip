// Cross attention: N query tokens a head against M encoder states, of which batch entry b shows those with j < kv_len[b] and
// key_mask[b, j] != 0.  With s_j = scale q.k_j:  P = softmax over the states that are seen, O = P V, lse = log sum exp(s).  Backward, with
// P = exp(s - lse), D = dO.O, dP = dO V^T, dS = P (dP - D):  dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.
//
// The kernels of a type are in cross_bf16.hip and cross_f32.hip (what they share: cross_dev.h); here are those that add up partial results and the rules by which the
// host shares the work.  Query rows stay in registers and tiles of states come by (forward, dQ), or states stay and tiles of query rows come by (dK, dV).  The query
// heads of a key head are rows of one matrix where that fills tiles better (cross_flat; merge_heads in api.hip).
// No atomics: sums over workgroups are written as partial results and added in a fixed order.
#include "cross_dev.h"

namespace psa {

// Rows of a part each -> the row: O = sum w O_part / sum w, w = exp(lse_part - their maximum).  Eight parts' loads at a time: the kernel is latency.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_join_kernel(const float* __restrict__ Opart, const float* __restrict__ stats, T* __restrict__ O, float* __restrict__ lse, CrossArgs a) {
  constexpr int LANES = D / 4, AHEAD = 8;
  const int64_t total = (int64_t)a.B * a.Hkv * a.rows, x = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (x >= total) return;
  const int c = threadIdx.x % LANES;
  // One pass with the running maximum of a softmax, a batch at a time
  float top = -INFINITY, weight = 0.f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.parts; s0 += AHEAD) {
    float l[AHEAD];
    f32x4 o[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int s = s0 + u < a.parts ? s0 + u : a.parts - 1;
      l[u] = stats[s * total + x];
      o[u] = *reinterpret_cast<const f32x4*>(Opart + (s * total + x) * D + c * 4);
    }
    float most = top;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) most = fmaxf(most, l[u]);
    const float base = most == -INFINITY ? 0.f : most;      // (parts that see nothing have weight 0, one that is not a number spoils the row)
    const float keep = __builtin_amdgcn_exp2f((top - base) * CROSS_LOG2E);
    weight *= keep;
    sum *= keep;
    top = most;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const float w = __builtin_amdgcn_exp2f((l[u] - base) * CROSS_LOG2E);
      if (s0 + u < a.parts) {
        weight += w;
        sum += o[u] * w;
      }
    }
  }
  const float inv = weight == 0.f ? 0.f : 1.f / weight;
  const int bh = (int)(x / a.rows), row = (int)(x - (int64_t)bh * a.rows), b = bh / a.Hkv, hk = bh % a.Hkv;
  const CrossRow r = cross_row(a, row);
  Four<T>::store(O + b * a.o.b + (int64_t)(hk * a.group + r.g) * a.o.h + r.n * a.o.n + c * 4, sum * inv);
  if (lse && c == 0) lse[((int64_t)b * a.Hq + hk * a.group) * a.N + row] = weight == 0.f ? -INFINITY : top + log2f(weight) * CROSS_LN2;
}

// out[b, h, l, :] = factor * sum over the parts, in their order; up to three tensors in one launch (blockIdx.y)
template <typename T> struct CrossSum {
  struct One {
    const float* part;
    T* out;
    int64_t rows;
    Strides to;
    int H, L, parts;
    float factor;
  } of[3];
};
template <typename T, int D> __global__ __launch_bounds__(256) void cross_sum_kernel(CrossSum<T> p) {
  constexpr int LANES = D / 4, AHEAD = 8;
  const auto& o = p.of[blockIdx.y];
  const int64_t x = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (x >= o.rows) return;
  const int c = threadIdx.x % LANES;
  const float* part = o.part + x * D + c * 4;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < o.parts; s0 += AHEAD) {
    f32x4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) v[u] = *reinterpret_cast<const f32x4*>(part + (s0 + u < o.parts ? s0 + u : o.parts - 1) * o.rows * D);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u < o.parts) sum += v[u];
  }
  const int64_t bh = x / o.L;
  Four<T>::store(o.out + bh / o.H * o.to.b + bh % o.H * o.to.h + (x - bh * o.L) * o.to.n + c * 4, sum * o.factor);
}

// ---- host

// Wavefronts of a workgroup by the rows that a key head has: no more than have rows.
static int cross_waves(const Plan& pl) {
  const int64_t rows = (int64_t)pl.group * pl.N;
  return rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
}
// Blocks of rows that hold rows of several heads: float32; bfloat16, whose rows of one head are addressed as one range, only where heads are so short that their last blocks, partly empty, would cost an eighth of the work.
static bool cross_flat(const Plan& pl) {
  if (pl.dtype != PSA_BF16) return true;
  const int64_t per = cross_waves(pl) * 32;
  return pl.group > 1 && (pl.N + per - 1) / per * per * 8 > (int64_t)pl.N * 9;
}
static int cross_tile(const Plan& pl) { return pl.dtype == PSA_BF16 ? cross_keys<bf16_t>() : cross_keys<float>(); }

// How many workgroups share the tiles of a block (the keys of a block of rows, the rows of a block of keys), each leaving a partial result that is read and added up by
// another kernel.  The number that is expected to take least: with w workgroups on a compute unit a tile takes them w * busy, but no less than `lone`, a
// workgroup costs `start` besides (as many as fit at one time: once), and the parts cost what they move and 5 us for the launch.
struct CrossCost { double busy, lone, start; int fit; };                 // us
static int cross_parts(int64_t blocks, int64_t tiles, const CrossCost& c, double part_bytes) {
  int best = 1;
  double least = 0.0;
  for (int64_t p = 1; p <= 128 && p <= (tiles > 1 ? tiles : 1); ++p) {
    if (p > 1 && c.lone + c.start + 5.0 + (double)p * part_bytes / 1.75e6 >= least) break;      // more parts take longer than the best
    const int64_t w = (blocks * p + 255) / 256, each = (tiles + p - 1) / p;
    const double us = (double)each * (w * c.busy > c.lone ? w * c.busy : c.lone) + (double)((w + c.fit - 1) / c.fit) * c.start + (p > 1 ? 5.0 + (double)p * part_bytes / 1.75e6 : 0.0);
    if (p == 1 || us < least) {
      least = us;
      best = (int)p;
    }
  }
  return best;
}
// Measured: bfloat16, us of a tile of 64 with the chip full and for a workgroup alone; float32: the rate of its matrix instructions (0.98 us of 32 x 32 x 64 on a SIMD).
int cross_key_parts(const Plan& pl, int M, bool gradient) {
  const int nw = cross_waves(pl);
  const int64_t per = nw * 32, blocks = (cross_flat(pl) ? ((int64_t)pl.group * pl.N + per - 1) / per : pl.group * ((pl.N + per - 1) / per)) * pl.B * pl.Hkv;
  const int64_t tiles = ((int64_t)M + cross_tile(pl) - 1) / cross_tile(pl);
  CrossCost c;
  if (pl.dtype == PSA_BF16) {
    if (pl.d == 128) c = gradient ? CrossCost{1.35, 2.0, 5.0, 2} : CrossCost{0.9, 1.3, 4.0, 2};
    else c = gradient ? CrossCost{0.75, 1.4, 5.0, 2} : CrossCost{0.47, 1.0, 4.0, nw == 4 ? 3 : 5};
    c.busy *= nw / 4.0;
  } else {
    const double us = (gradient ? 3 : 2) * (pl.d == 128 ? 1.96 : 0.98);
    c = CrossCost{us * nw / 4.0, us, 4.0, pl.d == 128 ? (gradient ? 1 : 2) : (gradient ? 2 : 4)};
  }
  return cross_parts(blocks, tiles, c, 4.0 * pl.B * pl.Hq * (double)pl.N * pl.d);
}
int cross_row_parts(const Plan& pl, int M) {
  const int64_t blocks = ((int64_t)M + 127) / 128 * pl.B * pl.Hkv, tiles = (int64_t)pl.group * ((pl.N + cross_tile(pl) - 1) / cross_tile(pl));
  if (blocks == 0) return 1;
  CrossCost c;
  if (pl.dtype == PSA_BF16) c = pl.d == 128 ? CrossCost{1.5, 2.2, 5.0, 2} : CrossCost{0.8, 1.5, 5.0, 3};
  else c = pl.d == 128 ? CrossCost{7.8, 7.8, 5.0, 1} : CrossCost{3.9, 3.9, 5.0, 2};
  return cross_parts(blocks, tiles, c, 8.0 * pl.B * pl.Hkv * (double)M * pl.d);
}

static CrossArgs cross_args(const Plan& pl, const CrossCall& c) {
  CrossArgs a;
  a.B = pl.B; a.Hq = pl.Hq; a.Hkv = pl.Hkv; a.group = pl.group; a.N = pl.N; a.M = c.M; a.rows = pl.group * pl.N;
  a.scale = pl.scale; a.scale_log2 = pl.scale * CROSS_LOG2E;
  a.q = c.q; a.k = c.k; a.v = c.v; a.o = c.o; a.gq = c.gq; a.gk = c.gk; a.gv = c.gv; a.go = c.go;
  a.kv_len = c.kv_len; a.mask = c.key_mask;
  a.chunks = (pl.N + cross_tile(pl) - 1) / cross_tile(pl);
  a.flat = cross_flat(pl);
  a.once = a.parts = a.tiles_per_part = 0;
  return a;
}
static void cross_share(CrossArgs& a, int parts, int tiles) {
  a.parts = parts;
  a.tiles_per_part = parts > 0 ? (tiles + parts - 1) / parts : tiles;
}

static dim3 cross_row_grid(const Plan& pl, const CrossArgs& a, int nw) {
  return dim3((unsigned)(a.flat ? (a.rows + nw * 32 - 1) / (nw * 32) : pl.group * ((pl.N + nw * 32 - 1) / (nw * 32))), (unsigned)(pl.B * pl.Hkv), (unsigned)a.parts);
}
static unsigned cross_rows_of_256(int64_t rows, int d) { return (unsigned)((rows + 1024 / d - 1) / (1024 / d)); }      // four channels a thread

template <typename T>
static void launch_cross_fwd_t(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, void* O, float* lse, float* part, float* stats, hipStream_t s) {
  CrossArgs a = cross_args(pl, c);
  const int nw = cross_waves(pl);
  cross_share(a, c.key_parts, (c.M + cross_keys<T>() - 1) / cross_keys<T>());
  const bool split = a.parts > 1;
  const dim3 grid = cross_row_grid(pl, a, nw);
  // Keys, values and partial results that do not fit the memory-side cache (256 MB) together: reading them past it costs what is still there and saves the writing back.  2 x 16 heads
  // x 64 rows, d = 64, us with / without, states last used long ago: 134 MB 39 / 43, 268 MB 64 / 71, 402 MB 87 / 93; just used: 40 / 34, 64 / 57, 87 / 93.
  // (Not in the backward call, whose kernels both read keys and values: 8190 states 52 / 46.)
  a.once = grid.x == 1 && pl.esize * 2 * (int64_t)pl.B * pl.Hkv * c.M * pl.d + 4 * (int64_t)a.parts * pl.B * pl.Hq * pl.N * pl.d > ((int64_t)256 << 20);
  T* o = static_cast<T*>(O);
  cross_fwd(a, pl.d, grid, nw, split, static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V), o, split ? stats : lse, part, s);
  if (!split) return;
  const unsigned blocks = cross_rows_of_256((int64_t)pl.B * pl.Hq * pl.N, pl.d);
  if (pl.d == 128) cross_join_kernel<T, 128><<<blocks, 256, 0, s>>>(part, stats, o, lse, a);
  else cross_join_kernel<T, 64><<<blocks, 256, 0, s>>>(part, stats, o, lse, a);
}

hipError_t launch_cross_fwd(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, void* O, float* lse, float* part, float* stats, hipStream_t s) {
  if (pl.dtype == PSA_BF16) launch_cross_fwd_t<bf16_t>(pl, c, Q, K, V, O, lse, part, stats, s);
  else launch_cross_fwd_t<float>(pl, c, Q, K, V, O, lse, part, stats, s);
  return hipGetLastError();
}

template <typename T>
static void launch_cross_bwd_t(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, const void* O, const float* lse, const void* dO, void* dQ, void* dK,
                               void* dV, float* Dr, float* dQpart, float* dKpart, float* dVpart, hipStream_t s) {
  CrossArgs a = cross_args(pl, c);
  const T *q = static_cast<const T*>(Q), *k = static_cast<const T*>(K), *v = static_cast<const T*>(V), *o = static_cast<const T*>(O), *g = static_cast<const T*>(dO);
  T *gq = static_cast<T*>(dQ), *gk = static_cast<T*>(dK), *gv = static_cast<T*>(dV);
  const int nw = cross_waves(pl);
  CrossSum<T> sums;
  int tensors = 0;
  int64_t most = 0;
  auto add = [&](const float* part, T* out, int H, int L, const Strides& to, float factor) {
    const int64_t rows = (int64_t)pl.B * H * L;
    sums.of[tensors++] = {part, out, rows, to, H, L, a.parts, factor};
    if (rows > most) most = rows;
  };
  cross_share(a, c.key_parts, (c.M + cross_keys<T>() - 1) / cross_keys<T>());
  cross_dq(a, pl.d, cross_row_grid(pl, a, nw), nw, a.parts > 1, q, k, v, o, lse, g, Dr, gq, dQpart, s);
  if (a.parts > 1) add(dQpart, gq, pl.Hq, pl.N, c.gq, pl.scale);
  if (c.M > 0) {
    cross_share(a, c.row_parts, pl.group * a.chunks);
    cross_dkv(a, pl.d, dim3((unsigned)((c.M + 127) / 128), (unsigned)(pl.B * pl.Hkv), (unsigned)a.parts), a.parts > 1, q, k, v, Dr, g, gk, gv, dKpart, dVpart, s);
    if (a.parts > 1) {
      add(dKpart, gk, pl.Hkv, c.M, c.gk, pl.scale);
      add(dVpart, gv, pl.Hkv, c.M, c.gv, 1.f);
    }
  }
  if (tensors == 0) return;
  for (int i = tensors; i < 3; ++i) sums.of[i] = sums.of[0];
  const dim3 grid(cross_rows_of_256(most, pl.d), (unsigned)tensors);
  if (pl.d == 128) cross_sum_kernel<T, 128><<<grid, 256, 0, s>>>(sums);
  else cross_sum_kernel<T, 64><<<grid, 256, 0, s>>>(sums);
}

hipError_t launch_cross_bwd(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, const void* O, const float* lse, const void* dO, void* dQ, void* dK,
                            void* dV, float* Dr, float* dQpart, float* dKpart, float* dVpart, hipStream_t s) {
  if (pl.dtype == PSA_BF16) launch_cross_bwd_t<bf16_t>(pl, c, Q, K, V, O, lse, dO, dQ, dK, dV, Dr, dQpart, dKpart, dVpart, s);
  else launch_cross_bwd_t<float>(pl, c, Q, K, V, O, lse, dO, dQ, dK, dV, Dr, dQpart, dKpart, dVpart, s);
  return hipGetLastError();
}

}  // namespace psa
