// Rotary positions with several axes: pair i of a row's d / 2 channel pairs turns by pos[axis(i)] * freq(i) radians,
//   y0 = x0 cos - x1 sin,  y1 = x0 sin + x1 cos,
// Q and K of a token in one launch, optionally in the order of a permutation (a token's row is read where the projection left it and
// written where the attention wants it); inverse: the same with the angle's sign and the two sides exchanged, which is also the gradient.
//
// Bound by HBM: every row is read and written once, 16 bytes a lane and access.  A thread keeps one place in the row for a run of heads, so
// that the sines and cosines of a token, the only arithmetic worth counting, are made once for several rows (in registers, never in memory).
#include "psa_dev.h"
#include "psa_internal.h"

namespace psa {

struct RotaryArgs {
  int N, Hq, Hkv, heads, groups, per_group;   // heads = Hq + Hkv; groups of per_group of them (the last may be short)
  uint32_t rows;                              // B * groups * N
  int once;                                   // the inputs do not fit the memory-side cache
  int64_t pos_stride;
  Strides q, k;                               // the projections' side
  double quarters[ROTARY_PAIRS];              // quarter turns a position
  uint8_t axis[ROTARY_PAIRS];                 // 255: the pair is not turned
};

// Cosine and sine of pos * quarters quarter turns.  The whole quarters and what is left over in 64 bits (position 10^6 on the fastest channel is 6 10^5 quarters, of which 32 bits
// would keep 1/16): at 1.5 2^52 a sum is rounded to a whole number, whose last bits it holds (|pos * quarters| < 2^51).  Then Taylor's series on +- pi / 4: the
// first terms left out are below 2^-29.
__device__ __forceinline__ void cos_sin(double quarters, int pos, float& c, float& s) {
  constexpr double WHOLE = 6755399441055744.0;
  const double turned = fma(quarters, (double)pos, WHOLE), whole = turned - WHOLE;
  const int n = (int)(__double_as_longlong(turned) & 3);
  const float a = (float)fma(quarters, (double)pos, -whole) * 1.57079632679489661923f, a2 = a * a;
  const float sn = fmaf(a * a2, fmaf(a2, fmaf(a2, fmaf(a2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), a);
  const float cs = fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  c = n & 1 ? sn : cs;
  s = n & 1 ? cs : sn;
  if (n == 1 || n == 2) c = -c;
  if (n >= 2) s = -s;
}

// 16 bytes at any element's address.  Stores are non-temporal, so that what is written does not push out of the memory-side cache (256 MB) what a projection left
// there; loads are where the inputs do not fit it (12 + 12 heads x 32760 tokens, 201 MB, permuted, us, inputs in the cache / in memory: neither - / 80.7, stores
// 62 / 75, both 73 / 73.6; 1.5 GB, inverse: 580 -> 572).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
template <bool ONCE, typename T> __device__ __forceinline__ u32x4 load16(const T* p) {
  const u32x4_any* q = reinterpret_cast<const u32x4_any*>(p);
  if constexpr (ONCE) return __builtin_nontemporal_load(q);
  else return *q;
}
template <typename T> __device__ __forceinline__ void store16(T* p, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(p)); }

// HALVES: pair i is channels i, i + d / 2, and a thread has a chunk of each half; otherwise channels 2i, 2i + 1 and one chunk.
template <typename T, int D, bool HALVES, bool INVERSE>
__global__ __launch_bounds__(256) void rotary_kernel(const T* __restrict__ Qin, const T* __restrict__ Kin, T* __restrict__ Qout, T* __restrict__ Kout,
                                                     const int32_t* __restrict__ pos, const int32_t* __restrict__ perm, RotaryArgs a) {
  constexpr int VEC = Elem<T>::VEC, PAIRS = HALVES ? VEC : VEC / 2, LANES = D / 2 / PAIRS, AHEAD = HALVES ? 2 : 4;
  const int c = threadIdx.x % LANES;
  const uint32_t row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (row >= a.rows) return;
  const uint32_t bg = row / (uint32_t)a.N;
  const int k = (int)(row - bg * (uint32_t)a.N), b = (int)(bg / (uint32_t)a.groups), h0 = (int)(bg % (uint32_t)a.groups) * a.per_group;
  const int h1 = h0 + a.per_group < a.heads ? h0 + a.per_group : a.heads;
  int t = k;
  if (perm) {
    t = perm[k];
    if ((uint32_t)t >= (uint32_t)a.N) return;
  }
  const int first = c * VEC, second = D / 2 + c * VEC;
  const int64_t tight_q = (int64_t)b * a.Hq * a.N + k, tight_k = (int64_t)b * a.Hkv * a.N + k;
  const int64_t loose_q = b * a.q.b + t * a.q.n, loose_k = b * a.k.b + t * a.k.n;
  auto place = [&](int h, const T*& src, T*& dst) __attribute__((always_inline)) {
    const bool is_q = h < a.Hq;
    const int hh = is_q ? h : h - a.Hq;
    const int64_t tight = ((is_q ? tight_q : tight_k) + (int64_t)hh * a.N) * D, loose = is_q ? loose_q + hh * a.q.h : loose_k + hh * a.k.h;
    src = (is_q ? Qin : Kin) + (INVERSE ? tight : loose);
    dst = (is_q ? Qout : Kout) + (INVERSE ? loose : tight);
  };
  u32x4 v[AHEAD][HALVES ? 2 : 1];
  T* dst[AHEAD];
  auto load_as = [&](auto once, int h) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const T* src;
      place(h + u < h1 ? h + u : h1 - 1, src, dst[u]);
      v[u][0] = load16<decltype(once)::value>(src + first);
      if (HALVES) v[u][HALVES ? 1 : 0] = load16<decltype(once)::value>(src + second);
    }
  };
  auto load = [&](int h) __attribute__((always_inline)) {
    if (a.once) load_as(std::integral_constant<bool, true>{}, h);
    else load_as(std::integral_constant<bool, false>{}, h);
  };
  // The angles are worked out while the first rows are on their way: what they need is requested before (12 + 12 heads x 32760 tokens 84 -> 75 us; inverse
  // calls, whose scattered side is the written one, gain nothing and lose 2 % of the largest pass).
  int at[PAIRS];
  double quarters[PAIRS];
  uint32_t still = 0u;
#pragma unroll
  for (int u = 0; u < PAIRS; ++u) {
    const int ax = a.axis[c * PAIRS + u];
    still |= (uint32_t)(ax == 255) << u;
    quarters[u] = a.quarters[c * PAIRS + u];
    at[u] = pos[b * a.pos_stride + (int64_t)(ax == 255 ? 0 : ax) * a.N + t];
  }
  if (!INVERSE) load(h0);
  float cs[PAIRS], sn[PAIRS];
#pragma unroll
  for (int u = 0; u < PAIRS; ++u) {
    cos_sin(quarters[u], at[u], cs[u], sn[u]);
    if (INVERSE) sn[u] = -sn[u];
  }
  for (int h = h0; h < h1; h += AHEAD) {
    if (INVERSE || h > h0) load(h);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (h + u >= h1) break;
      float x[HALVES ? 2 : 1][VEC];
      Elem<T>::widen(v[u][0], x[0]);
      if (HALVES) Elem<T>::widen(v[u][HALVES ? 1 : 0], x[HALVES ? 1 : 0]);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        float& x0 = HALVES ? x[0][i] : x[0][2 * i % VEC];
        float& x1 = HALVES ? x[HALVES ? 1 : 0][i] : x[0][(2 * i + 1) % VEC];
        const float y0 = fmaf(x0, cs[i], -(x1 * sn[i])), y1 = fmaf(x0, sn[i], x1 * cs[i]);
        if (!(still >> i & 1u)) {          // (a pair that is not turned keeps its bits, also where one of it is not finite)
          x0 = y0;
          x1 = y1;
        }
      }
      store16(dst[u] + first, Elem<T>::pack(x[0]));
      if (HALVES) store16(dst[u] + second, Elem<T>::pack(x[HALVES ? 1 : 0]));
    }
  }
}

template <typename T, int D>
static void launch_rotary_t(RotaryArgs& a, int B, bool halves, bool inverse, const void* Qin, const void* Kin, void* Qout, void* Kout, const int32_t* pos,
                            const int32_t* perm, hipStream_t s) {
  const int lanes = D / 2 / (halves ? Elem<T>::VEC : Elem<T>::VEC / 2), per_block = 256 / lanes;
  // Heads a thread: as many as leave four workgroups to a compute unit, at most 4 (us at 2 / 4 / 8: 12 + 12 heads x 32760 tokens 93 / 75 / 76, the largest pass 631 / 580 / 598).
  const int64_t all = (int64_t)B * a.heads * a.N / per_block;
  int per = 1;
  while (per < 4 && per < a.heads && all / (2 * per) >= 1024) per *= 2;
  a.per_group = per;
  a.groups = (a.heads + per - 1) / per;
  a.rows = (uint32_t)((int64_t)B * a.groups * a.N);
  a.once = (int64_t)B * a.heads * a.N * D * (int64_t)sizeof(T) > ((int64_t)256 << 20);
  const unsigned grid = (unsigned)((a.rows + (int64_t)per_block - 1) / per_block);
  auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, s>>>(static_cast<const T*>(Qin), static_cast<const T*>(Kin), static_cast<T*>(Qout), static_cast<T*>(Kout), pos, perm, a);
  };
  if (halves) inverse ? go(rotary_kernel<T, D, true, true>) : go(rotary_kernel<T, D, true, false>);
  else inverse ? go(rotary_kernel<T, D, false, true>) : go(rotary_kernel<T, D, false, false>);
}

hipError_t launch_rotary(const Plan& pl, const psa_rotary_spec& r, int Hq, int Hkv, const Strides& q, const Strides& k, const int32_t* pos, int64_t pos_stride,
                         const int32_t* perm, bool inverse, const void* Qin, const void* Kin, void* Qout, void* Kout, hipStream_t s) {
  RotaryArgs a;
  a.N = pl.N; a.Hq = Hq; a.Hkv = Hkv; a.heads = Hq + Hkv; a.pos_stride = pos_stride; a.q = q; a.k = k;
  for (int i = 0; i < ROTARY_PAIRS; ++i) {
    a.axis[i] = i < pl.d / 2 ? r.axis[i] : 255;
    a.quarters[i] = a.axis[i] != 255 ? r.freq[i] * 0.63661977236758134308 : 0.0;   // 2 / pi
  }
  const bool halves = r.pairing == PSA_ROTARY_HALVES;
  if (pl.dtype == PSA_BF16) {
    if (pl.d == 128) launch_rotary_t<bf16_t, 128>(a, pl.B, halves, inverse, Qin, Kin, Qout, Kout, pos, perm, s);
    else launch_rotary_t<bf16_t, 64>(a, pl.B, halves, inverse, Qin, Kin, Qout, Kout, pos, perm, s);
  } else {
    if (pl.d == 128) launch_rotary_t<float, 128>(a, pl.B, halves, inverse, Qin, Kin, Qout, Kout, pos, perm, s);
    else launch_rotary_t<float, 64>(a, pl.B, halves, inverse, Qin, Kin, Qout, Kout, pos, perm, s);
  }
  return hipGetLastError();
}

// Axis and frequency of every pair: axis 0's pairs first, then axis 1's; what is left over is not turned.
void rotary_spectrum_host(int d, int axes, const int32_t* pairs, double base, bool shared, psa_rotary_spec* r) {
  int i = 0;
  for (int ax = 0; ax < axes; ++ax)
    for (int j = 0; j < pairs[ax]; ++j, ++i) {
      r->axis[i] = (uint8_t)ax;
      r->freq[i] = pow(base, shared ? -(double)i / (d / 2) : -(double)j / pairs[ax]);
    }
  for (; i < ROTARY_PAIRS; ++i) {
    r->axis[i] = PSA_ROTARY_STILL;
    r->freq[i] = 0.0;
  }
  r->axes = axes;
}

}  // namespace psa
