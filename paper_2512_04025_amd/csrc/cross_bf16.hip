// Cross attention and its gradients (see cross.hip), bfloat16: the order of a tile fixed by hand.
#include "cross_dev.h"

namespace psa {

// Forward.  A step makes the scores of tile t + 1 and the second product of tile t, and every MFMA is
// followed by a slice of the vector work (exponentials of tile t, maximum of tile t + 1), about one weight a lane per MFMA, so that
// one wavefront keeps both pipes busy; K is loaded a tile further ahead than V.
template <int D, int NW, bool PART>
__global__ __launch_bounds__(NW * 64, D == 64 ? 3 : 2) void cross_fwd_bf16_kernel(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V,
                                                                     bf16_t* __restrict__ O, float* __restrict__ lse, float* __restrict__ Opart, CrossArgs a) {
  typedef Mma<bf16_t, D> X;
  constexpr int BN = 64, TILEB = BN * X::ROWB, OFF_V = 2 * TILEB, NA = 2 * X::KS, NB = 4 * X::MD, NPAIR = 16, NPA = 10, BSTRIDE = NB / 8, PF = 2;
  static_assert((NPAIR - NPA - 1) * BSTRIDE < X::MD * 3 && 1 * BSTRIDE < X::MD * 2, "late weights are ready before the products that take them");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB];   // K, K, V, V
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y, b = bh / a.Hkv, hk = bh - b * a.Hkv, part = blockIdx.z;
  const int len = __builtin_amdgcn_readfirstlane(seen_states(a, b));
  const int t0 = part * a.tiles_per_part, tiles = (len + BN - 1) / BN, n = (t0 + a.tiles_per_part < tiles ? t0 + a.tiles_per_part : tiles) - t0;
  const uint32_t lds = lds_address(smem);
  TileStream<bf16_t, D, BN, NW> ks(K + b * a.k.b + hk * a.k.h + (int64_t)t0 * BN * a.k.n, (uint32_t)(a.k.n * 2), a.M - t0 * BN, wave, lane);
  TileStream<bf16_t, D, BN, NW> vs(V + b * a.v.b + hk * a.v.h + (int64_t)t0 * BN * a.v.n, (uint32_t)(a.v.n * 2), a.M - t0 * BN, wave, lane);
  auto byte_of = [&](int i) __attribute__((always_inline)) { return a.mask && i < n ? mask_byte(a, b, (t0 + i) * BN, len, lane) : 1; };
  auto seen_of = [&](int byte, int i) __attribute__((always_inline)) -> uint64_t {
    if (a.mask) return seen_bits(byte, (t0 + i) * BN, len, BN, lane);
    const int have = len - (t0 + i) * BN;
    return have >= 64 ? ~0ull : (1ull << have) - 1ull;
  };
  const bool once = NW < 4 && a.once != 0;
  if (n > 0) ks.next(lds, wave, once);
  int byte = byte_of(0), byte_next = byte_of(1);

  // the wavefront's rows: of one head, or (flat) the next 32 of the key head's rows
  const int head_blocks = a.flat ? 0x7fffffff : (a.N + NW * 32 - 1) / (NW * 32);
  const int g = a.group == 1 || a.flat ? 0 : (int)blockIdx.x / head_blocks;
  const int n0 = ((int)blockIdx.x - (a.flat ? 0 : g * head_blocks)) * (NW * 32) + wave * 32, row = n0 + l32;   // flat: rows of the key head
  const int have = (a.flat ? a.rows : a.N) - n0;
  typename X::Frag qf[X::KS];
  if (a.flat) {
    const CrossRow r = cross_row(a, row);
    row_frags<D>(qf, Q + b * a.q.b + (int64_t)(hk * a.group + r.g) * a.q.h + r.n * a.q.n, hf, l32 < have);
  } else {
    const uint32_t step = (uint32_t)(a.q.n * 2);
    const auto rsrc = rows_rsrc(Q + b * a.q.b + (int64_t)(hk * a.group + g) * a.q.h + (int64_t)n0 * a.q.n, step, have, X::ROWB);
#pragma unroll
    for (int k = 0; k < X::KS; ++k)
      qf[k] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)((uint32_t)l32 * step) + hf * 16 + k * 32, 0, 0));
  }
  f32x16 acc[X::MD];
#pragma unroll
  for (int md = 0; md < X::MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[md][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f, shift = 0.f;
  if (n > 0) {
    vs.next(lds + OFF_V, wave, once);
    if (n > 1) ks.next(lds + TILEB, wave, once);
    const uint32_t rbase = rows_base<bf16_t, D>(lane), cbase = X::cols_base(lane);
    uint64_t seen = seen_of(byte, 0), seen_next = 0;
    auto advance = [&](float top) __attribute__((always_inline)) {
      float p, q;
      halves(top * a.scale_log2, p, q);
      top = fmaxf(p, q);
      const bool up = top - m_run > CROSS_LAZY;
      if (__any(up)) {                        // (a row's own maximum decides: its bits do not depend on the rows beside it)
        const float alpha = up ? __builtin_amdgcn_exp2f(m_run - top) : 1.f;
        l_run *= alpha;
#pragma unroll
        for (int md = 0; md < X::MD; ++md)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[md][v] *= alpha;
        m_run = up ? top : m_run;
      }
      shift = m_run == -INFINITY ? 0.f : -m_run;
    };
    auto read_k = [&](int j, int buf) __attribute__((always_inline)) {       // product j: half j % 2 of the keys, k-step j / 2
      return *reinterpret_cast<const bf16x8*>(smem + buf * TILEB + (j % 2) * 32 * X::ROWB + (rbase ^ (uint32_t)((j / 2) << 5)));
    };
    // weights 2q, 2q + 1 of the lane: registers of half q / 8
    auto exp_pair = [&](const f32x16 (&s)[2], uint32_t (&w)[NPAIR], int q) __attribute__((always_inline)) {
      const int u = q >> 3, v = 2 * (q & 7);
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[u][v], a.scale_log2, shift));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(s[u][v + 1], a.scale_log2, shift));
      l_run += p0;
      l_run += p1;
      uint32_t bits = f32_to_bf16_pair(p0, p1);
      asm volatile("" : "+v"(bits), "+v"(l_run));     // made here, not where it is used
      w[q] = bits;
    };
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

    auto step = [&](auto parity, auto more_tag, f32x16 (&sc)[2], f32x16 (&sn)[2], int i) __attribute__((always_inline)) {
      constexpr int PAR = decltype(parity)::value;
      constexpr bool MORE = decltype(more_tag)::value;
      tile_arrived();                         // K(i + 1), V(i)
      if (MORE) {
        seen_next = seen_of(byte_next, i + 1);
        byte_next = byte_of(i + 2);
        if (i + 2 < n) ks.next(lds + PAR * TILEB, wave, once);
        vs.next(lds + OFF_V + (PAR ^ 1) * TILEB, wave, once);
      }
      unsigned char* vt = smem + OFF_V + PAR * TILEB;
      if (seen != ~0ull) {
        blank<bf16_t, D, NW * 64>(vt, BN, seen, tid);
        lds_ready();
      }
      uint32_t w[NPAIR];
      bf16x8 fr[4];
      __builtin_amdgcn_sched_barrier(0);
      if (MORE) {
#pragma unroll
        for (int j = 0; j < PF; ++j) fr[j] = read_k(j, PAR ^ 1);
      }
#pragma unroll
      for (int j = 0; j < NA; ++j) {
        if (MORE) {
          if (j + PF < NA) fr[(j + PF) & 3] = read_k(j + PF, PAR ^ 1);
          sn[j % 2] = X::mul(fr[j & 3], qf[j / 2], j < 2 ? zero : sn[j % 2]);
        }
#pragma unroll
        for (int q = j * NPA / NA; q < (j + 1) * NPA / NA; ++q) exp_pair(sc, w, q);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (MORE && seen_next != ~0ull) {
#pragma unroll
        for (int u = 0; u < 2; ++u) hide(sn[u], (uint32_t)(seen_next >> (32 * u)), hf);
      }
      cs16x4 lo[4], hi[4];
      auto read_v = [&](int j) __attribute__((always_inline)) {              // product j: channels j % MD, 16 keys j / MD
        const uint32_t x = cbase ^ (uint32_t)((j % X::MD) << 6);
        lo[j & 3] = X::read_t(vt + (j / X::MD) * 16 * X::ROWB + x);
        hi[j & 3] = X::read_t(vt + ((j / X::MD) * 16 + 8) * X::ROWB + (x ^ 32u));
      };
      float top = -INFINITY;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < PF; ++j) read_v(j);
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if (j + PF < NB) read_v(j + PF);
        const int md = j % X::MD, f = j / X::MD;
        const bf16x8 pf = __builtin_bit_cast(bf16x8, (u32x4{w[4 * f], w[4 * f + 1], w[4 * f + 2], w[4 * f + 3]}));
        acc[md] = X::mul(__builtin_bit_cast(bf16x8, (cs16x8)__builtin_shufflevector(lo[j & 3], hi[j & 3], 0, 1, 2, 3, 4, 5, 6, 7)), pf, acc[md]);
        if (j % BSTRIDE == 0 && NPA + j / BSTRIDE < NPAIR) exp_pair(sc, w, NPA + j / BSTRIDE);
        if (MORE) {
#pragma unroll
          for (int e = j * NPAIR / NB; e < (j + 1) * NPAIR / NB; ++e) top = fmaxf(top, fmaxf(sn[e >> 3][2 * (e & 7)], sn[e >> 3][2 * (e & 7) + 1]));
          asm volatile("" ::"v"(top));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (MORE) {
        advance(top);
        seen = seen_next;
      }
    };

    f32x16 sa[2], sb[2];
    tile_arrived();                           // K(0) (and what was requested with it)
#pragma unroll
    for (int j = 0; j < NA; ++j) sa[j % 2] = X::mul(read_k(j, 0), qf[j / 2], j < 2 ? zero : sa[j % 2]);
    if (seen != ~0ull) {
#pragma unroll
      for (int u = 0; u < 2; ++u) hide(sa[u], (uint32_t)(seen >> (32 * u)), hf);
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, sa[u][v]);
    advance(top);
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    const std::integral_constant<bool, true> more;
    const std::integral_constant<bool, false> last;
    int i = 0;
    for (; i + 2 < n; i += 2) {
      step(even, more, sa, sb, i);
      step(odd, more, sb, sa, i + 1);
    }
    if (i + 1 < n) {
      step(even, more, sa, sb, i);
      step(odd, last, sb, sa, i + 1);
    } else {
      step(even, last, sa, sb, i);
    }
  }

  // ---- the rows' sums and outputs
  {
    float p, q;
    halves(l_run, p, q);
    l_run = p + q;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  const float stat = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * CROSS_LN2;
  if constexpr (PART) {
    if (l32 >= have) return;
    const int64_t at = ((int64_t)part * a.B * a.Hkv + bh) * a.rows + (int64_t)g * a.N + row;
    float* po = Opart + at * D;
    if (hf == 0) lse[at] = stat;
#pragma unroll
    for (int md = 0; md < X::MD; ++md)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4*>(po + md * 32 + g4 * 8 + hf * 4) = f32x4{acc[md][g4 * 4], acc[md][g4 * 4 + 1], acc[md][g4 * 4 + 2], acc[md][g4 * 4 + 3]} * inv;
  } else {
    if (lse && hf == 0 && l32 < have) lse[((int64_t)b * a.Hq + hk * a.group + g) * a.N + row] = stat;
    lds_ready();                              // everyone has read the last tile
    if (a.flat) {
      rows_out<bf16_t, D>(acc, inv, smem + wave * 32 * X::ROWB, lane, [&](int r) __attribute__((always_inline)) -> bf16_t* {
        if (r >= have) return nullptr;
        const CrossRow c = cross_row(a, n0 + r);
        return O + b * a.o.b + (int64_t)(hk * a.group + c.g) * a.o.h + c.n * a.o.n;
      });
    } else {
      rows_out_head<D>(acc, inv, smem + wave * 32 * X::ROWB, lane, O + b * a.o.b + (int64_t)(hk * a.group + g) * a.o.h + (int64_t)n0 * a.o.n, (uint32_t)(a.o.n * 2), have);
    }
  }
}

// ---- bfloat16 gradients with the order of a tile fixed by hand: every operand fragment is requested two MFMAs ahead, and a slice of the vector work stands behind each MFMA.

// A rounding of P or dS to bfloat16 costs a gradient about as much as its own rounding to bfloat16 does (of the norm: 0.0017 each, 0.0024 together).  Where many rows or states add up it
// is one rounding.  Where few do, so that an outlying one can be most of the result (twice the error was seen), a second bfloat16 number holds what the first leaves over, and a second
// product adds it: dQ with at most 64 query rows to a key head (less than four wavefronts), dK and dV with at most 32.  The matrix instructions are not what bounds the kernels there:
// 2 x 16 heads x 64 rows x 8190 states, d = 64: dQ 17 -> 19 us; with dK and dV so too it would be 22 -> 29 us for these, hence 32.
// What (x, y) leave over when rounded to the pair `bits`
__device__ __forceinline__ uint32_t left_over(float x, float y, uint32_t bits) {
  return f32_to_bf16_pair(x - __uint_as_float(bits << 16), y - __uint_as_float(bits & 0xffff0000u));
}

// 32 x 32 scores' fragments for the second products: pairs q = 0 .. 7 of registers 2q, 2q + 1
template <bool TWO> struct WeightPairs {
  uint32_t w[8], rest[TWO ? 8 : 1];
  __device__ __forceinline__ void put(int q, float x, float y) {
    uint32_t bits = f32_to_bf16_pair(x, y);
    asm volatile("" : "+v"(bits));            // made here, not where it is used
    w[q] = bits;
    if constexpr (TWO) {
      bits = left_over(x, y, bits);
      asm volatile("" : "+v"(bits));
      rest[q] = bits;
    }
  }
  // acc + rows x weights 16 f .. 16 f + 15
  template <typename X> __device__ __forceinline__ f32x16 mul(bf16x8 rows, int f, f32x16 acc) const {
    acc = X::mul(rows, __builtin_bit_cast(bf16x8, (u32x4{w[4 * f], w[4 * f + 1], w[4 * f + 2], w[4 * f + 3]})), acc);
    if constexpr (TWO) acc = X::mul(rows, __builtin_bit_cast(bf16x8, (u32x4{rest[4 * f], rest[4 * f + 1], rest[4 * f + 2], rest[4 * f + 3]})), acc);
    return acc;
  }
};
// The operand fragments that are on their way, by the slot that takes them: of rows (16 bytes a lane) or of columns (two transposing reads).  AGAIN: a fragment's
// address is made for each request, where the compiler would hold those that come again over the tile.
template <int D, bool AGAIN> struct Fragments {
  typedef Mma<bf16_t, D> X;
  u32x4 f[3];
  template <int C> static __device__ __forceinline__ uint32_t turned(uint32_t x) {
    if constexpr (AGAIN) return flip<C>(x);
    else return x ^ (uint32_t)C;
  }
  template <int SLOT, int K> __device__ __forceinline__ void row(const unsigned char* tile, uint32_t base) {
    f[SLOT % 3] = *reinterpret_cast<const u32x4*>(tile + turned<(K << 5)>(base));
  }
  template <int SLOT, int J> __device__ __forceinline__ void col(const unsigned char* tile, uint32_t base) {   // channels J % MD, rows J / MD * 16 ..
    constexpr int C = (J % X::MD) << 6;
    const u32x2 lo = __builtin_bit_cast(u32x2, X::read_t(tile + (J / X::MD) * 16 * X::ROWB + turned<C>(base))),
                hi = __builtin_bit_cast(u32x2, X::read_t(tile + ((J / X::MD) * 16 + 8) * X::ROWB + turned<C ^ 32>(base)));
    f[SLOT % 3] = u32x4{lo.x, lo.y, hi.x, hi.y};
  }
  template <int SLOT> __device__ __forceinline__ bf16x8 get() const { return __builtin_bit_cast(bf16x8, f[SLOT % 3]); }
};

// dQ; and for the kernel after it -D and -lse log2(e) of every row (parts: the first one's).  Of a tile's two halves: S0, dP0 (beside the weights of half 0), S1 (beside dS0),
// dP1 (beside the weights of half 1), the product with half 0 (beside dS1), with half 1.
template <int D, int NW, bool PART>
__global__ __launch_bounds__(NW * 64, 2) void cross_dq_bf16_kernel(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const bf16_t* __restrict__ O,
                                                                   const float* __restrict__ lse, const bf16_t* __restrict__ dO, float* __restrict__ stats, bf16_t* __restrict__ dQ,
                                                                   float* __restrict__ dQpart, CrossArgs a) {
  typedef Mma<bf16_t, D> X;
  constexpr int BN = 64, TILEB = BN * X::ROWB, KS = X::KS, MD = X::MD, PF = 2;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB];   // K, V; K, V
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y, b = bh / a.Hkv, hk = bh - b * a.Hkv, part = blockIdx.z;
  const int len = __builtin_amdgcn_readfirstlane(seen_states(a, b));
  const int t0 = part * a.tiles_per_part, tiles = (len + BN - 1) / BN, n = (t0 + a.tiles_per_part < tiles ? t0 + a.tiles_per_part : tiles) - t0;
  const uint32_t lds = lds_address(smem);
  TileStream<bf16_t, D, BN, NW> ks(K + b * a.k.b + hk * a.k.h + (int64_t)t0 * BN * a.k.n, (uint32_t)(a.k.n * 2), a.M - t0 * BN, wave, lane);
  TileStream<bf16_t, D, BN, NW> vs(V + b * a.v.b + hk * a.v.h + (int64_t)t0 * BN * a.v.n, (uint32_t)(a.v.n * 2), a.M - t0 * BN, wave, lane);
  auto byte_of = [&](int i) __attribute__((always_inline)) { return a.mask && i < n ? mask_byte(a, b, (t0 + i) * BN, len, lane) : 1; };
  auto seen_of = [&](int byte, int i) __attribute__((always_inline)) -> uint64_t {
    if (a.mask) return seen_bits(byte, (t0 + i) * BN, len, BN, lane);
    const int have = len - (t0 + i) * BN;
    return have >= 64 ? ~0ull : (1ull << have) - 1ull;
  };
  if (n > 0) {
    ks.next(lds, wave);
    vs.next(lds + TILEB, wave);
  }
  int byte = byte_of(0);
  const int head_blocks = a.flat ? 0x7fffffff : (a.N + NW * 32 - 1) / (NW * 32);
  const int g = a.group == 1 || a.flat ? 0 : (int)blockIdx.x / head_blocks;
  const int n0 = ((int)blockIdx.x - (a.flat ? 0 : g * head_blocks)) * (NW * 32) + wave * 32, row = n0 + l32;
  const int have = (a.flat ? a.rows : a.N) - n0, head = hk * a.group + g;
  const bool active = l32 < have;
  const int64_t stat_at = ((int64_t)b * a.Hq + head) * a.N + row;
  typename X::Frag qf[KS], gf[KS];
  float dot = 0.f;
  {
    u32x4 of[KS];
    if (a.flat) {
      const CrossRow r = cross_row(a, row);
      row_frags<D>(qf, Q + b * a.q.b + (int64_t)(head + r.g) * a.q.h + r.n * a.q.n, hf, active);
      row_frags<D>(gf, dO + b * a.go.b + (int64_t)(head + r.g) * a.go.h + r.n * a.go.n, hf, active);
      typename X::Frag x[KS];
      row_frags<D>(x, O + b * a.o.b + (int64_t)(head + r.g) * a.o.h + r.n * a.o.n, hf, active);
#pragma unroll
      for (int k = 0; k < KS; ++k) of[k] = __builtin_bit_cast(u32x4, x[k]);
    } else {
      auto rows_of = [&](const bf16_t* base, const Strides& st, auto&& put) __attribute__((always_inline)) {
        const uint32_t step = (uint32_t)(st.n * 2);
        const auto rsrc = rows_rsrc(base + b * st.b + (int64_t)head * st.h + (int64_t)n0 * st.n, step, have, X::ROWB);
#pragma unroll
        for (int k = 0; k < KS; ++k) put(k, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)((uint32_t)l32 * step) + hf * 16 + k * 32, 0, 0));
      };
      rows_of(dO, a.go, [&](int k, u32x4 x) __attribute__((always_inline)) { gf[k] = __builtin_bit_cast(bf16x8, x); });
      rows_of(O, a.o, [&](int k, u32x4 x) __attribute__((always_inline)) { of[k] = x; });
      rows_of(Q, a.q, [&](int k, u32x4 x) __attribute__((always_inline)) { qf[k] = __builtin_bit_cast(bf16x8, x); });
    }
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      float x[8], y[8], sum = 0.f;
      Elem<bf16_t>::widen(of[k], x);
      Elem<bf16_t>::widen(__builtin_bit_cast(u32x4, gf[k]), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(x[e], y[e], sum);
      dot += sum;
    }
    float p, q;
    halves(dot, p, q);
    dot = p + q;
  }
  float shift = -INFINITY;                    // weights of 0 for a row that sees nothing
  if (active) {
    const float l = lse[stat_at];
    if (l != -INFINITY) shift = -l * CROSS_LOG2E;
    if (part == 0 && hf == 0) {
      stats[stat_at] = shift;
      stats[(int64_t)a.B * a.Hq * a.N + stat_at] = -dot;
    }
  }
  f32x16 acc[MD], ndot;
#pragma unroll
  for (int v = 0; v < 16; ++v) ndot[v] = -dot;
#pragma unroll
  for (int md = 0; md < MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[md][v] = 0.f;
  const uint32_t rbase = rows_base<bf16_t, D>(lane), cbase = X::cols_base(lane);
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < n; ++i) {
    unsigned char* tile = smem + (i & 1) * 2 * TILEB;
    const uint64_t seen = seen_of(byte, i);
    tile_arrived();
    if (i + 1 < n) {
      byte = byte_of(i + 1);
      const uint32_t to = lds + (uint32_t)((~i & 1) * 2 * TILEB);
      ks.next(to, wave);
      vs.next(to + TILEB, wave);
    }
    const bool whole = seen == ~0ull;
    if (!whole) {
      if (seen == 0) continue;
      blank<bf16_t, D, NW * 64>(tile, BN, seen, tid);
      blank<bf16_t, D, NW * 64>(tile + TILEB, BN, seen, tid);
      lds_ready();
    }
    constexpr int HALF = 32 * X::ROWB, NF = 4 * KS + 4 * MD;
    Fragments<D, false> fr;
    f32x16 s[2], dp[2];
    WeightPairs<NW < 4> w[2];
    auto request = [&](auto tag) __attribute__((always_inline)) {
      constexpr int j = decltype(tag)::value;
      if constexpr (j < 4 * KS) fr.template row<j, j % KS>(tile + (j / KS & 1) * TILEB + j / (2 * KS) * HALF, rbase);
      else if constexpr (j < NF) fr.template col<j, (j - 4 * KS) % (2 * MD)>(tile + (j - 4 * KS) / (2 * MD) * HALF, cbase);
    };
    // f(0) .. f(COUNT - 1) spread over the slots FROM .. TO - 1
    auto spread = [&](auto slot_tag, auto from_tag, auto to_tag, auto count_tag, auto&& f) __attribute__((always_inline)) {
      constexpr int J = decltype(slot_tag)::value, FROM = decltype(from_tag)::value, TO = decltype(to_tag)::value, COUNT = decltype(count_tag)::value;
      if constexpr (J >= FROM && J < TO)
#pragma unroll
        for (int e = COUNT * (J - FROM) / (TO - FROM); e < COUNT * (J + 1 - FROM) / (TO - FROM); ++e) f(e);
    };
    using std::integral_constant;
    __builtin_amdgcn_sched_barrier(0);
    each<PF>([&](auto tag) __attribute__((always_inline)) { request(tag); });
    each<NF>([&](auto tag) __attribute__((always_inline)) {
      constexpr int j = decltype(tag)::value;
      request(integral_constant<int, j + PF>{});
      if constexpr (j < 4 * KS) {
        constexpr int u = j / (2 * KS), k = j % KS;
        if constexpr ((j / KS & 1) == 0) s[u] = X::mul(fr.template get<j>(), qf[k], k == 0 ? zero : s[u]);
        else dp[u] = X::mul(fr.template get<j>(), gf[k], k == 0 ? ndot : dp[u]);
      } else {
        constexpr int u = (j - 4 * KS) / (2 * MD), c = (j - 4 * KS) % (2 * MD);
        acc[c % MD] = w[u].template mul<X>(fr.template get<j>(), c / MD, acc[c % MD]);
      }
      if constexpr (j == KS || j == 3 * KS) {
        constexpr int u = j / (2 * KS);
        if (!whole) hide(s[u], (uint32_t)(seen >> (32 * u)), hf);
      }
      auto weight = [&](int u, int e) __attribute__((always_inline)) {
        float x = __builtin_amdgcn_exp2f(fmaf(s[u][e], a.scale_log2, shift));
        asm volatile("" : "+v"(x));
        s[u][e] = x;
      };
      auto dscore = [&](int u, int q) __attribute__((always_inline)) { w[u].put(q, s[u][2 * q] * dp[u][2 * q], s[u][2 * q + 1] * dp[u][2 * q + 1]); };
      spread(tag, integral_constant<int, KS + 1>{}, integral_constant<int, 2 * KS>{}, integral_constant<int, 16>{}, [&](int e) __attribute__((always_inline)) { weight(0, e); });
      spread(tag, integral_constant<int, 2 * KS + 1>{}, integral_constant<int, 3 * KS>{}, integral_constant<int, 8>{}, [&](int q) __attribute__((always_inline)) { dscore(0, q); });
      spread(tag, integral_constant<int, 3 * KS + 1>{}, integral_constant<int, 4 * KS>{}, integral_constant<int, 16>{}, [&](int e) __attribute__((always_inline)) { weight(1, e); });
      spread(tag, integral_constant<int, 4 * KS + 1>{}, integral_constant<int, 4 * KS + 2 * MD>{}, integral_constant<int, 8>{}, [&](int q) __attribute__((always_inline)) { dscore(1, q); });
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  if constexpr (PART) {
    if (!active) return;
    float* po = dQpart + (((int64_t)part * a.B * a.Hkv + bh) * a.rows + (int64_t)g * a.N + row) * D;
#pragma unroll
    for (int md = 0; md < MD; ++md)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4*>(po + md * 32 + g4 * 8 + hf * 4) = f32x4{acc[md][g4 * 4], acc[md][g4 * 4 + 1], acc[md][g4 * 4 + 2], acc[md][g4 * 4 + 3]};
  } else {
    lds_ready();
    if (a.flat) {
      rows_out<bf16_t, D>(acc, a.scale, smem + wave * 32 * X::ROWB, lane, [&](int x) __attribute__((always_inline)) -> bf16_t* {
        if (x >= have) return nullptr;
        const CrossRow c = cross_row(a, n0 + x);
        return dQ + b * a.gq.b + (int64_t)(hk * a.group + c.g) * a.gq.h + c.n * a.gq.n;
      });
    } else {
      rows_out_head<D>(acc, a.scale, smem + wave * 32 * X::ROWB, lane, dQ + b * a.gq.b + (int64_t)head * a.gq.h + (int64_t)n0 * a.gq.n, (uint32_t)(a.gq.n * 2), have);
    }
  }
}

// dK, dV of 32 keys a wavefront.  Of 32 query rows: S, dP (beside the weights), the product for dV (beside dS), for dK.
template <int D, bool PART, bool TWO>
__global__ __launch_bounds__(256, D == 64 ? (TWO ? 2 : 3) : 2) void cross_dkv_bf16_kernel(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const float* __restrict__ stats,
                                                                const bf16_t* __restrict__ dO, bf16_t* __restrict__ dK, bf16_t* __restrict__ dV, float* __restrict__ dKpart,
                                                                float* __restrict__ dVpart, CrossArgs a) {
  typedef Mma<bf16_t, D> X;
  constexpr int NW = 4, BN = 64, TILEB = BN * X::ROWB, OFF_STAT = 4 * TILEB, KS = X::KS, MD = X::MD, PF = 2;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB + 2 * 2 * BN * 4];   // Q, dO; Q, dO; -lse log2(e), -D; the same
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y, b = bh / a.Hkv, hk = bh - b * a.Hkv, part = blockIdx.z;
  const int key0 = (int)(blockIdx.x * (NW * 32) + wave * 32), key = key0 + l32;
  const int len = __builtin_amdgcn_readfirstlane(seen_states(a, b));
  const bool seen = key < len && (!a.mask || a.mask[(int64_t)b * a.M + key] != 0);
  const bool any = __syncthreads_or(seen), mine = __any(seen);       // a wavefront none of whose keys is seen loads for the others
  const int all = any ? a.group * a.chunks : 0;
  const int t0 = part * a.tiles_per_part, t1 = t0 + a.tiles_per_part < all ? t0 + a.tiles_per_part : all;
  const uint32_t lds = lds_address(smem);
  f32x16 dk[MD], dv[MD];
#pragma unroll
  for (int md = 0; md < MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[md][v] = dv[md][v] = 0.f;
  if (t0 < t1) {
    TileStream<bf16_t, D, BN, NW> qs(Q, (uint32_t)(a.q.n * 2), 0, wave, lane), gs(dO, (uint32_t)(a.go.n * 2), 0, wave, lane);
    uint64_t st = 0;                          // the wavefront's statistics (0: -lse log2(e), 1: -D) of the next tile
    const uint64_t plane = (uint64_t)a.B * a.Hq * a.N * 4;
    int g = t0 / a.chunks, c = t0 - g * a.chunks;        // next tile: of head g of the group, chunk c
    auto head_at = [&]() __attribute__((always_inline)) {
      const int head = hk * a.group + g;
      qs.base = (uint64_t)(Q + b * a.q.b + (int64_t)head * a.q.h + (int64_t)c * BN * a.q.n);
      gs.base = (uint64_t)(dO + b * a.go.b + (int64_t)head * a.go.h + (int64_t)c * BN * a.go.n);
      qs.left = gs.left = a.N - c * BN;
      st = (uint64_t)stats + ((uint64_t)b * a.Hq + head) * a.N * 4 + (uint64_t)c * BN * 4 + (wave == 1 ? plane : 0);
    };
    head_at();
    auto fire = [&](int at) __attribute__((always_inline)) {
      const uint32_t to = lds + (uint32_t)(at * 2 * TILEB);
      if (wave < 2) {
        const rsrc_words rsrc = make_rsrc((const void*)st, (uint32_t)(qs.left < BN ? qs.left : BN) * 4);
        load_lds4(rsrc, lds + (uint32_t)(OFF_STAT + (at * 2 + wave) * BN * 4), lane_again() * 4, 0);
      }
      qs.again(wave);
      qs.next(to, wave);
      gs.again(wave);
      gs.next(to + TILEB, wave);
      st += BN * 4;
      if (++c == a.chunks) {
        c = 0;
        ++g;
        head_at();
      }
    };
    int have = qs.left, have_next = 0;        // rows of this tile and of the one being loaded
    fire(0);
    typename X::Frag kf[KS], vf[KS];
    row_frags<D>(kf, K + b * a.k.b + hk * a.k.h + key * a.k.n, hf, seen);
    row_frags<D>(vf, V + b * a.v.b + hk * a.v.h + key * a.v.n, hf, seen);
    const uint32_t rbase = rows_base<bf16_t, D>(lane), cbase = X::cols_base(lane);
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int t = t0; t < t1; ++t, have = have_next) {
      const int at = (t - t0) & 1;
      unsigned char* tile = smem + at * 2 * TILEB;
      float* stat = reinterpret_cast<float*>(smem + OFF_STAT + at * 2 * BN * 4);
      tile_arrived();
      if (t + 1 < t1) {
        have_next = qs.left;
        fire(at ^ 1);
      }
      if (have < BN) {
        const int tid = wave * 64 + lane_again();
        const uint64_t keep = (1ull << have) - 1ull;
        blank<bf16_t, D, 256>(tile, BN, keep, tid);
        blank<bf16_t, D, 256>(tile + TILEB, BN, keep, tid);
        if (tid < BN && tid >= have) {
          stat[tid] = -INFINITY;
          stat[BN + tid] = 0.f;
        }
        lds_ready();
      }
#pragma unroll 1
      for (int u = 0; u < 2; ++u) {
        if (u * 32 >= have || !mine) break;
        const unsigned char* qt = tile + u * 32 * X::ROWB;
        const float* sl = stat + u * 32 + (lane_again() >> 5) * 4;
        Fragments<D, D == 128> fr;
        f32x16 s, dp;
        WeightPairs<TWO> w;
        f32x4 l[2];
        constexpr int NF = 2 * KS + 4 * MD;
        auto request = [&](auto tag) __attribute__((always_inline)) {
          constexpr int j = decltype(tag)::value;
          if constexpr (j < 2 * KS) fr.template row<j, j % KS>(qt + j / KS * TILEB, rbase);
          else if constexpr (j < 2 * KS + 2 * MD) fr.template col<j, j - 2 * KS>(qt + TILEB, cbase);
          else if constexpr (j < NF) fr.template col<j, j - 2 * KS - 2 * MD>(qt, cbase);
        };
        auto spread = [&](auto slot_tag, auto from_tag, auto to_tag, auto count_tag, auto&& f) __attribute__((always_inline)) {
          constexpr int J = decltype(slot_tag)::value, FROM = decltype(from_tag)::value, TO = decltype(to_tag)::value, COUNT = decltype(count_tag)::value;
          if constexpr (J >= FROM && J < TO)
#pragma unroll
            for (int e = COUNT * (J - FROM) / (TO - FROM); e < COUNT * (J + 1 - FROM) / (TO - FROM); ++e) f(e);
        };
        using std::integral_constant;
        __builtin_amdgcn_sched_barrier(0);
        each<PF>([&](auto tag) __attribute__((always_inline)) { request(tag); });
        each<NF>([&](auto tag) __attribute__((always_inline)) {
          constexpr int j = decltype(tag)::value;
          request(integral_constant<int, j + PF>{});
          if constexpr (j == KS - 2) {        // -D straight into the accumulators
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
              const f32x4 d = *reinterpret_cast<const f32x4*>(sl + BN + g4 * 8);
#pragma unroll
              for (int e = 0; e < 4; ++e) dp[g4 * 4 + e] = d[e];
            }
          }
          if constexpr (j == KS - 1) l[0] = *reinterpret_cast<const f32x4*>(sl);
          if constexpr (j < KS) s = X::mul(fr.template get<j>(), kf[j], j == 0 ? zero : s);
          else if constexpr (j < 2 * KS) dp = X::mul(fr.template get<j>(), vf[j - KS], dp);
          else if constexpr (j < 2 * KS + 2 * MD) dv[(j - 2 * KS) % MD] = w.template mul<X>(fr.template get<j>(), (j - 2 * KS) / MD, dv[(j - 2 * KS) % MD]);
          else dk[(j - 2 * KS) % MD] = w.template mul<X>(fr.template get<j>(), (j - 2 * KS - 2 * MD) / MD, dk[(j - 2 * KS) % MD]);
          spread(tag, integral_constant<int, KS + 1>{}, integral_constant<int, 2 * KS>{}, integral_constant<int, 16>{}, [&](int e) __attribute__((always_inline)) {
            if (e % 4 == 0 && e < 12) l[(e / 4 + 1) & 1] = *reinterpret_cast<const f32x4*>(sl + (e / 4 + 1) * 8);
            float x = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, l[(e / 4) & 1][e % 4]));
            asm volatile("" : "+v"(x));
            s[e] = x;
          });
          // (P and dS are packed when they are whole: sooner, the packed ones beside the others do not fit the registers)
          spread(tag, integral_constant<int, 2 * KS + MD>{}, integral_constant<int, 2 * KS + 2 * MD>{}, integral_constant<int, 16>{}, [&](int e) __attribute__((always_inline)) {
            float x = s[e] * dp[e];
            asm volatile("" : "+v"(x));
            s[e] = x;
          });
          if constexpr (j == 2 * KS - 1 || j == 2 * KS + 2 * MD - 1) {
#pragma unroll
            for (int q = 0; q < 8; ++q) w.put(q, s[2 * q], s[2 * q + 1]);
          }
          __builtin_amdgcn_sched_barrier(0);
        });
      }
    }
  }
  const int lane_end = lane_again(), key_end = key0 + (lane_end & 31);
  const bool seen_end = key_end < len && (!a.mask || a.mask[(int64_t)b * a.M + key_end] != 0);
  if constexpr (PART) {
    const int key = key_end, hf = lane_end >> 5;
    const bool seen = seen_end;
    if (key >= a.M) return;
    const int64_t to = (((int64_t)part * a.B * a.Hkv + bh) * a.M + key) * D;
#pragma unroll
    for (int md = 0; md < MD; ++md)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const int c = md * 32 + g4 * 8 + hf * 4;
        f32x4 x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = seen ? dk[md][g4 * 4 + e] : 0.f;
          y[e] = seen ? dv[md][g4 * 4 + e] : 0.f;
        }
        *reinterpret_cast<f32x4*>(dKpart + to + c) = x;
        *reinterpret_cast<f32x4*>(dVpart + to + c) = y;
      }
  } else {
    const int lane = lane_end;
    if (!seen_end) {
#pragma unroll
      for (int md = 0; md < MD; ++md)
#pragma unroll
        for (int v = 0; v < 16; ++v) dk[md][v] = dv[md][v] = 0.f;
    }
    lds_ready();
    unsigned char* mine = smem + wave * 32 * X::ROWB;
    rows_out_head<D>(dk, a.scale, mine, lane, dK + b * a.gk.b + hk * a.gk.h + (int64_t)key0 * a.gk.n, (uint32_t)(a.gk.n * 2), a.M - key0);
    rows_out_head<D>(dv, 1.f, mine, lane, dV + b * a.gv.b + hk * a.gv.h + (int64_t)key0 * a.gv.n, (uint32_t)(a.gv.n * 2), a.M - key0);
  }
}

template <int D> static void fwd_d(const CrossArgs& a, dim3 grid, int nw, bool part, const bf16_t* Q, const bf16_t* K, const bf16_t* V, bf16_t* O, float* lse, float* Opart, hipStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, nw * 64, 0, s>>>(Q, K, V, O, lse, Opart, a); };
  if (nw == 1) part ? go(cross_fwd_bf16_kernel<D, 1, true>) : go(cross_fwd_bf16_kernel<D, 1, false>);
  else if (nw == 2) part ? go(cross_fwd_bf16_kernel<D, 2, true>) : go(cross_fwd_bf16_kernel<D, 2, false>);
  else part ? go(cross_fwd_bf16_kernel<D, 4, true>) : go(cross_fwd_bf16_kernel<D, 4, false>);
}
void cross_fwd(const CrossArgs& a, int d, dim3 grid, int nw, bool part, const bf16_t* Q, const bf16_t* K, const bf16_t* V, bf16_t* O, float* lse, float* Opart, hipStream_t s) {
  d == 128 ? fwd_d<128>(a, grid, nw, part, Q, K, V, O, lse, Opart, s) : fwd_d<64>(a, grid, nw, part, Q, K, V, O, lse, Opart, s);
}

template <int D> static void dq_d(const CrossArgs& a, dim3 grid, int nw, bool part, const bf16_t* Q, const bf16_t* K, const bf16_t* V, const bf16_t* O, const float* lse, const bf16_t* dO,
                                  float* stats, bf16_t* dQ, float* dQpart, hipStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, nw * 64, 0, s>>>(Q, K, V, O, lse, dO, stats, dQ, dQpart, a); };
  if (nw == 1) part ? go(cross_dq_bf16_kernel<D, 1, true>) : go(cross_dq_bf16_kernel<D, 1, false>);
  else if (nw == 2) part ? go(cross_dq_bf16_kernel<D, 2, true>) : go(cross_dq_bf16_kernel<D, 2, false>);
  else part ? go(cross_dq_bf16_kernel<D, 4, true>) : go(cross_dq_bf16_kernel<D, 4, false>);
}
void cross_dq(const CrossArgs& a, int d, dim3 grid, int nw, bool part, const bf16_t* Q, const bf16_t* K, const bf16_t* V, const bf16_t* O, const float* lse, const bf16_t* dO, float* stats,
              bf16_t* dQ, float* dQpart, hipStream_t s) {
  d == 128 ? dq_d<128>(a, grid, nw, part, Q, K, V, O, lse, dO, stats, dQ, dQpart, s) : dq_d<64>(a, grid, nw, part, Q, K, V, O, lse, dO, stats, dQ, dQpart, s);
}

void cross_dkv(const CrossArgs& a, int d, dim3 grid, bool part, const bf16_t* Q, const bf16_t* K, const bf16_t* V, const float* stats, const bf16_t* dO, bf16_t* dK, bf16_t* dV, float* dKpart,
               float* dVpart, hipStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(Q, K, V, stats, dO, dK, dV, dKpart, dVpart, a); };
  const bool few = a.rows <= 32;
  if (d == 128) {
    if (few) part ? go(cross_dkv_bf16_kernel<128, true, true>) : go(cross_dkv_bf16_kernel<128, false, true>);
    else part ? go(cross_dkv_bf16_kernel<128, true, false>) : go(cross_dkv_bf16_kernel<128, false, false>);
  } else {
    if (few) part ? go(cross_dkv_bf16_kernel<64, true, true>) : go(cross_dkv_bf16_kernel<64, false, true>);
    else part ? go(cross_dkv_bf16_kernel<64, true, false>) : go(cross_dkv_bf16_kernel<64, false, false>);
  }
}

}  // namespace psa
