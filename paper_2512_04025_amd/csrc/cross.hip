// Cross attention: N query tokens a head against M encoder states, of which batch entry b shows those with j < kv_len[b] and
// key_mask[b, j] != 0.  With s_j = scale q.k_j:  P = softmax over the states that are seen, O = P V, lse = log sum exp(s).  Backward, with
// P = exp(s - lse), D = dO.O, dP = dO V^T, dS = P (dP - D):  dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.
//
// All three kernels are made of two products on 32x32 MFMA tiles with fp32 accumulation (see Mma):
//   rows:  [32 rows of a tile in LDS] x [32 rows in registers]^T   -> one register row in each lane, the tile's rows in its registers
//   cols:  [32 rows of a tile in LDS]^T x [that result]            -> the result is the second operand as it lies, no lane exchange
// forward, dQ: the tile is a piece of K or V, the registers hold the query rows; dK, dV: the tile is a piece of Q or dO, the registers hold
// keys and values.  The query heads of a key head are rows of one matrix (row = head in group * N + token), so that few tokens of many
// heads fill a tile.  Tiles come straight into LDS, double buffered, one tile ahead; one barrier a tile.
// No atomics: sums over workgroups are written as partial results and added in a fixed order.
#include "psa_dev.h"
#include "psa_internal.h"

namespace psa {

struct CrossArgs {
  int B, Hq, Hkv, group, N, M;
  int rows;                                   // group * N: query rows of a key head
  int flat;                                   // a block of rows may hold rows of several heads
  int parts, tiles_per_part;                  // workgroups that share a row's keys (forward, dQ) or a key's rows (dK, dV)
  int chunks;                                 // dK, dV: tiles of one head's tokens
  float scale, scale_log2;
  Strides q, k, v, o, gq, gk, gv, go;         // g: gradients
  const int32_t* kv_len;
  const uint8_t* mask;
};

constexpr float CROSS_LOG2E = 1.44269504088896340736f, CROSS_LN2 = 0.69314718055994530942f;
constexpr float CROSS_LAZY = 8.f;             // the running maximum moves when it grows by more than 2^8

typedef __attribute__((ext_vector_type(4))) short cs16x4;
typedef __attribute__((ext_vector_type(8))) short cs16x8;
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));

// Tiles are rows of D elements; the 16-byte chunks of a row are permuted (XOR with swz(row), which has period 16), on the way into LDS, so that
// neither the row reads nor the column reads meet in a bank.
template <typename T, int D> struct Mma;

template <int D> struct Mma<bf16_t, D> {
  static constexpr int ROWB = D * 2, CPR = D / 8, KS = D / 16, MD = D / 32, VEC = 8;
  typedef bf16x8 Frag;
  static __device__ __forceinline__ int swz(int row) { return row_swizzle32<D>(row); }
  static __device__ __forceinline__ f32x16 mul(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  // 32 rows x 32 channels transposed: 16 lanes take 4 rows x 32 bytes, a lane gets one channel of them
  static __device__ __forceinline__ uint32_t cols_base(int lane) {
    const int hf = lane >> 5, s16 = lane & 15, row = hf * 4 + (s16 >> 2), chunk = ((lane >> 4) & 1) * 2 + ((s16 & 3) >> 1);
    return (uint32_t)(row * ROWB + ((chunk ^ swz(row)) << 4) + (s16 & 1) * 8);
  }
  static __device__ __forceinline__ cs16x4 read_t(const unsigned char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) cs16x4*)p);
  }
  struct Weights { bf16x8 f[2]; };            // rounded once: the products take bfloat16
  static __device__ __forceinline__ Weights weights(const f32x16& p) {
    Weights w;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w.f[i] = __builtin_bit_cast(bf16x8, (u32x4{f32_to_bf16_pair(p[8 * i], p[8 * i + 1]), f32_to_bf16_pair(p[8 * i + 2], p[8 * i + 3]),
                                                 f32_to_bf16_pair(p[8 * i + 4], p[8 * i + 5]), f32_to_bf16_pair(p[8 * i + 6], p[8 * i + 7])}));
    return w;
  }
  static __device__ __forceinline__ void cols(f32x16 (&acc)[MD], const unsigned char* tile, uint32_t base, const Weights& w) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int md = 0; md < MD; ++md) {
        const uint32_t x = base ^ (uint32_t)(md << 6);
        const cs16x4 lo = read_t(tile + i * 16 * ROWB + x), hi = read_t(tile + (i * 16 + 8) * ROWB + (x ^ 32u));
        acc[md] = mul(__builtin_bit_cast(bf16x8, (cs16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), w.f[i], acc[md]);
      }
  }
};

template <int D> struct Mma<float, D> {
  static constexpr int ROWB = D * 4, CPR = D / 4, KS = D / 8, MD = D / 32, VEC = 4;
  typedef f32x4 Frag;                         // four products of 32x32x2; a lane half has every other chunk
  static __device__ __forceinline__ int swz(int row) { return row & 15; }
  static __device__ __forceinline__ f32x16 mul(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ uint32_t cols_base(int lane) {
    const int hf = lane >> 5, l32 = lane & 31;
    return (uint32_t)(hf * 4 * ROWB + (((l32 >> 2) ^ (hf * 4)) << 4) + (l32 & 3) * 4);
  }
  struct Weights { f32x16 f; };
  static __device__ __forceinline__ Weights weights(const f32x16& p) { return {p}; }
  static __device__ __forceinline__ void cols(f32x16 (&acc)[MD], const unsigned char* tile, uint32_t base, const Weights& w) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {            // register v: rows (v / 4) * 8 + v % 4 and 4 after it
      const int row = (v >> 2) * 8 + (v & 3);
#pragma unroll
      for (int md = 0; md < MD; ++md) {
        const float x = *reinterpret_cast<const float*>(tile + row * ROWB + (base ^ (uint32_t)(((row & 15) ^ (md * 8)) << 4)));
        acc[md] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w.f[v], acc[md], 0, 0, 0);
      }
    }
  }
};

template <typename T, int D> using RowFrags = typename Mma<T, D>::Frag[Mma<T, D>::KS];
template <typename T, int D> __device__ __forceinline__ uint32_t rows_base(int lane) {
  typedef Mma<T, D> X;
  const int l32 = lane & 31, hf = lane >> 5;
  return (uint32_t)(l32 * X::ROWB + ((hf ^ X::swz(l32)) << 4));
}
template <typename T, int D> __device__ __forceinline__ f32x16 rows(const unsigned char* tile, uint32_t base, const RowFrags<T, D>& f) {
  typedef Mma<T, D> X;
  f32x16 acc = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int ks = 0; ks < X::KS; ++ks) acc = X::mul(*reinterpret_cast<const typename X::Frag*>(tile + (base ^ (uint32_t)(ks << 5))), f[ks], acc);
  return acc;
}
// the lane's row (p: its first element) as the operand of rows(); ok: false gives zeros
template <typename T, int D> __device__ __forceinline__ void row_frags(RowFrags<T, D>& f, const T* p, int hf, bool ok) {
  typedef Mma<T, D> X;
#pragma unroll
  for (int ks = 0; ks < X::KS; ++ks) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (ok) x = *reinterpret_cast<const u32x4_at2*>(p + (2 * ks + hf) * X::VEC);
    f[ks] = __builtin_bit_cast(typename X::Frag, x);
  }
}

// R rows from `base` on, `step` bytes apart, of which `have` exist, straight into LDS at `to`, by NW wavefronts.  Rows that do not exist are out of the
// descriptor's range; what their places in LDS then hold is not relied on (see blank()).
template <typename T, int D, int R, int NW> struct Stage {
  typedef Mma<T, D> X;
  static constexpr int RPI = 64 / X::CPR, NI = R / (RPI * NW);
  static_assert(NI * RPI * NW == R, "rows split evenly over the wavefronts");
  static __device__ __forceinline__ int lane_offset(int k, int wave, int lane, uint32_t step) {
    const int lrow = lane / X::CPR, r = (k * NW + wave) * RPI + lrow;
    return (int)((uint32_t)lrow * step) + (((lane % X::CPR) ^ X::swz(r)) << 4);
  }
  static __device__ __forceinline__ void go(const T* base, uint32_t step, int have, uint32_t to, int wave, int lane) {
    const uint32_t bytes = have > 0 ? (uint32_t)((have < R ? have : R) - 1) * step + X::ROWB : 0u;
    const rsrc_words rsrc = make_rsrc(base, bytes);
#pragma unroll
    for (int k = 0; k < NI; ++k)
      load_lds16(rsrc, to + (uint32_t)((k * NW + wave) * RPI * X::ROWB), lane_offset(k, wave, lane, step), (int)((uint32_t)((k * NW + wave) * RPI) * step));
  }
};
// Zeros in the tile's rows that are not in `keep` (bit: row): a weight of 0 times what lies there has to be 0.
template <typename T, int D, int NT> __device__ __forceinline__ void blank(unsigned char* tile, int R, uint64_t keep, int tid) {
  typedef Mma<T, D> X;
  for (int x = tid; x < R * X::CPR; x += NT)
    if (!(keep >> (x / X::CPR) & 1u)) *reinterpret_cast<u32x4*>(tile + x * 16) = u32x4{0u, 0u, 0u, 0u};
}
__device__ __forceinline__ void tile_arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void lds_ready() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

__device__ __forceinline__ void halves(float x, float& p, float& q) {   // the values of the lane and of the one 32 apart, the lower first
  const uint32_t u = __float_as_uint(x);
  uint32_t u2 = u;
  asm volatile("" : "+v"(u2));                // (two operands: with one value twice both results are taken to be equal)
  const auto r = __builtin_amdgcn_permlane32_swap(u, u2, false, false);
  p = __uint_as_float(r[0]);
  q = __uint_as_float(r[1]);
}

__device__ __forceinline__ int seen_states(const CrossArgs& a, int b) {
  const int n = a.kv_len ? a.kv_len[b] : a.M;
  return n < 0 ? 0 : n < a.M ? n : a.M;
}
// which of R keys from j0 on are seen; `byte`: the lane's byte of the mask (1 without one)
__device__ __forceinline__ uint64_t seen_bits(int byte, int j0, int len, int R, int lane) { return __ballot(lane < R && j0 + lane < len && byte != 0); }
__device__ __forceinline__ int mask_byte(const CrossArgs& a, int b, int j0, int len, int lane) {
  return a.mask && j0 + lane < len ? (int)a.mask[(int64_t)b * a.M + j0 + lane] : 1;
}
// a register's key in a tile of 32: (v / 4) * 8 + hf * 4 + v % 4
__device__ __forceinline__ void hide(f32x16& s, uint32_t bits, int hf) {
  const uint32_t mine = bits >> (hf * 4);
#pragma unroll
  for (int v = 0; v < 16; ++v)
    if (!(mine >> ((v >> 2) * 8 + (v & 3)) & 1u)) s[v] = -INFINITY;
}

template <typename T> constexpr int cross_keys() { return sizeof(T) == 2 ? 64 : 32; }   // keys of a tile

struct CrossRow { int g, n; };
__device__ __forceinline__ CrossRow cross_row(const CrossArgs& a, int r) {
  if (a.group == 1) return {0, r};
  const int g = (int)((uint32_t)r / (uint32_t)a.N);
  return {g, r - g * a.N};
}

// Tiles of consecutive rows, one after the other, straight into LDS: what is fixed is made once.
template <typename T, int D, int R, int NW> struct TileStream {
  typedef Mma<T, D> X;
  static constexpr int RPI = 64 / X::CPR, NI = R / (RPI * NW), OFFS = (16 / RPI + NW - 1) / NW;   // (the permutation of the chunks has period 16)
  uint64_t base;
  uint32_t step;                              // bytes from one row to the next
  int left;                                   // rows from the next tile's first on
  int off[OFFS];
  __device__ __forceinline__ TileStream(const T* from, uint32_t step_, int left_, int wave, int lane) : base((uint64_t)from), step(step_), left(left_) {
#pragma unroll
    for (int k = 0; k < OFFS; ++k) off[k] = Stage<T, D, R, NW>::lane_offset(k, wave, lane, step);
  }
  // the lane's offsets made again, for a caller that has no registers to hold them
  __device__ __forceinline__ void again(int wave) {
#pragma unroll
    for (int k = 0; k < OFFS; ++k) off[k] = Stage<T, D, R, NW>::lane_offset(k, wave, lane_again(), step);
  }
  __device__ __forceinline__ void next(uint32_t to, int wave) {       // `left` > 0
    const rsrc_words rsrc = make_rsrc((const void*)base, (uint32_t)((left < R ? left : R) - 1) * step + X::ROWB);
#pragma unroll
    for (int k = 0; k < NI; ++k)
      load_lds16(rsrc, to + (uint32_t)((k * NW + wave) * RPI * X::ROWB), off[k % OFFS], (int)((uint32_t)((k * NW + wave) * RPI) * step));
    base += (uint64_t)R * step;
    left -= R;
  }
};

// 32 rows of one head, a row in each lane, through a buffer descriptor whose range ends with the head's rows: rows behind it are read as zeros and not written.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const void* base, uint32_t step, int have, int rowb) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, have > 0 ? (int)((uint32_t)((have < 32 ? have : 32) - 1) * step + (uint32_t)rowb) : 0, 0x00020000);
}

// 32 rows of accumulators (one in each lane) to memory through the wavefront's LDS, 16 bytes a lane: at(row) gives the row's address or null
template <typename T, int D, typename F> __device__ __forceinline__ void rows_out(const f32x16 (&acc)[D / 32], float factor, unsigned char* mine, int lane, F&& at) {
  typedef Mma<T, D> X;
  const int l32 = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int md = 0; md < D / 32; ++md)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = acc[md][g4 * 4 + e] * factor;
      const int c = md * 32 + g4 * 8 + hf * 4, chunk = c / X::VEC;
      unsigned char* to = mine + l32 * X::ROWB + ((chunk ^ (l32 & (X::CPR - 1))) << 4);
      if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(to + (c % 8) * 2) = u32x2{f32_to_bf16_pair(x[0], x[1]), f32_to_bf16_pair(x[2], x[3])};
      else *reinterpret_cast<f32x4*>(to) = x;
    }
  constexpr int RPI = 64 / X::CPR;
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int row = i * RPI + lane / X::CPR, chunk = lane % X::CPR;
    T* p = at(row);
    if (p) *reinterpret_cast<u32x4_at2*>(p + chunk * X::VEC) = *reinterpret_cast<const u32x4*>(mine + row * X::ROWB + ((chunk ^ (row & (X::CPR - 1))) << 4));
  }
}

// ... of one head, of which `have` exist, bfloat16: rows behind them are out of the descriptor's range
template <int D> __device__ __forceinline__ void rows_out_head(const f32x16 (&acc)[D / 32], float factor, unsigned char* mine, int lane, bf16_t* to, uint32_t step, int have) {
  typedef Mma<bf16_t, D> X;
  const int l32 = lane & 31, hf = lane >> 5;
  // chunk md * 4 + g4 of the lane's row, at (chunk ^ row) * 16
  unsigned char* row = mine + l32 * X::ROWB + hf * 8;
  const uint32_t turn = (uint32_t)(l32 & (X::CPR - 1)) << 4;
#pragma unroll
  for (int md = 0; md < D / 32; ++md)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      *reinterpret_cast<u32x2*>(row + (turn ^ (uint32_t)((md * 4 + g4) << 4))) =
          u32x2{f32_to_bf16_pair(acc[md][g4 * 4] * factor, acc[md][g4 * 4 + 1] * factor), f32_to_bf16_pair(acc[md][g4 * 4 + 2] * factor, acc[md][g4 * 4 + 3] * factor)};
  constexpr int RPI = 64 / X::CPR;
  const int r0 = lane / X::CPR, chunk = lane % X::CPR;
  const auto rsrc = rows_rsrc(to, step, have, X::ROWB);
  const int off = (int)((uint32_t)r0 * step) + chunk * 16;
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i)
    __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4*>(mine + (i * RPI + r0) * X::ROWB + ((chunk ^ ((i * RPI + r0) & (X::CPR - 1))) << 4)), rsrc, off,
                                           (int)((uint32_t)(i * RPI) * step), 0);
}
// Row sums and outputs of a wavefront's 32 rows; l: the lane's half of the sum.
template <typename T, int D, bool PART>
__device__ __forceinline__ void fwd_out(const f32x16 (&acc)[D / 32], float m_run, float l_run, unsigned char* smem, T* O, float* lse, float* Opart, const CrossArgs& a, int bh, int part,
                                        int wave, int lane, int row0) {
  typedef Mma<T, D> X;
  const int l32 = lane & 31, hf = lane >> 5, row = row0 + l32, b = bh / a.Hkv, hk = bh % a.Hkv;
  const bool active = row < a.rows;
  {
    float p, q;
    halves(l_run, p, q);
    l_run = p + q;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  const float stat = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * CROSS_LN2;
  if constexpr (PART) {
    if (!active) return;
    const int64_t at = ((int64_t)part * a.B * a.Hkv + bh) * a.rows + row;
    float* po = Opart + at * D;
#pragma unroll
    for (int md = 0; md < X::MD; ++md)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4*>(po + md * 32 + g4 * 8 + hf * 4) = f32x4{acc[md][g4 * 4], acc[md][g4 * 4 + 1], acc[md][g4 * 4 + 2], acc[md][g4 * 4 + 3]} * inv;
    if (hf == 0) lse[at] = stat;
  } else {
    if (lse && active && hf == 0) lse[((int64_t)b * a.Hq + hk * a.group) * a.N + row] = stat;
    lds_ready();                              // everyone has read the last tile
    rows_out<T, D>(acc, inv, smem + wave * 32 * X::ROWB, lane, [&](int r) __attribute__((always_inline)) -> T* {
      if (row0 + r >= a.rows) return nullptr;
      const CrossRow c = cross_row(a, row0 + r);
      return O + b * a.o.b + (int64_t)(hk * a.group + c.g) * a.o.h + c.n * a.o.n;
    });
  }
}

template <typename T, int D, int NW, bool PART>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) void cross_fwd_kernel(const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ O,
                                                                float* __restrict__ lse, float* __restrict__ Opart, CrossArgs a) {
  typedef Mma<T, D> X;
  constexpr int BN = cross_keys<T>(), TILEB = BN * X::ROWB, HALVES = BN / 32;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB];   // K, V; K, V
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y, b = bh / a.Hkv, hk = bh % a.Hkv, part = blockIdx.z;
  const int row0 = (int)(blockIdx.x * (NW * 32) + wave * 32), row = row0 + l32;
  const bool active = row < a.rows;
  const int len = seen_states(a, b);
  const int t0 = part * a.tiles_per_part, tiles = (len + BN - 1) / BN, t1 = t0 + a.tiles_per_part < tiles ? t0 + a.tiles_per_part : tiles;
  const T* kb = K + b * a.k.b + hk * a.k.h;
  const T* vb = V + b * a.v.b + hk * a.v.h;
  const uint32_t kstep = (uint32_t)(a.k.n * (int64_t)sizeof(T)), vstep = (uint32_t)(a.v.n * (int64_t)sizeof(T));
  const uint32_t lds = lds_address(smem);
  auto fire = [&](int t) __attribute__((always_inline)) {
    const uint32_t to = lds + (uint32_t)((t - t0) & 1) * 2 * TILEB;
    Stage<T, D, BN, NW>::go(kb + (int64_t)t * BN * a.k.n, kstep, a.M - t * BN, to, wave, lane);
    Stage<T, D, BN, NW>::go(vb + (int64_t)t * BN * a.v.n, vstep, a.M - t * BN, to + TILEB, wave, lane);
  };
  int byte = 1;
  if (t0 < t1) {
    byte = mask_byte(a, b, t0 * BN, len, lane);
    fire(t0);
  }
  typename X::Frag qf[X::KS];
  {
    const CrossRow r = cross_row(a, row);
    row_frags<T, D>(qf, Q + b * a.q.b + (int64_t)(hk * a.group + r.g) * a.q.h + r.n * a.q.n, hf, active);
  }
  f32x16 acc[X::MD];
#pragma unroll
  for (int md = 0; md < X::MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[md][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const uint32_t rbase = rows_base<T, D>(lane), cbase = X::cols_base(lane);
  for (int t = t0; t < t1; ++t) {
    unsigned char* tile = smem + ((t - t0) & 1) * 2 * TILEB;
    const uint64_t seen = seen_bits(byte, t * BN, len, BN, lane);
    tile_arrived();
    if (t + 1 < t1) {
      byte = mask_byte(a, b, (t + 1) * BN, len, lane);
      fire(t + 1);
    }
    const bool whole = seen == (BN == 64 ? ~0ull : 0xffffffffull);
    if (!whole) {
      if (seen == 0) continue;
      blank<T, D, NW * 64>(tile + TILEB, BN, seen, tid);
      lds_ready();
    }
    f32x16 s[HALVES];
#pragma unroll
    for (int u = 0; u < HALVES; ++u) s[u] = rows<T, D>(tile + u * 32 * X::ROWB, rbase, qf);
    if (!whole) {
#pragma unroll
      for (int u = 0; u < HALVES; ++u) hide(s[u], (uint32_t)(seen >> (32 * u)), hf);
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < HALVES; ++u)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, s[u][v]);
    {
      float p, q;
      halves(top * a.scale_log2, p, q);
      top = fmaxf(p, q);
    }
    const bool up = top - m_run > CROSS_LAZY;
    if (__any(up)) {                          // (a row's own maximum decides: its bits do not depend on the rows beside it)
      const float alpha = up ? __builtin_amdgcn_exp2f(m_run - top) : 1.f;
      l_run *= alpha;
#pragma unroll
      for (int md = 0; md < X::MD; ++md)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[md][v] *= alpha;
      m_run = up ? top : m_run;
    }
    const float shift = m_run == -INFINITY ? 0.f : -m_run;
#pragma unroll
    for (int u = 0; u < HALVES; ++u) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[u][v] = __builtin_amdgcn_exp2f(fmaf(s[u][v], a.scale_log2, shift));
        l_run += s[u][v];
      }
      X::cols(acc, tile + TILEB + u * 32 * X::ROWB, cbase, X::weights(s[u]));
    }
  }
  fwd_out<T, D, PART>(acc, m_run, l_run, smem, O, lse, Opart, a, bh, part, wave, lane, row0);
}

// bfloat16: the same, with the order of a tile fixed by hand.  A step makes the scores of tile t + 1 and the second product of tile t, and every MFMA is
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
  const int len = seen_states(a, b);
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
  if (n > 0) ks.next(lds, wave);
  int byte = byte_of(0), byte_next = byte_of(1);

  // the wavefront's rows: of one head, or (flat) the next 32 of the key head's rows
  const int head_blocks = a.flat ? 0x7fffffff : (a.N + NW * 32 - 1) / (NW * 32);
  const int g = a.group == 1 || a.flat ? 0 : (int)blockIdx.x / head_blocks;
  const int n0 = ((int)blockIdx.x - (a.flat ? 0 : g * head_blocks)) * (NW * 32) + wave * 32, row = n0 + l32;   // flat: rows of the key head
  const int have = (a.flat ? a.rows : a.N) - n0;
  typename X::Frag qf[X::KS];
  if (a.flat) {
    const CrossRow r = cross_row(a, row);
    row_frags<bf16_t, D>(qf, Q + b * a.q.b + (int64_t)(hk * a.group + r.g) * a.q.h + r.n * a.q.n, hf, l32 < have);
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
    vs.next(lds + OFF_V, wave);
    if (n > 1) ks.next(lds + TILEB, wave);
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
        if (i + 2 < n) ks.next(lds + PAR * TILEB, wave);
        vs.next(lds + OFF_V + (PAR ^ 1) * TILEB, wave);
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

// dQ of 32 rows a wavefront, and D = dO.O for the kernel after it (parts: the first one's).
template <typename T, int D, int NW, bool PART>
__global__ __launch_bounds__(NW * 64, NW == 4 && (sizeof(T) == 2 || D == 64) ? 2 : 1) void cross_dq_kernel(const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const T* __restrict__ O,
                                                               const float* __restrict__ lse, const T* __restrict__ dO, float* __restrict__ Dr, T* __restrict__ dQ,
                                                               float* __restrict__ dQpart, CrossArgs a) {
  typedef Mma<T, D> X;
  constexpr int BN = cross_keys<T>(), TILEB = BN * X::ROWB, HALVES = BN / 32;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y, b = bh / a.Hkv, hk = bh % a.Hkv, part = blockIdx.z;
  const int row0 = (int)(blockIdx.x * (NW * 32) + wave * 32), row = row0 + l32;
  const bool active = row < a.rows;
  const int len = seen_states(a, b);
  const int t0 = part * a.tiles_per_part, tiles = (len + BN - 1) / BN, t1 = t0 + a.tiles_per_part < tiles ? t0 + a.tiles_per_part : tiles;
  const T* kb = K + b * a.k.b + hk * a.k.h;
  const T* vb = V + b * a.v.b + hk * a.v.h;
  const uint32_t kstep = (uint32_t)(a.k.n * (int64_t)sizeof(T)), vstep = (uint32_t)(a.v.n * (int64_t)sizeof(T));
  const uint32_t lds = lds_address(smem);
  auto fire = [&](int t) __attribute__((always_inline)) {
    const uint32_t to = lds + (uint32_t)((t - t0) & 1) * 2 * TILEB;
    Stage<T, D, BN, NW>::go(kb + (int64_t)t * BN * a.k.n, kstep, a.M - t * BN, to, wave, lane);
    Stage<T, D, BN, NW>::go(vb + (int64_t)t * BN * a.v.n, vstep, a.M - t * BN, to + TILEB, wave, lane);
  };
  int byte = 1;
  if (t0 < t1) {
    byte = mask_byte(a, b, t0 * BN, len, lane);
    fire(t0);
  }
  typename X::Frag qf[X::KS], gf[X::KS];
  const CrossRow r = cross_row(a, row);
  const int head = hk * a.group + r.g;
  const int64_t stat_at = ((int64_t)b * a.Hq + hk * a.group) * a.N + row;
  row_frags<T, D>(qf, Q + b * a.q.b + (int64_t)head * a.q.h + r.n * a.q.n, hf, active);
  row_frags<T, D>(gf, dO + b * a.go.b + (int64_t)head * a.go.h + r.n * a.go.n, hf, active);
  float dot = 0.f;
  {
    const T* op = O + b * a.o.b + (int64_t)head * a.o.h + r.n * a.o.n;
#pragma unroll
    for (int ks = 0; ks < X::KS; ++ks) {
      float x[X::VEC], y[X::VEC];
      u32x4 raw = {0u, 0u, 0u, 0u};
      if (active) raw = *reinterpret_cast<const u32x4_at2*>(op + (2 * ks + hf) * X::VEC);
      Elem<T>::widen(raw, x);
      Elem<T>::widen(__builtin_bit_cast(u32x4, gf[ks]), y);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < X::VEC; ++e) sum = fmaf(x[e], y[e], sum);
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
    if (part == 0 && hf == 0) Dr[stat_at] = dot;
  }
  f32x16 acc[X::MD];
#pragma unroll
  for (int md = 0; md < X::MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[md][v] = 0.f;
  const uint32_t rbase = rows_base<T, D>(lane), cbase = X::cols_base(lane);
  for (int t = t0; t < t1; ++t) {
    unsigned char* tile = smem + ((t - t0) & 1) * 2 * TILEB;
    const uint64_t seen = seen_bits(byte, t * BN, len, BN, lane);
    tile_arrived();
    if (t + 1 < t1) {
      byte = mask_byte(a, b, (t + 1) * BN, len, lane);
      fire(t + 1);
    }
    const bool whole = seen == (BN == 64 ? ~0ull : 0xffffffffull);
    if (!whole) {
      if (seen == 0) continue;
      blank<T, D, NW * 64>(tile, BN, seen, tid);
      blank<T, D, NW * 64>(tile + TILEB, BN, seen, tid);
      lds_ready();
    }
#pragma unroll
    for (int u = 0; u < HALVES; ++u) {
      const unsigned char* kt = tile + u * 32 * X::ROWB;
      f32x16 s = rows<T, D>(kt, rbase, qf);
      const f32x16 g = rows<T, D>(kt + TILEB, rbase, gf);
      if (!whole) hide(s, (uint32_t)(seen >> (32 * u)), hf);
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, shift)) * (g[v] - dot);
      X::cols(acc, kt, cbase, X::weights(s));
    }
  }
  if constexpr (PART) {
    if (!active) return;
    float* po = dQpart + (((int64_t)part * a.B * a.Hkv + bh) * a.rows + row) * D;
#pragma unroll
    for (int md = 0; md < X::MD; ++md)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4)
        *reinterpret_cast<f32x4*>(po + md * 32 + g4 * 8 + hf * 4) = f32x4{acc[md][g4 * 4], acc[md][g4 * 4 + 1], acc[md][g4 * 4 + 2], acc[md][g4 * 4 + 3]};
  } else {
    lds_ready();
    rows_out<T, D>(acc, a.scale, smem + wave * 32 * X::ROWB, lane, [&](int x) __attribute__((always_inline)) -> T* {
      if (row0 + x >= a.rows) return nullptr;
      const CrossRow c = cross_row(a, row0 + x);
      return dQ + b * a.gq.b + (int64_t)(hk * a.group + c.g) * a.gq.h + c.n * a.gq.n;
    });
  }
}

// dK, dV of 32 keys a wavefront: the query rows of the key's group, a head after the other, in tiles of BN tokens.
template <typename T, int D, bool PART>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void cross_dkv_kernel(const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V, const float* __restrict__ lse,
                                                       const T* __restrict__ dO, const float* __restrict__ Dr, T* __restrict__ dK, T* __restrict__ dV,
                                                       float* __restrict__ dKpart, float* __restrict__ dVpart, CrossArgs a) {
  typedef Mma<T, D> X;
  constexpr int NW = 4, BN = cross_keys<T>(), TILEB = BN * X::ROWB, OFF_STAT = 4 * TILEB, STATS = 64;   // (a load of the statistics is 64 lanes wide)
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB + 2 * 2 * STATS * 4];   // Q, dO; Q, dO; lse, D; lse, D
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y, b = bh / a.Hkv, hk = bh % a.Hkv, part = blockIdx.z;
  const int key0 = (int)(blockIdx.x * (NW * 32) + wave * 32), key = key0 + l32;
  const int len = seen_states(a, b);
  const bool seen = key < len && (!a.mask || a.mask[(int64_t)b * a.M + key] != 0);
  const bool any = __syncthreads_or(seen);
  const int all = any ? a.group * a.chunks : 0;
  const int t0 = part * a.tiles_per_part, t1 = t0 + a.tiles_per_part < all ? t0 + a.tiles_per_part : all;
  const uint32_t qstep = (uint32_t)(a.q.n * (int64_t)sizeof(T)), gstep = (uint32_t)(a.go.n * (int64_t)sizeof(T));
  const uint32_t lds = lds_address(smem);
  auto fire = [&](int t) __attribute__((always_inline)) {
    const int g = t / a.chunks, n0 = (t - g * a.chunks) * BN, head = hk * a.group + g, at = (t - t0) & 1;
    const uint32_t to = lds + (uint32_t)at * 2 * TILEB;
    Stage<T, D, BN, NW>::go(Q + b * a.q.b + (int64_t)head * a.q.h + (int64_t)n0 * a.q.n, qstep, a.N - n0, to, wave, lane);
    Stage<T, D, BN, NW>::go(dO + b * a.go.b + (int64_t)head * a.go.h + (int64_t)n0 * a.go.n, gstep, a.N - n0, to + TILEB, wave, lane);
    if (wave < 2) {
      const float* from = (wave ? Dr : lse) + ((int64_t)b * a.Hq + head) * a.N + n0;
      const int have = a.N - n0 < BN ? a.N - n0 : BN;
      const rsrc_words rsrc = make_rsrc(from, (uint32_t)have * 4);
      load_lds4(rsrc, lds + (uint32_t)(OFF_STAT + (at * 2 + wave) * STATS * 4), lane * 4, 0);
    }
  };
  if (t0 < t1) fire(t0);
  typename X::Frag kf[X::KS], vf[X::KS];
  row_frags<T, D>(kf, K + b * a.k.b + hk * a.k.h + key * a.k.n, hf, seen);
  row_frags<T, D>(vf, V + b * a.v.b + hk * a.v.h + key * a.v.n, hf, seen);
  f32x16 dk[X::MD], dv[X::MD];
#pragma unroll
  for (int md = 0; md < X::MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[md][v] = dv[md][v] = 0.f;
  const uint32_t rbase = rows_base<T, D>(lane), cbase = X::cols_base(lane);
  for (int t = t0; t < t1; ++t) {
    const int at = (t - t0) & 1, have = a.N - t % a.chunks * BN;
    unsigned char* tile = smem + at * 2 * TILEB;
    float* stat = reinterpret_cast<float*>(smem + OFF_STAT + at * 2 * STATS * 4);
    tile_arrived();
    if (t + 1 < t1) fire(t + 1);
    if (have < BN) {
      const uint64_t keep = (1ull << have) - 1ull;
      blank<T, D, 256>(tile, BN, keep, tid);
      blank<T, D, 256>(tile + TILEB, BN, keep, tid);
      if (tid < BN && tid >= have) {
        stat[tid] = INFINITY;
        stat[STATS + tid] = 0.f;
      }
      lds_ready();
    }
#pragma unroll
    for (int u = 0; u < BN / 32; ++u) {
      const unsigned char* qt = tile + u * 32 * X::ROWB;
      f32x16 s = rows<T, D>(qt, rbase, kf), g = rows<T, D>(qt + TILEB, rbase, vf);
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const f32x4 l = *reinterpret_cast<const f32x4*>(stat + u * 32 + g4 * 8 + hf * 4), d = *reinterpret_cast<const f32x4*>(stat + STATS + u * 32 + g4 * 8 + hf * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int v = g4 * 4 + e;
          s[v] = l[e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, -l[e] * CROSS_LOG2E));
          g[v] = s[v] * (g[v] - d[e]);
        }
      }
      X::cols(dv, qt + TILEB, cbase, X::weights(s));
      X::cols(dk, qt, cbase, X::weights(g));
    }
  }
  if constexpr (PART) {
    if (key >= a.M) return;
    const int64_t to = (((int64_t)part * a.B * a.Hkv + bh) * a.M + key) * D;
#pragma unroll
    for (int md = 0; md < X::MD; ++md)
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
    if (!seen) {
#pragma unroll
      for (int md = 0; md < X::MD; ++md)
#pragma unroll
        for (int v = 0; v < 16; ++v) dk[md][v] = dv[md][v] = 0.f;
    }
    lds_ready();
    unsigned char* mine = smem + wave * 32 * X::ROWB;
    rows_out<T, D>(dk, a.scale, mine, lane, [&](int x) __attribute__((always_inline)) -> T* {
      return key0 + x < a.M ? dK + b * a.gk.b + hk * a.gk.h + (int64_t)(key0 + x) * a.gk.n : nullptr;
    });
    rows_out<T, D>(dv, 1.f, mine, lane, [&](int x) __attribute__((always_inline)) -> T* {
      return key0 + x < a.M ? dV + b * a.gv.b + hk * a.gv.h + (int64_t)(key0 + x) * a.gv.n : nullptr;
    });
  }
}

// ---- bfloat16 gradients with the order of a tile fixed by hand: every operand fragment is requested two MFMAs ahead, and a slice of the vector work stands behind each MFMA.

// 32 x 32 scores' fragments for the second products: pairs q = 0 .. 7 of registers 2q, 2q + 1
struct WeightPairs {
  uint32_t w[8];
  __device__ __forceinline__ void put(int q, float x, float y) {
    uint32_t bits = f32_to_bf16_pair(x, y);
    asm volatile("" : "+v"(bits));            // made here, not where it is used
    w[q] = bits;
  }
  __device__ __forceinline__ bf16x8 frag(int f) const { return __builtin_bit_cast(bf16x8, (u32x4{w[4 * f], w[4 * f + 1], w[4 * f + 2], w[4 * f + 3]})); }
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
      row_frags<bf16_t, D>(qf, Q + b * a.q.b + (int64_t)(head + r.g) * a.q.h + r.n * a.q.n, hf, active);
      row_frags<bf16_t, D>(gf, dO + b * a.go.b + (int64_t)(head + r.g) * a.go.h + r.n * a.go.n, hf, active);
      typename X::Frag x[KS];
      row_frags<bf16_t, D>(x, O + b * a.o.b + (int64_t)(head + r.g) * a.o.h + r.n * a.o.n, hf, active);
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
    WeightPairs w[2];
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
        acc[c % MD] = X::mul(fr.template get<j>(), w[u].frag(c / MD), acc[c % MD]);
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
template <int D, bool PART>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void cross_dkv_bf16_kernel(const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const float* __restrict__ stats,
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
  const bool any = __syncthreads_or(seen);
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
    row_frags<bf16_t, D>(kf, K + b * a.k.b + hk * a.k.h + key * a.k.n, hf, seen);
    row_frags<bf16_t, D>(vf, V + b * a.v.b + hk * a.v.h + key * a.v.n, hf, seen);
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
        if (u * 32 >= have) break;
        const unsigned char* qt = tile + u * 32 * X::ROWB;
        const float* sl = stat + u * 32 + (lane_again() >> 5) * 4;
        Fragments<D, D == 128> fr;
        f32x16 s, dp;
        WeightPairs w;
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
          else if constexpr (j < 2 * KS + 2 * MD) dv[(j - 2 * KS) % MD] = X::mul(fr.template get<j>(), w.frag((j - 2 * KS) / MD), dv[(j - 2 * KS) % MD]);
          else dk[(j - 2 * KS) % MD] = X::mul(fr.template get<j>(), w.frag((j - 2 * KS - 2 * MD) / MD), dk[(j - 2 * KS) % MD]);
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

// out[b, h, l, :] = factor * sum over the parts, in their order; two tensors of one shape in one launch (blockIdx.y)
template <typename T> struct CrossSum {
  const float* part[2];
  T* out[2];
  float factor[2];
  Strides to[2];
  int H, L, parts;
  int64_t total;                              // rows
};
template <typename T, int D> __global__ __launch_bounds__(256) void cross_sum_kernel(CrossSum<T> p) {
  constexpr int LANES = D / 4, AHEAD = 8;
  const int64_t x = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (x >= p.total) return;
  const int c = threadIdx.x % LANES, which = blockIdx.y;
  const float* part = p.part[which] + x * D + c * 4;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < p.parts; s0 += AHEAD) {
    f32x4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) v[u] = *reinterpret_cast<const f32x4*>(part + (s0 + u < p.parts ? s0 + u : p.parts - 1) * p.total * D);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u < p.parts) sum += v[u];
  }
  const Strides to = p.to[which];
  const int64_t bh = x / p.L;
  Four<T>::store(p.out[which] + bh / p.H * to.b + bh % p.H * to.h + (x - bh * p.L) * to.n + c * 4, sum * p.factor[which]);
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
  return a;
}
static void cross_share(CrossArgs& a, int parts, int tiles) {
  a.parts = parts;
  a.tiles_per_part = parts > 0 ? (tiles + parts - 1) / parts : tiles;
}

template <typename T, int D>
static void launch_cross_fwd_t(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, void* O, float* lse, float* part, float* stats, hipStream_t s) {
  CrossArgs a = cross_args(pl, c);
  const int nw = cross_waves(pl);
  cross_share(a, cross_key_parts(pl, c.M, false), (c.M + cross_keys<T>() - 1) / cross_keys<T>());
  a.flat = cross_flat(pl);
  const dim3 grid((unsigned)(a.flat ? (a.rows + nw * 32 - 1) / (nw * 32) : pl.group * ((pl.N + nw * 32 - 1) / (nw * 32))), (unsigned)(pl.B * pl.Hkv), (unsigned)a.parts);
  const bool split = a.parts > 1;
  auto go = [&](auto kernel) {
    kernel<<<grid, nw * 64, 0, s>>>(static_cast<const T*>(Q), static_cast<const T*>(K), static_cast<const T*>(V), static_cast<T*>(O), split ? stats : lse, part, a);
  };
  if constexpr (sizeof(T) == 2) {
    if (nw == 1) split ? go(cross_fwd_bf16_kernel<D, 1, true>) : go(cross_fwd_bf16_kernel<D, 1, false>);
    else if (nw == 2) split ? go(cross_fwd_bf16_kernel<D, 2, true>) : go(cross_fwd_bf16_kernel<D, 2, false>);
    else split ? go(cross_fwd_bf16_kernel<D, 4, true>) : go(cross_fwd_bf16_kernel<D, 4, false>);
  } else {
    if (nw == 1) split ? go(cross_fwd_kernel<T, D, 1, true>) : go(cross_fwd_kernel<T, D, 1, false>);
    else if (nw == 2) split ? go(cross_fwd_kernel<T, D, 2, true>) : go(cross_fwd_kernel<T, D, 2, false>);
    else split ? go(cross_fwd_kernel<T, D, 4, true>) : go(cross_fwd_kernel<T, D, 4, false>);
  }
  if (!split) return;
  const int64_t total = (int64_t)pl.B * pl.Hq * pl.N, per = 256 / (D / 4);
  cross_join_kernel<T, D><<<(unsigned)((total + per - 1) / per), 256, 0, s>>>(part, stats, static_cast<T*>(O), lse, a);
}

hipError_t launch_cross_fwd(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, void* O, float* lse, float* part, float* stats, hipStream_t s) {
  if (pl.dtype == PSA_BF16) pl.d == 128 ? launch_cross_fwd_t<bf16_t, 128>(pl, c, Q, K, V, O, lse, part, stats, s) : launch_cross_fwd_t<bf16_t, 64>(pl, c, Q, K, V, O, lse, part, stats, s);
  else pl.d == 128 ? launch_cross_fwd_t<float, 128>(pl, c, Q, K, V, O, lse, part, stats, s) : launch_cross_fwd_t<float, 64>(pl, c, Q, K, V, O, lse, part, stats, s);
  return hipGetLastError();
}

template <typename T, int D>
static void launch_cross_bwd_t(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, const void* O, const float* lse, const void* dO, void* dQ, void* dK,
                               void* dV, float* Dr, float* dQpart, float* dKpart, float* dVpart, hipStream_t s) {
  CrossArgs a = cross_args(pl, c);
  const T *q = static_cast<const T*>(Q), *k = static_cast<const T*>(K), *v = static_cast<const T*>(V), *o = static_cast<const T*>(O), *g = static_cast<const T*>(dO);
  const int nw = cross_waves(pl), per = 256 / (D / 4);
  cross_share(a, cross_key_parts(pl, c.M, true), (c.M + cross_keys<T>() - 1) / cross_keys<T>());
  a.flat = cross_flat(pl);
  {
    const dim3 grid((unsigned)(a.flat ? (a.rows + nw * 32 - 1) / (nw * 32) : pl.group * ((pl.N + nw * 32 - 1) / (nw * 32))), (unsigned)(pl.B * pl.Hkv), (unsigned)a.parts);
    const bool split = a.parts > 1;
    auto go = [&](auto kernel) { kernel<<<grid, nw * 64, 0, s>>>(q, k, v, o, lse, g, Dr, static_cast<T*>(dQ), dQpart, a); };
    if constexpr (sizeof(T) == 2) {
      if (nw == 1) split ? go(cross_dq_bf16_kernel<D, 1, true>) : go(cross_dq_bf16_kernel<D, 1, false>);
      else if (nw == 2) split ? go(cross_dq_bf16_kernel<D, 2, true>) : go(cross_dq_bf16_kernel<D, 2, false>);
      else split ? go(cross_dq_bf16_kernel<D, 4, true>) : go(cross_dq_bf16_kernel<D, 4, false>);
    } else {
      if (nw == 1) split ? go(cross_dq_kernel<T, D, 1, true>) : go(cross_dq_kernel<T, D, 1, false>);
      else if (nw == 2) split ? go(cross_dq_kernel<T, D, 2, true>) : go(cross_dq_kernel<T, D, 2, false>);
      else split ? go(cross_dq_kernel<T, D, 4, true>) : go(cross_dq_kernel<T, D, 4, false>);
    }
    const int64_t total = (int64_t)pl.B * pl.Hq * pl.N;
    if (split)
      cross_sum_kernel<T, D><<<dim3((unsigned)((total + per - 1) / per), 1), 256, 0, s>>>(
          CrossSum<T>{{dQpart, nullptr}, {static_cast<T*>(dQ), nullptr}, {pl.scale, 0.f}, {c.gq, c.gq}, pl.Hq, pl.N, a.parts, total});
  }
  if (c.M == 0) return;
  cross_share(a, cross_row_parts(pl, c.M), pl.group * a.chunks);
  const dim3 grid((unsigned)((c.M + 127) / 128), (unsigned)(pl.B * pl.Hkv), (unsigned)a.parts);
  auto go = [&](auto kernel) {
    if constexpr (sizeof(T) == 2) kernel<<<grid, 256, 0, s>>>(q, k, v, Dr, g, static_cast<T*>(dK), static_cast<T*>(dV), dKpart, dVpart, a);
    else kernel<<<grid, 256, 0, s>>>(q, k, v, lse, g, Dr, static_cast<T*>(dK), static_cast<T*>(dV), dKpart, dVpart, a);
  };
  auto gradients = [&](auto split) {
    if constexpr (sizeof(T) == 2) go(cross_dkv_bf16_kernel<D, decltype(split)::value>);
    else go(cross_dkv_kernel<T, D, decltype(split)::value>);
  };
  if (a.parts > 1) {
    gradients(std::true_type{});
    const int64_t total = (int64_t)pl.B * pl.Hkv * c.M;
    cross_sum_kernel<T, D><<<dim3((unsigned)((total + per - 1) / per), 2), 256, 0, s>>>(
        CrossSum<T>{{dKpart, dVpart}, {static_cast<T*>(dK), static_cast<T*>(dV)}, {pl.scale, 1.f}, {c.gk, c.gv}, pl.Hkv, c.M, a.parts, total});
  } else {
    gradients(std::false_type{});
  }
}

hipError_t launch_cross_bwd(const Plan& pl, const CrossCall& c, const void* Q, const void* K, const void* V, const void* O, const float* lse, const void* dO, void* dQ, void* dK,
                            void* dV, float* Dr, float* dQpart, float* dKpart, float* dVpart, hipStream_t s) {
  auto go = [&](auto f) { f(pl, c, Q, K, V, O, lse, dO, dQ, dK, dV, Dr, dQpart, dKpart, dVpart, s); };
  if (pl.dtype == PSA_BF16) pl.d == 128 ? go(launch_cross_bwd_t<bf16_t, 128>) : go(launch_cross_bwd_t<bf16_t, 64>);
  else pl.d == 128 ? go(launch_cross_bwd_t<float, 128>) : go(launch_cross_bwd_t<float, 64>);
  return hipGetLastError();
}

}  // namespace psa
