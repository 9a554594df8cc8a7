// Cross attention on the matrix cores: what the kernels of cross_bf16.hip and cross_f32.hip share.  Both are made of two products on 32 x 32 tiles:
//   rows:  [32 rows of a tile in LDS] x [32 rows in registers]^T   -> one register row in each lane, the tile's rows in its registers
//   cols:  [32 rows of a tile in LDS]^T x [that result]            -> the result is the second operand as it lies, no lane exchange
#pragma once
#include "psa_dev.h"
#include "psa_internal.h"

namespace psa {

struct CrossArgs {
  int B, Hq, Hkv, group, N, M;
  int rows;                                   // group * N: query rows of a key head
  int flat;                                   // a block of rows may hold rows of several heads
  int once;                                   // forward: the keys and values are read by one workgroup each and do not fit the memory-side cache
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
};

template <int D> struct Mma<float, D> {
  static constexpr int ROWB = D * 4, CPR = D / 4, MD = D / 32, VEC = 4;
  static __device__ __forceinline__ int swz(int row) { return row & 15; }
};

// the lane's part of a row of 32 in LDS, 16 bytes; chunk 2 k further on: base ^ k * 32
template <typename T, int D> __device__ __forceinline__ uint32_t rows_base(int lane) {
  typedef Mma<T, D> X;
  const int l32 = lane & 31, hf = lane >> 5;
  return (uint32_t)(l32 * X::ROWB + ((hf ^ X::swz(l32)) << 4));
}
// the lane's row (p: its first element) as the operand of the products with rows, bfloat16; ok: false gives zeros
template <int D> __device__ __forceinline__ void row_frags(bf16x8 (&f)[D / 16], const bf16_t* p, int hf, bool ok) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (ok) x = *reinterpret_cast<const u32x4_at2*>(p + (2 * ks + hf) * 8);
    f[ks] = __builtin_bit_cast(bf16x8, x);
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
  __device__ __forceinline__ void next(uint32_t to, int wave, bool once = false) {       // `left` > 0
    const rsrc_words rsrc = make_rsrc((const void*)base, (uint32_t)((left < R ? left : R) - 1) * step + X::ROWB);
    auto load = [&](auto&& from) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < NI; ++k)
        from(rsrc, to + (uint32_t)((k * NW + wave) * RPI * X::ROWB), off[k % OFFS], (int)((uint32_t)((k * NW + wave) * RPI) * step));
    };
    if (once) load(load_lds16_once);
    else load(load_lds16);
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

// ... of one head, of which `have` exist, bfloat16: rows behind them are out of the descriptor's range.  The stores are non-temporal (40 heads x 75600 tokens x 512 states
// 947 -> 915 us).
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
                                           (int)((uint32_t)(i * RPI) * step), 2);
}
// Launches of one type's kernels.  part: partial results into Opart (lse: theirs), dQpart, dKpart, dVpart; stats: -lse log2(e) of every query row, then -D.
#define CROSS_LAUNCHES(T)                                                                                                                                                        \
  void cross_fwd(const CrossArgs& a, int d, dim3 grid, int nw, bool part, const T* Q, const T* K, const T* V, T* O, float* lse, float* Opart, hipStream_t s);                      \
  void cross_dq(const CrossArgs& a, int d, dim3 grid, int nw, bool part, const T* Q, const T* K, const T* V, const T* O, const float* lse, const T* dO, float* stats, T* dQ,       \
                float* dQpart, hipStream_t s);                                                                                                                                    \
  void cross_dkv(const CrossArgs& a, int d, dim3 grid, bool part, const T* Q, const T* K, const T* V, const float* stats, const T* dO, T* dK, T* dV, float* dKpart, float* dVpart, \
                 hipStream_t s);
CROSS_LAUNCHES(bf16_t)
CROSS_LAUNCHES(float)
#undef CROSS_LAUNCHES

}  // namespace psa
