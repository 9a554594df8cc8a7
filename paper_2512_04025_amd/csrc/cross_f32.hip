// Cross attention and its gradients (see cross.hip), float32.
//
// The fp32 matrix instructions (32x32x2: 64 cycles for 2 channels, bfloat16's 32 for 16: a sixteenth of the rate) bound every kernel here: 4096 cycles for 32 x 32 x 128 on a SIMD.  Operands
// are requested a step ahead, and where two products share their shape their instructions take turns.  (Three bfloat16 planes of every operand, made from the tile
// for each product, were slower: gradients of 12 heads x 1000 tokens x 301 states at d = 128 107 -> 132 us.)
#include "cross_dev.h"

namespace psa {

// 32 rows in registers, one in each pair of lanes 32 apart: of every eight channels a lane half has four
template <int D> struct RowSide {
  f32x4 f[D / 8];
  __device__ __forceinline__ void load(const float* p, int lane, bool ok) {
#pragma unroll
    for (int k = 0; k < D / 8; ++k) {
      f[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (ok) f[k] = Four<float>::load(p + k * 8 + (lane >> 5) * 4);
    }
  }
};

// acc[i] = [32 rows at tile[i]] x [rows in registers]^T, of one or two pairs at a time
template <int D, int N> __device__ __forceinline__ void rows(f32x16 (&acc)[N], const unsigned char* const (&tile)[N], int lane, const RowSide<D>* const (&r)[N]) {
  const uint32_t base = rows_base<float, D>(lane);
  f32x4 v[2][N];
  auto read = [&](int k) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[k & 1][i] = *reinterpret_cast<const f32x4*>(tile[i] + (base ^ (uint32_t)(k << 5)));
  };
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
  read(0);
#pragma unroll
  for (int k = 0; k < D / 8; ++k) {
    if (k + 1 < D / 8) read(k + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[k & 1][i][c], r[i]->f[k][c], acc[i], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// acc += [32 rows at `tile`]^T x p
template <int D> __device__ __forceinline__ void cols(f32x16 (&acc)[D / 32], const unsigned char* tile, int lane, const f32x16& p) {
  typedef Mma<float, D> X;
  constexpr int MD = D / 32;
  const int l32 = lane & 31, hf = lane >> 5;
  // register v of p: row (v / 4) * 8 + v % 4, and in the upper lanes 4 after it
  const uint32_t base = (uint32_t)(hf * 4 * X::ROWB + (((l32 >> 2) ^ (hf * 4)) << 4) + (l32 & 3) * 4);
  float x[2][MD];
  auto read = [&](int v) __attribute__((always_inline)) {
    const int row = (v >> 2) * 8 + (v & 3);
#pragma unroll
    for (int md = 0; md < MD; ++md) x[v & 1][md] = *reinterpret_cast<const float*>(tile + row * X::ROWB + (base ^ (uint32_t)(((row & 15) ^ (md * 8)) << 4)));
  };
  read(0);
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    if (v + 1 < 16) read(v + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int md = 0; md < MD; ++md) acc[md] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[v & 1][md], p[v], acc[md], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}

constexpr int BN = 32;                        // rows of a tile

// Of a forward or dQ workgroup: its rows, its tiles of keys, their loads
template <int D, int NW> struct KeyWalk {
  typedef Mma<float, D> X;
  static constexpr int TILEB = BN * X::ROWB;
  int lane, wave, b, hk, bh, part, len, t0, t1, row0, row;
  bool active;
  int byte;
  uint32_t lds;
  TileStream<float, D, BN, NW> ks, vs;
  __device__ __forceinline__ KeyWalk(const float* K, const float* V, const CrossArgs& a, unsigned char* smem)
      : lane(threadIdx.x & 63), wave(NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), ks(K, (uint32_t)(a.k.n * 4), a.M, wave, lane), vs(V, (uint32_t)(a.v.n * 4), a.M, wave, lane) {
    bh = blockIdx.y;
    b = bh / a.Hkv;
    hk = bh - b * a.Hkv;
    part = blockIdx.z;
    row0 = (int)(blockIdx.x * (NW * 32) + wave * 32);
    row = row0 + (lane & 31);
    active = row < a.rows;
    len = __builtin_amdgcn_readfirstlane(seen_states(a, b));
    t0 = part * a.tiles_per_part;
    const int tiles = (len + BN - 1) / BN;
    t1 = t0 + a.tiles_per_part < tiles ? t0 + a.tiles_per_part : tiles;
    ks.base = (uint64_t)(K + b * a.k.b + hk * a.k.h + (int64_t)t0 * BN * a.k.n);
    vs.base = (uint64_t)(V + b * a.v.b + hk * a.v.h + (int64_t)t0 * BN * a.v.n);
    ks.left = vs.left = a.M - t0 * BN;
    lds = lds_address(smem);
    byte = 1;
    if (t0 < t1) {
      byte = mask_byte(a, b, t0 * BN, len, lane);
      fire(t0);
    }
  }
  __device__ __forceinline__ void fire(int t) {
    const uint32_t to = lds + (uint32_t)((t - t0) & 1) * 2 * TILEB;
    ks.next(to, wave);
    vs.next(to + TILEB, wave);
  }
  // Tile t has arrived and the next is requested; which keys of it are seen.  Rows that are not are zeros then.
  __device__ __forceinline__ uint32_t arrive(int t, const CrossArgs& a, unsigned char* smem) {
    unsigned char* tile = smem + ((t - t0) & 1) * 2 * TILEB;
    const uint32_t seen = (uint32_t)seen_bits(byte, t * BN, len, BN, lane);
    tile_arrived();
    if (t + 1 < t1) {
      byte = mask_byte(a, b, (t + 1) * BN, len, lane);
      fire(t + 1);
    }
    if (seen != 0xffffffffu && seen != 0u) {
      blank<float, D, NW * 64>(tile, BN, seen, threadIdx.x);
      blank<float, D, NW * 64>(tile + TILEB, BN, seen, threadIdx.x);
      lds_ready();
    }
    return seen;
  }
};

template <int D, int NW, bool PART>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) void cross_fwd_f32_kernel(const float* __restrict__ Q, const float* __restrict__ K, const float* __restrict__ V, float* __restrict__ O,
                                                                                float* __restrict__ lse, float* __restrict__ Opart, CrossArgs a) {
  typedef Mma<float, D> X;
  constexpr int TILEB = BN * X::ROWB;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB];   // K, V; K, V
  KeyWalk<D, NW> k(K, V, a, smem);
  const int lane = k.lane, hf = lane >> 5;
  RowSide<D> q;
  {
    const CrossRow r = cross_row(a, k.row);
    q.load(Q + k.b * a.q.b + (int64_t)(k.hk * a.group + r.g) * a.q.h + r.n * a.q.n, lane, k.active);
  }
  f32x16 acc[X::MD];
#pragma unroll
  for (int md = 0; md < X::MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[md][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  for (int t = k.t0; t < k.t1; ++t) {
    const unsigned char* tile = smem + ((t - k.t0) & 1) * 2 * TILEB;
    const uint32_t seen = k.arrive(t, a, smem);
    if (seen == 0u) continue;
    f32x16 one[1];
    rows<D, 1>(one, {tile}, lane, {&q});
    f32x16& s = one[0];
    if (seen != 0xffffffffu) hide(s, seen, hf);
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; ++v) top = fmaxf(top, s[v]);
    {
      float x, y;
      halves(top * a.scale_log2, x, y);
      top = fmaxf(x, y);
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
    for (int v = 0; v < 16; ++v) {
      s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, shift));
      l_run += s[v];
    }
    cols<D>(acc, tile + TILEB, lane, s);
  }
  {
    float x, y;
    halves(l_run, x, y);
    l_run = x + y;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  const float stat = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * CROSS_LN2;
  const int64_t at = ((int64_t)k.part * a.B * a.Hkv + k.bh) * a.rows + k.row0;
  if (lse && k.active && hf == 0) lse[PART ? at + (lane & 31) : ((int64_t)k.b * a.Hq + k.hk * a.group) * a.N + k.row] = stat;
  lds_ready();                                // everyone has read the last tile
  rows_out<float, D>(acc, inv, smem + k.wave * 32 * X::ROWB, lane, [&](int r) __attribute__((always_inline)) -> float* {
    if (k.row0 + r >= a.rows) return nullptr;
    if constexpr (PART) return Opart + (at + r) * D;
    const CrossRow c = cross_row(a, k.row0 + r);
    return O + k.b * a.o.b + (int64_t)(k.hk * a.group + c.g) * a.o.h + c.n * a.o.n;
  });
}

// dQ of 32 rows a wavefront; and for the kernel after it -D, D = dO.O, and -lse log2(e) of every row (parts: the first one's)
template <int D, int NW, bool PART>
__global__ __launch_bounds__(NW * 64, NW == 4 && D == 64 ? 2 : 1) void cross_dq_f32_kernel(const float* __restrict__ Q, const float* __restrict__ K, const float* __restrict__ V,
                                                                                          const float* __restrict__ O, const float* __restrict__ lse, const float* __restrict__ dO,
                                                                                          float* __restrict__ stats, float* __restrict__ dQ, float* __restrict__ dQpart, CrossArgs a) {
  typedef Mma<float, D> X;
  constexpr int TILEB = BN * X::ROWB;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILEB];
  KeyWalk<D, NW> k(K, V, a, smem);
  const int lane = k.lane, hf = lane >> 5;
  const CrossRow r = cross_row(a, k.row);
  const int head = k.hk * a.group + r.g;
  const int64_t stat_at = ((int64_t)k.b * a.Hq + k.hk * a.group) * a.N + k.row;
  RowSide<D> q, g;
  float dot = 0.f;
  {
    RowSide<D> o;
    g.load(dO + k.b * a.go.b + (int64_t)head * a.go.h + r.n * a.go.n, lane, k.active);
    o.load(O + k.b * a.o.b + (int64_t)head * a.o.h + r.n * a.o.n, lane, k.active);
    q.load(Q + k.b * a.q.b + (int64_t)head * a.q.h + r.n * a.q.n, lane, k.active);
#pragma unroll
    for (int c = 0; c < D / 8; ++c) dot += fmaf(o.f[c][0], g.f[c][0], o.f[c][1] * g.f[c][1]) + fmaf(o.f[c][2], g.f[c][2], o.f[c][3] * g.f[c][3]);
  }
  {
    float x, y;
    halves(dot, x, y);
    dot = x + y;
  }
  float shift = -INFINITY;                    // weights of 0 for a row that sees nothing
  if (k.active) {
    const float l = lse[stat_at];
    if (l != -INFINITY) shift = -l * CROSS_LOG2E;
    if (k.part == 0 && hf == 0) {
      stats[stat_at] = shift;
      stats[(int64_t)a.B * a.Hq * a.N + stat_at] = -dot;
    }
  }
  f32x16 acc[X::MD];
#pragma unroll
  for (int md = 0; md < X::MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[md][v] = 0.f;
  for (int t = k.t0; t < k.t1; ++t) {
    const unsigned char* tile = smem + ((t - k.t0) & 1) * 2 * TILEB;
    const uint32_t seen = k.arrive(t, a, smem);
    if (seen == 0u) continue;
    f32x16 two[2];
    rows<D, 2>(two, {tile, tile + TILEB}, lane, {&q, &g});
    f32x16 &s = two[0], &dp = two[1];
    if (seen != 0xffffffffu) hide(s, seen, hf);
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, shift)) * (dp[v] - dot);
    cols<D>(acc, tile, lane, s);
  }
  lds_ready();                                // everyone has read the last tile
  rows_out<float, D>(acc, PART ? 1.f : a.scale, smem + k.wave * 32 * X::ROWB, lane, [&](int x) __attribute__((always_inline)) -> float* {
    if (k.row0 + x >= a.rows) return nullptr;
    if constexpr (PART) return dQpart + (((int64_t)k.part * a.B * a.Hkv + k.bh) * a.rows + k.row0 + x) * D;
    const CrossRow c = cross_row(a, k.row0 + x);
    return dQ + k.b * a.gq.b + (int64_t)(k.hk * a.group + c.g) * a.gq.h + c.n * a.gq.n;
  });
}

// dK, dV of 32 keys a wavefront: the query rows of the key's group, a head after the other, in tiles of 32 tokens
template <int D, bool PART>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void cross_dkv_f32_kernel(const float* __restrict__ Q, const float* __restrict__ K, const float* __restrict__ V, const float* __restrict__ stats,
                                                                            const float* __restrict__ dO, float* __restrict__ dK, float* __restrict__ dV, float* __restrict__ dKpart,
                                                                            float* __restrict__ dVpart, CrossArgs a) {
  typedef Mma<float, D> X;
  constexpr int NW = 4, TILEB = BN * X::ROWB, OFF_STAT = 4 * TILEB, STATS = 64;     // (a load of the statistics is 64 lanes wide)
  __shared__ __attribute__((aligned(1024))) unsigned char smem[OFF_STAT + 2 * 2 * STATS * 4];   // Q, dO; Q, dO; -lse log2(e), -D; the same
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.y, b = bh / a.Hkv, hk = bh - b * a.Hkv, part = blockIdx.z;
  const int key0 = (int)(blockIdx.x * (NW * 32) + wave * 32), key = key0 + l32;
  const int len = __builtin_amdgcn_readfirstlane(seen_states(a, b));
  const bool seen = key < len && (!a.mask || a.mask[(int64_t)b * a.M + key] != 0);
  const bool any = __syncthreads_or(seen), mine = __any(seen);       // a wavefront none of whose keys is seen loads for the others
  const int all = any ? a.group * a.chunks : 0;
  const int t0 = part * a.tiles_per_part, t1 = t0 + a.tiles_per_part < all ? t0 + a.tiles_per_part : all;
  const uint32_t lds = lds_address(smem), qstep = (uint32_t)(a.q.n * 4), gstep = (uint32_t)(a.go.n * 4);
  auto fire = [&](int t) __attribute__((always_inline)) {
    const int g = t / a.chunks, n0 = (t - g * a.chunks) * BN, head = hk * a.group + g, at = (t - t0) & 1;
    const uint32_t to = lds + (uint32_t)at * 2 * TILEB;
    Stage<float, D, BN, NW>::go(Q + b * a.q.b + (int64_t)head * a.q.h + (int64_t)n0 * a.q.n, qstep, a.N - n0, to, wave, lane);
    Stage<float, D, BN, NW>::go(dO + b * a.go.b + (int64_t)head * a.go.h + (int64_t)n0 * a.go.n, gstep, a.N - n0, to + TILEB, wave, lane);
    if (wave < 2) {
      const float* from = stats + (wave ? (int64_t)a.B * a.Hq * a.N : 0) + ((int64_t)b * a.Hq + head) * a.N + n0;
      const rsrc_words rsrc = make_rsrc(from, (uint32_t)(a.N - n0 < BN ? a.N - n0 : BN) * 4);
      load_lds4(rsrc, lds + (uint32_t)(OFF_STAT + (at * 2 + wave) * STATS * 4), lane * 4, 0);
    }
  };
  if (t0 < t1) fire(t0);
  RowSide<D> kr, vr;
  kr.load(K + b * a.k.b + hk * a.k.h + key * a.k.n, lane, seen);
  vr.load(V + b * a.v.b + hk * a.v.h + key * a.v.n, lane, seen);
  f32x16 dk[X::MD], dv[X::MD];
#pragma unroll
  for (int md = 0; md < X::MD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) dk[md][v] = dv[md][v] = 0.f;
  for (int t = t0; t < t1; ++t) {
    const int at = (t - t0) & 1, have = a.N - t % a.chunks * BN;
    unsigned char* tile = smem + at * 2 * TILEB;
    float* stat = reinterpret_cast<float*>(smem + OFF_STAT + at * 2 * STATS * 4);
    tile_arrived();
    if (t + 1 < t1) fire(t + 1);
    if (have < BN) {
      const uint64_t keep = (1ull << have) - 1ull;
      blank<float, D, 256>(tile, BN, keep, tid);
      blank<float, D, 256>(tile + TILEB, BN, keep, tid);
      if (tid < BN && tid >= have) {
        stat[tid] = -INFINITY;
        stat[STATS + tid] = 0.f;
      }
      lds_ready();
    }
    if (!mine) continue;
    f32x16 two[2];
    rows<D, 2>(two, {tile, tile + TILEB}, lane, {&kr, &vr});
    f32x16 &s = two[0], &g = two[1];
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
      const f32x4 l = *reinterpret_cast<const f32x4*>(stat + g4 * 8 + hf * 4), d = *reinterpret_cast<const f32x4*>(stat + STATS + g4 * 8 + hf * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = g4 * 4 + e;
        s[v] = __builtin_amdgcn_exp2f(fmaf(s[v], a.scale_log2, l[e]));
        g[v] = s[v] * (g[v] + d[e]);
      }
    }
    cols<D>(dv, tile + TILEB, lane, s);
    cols<D>(dk, tile, lane, g);
  }
  if (!seen) {
#pragma unroll
    for (int md = 0; md < X::MD; ++md)
#pragma unroll
      for (int v = 0; v < 16; ++v) dk[md][v] = dv[md][v] = 0.f;
  }
  lds_ready();
  unsigned char* rows_of = smem + wave * 32 * X::ROWB;
  const int64_t to = (((int64_t)part * a.B * a.Hkv + bh) * a.M + key0) * D;
  rows_out<float, D>(dk, PART ? 1.f : a.scale, rows_of, lane, [&](int x) __attribute__((always_inline)) -> float* {
    return key0 + x >= a.M ? nullptr : PART ? dKpart + to + x * D : dK + b * a.gk.b + hk * a.gk.h + (int64_t)(key0 + x) * a.gk.n;
  });
  rows_out<float, D>(dv, 1.f, rows_of, lane, [&](int x) __attribute__((always_inline)) -> float* {
    return key0 + x >= a.M ? nullptr : PART ? dVpart + to + x * D : dV + b * a.gv.b + hk * a.gv.h + (int64_t)(key0 + x) * a.gv.n;
  });
}

template <int D> static void fwd_d(const CrossArgs& a, dim3 grid, int nw, bool part, const float* Q, const float* K, const float* V, float* O, float* lse, float* Opart, hipStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, nw * 64, 0, s>>>(Q, K, V, O, lse, Opart, a); };
  if (nw == 1) part ? go(cross_fwd_f32_kernel<D, 1, true>) : go(cross_fwd_f32_kernel<D, 1, false>);
  else if (nw == 2) part ? go(cross_fwd_f32_kernel<D, 2, true>) : go(cross_fwd_f32_kernel<D, 2, false>);
  else part ? go(cross_fwd_f32_kernel<D, 4, true>) : go(cross_fwd_f32_kernel<D, 4, false>);
}
void cross_fwd(const CrossArgs& a, int d, dim3 grid, int nw, bool part, const float* Q, const float* K, const float* V, float* O, float* lse, float* Opart, hipStream_t s) {
  d == 128 ? fwd_d<128>(a, grid, nw, part, Q, K, V, O, lse, Opart, s) : fwd_d<64>(a, grid, nw, part, Q, K, V, O, lse, Opart, s);
}

template <int D> static void dq_d(const CrossArgs& a, dim3 grid, int nw, bool part, const float* Q, const float* K, const float* V, const float* O, const float* lse, const float* dO,
                                  float* stats, float* dQ, float* dQpart, hipStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, nw * 64, 0, s>>>(Q, K, V, O, lse, dO, stats, dQ, dQpart, a); };
  if (nw == 1) part ? go(cross_dq_f32_kernel<D, 1, true>) : go(cross_dq_f32_kernel<D, 1, false>);
  else if (nw == 2) part ? go(cross_dq_f32_kernel<D, 2, true>) : go(cross_dq_f32_kernel<D, 2, false>);
  else part ? go(cross_dq_f32_kernel<D, 4, true>) : go(cross_dq_f32_kernel<D, 4, false>);
}
void cross_dq(const CrossArgs& a, int d, dim3 grid, int nw, bool part, const float* Q, const float* K, const float* V, const float* O, const float* lse, const float* dO, float* stats,
              float* dQ, float* dQpart, hipStream_t s) {
  d == 128 ? dq_d<128>(a, grid, nw, part, Q, K, V, O, lse, dO, stats, dQ, dQpart, s) : dq_d<64>(a, grid, nw, part, Q, K, V, O, lse, dO, stats, dQ, dQpart, s);
}

void cross_dkv(const CrossArgs& a, int d, dim3 grid, bool part, const float* Q, const float* K, const float* V, const float* stats, const float* dO, float* dK, float* dV, float* dKpart,
               float* dVpart, hipStream_t s) {
  auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(Q, K, V, stats, dO, dK, dV, dKpart, dVpart, a); };
  if (d == 128) part ? go(cross_dkv_f32_kernel<128, true>) : go(cross_dkv_f32_kernel<128, false>);
  else part ? go(cross_dkv_f32_kernel<64, true>) : go(cross_dkv_f32_kernel<64, false>);
}

}  // namespace psa
