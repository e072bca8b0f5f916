// Attention that keeps its statistics, and its backward pass, in bfloat16 on MFMA 32x32x16, head dimension
// 64 or 128 (the formulas and the split into a query-side and a key-side kernel: attention_grad.hip).
//
// A wave owns 32 rows of its side, one to a lane pair (l, l + 32), as operands in registers, and walks
// 64-row tiles of the other side through two LDS buffers that direct global->LDS loads fill one tile ahead.
// Every product is computed transposed, D = A B with B the wave's own rows:
//   S^T = K Q^T, dP^T = V dO^T (query side), S = Q K^T, dP = dO V^T (key side): A = tile rows, over d
//   O^T += V^T P^T, dQ^T += K^T dS^T, dV^T += dO^T P, dK^T += Q^T dS:           A = tile columns, over its rows
// The accumulators of the first kind become the B operands of the second without a shuffle: tile rows are fed
// with bits 2 and 3 of their index swapped, and a lane's 8 accumulators of a 16-row slice are then rows
// 16 s + 8 (lane / 32) + 0..7, the B operand's slots.  Tile columns are read by the transposing LDS read (four
// rows of 16 columns to a 16-lane group; lane i gets column i).
//
// LDS: 16-byte chunk c of row r lies at chunk c ^ swz(r), which spreads both the 16 rows that a row read takes
// at once and the 4 rows x 64 bytes of a transposing read over all 64 banks.
#include <cmath>

#include "attention_grad.h"

namespace ff {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int KT = 64;   // rows of a tile

template <int D>
struct Tile {
  static constexpr int RB = 2 * D, CH = D / 8, BYTES = KT * RB;
  static __device__ __forceinline__ int swz(int r) {
    return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3);
  }
  // Row `row` (0 .. 63, already permuted), chunk c.
  static __device__ __forceinline__ bf16x8 row_frag(const char* t, int row, int c) {
    return *reinterpret_cast<const bf16x8*>(t + row * RB + ((c ^ swz(row)) << 4));
  }
  // Columns 32 db + lane % 32 of rows 16 s + 8 (lane / 32) + 0..7.
  static __device__ __forceinline__ bf16x8 col_frag(const char* t, int s, int db, int lane) {
    const int i = lane & 15, half = (lane >> 4) & 1, g = lane >> 5;
    union { s16x4 h[2]; bf16x8 v; } u;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = 16 * s + 8 * g + 4 * j + (i >> 2), c = 4 * db + 2 * half + ((i & 3) >> 1);
      u.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_s16x4*)(t + row * RB + ((c ^ swz(row)) << 4) + ((i & 1) << 3)));
    }
    return u.v;
  }
};

__device__ __forceinline__ int swap23(int l) { return (l & ~12) | ((l & 4) << 1) | ((l & 8) >> 1); }

// 64 lanes' 16 (4) bytes to LDS address `lds` on, lane after lane.  In inline assembly for the reason given at the
// forward kernel of ff_attention: the compiler would wait for every LDS read at each; completion is ordered by
// the waits below.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop
// Every load of this wave has landed, every LDS read has returned, and every wave has got here: the tile that the
// loads filled can be read, and the one read before can be filled.
__device__ __forceinline__ void tile_ready() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// This wave's share of a tile: rows n0 .. n0 + 63 of base, those past `last` replaced by it.
template <int D, int WAVES>
__device__ __forceinline__ void load_tile(uint32_t lds, const bf16_t* base, int64_t stride, int64_t n0, int64_t last, int wave, int lane) {
  constexpr int LOADS = Tile<D>::BYTES / 1024 / WAVES, RPL = 1024 / Tile<D>::RB;
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int r = (j * WAVES + wave) * RPL + lane / Tile<D>::CH;
    const int c = (lane % Tile<D>::CH) ^ Tile<D>::swz(r);
    const int64_t n = n0 + r < last ? n0 + r : last;
    dma16(base + n * stride + c * 8, __builtin_amdgcn_readfirstlane(lds + (j * WAVES + wave) * 1024));
  }
}
// Own row as operand: chunk 2 t + g of step t; zeros where not ok.
template <int D>
__device__ __forceinline__ void own_frags(const bf16_t* p, bool ok, int g, bf16x8 (&f)[D / 16]) {
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (ok) u = *reinterpret_cast<const uint4*>(p + 16 * t + 8 * g);
    f[t] = __builtin_bit_cast(bf16x8, u);
  }
}
__device__ __forceinline__ f32x16 splat(float v) {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = v;
  return z;
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
// acc + (rows 32 blk + 0..31 of the tile) x own^T
template <int D>
__device__ __forceinline__ f32x16 mul_rows(f32x16 acc, const char* t, int blk, const bf16x8 (&own)[D / 16], int prow, int g) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) acc = mfma(Tile<D>::row_frag(t, 32 * blk + prow, 2 * s + g), own[s], acc);
  return acc;
}
// acc[db] += (tile rows 32 blk + 0..31)^T x w, w the two 16-row slices of a block.
template <int D>
__device__ __forceinline__ void mul_cols(f32x16 (&acc)[D / 32], const char* t, int blk, const bf16x8 (&w)[2], int lane) {
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = mfma(Tile<D>::col_frag(t, 2 * blk + s, db, lane), w[s], acc[db]);
}
__device__ __forceinline__ void pack(const f32x16& x, bf16x8 (&w)[2]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    uint4 u;
    u.x = f2bf2(x[8 * s], x[8 * s + 1]);
    u.y = f2bf2(x[8 * s + 2], x[8 * s + 3]);
    u.z = f2bf2(x[8 * s + 4], x[8 * s + 5]);
    u.w = f2bf2(x[8 * s + 6], x[8 * s + 7]);
    w[s] = __builtin_bit_cast(bf16x8, u);
  }
}
// Tile row (within a block of 32) of accumulator r.
__device__ __forceinline__ int acc_row(int r, int g) { return 16 * (r >> 3) + 8 * g + (r & 7); }

template <int D>
__device__ __forceinline__ void store_bf16(bf16_t* p, const f32x16 (&acc)[D / 32], float f, int g) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      *reinterpret_cast<uint2*>(p + 32 * db + 8 * u + 4 * g) =
          make_uint2(f2bf2(acc[db][4 * u] * f, acc[db][4 * u + 1] * f), f2bf2(acc[db][4 * u + 2] * f, acc[db][4 * u + 3] * f));
}
template <int D>
__device__ __forceinline__ void store_f32(float* p, const f32x16 (&acc)[D / 32], float f, int g) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      *reinterpret_cast<float4*>(p + 32 * db + 8 * u + 4 * g) =
          make_float4(acc[db][4 * u] * f, acc[db][4 * u + 1] * f, acc[db][4 * u + 2] * f, acc[db][4 * u + 3] * f);
}
// Smallest and largest over the wave, in scalar registers.
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { const int u = __shfl_xor(v, o, 64); v = u < v ? u : v; }
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_top(int v) { return -wave_min(-v); }

// The running maximum m (log2 units) lags: a row keeps it until a score passes it by more than 8, so P is at
// most 256 and O is rescaled on few tiles.
template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void fwd_kernel(AttnGrad p) {
  constexpr int STAGE = 2 * Tile<D>::BYTES;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t smem_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane & 31, g = lane >> 5, prow = swap23(l);
  const QueryTile t = query_tile(p, 32 * WAVES);
  const OwnQuery q = own_query(p, t, t.row0 + wave * 32 + l);
  const bf16_t* K = key_base<bf16_t>(p.K, t);
  const bf16_t* V = key_base<bf16_t>(p.V, t);
  auto issue = [&](int64_t k0, int buf) {
    load_tile<D, WAVES>(smem_at + buf * STAGE, K, p.K.n, k0, t.key1 - 1, wave, lane);
    load_tile<D, WAVES>(smem_at + buf * STAGE + Tile<D>::BYTES, V, p.V.n, k0, t.key1 - 1, wave, lane);
  };
  if (t.key0 < t.key1) issue(t.key0, 0);
  bf16x8 qf[D / 16];
  own_frags<D>(q.at<bf16_t>(p.Q), q.ok, g, qf);
  const float c = fabsf(p.scale_log2);
  if (p.scale < 0.f) {   // the maximum of the scores is that of -q . k
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      uint4 u = __builtin_bit_cast(uint4, qf[s]);
      u.x ^= 0x80008000u; u.y ^= 0x80008000u; u.z ^= 0x80008000u; u.w ^= 0x80008000u;
      qf[s] = __builtin_bit_cast(bf16x8, u);
    }
  }
  const int lim_min = wave_min(q.lim), lim_top = wave_top(q.lim);
  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = splat(0.f);
  float m = -3e38f, sum = 0.f;
  int buf = 0;
  for (int64_t k0 = t.key0; k0 < t.key1; k0 += KT, buf ^= 1) {
    tile_ready();
    if (k0 + KT < t.key1) issue(k0 + KT, buf ^ 1);
    if (k0 >= lim_top) continue;
    const char* ks = smem + buf * STAGE;
    f32x16 s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) s[b] = mul_rows<D>(splat(0.f), ks, b, qf, prow, g);
    if (k0 + KT > lim_min) {
      const int left = q.lim - static_cast<int>(k0);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][r] = 32 * b + acc_row(r, g) < left ? s[b][r] : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c;
    if (__any(mx > m + 8.f)) {
      const float m_new = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      sum *= alpha;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
    }
    bf16x8 w[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = __builtin_amdgcn_exp2f(fmaf(s[b][r], c, -m));
        sum += s[b][r];
      }
      pack(s[b], w[b]);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) mul_cols<D>(o, ks + Tile<D>::BYTES, b, w[b], lane);
  }
  sum += __shfl_xor(sum, 32, 64);
  if (!q.ok) return;
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  const float lse = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
  if (p.splits > 1) {
    const int64_t row = split_row(p, t, q);
    store_f32<D>(p.part + row * D, o, inv, g);
    if (g == 0) p.part_lse[row] = lse;
  } else {
    store_bf16<D>(q.at<bf16_t>(p.O), o, inv, g);
    if (g == 0) p.lse[q.stat] = lse;
  }
}

template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void dq_kernel(AttnGrad p) {
  constexpr int STAGE = 2 * Tile<D>::BYTES;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t smem_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane & 31, g = lane >> 5, prow = swap23(l);
  const QueryTile t = query_tile(p, 32 * WAVES);
  const OwnQuery q = own_query(p, t, t.row0 + wave * 32 + l);
  const bf16_t* K = key_base<bf16_t>(p.K, t);
  const bf16_t* V = key_base<bf16_t>(p.V, t);
  auto issue = [&](int64_t k0, int buf) {
    load_tile<D, WAVES>(smem_at + buf * STAGE, K, p.K.n, k0, t.key1 - 1, wave, lane);
    load_tile<D, WAVES>(smem_at + buf * STAGE + Tile<D>::BYTES, V, p.V.n, k0, t.key1 - 1, wave, lane);
  };
  if (t.key0 < t.key1) issue(t.key0, 0);
  bf16x8 qf[D / 16], gf[D / 16];
  own_frags<D>(q.at<bf16_t>(p.Q), q.ok, g, qf);
  own_frags<D>(q.at<bf16_t>(p.dO), q.ok, g, gf);
  float delta = 0.f;
  {
    bf16x8 of[D / 16];
    own_frags<D>(q.at<bf16_t>(p.O), q.ok, g, of);
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(static_cast<float>(gf[s][j]), static_cast<float>(of[s][j]), delta);
  }
  delta += __shfl_xor(delta, 32, 64);
  const float lse = q.ok ? p.lse[q.stat] : 0.f;
  if (q.ok && g == 0 && t.split == 0) {
    // -lse / scale starts the dK, dV kernel's accumulators, and -D; exp2(scale_log2 x) is 0 for queries that see no
    // key and for those that only fill the last block
    float* st = p.delta + (t.b * p.heads + q.h) * stat_rows(p.n_q) * 2;
    const float none = p.scale > 0.f ? -INFINITY : INFINITY;
    const bool some = lse != -INFINITY;
    st[(q.i >> 5) * 64 + (q.i & 31)] = some ? -lse / p.scale : none;
    st[(q.i >> 5) * 64 + 32 + (q.i & 31)] = some ? -delta : 0.f;
    if (q.i == p.n_q - 1)
      for (int64_t i = p.n_q; i < stat_rows(p.n_q); ++i) {
        st[(i >> 5) * 64 + (i & 31)] = none;
        st[(i >> 5) * 64 + 32 + (i & 31)] = 0.f;
      }
  }
  const float lse2 = lse * 1.4426950408889634f;
  const int lim_min = wave_min(q.lim), lim_top = wave_top(q.lim);
  f32x16 dq[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dq[i] = splat(0.f);
  int buf = 0;
  for (int64_t k0 = t.key0; k0 < t.key1; k0 += KT, buf ^= 1) {
    tile_ready();
    if (k0 + KT < t.key1) issue(k0 + KT, buf ^ 1);
    if (k0 >= lim_top) continue;
    const char* ks = smem + buf * STAGE;
    const char* vs = ks + Tile<D>::BYTES;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 s = mul_rows<D>(splat(0.f), ks, b, qf, prow, g);
      const f32x16 dp = mul_rows<D>(splat(0.f), vs, b, gf, prow, g);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, -lse2)) * (dp[r] - delta);
      if (k0 + KT > lim_min) {
        const int left = q.lim - static_cast<int>(k0);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 32 * b + acc_row(r, g) < left ? s[r] : 0.f;
      }
      bf16x8 w[2];
      pack(s, w);
      mul_cols<D>(dq, ks, b, w, lane);
    }
  }
  if (!q.ok) return;
  if (p.splits > 1) store_f32<D>(p.part + split_row(p, t, q) * D, dq, p.scale, g);
  else store_bf16<D>(q.at<bf16_t>(p.dQ), dq, p.scale, g);
}

template <int D>
__global__ __launch_bounds__(256, 2) void dkv_kernel(AttnGrad p) {
  constexpr int STAGE = 2 * Tile<D>::BYTES + 512, WAVES = 4;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t smem_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane & 31, g = lane >> 5, prow = swap23(l);
  const KeyTile t = key_tile(p, 32 * WAVES);
  const int64_t wkey = t.key0 + wave * 32, key = wkey + l;
  const bool seen = key < t.len;
  TileWalk<KT> w(p, t);
  auto issue = [&](int buf) {
    const int64_t h = t.kvh * p.group + w.head, i0 = w.tile * KT;
    const uint32_t at = smem_at + buf * STAGE;
    load_tile<D, WAVES>(at, static_cast<const bf16_t*>(p.Q.p) + t.b * p.Q.b + h * p.Q.h, p.Q.n, i0, p.n_q - 1, wave, lane);
    load_tile<D, WAVES>(at + Tile<D>::BYTES, static_cast<const bf16_t*>(p.dO.p) + t.b * p.dO.b + h * p.dO.h, p.dO.n, i0, p.n_q - 1,
                        wave, lane);
    const float* st = p.delta + (t.b * p.heads + h) * stat_rows(p.n_q) * 2 + i0 * 2 + lane;
    if (wave < 2) dma4(st + wave * 64, __builtin_amdgcn_readfirstlane(at + 2 * Tile<D>::BYTES + wave * 256));
  };
  if (w.more()) issue(0);
  bf16x8 kf[D / 16], vf[D / 16];
  own_frags<D>(key_base<bf16_t>(p.K, t) + key * p.K.n, seen, g, kf);
  own_frags<D>(key_base<bf16_t>(p.V, t) + key * p.V.n, seen, g, vf);
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) { dk[i] = splat(0.f); dv[i] = splat(0.f); }
  // queries first .. n_q - 1 see this lane's key; the wave's first key has the smallest `first`
  const int64_t off = p.causal ? t.len - p.n_q : int64_t(1) << 40;
  const int64_t first = key - off, wfirst = wkey - off;
  int buf = 0;
  while (w.more()) {
    const int64_t i0 = w.tile * KT;
    w.next();
    tile_ready();
    if (w.more()) issue(buf ^ 1);
    const char* qs = smem + buf * STAGE;
    const char* gs = qs + Tile<D>::BYTES;
    const float* st = reinterpret_cast<const float*>(gs + Tile<D>::BYTES);
    buf ^= 1;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int64_t ib = i0 + 32 * b;
      if (ib + 31 < wfirst) continue;
      f32x16 s, dp;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int at = 64 * b + 16 * (u >> 1) + 8 * g + 4 * (u & 1);
        const float4 x = *reinterpret_cast<const float4*>(st + at), y = *reinterpret_cast<const float4*>(st + at + 32);
        s[4 * u] = x.x; s[4 * u + 1] = x.y; s[4 * u + 2] = x.z; s[4 * u + 3] = x.w;
        dp[4 * u] = y.x; dp[4 * u + 1] = y.y; dp[4 * u + 2] = y.z; dp[4 * u + 3] = y.w;
      }
      s = mul_rows<D>(s, qs, b, kf, prow, g);
      dp = mul_rows<D>(dp, gs, b, vf, prow, g);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * p.scale_log2);
      if (ib < wfirst + 31) {
        const int skip = static_cast<int>(first - ib);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = acc_row(r, g) >= skip ? s[r] : 0.f;
      }
      bf16x8 pw[2], dw[2];
      pack(s, pw);
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] *= s[r];
      pack(dp, dw);
      mul_cols<D>(dv, gs, b, pw, lane);
      mul_cols<D>(dk, qs, b, dw, lane);
    }
  }
  if (key >= p.n_kv) return;
  if (!seen) {   // no query sees it (its column may hold anything: its scores were those of a zero key)
#pragma unroll
    for (int i = 0; i < D / 32; ++i) { dk[i] = splat(0.f); dv[i] = splat(0.f); }
  }
  if (p.splits > 1) {
    const int64_t row = (((static_cast<int64_t>(t.split) * p.B + t.b) * p.kv_heads + t.kvh) * p.n_kv + key) * 2;
    store_f32<D>(p.part + row * D, dk, p.scale, g);
    store_f32<D>(p.part + (row + 1) * D, dv, 1.f, g);
  } else {
    store_bf16<D>(static_cast<bf16_t*>(p.dK.p) + t.b * p.dK.b + t.kvh * p.dK.h + key * p.dK.n, dk, p.scale, g);
    store_bf16<D>(static_cast<bf16_t*>(p.dV.p) + t.b * p.dV.b + t.kvh * p.dV.h + key * p.dV.n, dv, 1.f, g);
  }
}

template <int D> constexpr int kQuerySmem = 4 * Tile<D>::BYTES;
template <int D> constexpr int kKeySmem = 4 * Tile<D>::BYTES + 1024;

}  // namespace

// Raises the kernels' dynamic LDS limits (once a device).
int attn_bf16_prepare() {
  static std::atomic<uint64_t> done[10];
  const struct { const void* f; int bytes; } all[10] = {
      {reinterpret_cast<const void*>(&fwd_kernel<64, 1>), kQuerySmem<64>}, {reinterpret_cast<const void*>(&fwd_kernel<64, 4>), kQuerySmem<64>},
      {reinterpret_cast<const void*>(&fwd_kernel<128, 1>), kQuerySmem<128>}, {reinterpret_cast<const void*>(&fwd_kernel<128, 4>), kQuerySmem<128>},
      {reinterpret_cast<const void*>(&dq_kernel<64, 1>), kQuerySmem<64>}, {reinterpret_cast<const void*>(&dq_kernel<64, 4>), kQuerySmem<64>},
      {reinterpret_cast<const void*>(&dq_kernel<128, 1>), kQuerySmem<128>}, {reinterpret_cast<const void*>(&dq_kernel<128, 4>), kQuerySmem<128>},
      {reinterpret_cast<const void*>(&dkv_kernel<64>), kKeySmem<64>}, {reinterpret_cast<const void*>(&dkv_kernel<128>), kKeySmem<128>},
  };
  for (int i = 0; i < 10; ++i) FF_TRY(ensure_smem_limit(all[i].f, all[i].bytes, done[i]));
  return FF_OK;
}

#define FF_QUERY(KERNEL)                                                                                                   \
  const dim3 grid(static_cast<unsigned>(blocks));                                                                          \
  if (p.d == 128 && narrow) hipLaunchKernelGGL((KERNEL<128, 1>), grid, dim3(64), kQuerySmem<128>, s, p);                   \
  else if (p.d == 128) hipLaunchKernelGGL((KERNEL<128, 4>), grid, dim3(256), kQuerySmem<128>, s, p);                       \
  else if (narrow) hipLaunchKernelGGL((KERNEL<64, 1>), grid, dim3(64), kQuerySmem<64>, s, p);                              \
  else hipLaunchKernelGGL((KERNEL<64, 4>), grid, dim3(256), kQuerySmem<64>, s, p);

void attn_fwd_bf16(const AttnGrad& p, int64_t blocks, bool narrow, hipStream_t s) { FF_QUERY(fwd_kernel) }
void attn_dq_bf16(const AttnGrad& p, int64_t blocks, bool narrow, hipStream_t s) { FF_QUERY(dq_kernel) }
void attn_dkv_bf16(const AttnGrad& p, int64_t blocks, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(blocks));
  if (p.d == 128) hipLaunchKernelGGL(dkv_kernel<128>, grid, dim3(256), kKeySmem<128>, s, p);
  else hipLaunchKernelGGL(dkv_kernel<64>, grid, dim3(256), kKeySmem<64>, s, p);
}

}  // namespace ff
