// Attention that keeps its statistics, and its backward pass, in bfloat16 on MFMA 32x32x16, head dimension
// 64 or 128 (the formulas and the split into a query-side and a key-side kernel: attention_grad.hip).
//
// A wave owns 32 rows of its side, one to a lane pair (l, l + 32), as operands in registers, and walks
// tiles of the other side through LDS buffers that direct global->LDS loads fill ahead.
// Every product is computed transposed, D = A B with B the wave's own rows:
//   S^T = K Q^T, dP^T = V dO^T (query side), S = Q K^T, dP = dO V^T (key side): A = tile rows, over d
//   O^T += V^T P^T, dQ^T += K^T dS^T, dV^T += dO^T P, dK^T += Q^T dS:           A = tile columns, over its rows
// The accumulators of the first kind become the B operands of the second without a shuffle: tile rows are fed
// with bits 2 and 3 of their index swapped, and a lane's 8 accumulators of a 16-row slice are then rows
// 16 s + 8 (lane / 32) + 0..7, the B operand's slots.  Tile columns are read by the transposing LDS read (four
// rows of 16 columns to a 16-lane group; lane i gets column i).
//
// The operands of the second kind, P and dS, are rounded to bfloat16, as matrix products of this rate take them: each is off
// by up to 2^-8 relative, on its own, and the sums over keys or queries stay float32, so that the results are 0.0020 to
// 0.0025 of their norm off 64 bits, where rounding the results themselves makes 0.0017.  P and dS in two bfloat16 parts
// each would take one more product forward and three more than seven backward.  The sum of a row's P is taken before it is
// rounded.
//
// LDS: 16-byte chunk c of row r lies at chunk c ^ swz(r), which spreads both the 16 rows that a row read takes
// at once and the 4 rows x 64 bytes of a transposing read over all 64 banks.
#include <cmath>
#include <type_traits>

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
};

typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;

// A lane's addresses within a tile.  Rows: block of 32, row `row` of it, chunk 2 t + g.  Columns: 32 db + lane % 32 of
// rows 16 s + 8 g + 4 j + 0..3.  The swizzle depends on neither block, t, s nor db, and on j and g by their own bits,
// so one register each serves all reads: t, db and j enter by exclusive or, the rest by the instruction's offset.
struct Lane {
  uint32_t row, col;
};
template <int D>
__device__ __forceinline__ Lane lane_at(int lane, int row) {
  const int g = lane >> 5, i = lane & 15, half = (lane >> 4) & 1, r4 = 8 * g + (i >> 2);
  return {static_cast<uint32_t>(row * Tile<D>::RB + ((g ^ Tile<D>::swz(row)) << 4)),
          static_cast<uint32_t>(r4 * Tile<D>::RB + (((2 * half + ((i & 3) >> 1)) ^ Tile<D>::swz(r4)) << 4) + ((i & 1) << 3))};
}
// The same for a wave that keeps all of them: what is left for the instruction's offset is the tile.
template <int D>
struct Lanes {
  uint32_t row[D / 16], col[D / 32][2];
  __device__ __forceinline__ explicit Lanes(Lane at) {
#pragma unroll
    for (int t = 0; t < D / 16; ++t) row[t] = at.row ^ (t << 5);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 2; ++j) col[db][j] = at.col ^ (db << 6 | j << 4);
  }
  __device__ __forceinline__ bf16x8 row_frag(int tile, int t) const { return *reinterpret_cast<lds_bf16x8*>(row[t] + tile); }
  __device__ __forceinline__ bf16x8 col_frag(int tile, int s, int db) const {
    union { s16x4 h[2]; bf16x8 v; } u;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      u.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>(col[db][j] + (tile + (16 * s + 4 * j) * Tile<D>::RB)));
    return u.v;
  }
};
template <int D>
__device__ __forceinline__ bf16x8 row_frag(uint32_t row, int blk, int t) {
  return *reinterpret_cast<lds_bf16x8*>((row ^ (t << 5)) + blk * 32 * Tile<D>::RB);
}
template <int D>
__device__ __forceinline__ bf16x8 col_frag(uint32_t col, int s, int db) {
  union { s16x4 h[2]; bf16x8 v; } u;
#pragma unroll
  for (int j = 0; j < 2; ++j)
    u.h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        reinterpret_cast<lds_s16x4*>((col ^ (db << 6 | j << 4)) + (16 * s + 4 * j) * Tile<D>::RB));
  return u.v;
}

__device__ __forceinline__ int swap23(int l) { return (l & ~12) | ((l & 4) << 1) | ((l & 8) >> 1); }

// 64 lanes' 16 (4) bytes, at base + off, to LDS address `lds` on, lane after lane.  In inline assembly for the reason
// given at the forward kernel of ff_attention: the compiler would wait for every LDS read at each; completion is
// ordered by the waits below.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// ONCE: non-temporal, for what no other workgroup reads.
template <bool ONCE>
__device__ __forceinline__ void dma16(const void* base, uint32_t off, uint32_t lds) {
  if constexpr (ONCE)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
// Every load of this wave has landed, every LDS read has returned, and every wave has got here: the tile that the
// loads filled can be read, and the one read before can be filled.
// LEFT, READS: so many of the wave's latest loads and of its latest LDS reads may still be in flight.
template <int LEFT = 0, int READS = 0>
__device__ __forceinline__ void tile_ready() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)" ::"n"(LEFT), "n"(READS) : "memory");
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// The lane's index, computed anew where it is called (what is kept from one place to the next takes registers).
__device__ __forceinline__ int lane_id() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(l));
  return l;
}
// This wave's share of a tile: ROWS rows from `base` on, those past row `left` replaced by it.  Whole tiles take one
// offset register: the loads' rows are a scalar step apart (the host keeps 64 row strides below 2^32 bytes).
template <int D, int WAVES, int ROWS, bool ONCE = false>
__device__ __forceinline__ void load_tile(uint32_t lds, const bf16_t* base, int64_t stride, int left, int wave, int lane) {
  constexpr int LOADS = ROWS * Tile<D>::RB / 1024 / WAVES, RPL = 1024 / Tile<D>::RB, STEP = WAVES * RPL;
  static_assert(LOADS > 0, "every wave loads a part");
  const uint32_t bytes = static_cast<uint32_t>(stride) * 2;
  const int r0 = wave * RPL + lane / Tile<D>::CH;
  const uint32_t c0 = (lane % Tile<D>::CH ^ Tile<D>::swz(r0)) * 16;   // later loads' rows have further bits: swz is linear
  auto one = [&](int j, const void* from, int r) __attribute__((always_inline)) {
    dma16<ONCE>(from, r * bytes + (c0 ^ Tile<D>::swz(j * STEP) * 16), __builtin_amdgcn_readfirstlane(lds + (j * WAVES + wave) * 1024));
  };
  if (left >= ROWS - 1) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) one(j, reinterpret_cast<const char*>(base) + static_cast<uint64_t>(j * STEP) * bytes, r0);
  } else {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) one(j, base, r0 + j * STEP < left ? r0 + j * STEP : left);
  }
}
// Own row as operand: chunk 2 t + g of step t.
template <int D>
__device__ __forceinline__ void own_frags(const bf16_t* p, int g, bf16x8 (&f)[D / 16]) {
#pragma unroll
  for (int t = 0; t < D / 16; ++t) f[t] = *reinterpret_cast<const bf16x8*>(p + 16 * t + 8 * g);
}
__device__ __forceinline__ f32x16 splat(float v) {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = v;
  return z;
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
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
// Tile row (within a block of 32) of accumulator r of lanes 0 .. 31; the others' is 8 further on.
__device__ constexpr int acc_row(int r) { return 16 * (r >> 3) + (r & 7); }

// The wave's 32 rows as bfloat16, through LDS of its own (kTurn bytes): a lane holds pieces of four elements of one
// row, and rows leave as whole lines.  `at(r)` is the address of row r, or null.
template <int D> constexpr int kTurn = 32 * (2 * D + 8);
template <int D, typename At>
__device__ __forceinline__ void store_bf16(char* lds, const f32x16 (&acc)[D / 32], float f, int lane, At&& at) {
  constexpr int LD = 2 * D + 8, CH = D / 8;   // 8 bytes over: the pieces' and the rows' accesses spread over all banks
  char* mine = lds + (lane & 31) * LD + 8 * (lane >> 5);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      *reinterpret_cast<uint2*>(mine + 2 * (32 * db + 8 * u)) =
          make_uint2(f2bf2(acc[db][4 * u] * f, acc[db][4 * u + 1] * f), f2bf2(acc[db][4 * u + 2] * f, acc[db][4 * u + 3] * f));
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wave's own writes; no other wave is concerned
#pragma unroll
  for (int k = 0; k < CH / 2; ++k) {
    const int r = k * (64 / CH) + lane / CH, c = lane % CH;
    const uint2 x = *reinterpret_cast<const uint2*>(lds + r * LD + 16 * c), y = *reinterpret_cast<const uint2*>(lds + r * LD + 16 * c + 8);
    bf16_t* row = at(r);
    if (row) *reinterpret_cast<uint4*>(row + 8 * c) = make_uint4(x.x, x.y, y.x, y.y);
  }
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
// Address of row r of 32 rows from `row0` on of a key head's query rows (head-in-group * n_q + query), or null past them.
struct QueryRows {
  const AttnGrad& p;
  const Heads& t;
  int64_t b, h0, left;
  uint32_t i0;
  __device__ __forceinline__ QueryRows(const AttnGrad& p, const Heads& t, const QueryTile& q, int64_t row0)
      : p(p), t(t), b(q.b), left(p.group * p.n_q - row0) {
    const uint32_t n = static_cast<uint32_t>(p.n_q), h = static_cast<uint32_t>(row0) / n;
    h0 = q.kvh * p.group + h;
    i0 = static_cast<uint32_t>(row0) - h * n;
  }
  __device__ __forceinline__ bf16_t* operator()(int r) const {
    if (r >= left) return nullptr;
    const uint32_t n = static_cast<uint32_t>(p.n_q), i = i0 + r, h = i / n;
    return static_cast<bf16_t*>(t.p) + b * t.b + (h0 + h) * t.h + static_cast<int64_t>(i - h * n) * t.n;
  }
};
// f(0) .. f(E - 1) with compile-time arguments (an unroll pragma gives up on bodies of this size).
template <int E, int I = 0, typename F>
__device__ __forceinline__ void steps(F&& f) {
  if constexpr (I < E) {
    f(std::integral_constant<int, I>{});
    steps<E, I + 1>(f);
  }
}
__device__ __forceinline__ uint32_t add_here(uint32_t v, uint32_t scalar) {   // likewise computed where it stands
  uint32_t r;
  asm volatile("v_add_u32 %0, %1, %2" : "=v"(r) : "s"(scalar), "v"(v));
  return r;
}
// Slice and column block of product k of the second kind: neighbours differ in the block, and four share addresses.
__device__ constexpr int slice(int k) { return (k >> 1) & 1; }
__device__ constexpr int block(int k) { return 2 * (k >> 2) + (k & 1); }
// Smallest and largest over the wave, in scalar registers.
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { const int u = __shfl_xor(v, o, 64); v = u < v ? u : v; }
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_top(int v) { return -wave_min(-v); }

// Query side: tiles of 32 keys, K and V in a ring of four buffers each.  The operands of a block's first products are
// read before the barrier at its start, from tiles that landed a block earlier.
constexpr int QT = 32, RING = 4;
template <int D> constexpr int kQueryTile = QT * 2 * D;   // bytes of a tile

// Forward.  Block b: the N products O^T += V^T P^T of block b - 1, then the N products of block b + 1's scores; the
// exponentials of block b are spread over both.  Operands are read from LDS AHEAD products early.
// The running maximum m (log2 units) lags: P is exp2 of (score - m) for the m of the blocks before, without looking
// for a new maximum.  Where a lane's sum of a block exceeds 256, m moves to the block's maximum, O and the sum are
// rescaled and the block's P computed again (always on the first block, rare after it).
// Bound by the matrix pipes beside the exponentials: 16 x 24 heads, 1536^2, d 128 466 us, 1.00 PFLOP/s, pipes 51% busy.
// Single tokens (one wave, all query heads of a key head in its rows) are bound by HBM: 42 us (41 at best) for 206 MB, 4.9
// TB/s.
template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void fwd_kernel(AttnGrad p) {
  constexpr int TILE = kQueryTile<D>, V0 = RING * TILE, LPW = TILE / 512 / WAVES, N = D / 16, AHEAD = 4;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t smem_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 31, g = lane >> 5;
  const QueryTile t = query_tile(p, 32 * WAVES);
  const OwnQuery q = own_query(p, t, t.row0 + wave * 32 + l);
  const int key0 = static_cast<int>(t.key0), key1 = static_cast<int>(t.key1), n = (key1 - key0 + QT - 1) / QT;
  // Loads of the next K or V tile into buffer `ring`; past the last tile the last one again, which is not used.
  struct Next { const bf16_t* at; int left; };
  auto issue = [&](Next& x, int64_t stride, int to) __attribute__((always_inline)) {
    // One wave has all rows of its key head, so no other workgroup reads these keys (16 sequences of up to 4096, 8 key
    // heads, not in any cache: 46.9 us, plain loads 51.5).
    load_tile<D, WAVES, QT, WAVES == 1>(smem_at + to, x.at, stride, x.left, wave, lane);
    if (x.left >= QT) {
      x.at += QT * stride;
      x.left -= QT;
    }
  };
  Next kn{key_base<bf16_t>(p.K, t) + key0 * p.K.n, key1 - 1 - key0}, vn{key_base<bf16_t>(p.V, t) + key0 * p.V.n, key1 - 1 - key0};
  auto issue_k = [&](int ring) __attribute__((always_inline)) { issue(kn, p.K.n, ring * TILE); };
  auto issue_v = [&](int ring) __attribute__((always_inline)) { issue(vn, p.V.n, V0 + ring * TILE); };
  const Lanes<D> at(Lane{lane_at<D>(lane, swap23(l)).row + smem_at, lane_at<D>(lane, swap23(l)).col + smem_at});
  bf16x8 qf[N];
  own_frags<D>(q.at<bf16_t>(p.Q), g, qf);
  const float c = fabsf(p.scale_log2);
  if (p.scale < 0.f) {   // the maximum of the scores is that of -q . k
#pragma unroll
    for (int s = 0; s < N; ++s) {
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
  bf16x8 f[AHEAD];
  // Operand i of block b (b % RING = ring): columns of block b - 1's V, rows of block b + 1's K; then those of block b + 1.
  auto fetch = [&](auto ci, auto cr) __attribute__((always_inline)) {
    constexpr int i = decltype(ci)::value % (2 * N), k = i % N, ring = (decltype(cr)::value + decltype(ci)::value / (2 * N)) % RING;
    if constexpr (i < N) f[decltype(ci)::value % AHEAD] = at.col_frag(V0 + (ring + RING - 1) % RING * TILE, slice(k), block(k));
    else f[decltype(ci)::value % AHEAD] = at.row_frag((ring + 1) % RING * TILE, k);
  };
  // P of elements r, r + 1 of a block's scores.
  auto soft = [&](const f32x16& s, bf16x8 (&w)[2], int r, float& part) __attribute__((always_inline)) {
    const float a = __builtin_amdgcn_exp2f(fmaf(s[r], c, -m)), b = __builtin_amdgcn_exp2f(fmaf(s[r + 1], c, -m));
    part += a;
    part += b;
    uint4 u = __builtin_bit_cast(uint4, w[r >> 3]);
    const uint32_t x = f2bf2(a, b);
    if ((r & 7) == 0) u.x = x; else if ((r & 7) == 2) u.y = x; else if ((r & 7) == 4) u.z = x; else u.w = x;
    w[r >> 3] = __builtin_bit_cast(bf16x8, u);
  };
  auto block_step = [&](int k0, auto cr, auto cfirst, f32x16& s, f32x16& nx, const bf16x8 (&pw)[2], bf16x8 (&pn)[2])
      __attribute__((always_inline)) {
    constexpr int ring = decltype(cr)::value;
    constexpr bool first = decltype(cfirst)::value;
    constexpr int from = first ? N : 0;   // the first block has no products of one before it
    tile_ready<LPW, first ? 0 : 2 * AHEAD>();   // K of block b + 1 and V of block b are there
    issue_k((ring + 3) % RING);
    issue_v((ring + 2) % RING);
    if (k0 + QT > lim_min) {
      const int see = q.lim - k0 - 8 * g;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = acc_row(r) < see ? s[r] : -INFINITY;
    }
    float part = 0.f;
    if constexpr (first) steps<N + AHEAD, N>([&](auto ci) __attribute__((always_inline)) { fetch(ci, cr); });
    steps<2 * N, from>([&](auto ci) __attribute__((always_inline)) {
      constexpr int i = decltype(ci)::value, k = i % N;
      if constexpr (i < N) o[block(k)] = mfma(f[i % AHEAD], pw[slice(k)], o[block(k)]);
      else nx = mfma(f[i % AHEAD], qf[k], k == 0 ? splat(0.f) : nx);
      fetch(std::integral_constant<int, i + AHEAD>{}, cr);
      constexpr int lo = 8 * (i - from) / (2 * N - from), hi = 8 * (i + 1 - from) / (2 * N - from);
#pragma unroll
      for (int r = lo; r < hi; ++r) soft(s, pn, 2 * r, part);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (__any(part > 256.f)) {
      float mx = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c;
      const float m_new = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      sum *= alpha;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      part = 0.f;
#pragma unroll
      for (int r = 0; r < 16; r += 2) soft(s, pn, r, part);
    }
    sum += part;
  };
  if (n > 0) {
    issue_k(0);
    issue_k(1);
    issue_v(0);
    issue_k(2);
    issue_v(1);
    tile_ready<2 * LPW>();
    f32x16 sa = splat(0.f), sb = splat(0.f);
    bf16x8 pa[2], pb[2];
#pragma unroll
    for (int k = 0; k < N; ++k) sa = mfma(at.row_frag(0, k), qf[k], sa);
    // the wave's own blocks; then it keeps up with the others
    const int mine = lim_top <= key0 ? 0 : lim_top >= key1 ? n : (lim_top - key0 + QT - 1) / QT;
    if (mine > 0) {
      block_step(key0, std::integral_constant<int, 0>{}, std::true_type{}, sa, sb, pb, pa);
      int b = 1;
      // block b's P: pa where b is even, pb where it is odd
      auto step = [&](auto cr, f32x16& s, f32x16& nx, const bf16x8 (&pw)[2], bf16x8 (&pn)[2]) __attribute__((always_inline)) {
        if (b < mine) { block_step(key0 + b * QT, cr, std::false_type{}, s, nx, pw, pn); ++b; }
      };
      while (b < mine) {
        step(std::integral_constant<int, 1>{}, sb, sa, pa, pb);
        step(std::integral_constant<int, 2>{}, sa, sb, pb, pa);
        step(std::integral_constant<int, 3>{}, sb, sa, pa, pb);
        step(std::integral_constant<int, 0>{}, sa, sb, pb, pa);
      }
      // O of the last one, whose V is not being filled
      const uint32_t col = at.col[0][0] + V0 + ((mine - 1) % RING) * TILE;
      if (((mine - 1) & 1) != 0) { pa[0] = pb[0]; pa[1] = pb[1]; }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        o[block(k)] = mfma(col_frag<D>(col, slice(k), block(k)), pa[slice(k)], o[block(k)]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    for (int b = mine; b < n; ++b) {
      tile_ready<LPW>();
      issue_k((b + 3) % RING);
      issue_v((b + 2) % RING);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load is left behind
  }
  sum += __shfl_xor(sum, 32, 64);
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  const float lse = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
  if (p.splits > 1) {
    if (!q.ok) return;
    const int64_t at_row = split_row(p, t, q);
    store_f32<D>(p.part + at_row * D, o, inv, g);
    if (g == 0) p.part_lse[at_row] = lse;
  } else {
    tile_ready<>();   // every wave has read its last tile
    store_bf16<D>(smem + wave * kTurn<D>, o, inv, lane, QueryRows(p, p.O, t, t.row0 + wave * 32));
    if (q.ok && g == 0) p.lse[q.stat] = lse;
  }
}

// dQ.  A block: the N products of S, with dS = P (dP - D) of the block before between them; the N of dP, with the
// exponentials of S between; the N of dQ^T += K^T dS^T of the block before.  8 x 24 heads, 4352^2, d 128: 2.29 ms,
// 1.22 PFLOP/s of its three products, matrix pipes 66% busy.
template <int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void dq_kernel(AttnGrad p) {
  constexpr int HALF = kQueryTile<D>, STAGE = 2 * HALF, N = D / 16, AHEAD = 3, PER = 16 / N;   // a buffer holds K, then V
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t smem_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 31, g = lane >> 5;
  const QueryTile t = query_tile(p, 32 * WAVES);
  const OwnQuery q = own_query(p, t, t.row0 + wave * 32 + l);
  const int key0 = static_cast<int>(t.key0), key1 = static_cast<int>(t.key1), n = (key1 - key0 + QT - 1) / QT;
  const bf16_t* K = key_base<bf16_t>(p.K, t) + key0 * p.K.n;   // of the block that is loaded next
  const bf16_t* V = key_base<bf16_t>(p.V, t) + key0 * p.V.n;
  int left = key1 - 1 - key0;
  auto issue = [&](int ring) __attribute__((always_inline)) {
    const int ln = WAVES == 1 ? lane_id() : lane;   // a single wave's loads take more registers
    load_tile<D, WAVES, QT>(smem_at + ring * STAGE, K, p.K.n, left, wave, ln);
    load_tile<D, WAVES, QT>(smem_at + ring * STAGE + HALF, V, p.V.n, left, wave, ln);
    if (left >= QT) {
      K += QT * p.K.n;
      V += QT * p.V.n;
      left -= QT;
    }
  };
  const Lanes<D> at(Lane{lane_at<D>(lane, swap23(l)).row + smem_at, lane_at<D>(lane, swap23(l)).col + smem_at});
  bf16x8 qf[N], gf[N];
  own_frags<D>(q.at<bf16_t>(p.Q), g, qf);
  own_frags<D>(q.at<bf16_t>(p.dO), g, gf);
  float delta = 0.f;
  {
    bf16x8 of[N];
    own_frags<D>(q.at<bf16_t>(p.O), g, of);
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = fmaf(static_cast<float>(gf[s][j]), static_cast<float>(of[s][j]), delta);
  }
  delta += __shfl_xor(delta, 32, 64);
  const float lse = p.lse[q.stat];
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
  f32x16 dq[D / 32], pr, dp;   // pr, dp: P and dP of the block before
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dq[i] = splat(0.f);
  bf16x8 f[AHEAD], dw[2];
  // Operand i of the block in buffer `ring` (rows of its K, rows of its V, columns of K of the block before; then those
  // of the next block) into place `slot` of those read ahead.
  auto fetch = [&](auto ci, auto cr, int slot) __attribute__((always_inline)) {
    constexpr int i = decltype(ci)::value, k = i % N, ring = decltype(cr)::value, part = i / N;
    if constexpr (part == 2) f[slot] = at.col_frag((ring + RING - 1) % RING * STAGE, slice(k), block(k));
    else f[slot] = at.row_frag((part == 3 ? (ring + 1) % RING : ring) * STAGE + (part == 1 ? HALF : 0), k);
  };
  auto block_step = [&](int k0, auto cr, auto cfirst) __attribute__((always_inline)) {
    constexpr bool first = decltype(cfirst)::value;
    constexpr int from = first ? N : 0;   // the first block has no gradient of one before it
    static_assert(3 * N % AHEAD == 0, "a block's places follow the last one's");
    tile_ready<0, first ? 0 : AHEAD>();   // this block and the next are there
    issue((decltype(cr)::value + 2) % RING);
    f32x16 s;
    if constexpr (first)
      steps<AHEAD>([&](auto ci) __attribute__((always_inline)) { fetch(ci, cr, (from + decltype(ci)::value) % AHEAD); });
    steps<3 * N, from>([&](auto ci) __attribute__((always_inline)) {
      constexpr int i = decltype(ci)::value - from, slot = decltype(ci)::value % AHEAD, k = i % N;
      if constexpr (i < N) s = mfma(f[slot], qf[k], k == 0 ? splat(0.f) : s);
      else if constexpr (i < 2 * N) dp = mfma(f[slot], gf[k], k == 0 ? splat(0.f) : dp);
      else dq[block(k)] = mfma(f[slot], dw[slice(k)], dq[block(k)]);
      fetch(std::integral_constant<int, (i + AHEAD < 3 * N - from ? i + AHEAD : i + AHEAD + from)>{}, cr, slot);
      if constexpr (i < N && !first) {
#pragma unroll
        for (int r = PER * k; r < PER * (k + 1); ++r) pr[r] *= dp[r] - delta;
        if constexpr (k == N - 1) pack(pr, dw);
      } else if constexpr (i >= N && i < 2 * N) {
#pragma unroll
        for (int r = PER * k; r < PER * (k + 1); ++r) pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, -lse2));
        if constexpr (k == N - 1) {
          if (k0 + QT > lim_min) {
            const int see = q.lim - k0 - 8 * g;
#pragma unroll
            for (int r = 0; r < 16; ++r) pr[r] = acc_row(r) < see ? pr[r] : 0.f;
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  if (n > 0) {
    issue(0);
    issue(1);
    // the wave's own blocks; then it keeps up with the others
    const int mine = lim_top <= key0 ? 0 : lim_top >= key1 ? n : (lim_top - key0 + QT - 1) / QT;
    if (mine > 0) {
      block_step(key0, std::integral_constant<int, 0>{}, std::true_type{});
      int b = 1;
      auto step = [&](auto cr) __attribute__((always_inline)) {
        if (b < mine) { block_step(key0 + b * QT, cr, std::false_type{}); ++b; }
      };
      while (b < mine) {
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
        step(std::integral_constant<int, 0>{});
      }
      // dQ of the last one, whose buffer is not being filled
#pragma unroll
      for (int r = 0; r < 16; ++r) pr[r] *= dp[r] - delta;
      pack(pr, dw);
      const uint32_t col = lane_at<D>(lane, swap23(l)).col + smem_at + ((mine - 1) % RING) * STAGE;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        dq[block(k)] = mfma(col_frag<D>(col, slice(k), block(k)), dw[slice(k)], dq[block(k)]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    for (int b = mine; b < n; ++b) {
      tile_ready<>();
      issue((b + 2) % RING);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no load is left behind
  }
  if (p.splits > 1) {
    if (q.ok) store_f32<D>(p.part + split_row(p, t, q) * D, dq, p.scale, g);
  } else {
    tile_ready<>();   // every wave has read its last tile
    store_bf16<D>(smem + wave * kTurn<D>, dq, p.scale, lane, QueryRows(p, p.dQ, t, t.row0 + wave * 32));
  }
}

// The key-side kernel's operands of dP that wait in LDS: with all of K, V, dK and dV of head dimension 128 in registers
// (192) the rest does not fit into 256, and a spilled register's reload would wait for the tile loads in flight.
template <int D> constexpr int kVLds = D == 128 ? 3 : 0;
template <int D> constexpr int kQuerySmem = 2 * RING * kQueryTile<D>;   // the epilogue's rows, 4 kTurn, fit too
template <int D> constexpr int kKeyWork = 4 * Tile<D>::BYTES + 1024 + kVLds<D> * 4096;
template <int D> constexpr int kKeySmem = kKeyWork<D> > 8 * kTurn<D> ? kKeyWork<D> : 8 * kTurn<D>;

// Gradients of a key-side workgroup whose keys no query sees: zeros, and nothing of K and V is read.
template <int D>
__device__ __forceinline__ void unseen_keys(const AttnGrad& p, const KeyTile& t) {
  const int n = static_cast<int>(p.n_kv - t.key0 < kKeyRows ? p.n_kv - t.key0 : kKeyRows);
  if (p.splits > 1) {   // the partial results of dK and dV lie side by side
    const int64_t row = ((static_cast<int64_t>(t.split) * p.B + t.b) * p.kv_heads + t.kvh) * p.n_kv + t.key0;
    float4* to = reinterpret_cast<float4*>(p.part + row * 2 * D);
    for (int i = threadIdx.x; i < n * (D / 2); i += 256) to[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    return;
  }
  constexpr int CH = D / 8;
  for (int i = threadIdx.x; i < n * CH; i += 256) {
    const int64_t key = t.key0 + i / CH;
    for (const Heads& x : {p.dK, p.dV})
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(x.p) + t.b * x.b + t.kvh * x.h + key * x.n + i % CH * 8) = make_uint4(0, 0, 0, 0);
  }
}

// dK, dV: a wave holds its keys' K and V and both gradients, and walks tiles of 64 queries.  8 x 24 heads, 4352^2, d 128:
// 3.11 ms, 1.20 PFLOP/s of its four products, matrix pipes 61% busy.
template <int D>
__global__ __launch_bounds__(256, 2) void dkv_kernel(AttnGrad p) {
  constexpr int STAGE = 2 * Tile<D>::BYTES + 512, WAVES = kKeyRows / 32, VL = kVLds<D>, VR = D / 16 - VL;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t smem_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const KeyTile t = key_tile(p, kKeyRows);
  if (t.key0 >= t.len) return unseen_keys<D>(p, t);
  const int wkey = static_cast<int>(t.key0) + wave * 32, len = static_cast<int>(t.len);
  TileWalk<KT> w(p, t);
  auto issue = [&](int buf, int lane) {
    const int64_t h = t.kvh * p.group + w.head, i0 = w.tile * KT;
    const uint32_t to = smem_at + buf * STAGE;
    const int left = static_cast<int>(p.n_q - 1 - i0);
    load_tile<D, WAVES, KT>(to, static_cast<const bf16_t*>(p.Q.p) + t.b * p.Q.b + h * p.Q.h + i0 * p.Q.n, p.Q.n, left, wave, lane);
    load_tile<D, WAVES, KT>(to + Tile<D>::BYTES, static_cast<const bf16_t*>(p.dO.p) + t.b * p.dO.b + h * p.dO.h + i0 * p.dO.n, p.dO.n,
                        left, wave, lane);
    const float* st = p.delta + ((t.b * p.heads + h) * stat_rows(p.n_q) + i0) * 2;
    if (wave < 2) dma4(st, (wave * 64 + lane) * 4, __builtin_amdgcn_readfirstlane(to + 2 * Tile<D>::BYTES + wave * 256));
  };
  if (w.more()) issue(0, lane_id());
  bf16x8 kf[D / 16], vf[VR];   // the last key stands for those past it, whose gradients are set to 0 at the end
  {
    const int lane = lane_id(), key = wkey + (lane & 31), own = key < len ? key : len - 1;
    own_frags<D>(key_base<bf16_t>(p.K, t) + own * p.K.n, lane >> 5, kf);
    bf16x8 v[D / 16];
    own_frags<D>(key_base<bf16_t>(p.V, t) + own * p.V.n, lane >> 5, v);
#pragma unroll
    for (int i = 0; i < VR; ++i) vf[i] = v[i];
#pragma unroll
    for (int i = 0; i < VL; ++i) *reinterpret_cast<bf16x8*>(smem + 2 * STAGE + ((i * WAVES + wave) * 64 + lane) * 16) = v[VR + i];
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) { dk[i] = splat(0.f); dv[i] = splat(0.f); }
  // queries first .. n_q - 1 see a key; the wave's first key has the smallest `first`
  const int off = p.causal ? len - static_cast<int>(p.n_q) : 1 << 28;
  const int wfirst = wkey - off;
  // A block of 32 queries is 4 N products, each with one operand read from LDS `AHEAD` products before it:
  //   S = Q K^T, dP = dO V^T (with the exponentials of S between its products), dV += dO^T P (with the products
  //   P dP between), dK += Q^T dS.
  // The fences keep that order: left to itself the compiler holds dozens of addresses and spills K and V.
  constexpr int N = D / 16, STEPS = 4 * N, AHEAD = 3;
  int buf = 0;
  while (w.more()) {
    const int i0 = static_cast<int>(w.tile) * KT;
    w.next();
    tile_ready();
    const int lane = lane_id(), g = lane >> 5;   // what follows from it lives for one tile only
    if (w.more()) issue(buf ^ 1, lane);
    const uint32_t qs = smem_at + buf * STAGE, gs = qs + Tile<D>::BYTES, st = gs + Tile<D>::BYTES + 32 * g;
    buf ^= 1;
    if (i0 + KT - 1 < wfirst) continue;
    // The statistics start the accumulators: S - lse / scale and dP - D come out of the products.
    auto start = [&](f32x16& x, int b, int what) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 y = *reinterpret_cast<lds_f32x4*>(st + 4 * (64 * b + 32 * what + 16 * (u >> 1) + 4 * (u & 1)));
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * u + j] = y[j];
      }
    };
    const Lane at = lane_at<D>(lane, swap23(lane & 31));
    uint32_t row = 0, col = 0;
    bf16x8 f[AHEAD];
    auto fetch = [&](auto c) __attribute__((always_inline)) {   // the operand of product i of a tile
      constexpr int i = decltype(c)::value, b = i / STEPS, phase = i % STEPS / N, k = i % N;
      const uint32_t tile = phase == 1 || phase == 2 ? gs : qs;
      if constexpr (phase < 2) {
        if (k == 0) row = add_here(at.row, tile);
        f[i % AHEAD] = row_frag<D>(row, b, k);
      } else {
        if (k % 4 == 0) col = add_here(at.col, tile);
        f[i % AHEAD] = col_frag<D>(col, 2 * b + slice(k), block(k));
      }
    };
    f32x16 s, dp;
    bf16x8 pw[2], dw[2], vt[2];
    steps<AHEAD>(fetch);
    steps<2 * STEPS>([&](auto c) __attribute__((always_inline)) {
      constexpr int i = decltype(c)::value, b = i / STEPS, phase = i % STEPS / N, k = i % N, PER = 16 / N;
      if constexpr (phase == 0) {
        if (k == 0) start(s, b, 0);
        if (k == N - 1) start(dp, b, 1);
        s = mfma(f[i % AHEAD], kf[k], s);
      } else if constexpr (phase == 1) {
        dp = mfma(f[i % AHEAD], k < VR ? vf[k < VR ? k : 0] : vt[k % 2], dp);
        if constexpr (k + 2 >= VR && k + 2 < N)
          vt[k % 2] = *reinterpret_cast<lds_bf16x8*>(smem_at + 2 * STAGE + ((k + 2 - VR) * WAVES + wave) * 1024 + lane_id() * 16);
      } else if constexpr (phase == 2) {
        dv[block(k)] = mfma(f[i % AHEAD], pw[slice(k)], dv[block(k)]);
      } else {
        dk[block(k)] = mfma(f[i % AHEAD], dw[slice(k)], dk[block(k)]);
      }
      if constexpr (i + AHEAD < 2 * STEPS) fetch(std::integral_constant<int, i + AHEAD>{});
      if constexpr (phase == 1) {
#pragma unroll
        for (int r = PER * k; r < PER * (k + 1); ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * p.scale_log2);
        if constexpr (k == N - 1) {
          const int ib = i0 + 32 * b;
          if (ib < wfirst + 31) {
            const int own = lane_id(), skip = wfirst + (own & 31) - ib - 8 * (own >> 5);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = acc_row(r) >= skip ? s[r] : 0.f;
          }
          pack(s, pw);
        }
      } else if constexpr (phase == 2) {
#pragma unroll
        for (int r = PER * k; r < PER * (k + 1); ++r) s[r] *= dp[r];
        if constexpr (k == N - 1) pack(s, dw);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  const int lane = lane_id(), g = lane >> 5, key = wkey + (lane & 31);
  if (key >= len) {   // no query sees it
#pragma unroll
    for (int i = 0; i < D / 32; ++i) { dk[i] = splat(0.f); dv[i] = splat(0.f); }
  }
  if (p.splits > 1) {
    if (key >= p.n_kv) return;
    const int64_t row = (((static_cast<int64_t>(t.split) * p.B + t.b) * p.kv_heads + t.kvh) * p.n_kv + key) * 2;
    store_f32<D>(p.part + row * D, dk, p.scale, g);
    store_f32<D>(p.part + (row + 1) * D, dv, 1.f, g);
  } else {
    tile_ready<>();   // every wave has read its last tile
    auto rows = [&](const Heads& x) {
      return [&](int r) {
        return wkey + r < p.n_kv ? static_cast<bf16_t*>(x.p) + t.b * x.b + t.kvh * x.h + static_cast<int64_t>(wkey + r) * x.n : nullptr;
      };
    };
    store_bf16<D>(smem + wave * kTurn<D>, dk, p.scale, lane, rows(p.dK));
    store_bf16<D>(smem + (WAVES + wave) * kTurn<D>, dv, 1.f, lane, rows(p.dV));
  }
}

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
