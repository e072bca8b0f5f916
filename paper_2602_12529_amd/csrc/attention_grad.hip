// Attention that keeps its statistics, and its backward pass, for any head dimension up to 128 in float32
// arithmetic (float32 operands, and bfloat16 ones of the widths that attention_grad_bf16.hip leaves).
//
//   s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  O_i = sum_j exp(s_ij - lse_i) v_j
//   P = exp(S - lse),  D_i = dO_i . O_i,  dP = dO V^T,  dS = P (dP - D)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// The backward pass runs in two kernels, one whose waves own queries (dQ, two of its three products
// recompute S and dP) and one whose waves own keys (dK, dV): seven products where five would do, but no
// two workgroups add to the same element, so nothing is summed by atomics and a launch gives the same
// bits every time.
//
// A wave owns 32 rows of its side, one to a lane and its lane + 32, and walks 32-row tiles of the other
// side, staged in LDS as float32.  Every product is computed transposed on MFMA 32x32x2 (f32), so that the
// accumulators of S^T hold, lane by lane, the other operand of the next product: in the accumulators of a
// 32x32 product lane l has column l % 32 and rows row_of(r, l / 32), r = 0 .. 15, and a product over those
// rows may take them in any order, so step r takes row_of(r, 0) from lanes 0..31 and row_of(r, 1) from the
// others.  LDS rows are padded by one word: rows and columns are both read without bank conflicts.
// Between the products nothing branches by lane: masks are selects, and only where a tile needs them (a branch to
// each score, with its statistics read from LDS behind it, cost as much as the products).  Bound by the matrix pipes,
// at head dimensions below 64 by the exponentials beside them; backward, all seven products, of 154 TFLOP/s: 2 x 8 heads,
// 2048^2, d 128 1006 us, 120 (forward 310 us, 111); d 64 517 us, 116; 2 x 16 heads, 1463 x 4997 causal, d 16 650 us, 69 (98
// with the padding of 32-wide products).
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "attention_grad.h"

namespace ff {
namespace {

constexpr int kRows = 128;   // own rows of a workgroup: four waves of 32

__device__ __forceinline__ int row_of(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

template <typename T>
__device__ __forceinline__ float4 ld4(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const float4*>(p);
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
  }
}
template <typename T>
__device__ __forceinline__ void st4(T* p, float a, float b, float c, float d) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
  else *reinterpret_cast<uint2*>(p) = make_uint2(f2bf2(a, b), f2bf2(c, d));
}

// Rows n0 .. n0 + 31 of a [*, d] matrix on their way to LDS [32][DP + 1], in registers while the tile before is worked
// on; rows at and past n_end, and columns past d, are 0.
template <typename T, int DP>
struct Stage {
  static constexpr int PIECES = 32 * (DP / 4), PER = (PIECES + 255) / 256;   // pieces of four columns, a thread's
  float4 v[PER];
  __device__ __forceinline__ void load(const T* base, int64_t stride, int64_t n0, int64_t n_end, int d) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = threadIdx.x + 256 * i, r = e / (DP / 4), c = e % (DP / 4) * 4;
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (n0 + r < n_end && c < d && e < PIECES) v[i] = ld4(base + (n0 + r) * stride + c);
    }
  }
  __device__ __forceinline__ void put(float* lds) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = threadIdx.x + 256 * i;
      if (PIECES % 256 != 0 && e >= PIECES) break;
      float* o = lds + e / (DP / 4) * (DP + 1) + e % (DP / 4) * 4;
      o[0] = v[i].x; o[1] = v[i].y; o[2] = v[i].z; o[3] = v[i].w;
    }
  }
};
// Words of a tile; a column read past its last row's (32 columns at a time) stays within them.
template <int DP> constexpr int kTileWords = 32 * (DP + 1) + (DP < 32 ? 32 - DP : 0);
template <int DP> constexpr int kBlocks = (DP + 31) / 32;   // blocks of 32 of the head dimension in products over rows
// Lane (row, g)'s operand of a product over the head dimension: element 2 s + g of step s.
template <typename T, int DP>
__device__ __forceinline__ void own_row(const T* p, bool ok, int d, int g, float (&f)[DP / 2]) {
#pragma unroll
  for (int s = 0; s < DP / 2; ++s) f[s] = 0.f;
  if (!ok) return;
#pragma unroll
  for (int s = 0; s < DP / 2; ++s)
    if (2 * s < d) f[s] = ld1<sizeof(T) == 2>(p, 2 * s + g);
}
// acc += (rows of tile) x own^T over the head dimension.
template <int DP>
__device__ __forceinline__ void mul_rows(f32x16& acc, const float* tile, const float (&own)[DP / 2], int l, int g) {
#pragma unroll
  for (int s = 0; s < DP / 2; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[l * (DP + 1) + 2 * s + g], own[s], acc, 0, 0, 0);
}
// acc[db] += tile^T x w over the tile's 32 rows: (32 of the head dimension) x (own rows).
template <int DP>
__device__ __forceinline__ void mul_cols(f32x16 (&acc)[kBlocks<DP>], const float* tile, const f32x16& w, int l, int g) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int db = 0; db < kBlocks<DP>; ++db)
      acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[row_of(r, g) * (DP + 1) + 32 * db + l], w[r], acc[db], 0, 0, 0);
}
template <typename T, int DP>
__device__ __forceinline__ void store_row(T* p, const f32x16 (&acc)[kBlocks<DP>], float f, int d, int g) {
#pragma unroll
  for (int db = 0; db < kBlocks<DP>; ++db)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int c = 32 * db + 8 * u + 4 * g;
      if (c < d) st4(p + c, acc[db][4 * u] * f, acc[db][4 * u + 1] * f, acc[db][4 * u + 2] * f, acc[db][4 * u + 3] * f);
    }
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
// Smallest and largest over the lanes, in scalar registers.
__device__ __forceinline__ int lanes_min(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { const int u = __shfl_xor(v, o, 64); v = u < v ? u : v; }
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int lanes_max(int v) { return -lanes_min(-v); }

template <typename T, int DP>
__global__ __launch_bounds__(256, 2) void attn_fwd_f32math(AttnGrad p) {
  __shared__ float ks[kTileWords<DP>], vs[kTileWords<DP>];
  const int tid = threadIdx.x, lane = tid & 63, l = lane & 31, g = lane >> 5;
  const QueryTile t = query_tile(p, kRows);
  const OwnQuery q = own_query(p, t, t.row0 + (tid >> 6) * 32 + l);
  float qf[DP / 2];
  own_row<T, DP>(q.at<T>(p.Q), q.ok, p.d, g, qf);
  f32x16 o[kBlocks<DP>];
#pragma unroll
  for (int i = 0; i < kBlocks<DP>; ++i) o[i] = zero16();
  float m = -INFINITY, sum = 0.f;
  const int lim_min = lanes_min(q.lim);
  const float hidden = p.scale > 0.f ? -INFINITY : INFINITY;   // before the factor
  const T* K = key_base<T>(p.K, t);
  const T* V = key_base<T>(p.V, t);
  Stage<T, DP> kn, vn;
  kn.load(K, p.K.n, t.key0, t.key1, p.d);
  vn.load(V, p.V.n, t.key0, t.key1, p.d);
  for (int64_t k0 = t.key0; k0 < t.key1; k0 += 32) {
    __syncthreads();
    kn.put(ks);
    vn.put(vs);
    __syncthreads();
    kn.load(K, p.K.n, k0 + 32, t.key1, p.d);
    vn.load(V, p.V.n, k0 + 32, t.key1, p.d);
    f32x16 s = zero16();
    mul_rows<DP>(s, ks, qf, l, g);
    if (k0 + 32 > lim_min) {   // some query does not see all of the tile's keys
      const int left = q.lim - static_cast<int>(k0) - 4 * g;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = row_of(r, 0) < left ? s[r] : hidden;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] *= p.scale_log2;
      mx = fmaxf(mx, s[r]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m, mx), base = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m - base);
    float part = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(s[r] - base);
      part += s[r];
    }
    sum = fmaf(sum, alpha, part + __shfl_xor(part, 32, 64));
    m = m_new;
#pragma unroll
    for (int i = 0; i < kBlocks<DP>; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
    mul_cols<DP>(o, vs, s, l, g);
  }
  if (!q.ok) return;
  const float inv = sum > 0.f || sum != sum ? 1.0f / sum : 0.f;
  const float lse = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
  if (p.splits > 1) {
    const int64_t row = split_row(p, t, q);
    store_row<float, DP>(p.part + row * p.d, o, inv, p.d, g);
    if (g == 0) p.part_lse[row] = lse;
  } else {
    store_row<T, DP>(q.at<T>(p.O), o, inv, p.d, g);
    if (g == 0) p.lse[q.stat] = lse;
  }
}

template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 128 ? 1 : 2) void attn_dq_f32math(AttnGrad p) {
  __shared__ float ks[kTileWords<DP>], vs[kTileWords<DP>];
  const int tid = threadIdx.x, lane = tid & 63, l = lane & 31, g = lane >> 5;
  const QueryTile t = query_tile(p, kRows);
  const OwnQuery q = own_query(p, t, t.row0 + (tid >> 6) * 32 + l);
  float qf[DP / 2], gf[DP / 2];
  own_row<T, DP>(q.at<T>(p.Q), q.ok, p.d, g, qf);
  own_row<T, DP>(q.at<T>(p.dO), q.ok, p.d, g, gf);
  float delta = 0.f;
  {
    float of[DP / 2];
    own_row<T, DP>(q.at<T>(p.O), q.ok, p.d, g, of);
#pragma unroll
    for (int s = 0; s < DP / 2; ++s) delta = fmaf(gf[s], of[s], delta);
  }
  delta += __shfl_xor(delta, 32, 64);
  if (q.ok && g == 0 && t.split == 0) p.delta[q.stat] = delta;
  const float lse2 = q.ok ? p.lse[q.stat] * 1.4426950408889634f : 0.f;
  const int lim_min = lanes_min(q.lim);
  f32x16 dq[kBlocks<DP>];
#pragma unroll
  for (int i = 0; i < kBlocks<DP>; ++i) dq[i] = zero16();
  const T* K = key_base<T>(p.K, t);
  const T* V = key_base<T>(p.V, t);
  Stage<T, DP> kn, vn;
  kn.load(K, p.K.n, t.key0, t.key1, p.d);
  vn.load(V, p.V.n, t.key0, t.key1, p.d);
  for (int64_t k0 = t.key0; k0 < t.key1; k0 += 32) {
    __syncthreads();
    kn.put(ks);
    vn.put(vs);
    __syncthreads();
    kn.load(K, p.K.n, k0 + 32, t.key1, p.d);
    vn.load(V, p.V.n, k0 + 32, t.key1, p.d);
    f32x16 s = zero16(), dp = zero16();
    mul_rows<DP>(s, ks, qf, l, g);
    mul_rows<DP>(dp, vs, gf, l, g);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.scale_log2, -lse2)) * (dp[r] - delta);
    if (k0 + 32 > lim_min) {
      const int left = q.lim - static_cast<int>(k0) - 4 * g;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = row_of(r, 0) < left ? s[r] : 0.f;
    }
    mul_cols<DP>(dq, ks, s, l, g);
  }
  if (!q.ok) return;
  if (p.splits > 1) store_row<float, DP>(p.part + split_row(p, t, q) * p.d, dq, p.scale, p.d, g);
  else store_row<T, DP>(q.at<T>(p.dQ), dq, p.scale, p.d, g);
}

template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 128 ? 1 : 2) void attn_dkv_f32math(AttnGrad p) {
  __shared__ float qs[kTileWords<DP>], gs[kTileWords<DP>];
  __shared__ __attribute__((aligned(16))) float lse_s[32], del_s[32];
  const int tid = threadIdx.x, lane = tid & 63, l = lane & 31, g = lane >> 5;
  const KeyTile t = key_tile(p, kRows);
  const int64_t key = t.key0 + (tid >> 6) * 32 + l;
  const bool ok = key < p.n_kv, seen = key < t.len;
  float kf[DP / 2], vf[DP / 2];
  own_row<T, DP>(key_base<T>(p.K, t) + key * p.K.n, seen, p.d, g, kf);
  own_row<T, DP>(key_base<T>(p.V, t) + key * p.V.n, seen, p.d, g, vf);
  f32x16 dk[kBlocks<DP>], dv[kBlocks<DP>];
#pragma unroll
  for (int i = 0; i < kBlocks<DP>; ++i) { dk[i] = zero16(); dv[i] = zero16(); }
  // queries that see this key: first .. n_q - 1 (keys that none sees are set to 0 at the end)
  const int first = p.causal ? static_cast<int>(key - (t.len - p.n_q)) : 0;
  const int first_max = lanes_max(first);
  Stage<T, DP> qn, gn;
  float lse_n = 0.f, del_n = 0.f;
  TileWalk<32> w(p, t);
  auto load = [&]() {
    if (!w.more()) return;
    const int64_t h = t.kvh * p.group + w.head, i0 = w.tile * 32;
    qn.load(static_cast<const T*>(p.Q.p) + t.b * p.Q.b + h * p.Q.h, p.Q.n, i0, p.n_q, p.d);
    gn.load(static_cast<const T*>(p.dO.p) + t.b * p.dO.b + h * p.dO.h, p.dO.n, i0, p.n_q, p.d);
    if (tid < 32) {
      const int64_t st = (t.b * p.heads + h) * p.n_q + i0 + tid;
      const bool in = i0 + tid < p.n_q;
      // queries past the last, and those that see no key, have P = exp2(-inf)
      const float lse = in ? p.lse[st] : INFINITY;
      lse_n = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
      del_n = in ? p.delta[st] : 0.f;
    }
  };
  load();
  while (w.more()) {
    const int64_t i0 = w.tile * 32;
    __syncthreads();
    qn.put(qs);
    gn.put(gs);
    if (tid < 32) {
      lse_s[tid] = lse_n;
      del_s[tid] = del_n;
    }
    __syncthreads();
    w.next();
    load();
    f32x16 s = zero16(), dp = zero16();
    mul_rows<DP>(s, qs, kf, l, g);
    mul_rows<DP>(dp, gs, vf, l, g);
#pragma unroll
    for (int u = 0; u < 4; ++u) {   // rows row_of(4 u, g) .. + 3
      const float4 ls = *reinterpret_cast<const float4*>(lse_s + row_of(4 * u, g));
      s[4 * u] = __builtin_amdgcn_exp2f(fmaf(s[4 * u], p.scale_log2, -ls.x));
      s[4 * u + 1] = __builtin_amdgcn_exp2f(fmaf(s[4 * u + 1], p.scale_log2, -ls.y));
      s[4 * u + 2] = __builtin_amdgcn_exp2f(fmaf(s[4 * u + 2], p.scale_log2, -ls.z));
      s[4 * u + 3] = __builtin_amdgcn_exp2f(fmaf(s[4 * u + 3], p.scale_log2, -ls.w));
    }
    if (i0 < first_max) {
      const int skip = first - static_cast<int>(i0) - 4 * g;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = row_of(r, 0) >= skip ? s[r] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float4 de = *reinterpret_cast<const float4*>(del_s + row_of(4 * u, g));
      dp[4 * u] = s[4 * u] * (dp[4 * u] - de.x);
      dp[4 * u + 1] = s[4 * u + 1] * (dp[4 * u + 1] - de.y);
      dp[4 * u + 2] = s[4 * u + 2] * (dp[4 * u + 2] - de.z);
      dp[4 * u + 3] = s[4 * u + 3] * (dp[4 * u + 3] - de.w);
    }
    mul_cols<DP>(dv, gs, s, l, g);
    mul_cols<DP>(dk, qs, dp, l, g);
  }
  if (!ok) return;
  if (!seen) {
#pragma unroll
    for (int i = 0; i < kBlocks<DP>; ++i) { dk[i] = zero16(); dv[i] = zero16(); }
  }
  if (p.splits > 1) {
    const int64_t row = (((static_cast<int64_t>(t.split) * p.B + t.b) * p.kv_heads + t.kvh) * p.n_kv + key) * 2;
    store_row<float, DP>(p.part + row * p.d, dk, p.scale, p.d, g);
    store_row<float, DP>(p.part + (row + 1) * p.d, dv, 1.f, p.d, g);
  } else {
    store_row<T, DP>(static_cast<T*>(p.dK.p) + t.b * p.dK.b + t.kvh * p.dK.h + key * p.dK.n, dk, p.scale, p.d, g);
    store_row<T, DP>(static_cast<T*>(p.dV.p) + t.b * p.dV.b + t.kvh * p.dV.h + key * p.dV.n, dv, 1.f, p.d, g);
  }
}

// Joins of the partial results of `splits` workgroups, in an order that depends on their number alone.
// Forward: O = sum_s exp(lse_s - lse) O_s, a wave a row (b, head, query): lane s holds the weight of split s (at most
// 64), and 64 / (d / 4) groups of lanes take the splits in turn, four columns a lane.
constexpr int kMaxSplits = 64;
template <typename T>
__global__ __launch_bounds__(256) void attn_join_fwd(AttnGrad p) {
  const int64_t rows = p.B * p.heads * p.n_q;
  const int lane = threadIdx.x & 63, per = p.d / 4, groups = 64 / per, mine = lane / per;
  for (int64_t row = blockIdx.x * int64_t(4) + (threadIdx.x >> 6); row < rows; row += gridDim.x * int64_t(4)) {
    const float lse = lane < p.splits ? p.part_lse[lane * rows + row] : -INFINITY;
    const float top = wave_max(lse), base = top == -INFINITY ? 0.f : top;
    const float w = exp2f((lse - base) * 1.4426950408889634f), total = wave_sum(w);
    const int c = lane % per * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    // every lane takes every turn: a lane that had left would not hand out its weight
    for (int s0 = 0; s0 < p.splits; s0 += groups) {
      const int s = s0 + mine;
      const float f = __shfl(w, s & 63, 64);
      if (mine >= groups || s >= p.splits) continue;
      const float4 x = *reinterpret_cast<const float4*>(p.part + (s * rows + row) * p.d + c);
      o.x = fmaf(f, x.x, o.x); o.y = fmaf(f, x.y, o.y); o.z = fmaf(f, x.z, o.z); o.w = fmaf(f, x.w, o.w);
    }
    float4 all = o;   // the groups' sums, in order
    for (int k = 1; k < groups; ++k) {
      const int from = lane % per + k * per;
      all.x += __shfl(o.x, from, 64); all.y += __shfl(o.y, from, 64); all.z += __shfl(o.z, from, 64); all.w += __shfl(o.w, from, 64);
    }
    if (mine != 0) continue;
    const float inv = total == 0.f ? 0.f : 1.0f / total;
    const int64_t i = row % p.n_q, h = row / p.n_q % p.heads, b = row / p.n_q / p.heads;
    st4(static_cast<T*>(p.O.p) + b * p.O.b + h * p.O.h + i * p.O.n + c, all.x * inv, all.y * inv, all.z * inv, all.w * inv);
    if (c == 0) p.lse[row] = total == 0.f ? -INFINITY : base + logf(total);
  }
}
// Sums: part [splits][B][heads][n][outs][d] to out[0 .. outs - 1].
struct JoinSum {
  const float* part;
  int64_t splits, B, heads, n, d, outs;
  Heads out[2];
};
template <typename T>
__global__ __launch_bounds__(256) void attn_join_sum(JoinSum p) {
  const int64_t rows = p.B * p.heads * p.n * p.outs, per = p.d / 4;
  for (int64_t e = blockIdx.x * int64_t(256) + threadIdx.x; e < rows * per; e += gridDim.x * int64_t(256)) {
    const int64_t row = e / per, c = e % per * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int64_t s = 0; s < p.splits; ++s) {
      const float4 x = *reinterpret_cast<const float4*>(p.part + (s * rows + row) * p.d + c);
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    const Heads& t = p.out[row % p.outs];
    const int64_t r = row / p.outs, i = r % p.n, h = r / p.n % p.heads, b = r / p.n / p.heads;
    st4(static_cast<T*>(t.p) + b * t.b + h * t.h + i * t.n + c, o.x, o.y, o.z, o.w);
  }
}

unsigned join_blocks(int64_t threads) {
  const int64_t b = (threads + 255) / 256;
  return static_cast<unsigned>(b < 8192 ? b : 8192);
}

// How a launch is cut: own rows a workgroup, and splits of the other side's tiles where that is quicker.  The estimate
// counts in tiles of 64 rows: a compute unit works on two workgroups at once, and on a last one alone in 0.6 of a pair's
// time; a partial result of 128 rows, written and read, is worth 6 tiles and the join 3.  Causal work is uneven (half of
// it on average, the longest workgroups first): the longer of the longest workgroup and the units' share.  dK and dV,
// us with the join, bf16: 96 workgroups of 512 tiles (a video's cross-attention) 5 splits 400, 6 splits 540; 192 of 512 tiles
// 2 splits 895, 8 splits 795; 288 of 24 tiles 1 split 92, 2 splits 103; causal 256 of 128 tiles 1 split 188, 2 splits
// 149, 4 splits 113.  In float32 arithmetic a tile takes eight times as long, so that partial results cost little, and one
// workgroup nearly fills the unit's matrix pipes: a last one alone takes 0.53 of a pair's time (all of a backward pass:
// 132 workgroups of 24 tiles for dK and dV 1 split 208, 5 splits 157; 32 of 8 tiles 1 split 145, 2 splits 93; 256 of 32
// tiles 1 split 1007, 2 splits 1080; 12 of 7 tiles forward 1 split 70, 7 splits 24), and its first loads count as a tile
// (causal splits of fewer than four tiles do not pay: 128 workgroups of 16 tiles 4 splits 139, 6 splits 164).  bf16 splits
// of fewer than four tiles pay for few rows only (one token: 16 heads, 420 keys 1 split 14.4, 7 splits 10.9; 1024^2
// causal backward, 16 heads 4 splits 48, 8 splits 51).
// The estimate knows neither the samples' lengths (they count as n_kv) nor that the kernels of head dimension 64 leave
// registers and LDS for a third workgroup on a unit, and charges the partial result of a narrow tile with all its 32 rows.
struct Cut { int64_t blocks; int splits; };
Cut cut(int64_t bh, int64_t own, int rows, int64_t other, bool causal, bool f32math) {
  constexpr double units = 256;
  const double part_tiles = f32math ? 0.75 : 6, join_tiles = f32math ? 1 : 3, alone = f32math ? 0.53 : 0.6, begin = f32math ? 1 : 0;
  const int64_t blocks = bh * ((own + rows - 1) / rows), tiles = (other + 63) / 64;
  const int64_t shortest = rows == kNarrowRows || (f32math && !causal) ? 1 : 4, most = tiles / shortest < kMaxSplits ? tiles / shortest : kMaxSplits;
  Cut best{blocks, 1};
  double least = 0;
  for (int64_t s = 1; blocks > 0 && s <= (most < 1 ? 1 : most); ++s) {
    const double part = begin + (s > 1 ? part_tiles * rows / 128 : 0), one = static_cast<double>(tiles) / s, n = static_cast<double>(blocks) * s;
    const int64_t each = static_cast<int64_t>(std::ceil(n / units));
    const double even = (each / 2 + (each % 2 ? alone : 0.0)) * (one + part);
    const double uneven = std::max(one + part, n / units / 2 * (one / 2 + part));
    const double cost = (causal ? uneven : even) + (s > 1 ? join_tiles : 0);
    if (s == 1 || cost < least) { least = cost; best.splits = static_cast<int>(s); }
  }
  return best;
}

// bf16 of head dimension 64 or 128 runs on the bf16 matrix instructions.
bool wide_path(const ff_attn_shape& a) { return a.dtype == FF_BF16 && (a.head_dim == 64 || a.head_dim == 128); }

// Key heads whose causal workgroups run together, the longest first: as many as fill an XCD's 64 places twice, so that what
// runs last is short (causal 2047^2, 16 key heads of 64 tiles: see there).
int together(const ff_attn_shape& a, const Cut& c) {
  const int64_t bh = a.B * a.kv_heads, each = c.blocks / bh * c.splits;
  if (!a.causal) return 1;
  int g = 1;
  while (bh % (16 * g) == 0 && 2 * g * each <= 128) g *= 2;   // whole groups on each of the eight XCDs
  return g;
}

struct Plan { Cut fwd, dq, dkv; bool bf16, narrow; };
Plan plan(const ff_attn_shape& a) {
  const int64_t group = a.heads / a.kv_heads, bh = a.B * a.kv_heads, own = group * a.n_q;
  Plan p{};
  p.bf16 = wide_path(a);
  p.narrow = p.bf16 && own <= kNarrowRows;
  p.fwd = p.dq = cut(bh, own, p.narrow ? kNarrowRows : kRows, a.n_kv, a.causal != 0, !p.bf16);
  p.dkv = cut(bh, a.n_kv, kRows, group * ((a.n_q + 63) / 64) * 64, a.causal != 0, !p.bf16);
  return p;
}
// Workspace: forward partials; backward D, then the larger of the two kernels' partials.
struct Room { size_t part, lse, delta; };
Room room_fwd(const ff_attn_shape& a, const Plan& p) {
  const size_t rows = static_cast<size_t>(a.B * a.heads * a.n_q) * (p.fwd.splits > 1 ? p.fwd.splits : 0);
  return {rows * a.head_dim * 4, rows * 4, 0};
}
Room room_bwd(const ff_attn_shape& a, const Plan& p) {
  const size_t q = static_cast<size_t>(a.B * a.heads * a.n_q), k = static_cast<size_t>(a.B * a.kv_heads * a.n_kv) * 2;
  const size_t stat = p.bf16 ? static_cast<size_t>(a.B * a.heads * stat_rows(a.n_q)) * 2 : q;
  const size_t pq = p.dq.splits > 1 ? q * p.dq.splits : 0, pk = p.dkv.splits > 1 ? k * p.dkv.splits : 0;
  return {(pq > pk ? pq : pk) * a.head_dim * 4, 0, stat * 4};
}

size_t bytes_fwd(const Room& r) {
  Carver c(nullptr, 0);
  if (r.part) { c.take(r.part); c.take(r.lse); }
  return c.off;
}
size_t bytes_bwd(const Room& r) {
  Carver c(nullptr, 0);
  c.take(r.delta);
  c.take(r.part);
  return c.off;
}

// Pairs of a query and a key that it sees, for the profiler: causal, the last query sees n_kv keys and each one before it
// one fewer.  Every sample counts as n_kv keys, for their lengths lie on the device.
double seen_pairs(const ff_attn_shape& a) {
  const double n_kv = static_cast<double>(a.n_kv), rows = static_cast<double>(a.causal && a.n_kv < a.n_q ? a.n_kv : a.n_q);
  return static_cast<double>(a.B) * a.heads * (rows * n_kv - (a.causal ? rows * (rows - 1) / 2 : 0.0));
}

Heads view(const ff_heads& t) { return {t.data, t.batch, t.head, t.token}; }

AttnGrad args(const ff_attn_shape& a, const ff_heads& Q, const ff_heads& K, const ff_heads& V) {
  AttnGrad p{};
  p.B = a.B; p.heads = a.heads; p.kv_heads = a.kv_heads; p.group = a.heads / a.kv_heads;
  p.n_q = a.n_q; p.n_kv = a.n_kv; p.d = static_cast<int>(a.head_dim);
  p.causal = a.causal;
  p.kv_len = a.kv_len;
  const double scale = a.scale != 0.f ? static_cast<double>(a.scale) : 1.0 / std::sqrt(static_cast<double>(a.head_dim));
  p.scale = static_cast<float>(scale);
  p.scale_log2 = static_cast<float>(scale * 1.4426950408889634);
  p.Q = view(Q); p.K = view(K); p.V = view(V);
  return p;
}

#define FF_WIDTHS(KERNEL)                                                                                          \
  do {                                                                                                             \
    const dim3 grid(static_cast<unsigned>(blocks));                                                                \
    if (a.dtype == FF_BF16) {                                                                                      \
      if (p.d <= 16) hipLaunchKernelGGL((KERNEL<bf16_t, 16>), grid, dim3(256), 0, s, p);                           \
      else if (p.d <= 32) hipLaunchKernelGGL((KERNEL<bf16_t, 32>), grid, dim3(256), 0, s, p);                      \
      else if (p.d <= 64) hipLaunchKernelGGL((KERNEL<bf16_t, 64>), grid, dim3(256), 0, s, p);                      \
      else hipLaunchKernelGGL((KERNEL<bf16_t, 128>), grid, dim3(256), 0, s, p);                                    \
    } else {                                                                                                       \
      if (p.d <= 16) hipLaunchKernelGGL((KERNEL<float, 16>), grid, dim3(256), 0, s, p);                            \
      else if (p.d <= 32) hipLaunchKernelGGL((KERNEL<float, 32>), grid, dim3(256), 0, s, p);                       \
      else if (p.d <= 64) hipLaunchKernelGGL((KERNEL<float, 64>), grid, dim3(256), 0, s, p);                       \
      else hipLaunchKernelGGL((KERNEL<float, 128>), grid, dim3(256), 0, s, p);                                     \
    }                                                                                                              \
  } while (0)

int check_shape(const char* fn, const ff_attn_shape* a) {
  if (!a) return fail(FF_EINVAL, "%s: null shape", fn);
  if (a->dtype != FF_F32 && a->dtype != FF_BF16) return fail(FF_EINVAL, "%s: bad dtype %d", fn, a->dtype);
  if (a->B < 0 || a->heads < 1 || a->kv_heads < 1 || a->n_q < 0 || a->n_kv < 0 || a->head_dim < 1)
    return fail(FF_EINVAL, "%s: bad shape", fn);
  if (a->heads % a->kv_heads) return fail(FF_EINVAL, "%s: heads %lld not a multiple of kv_heads %lld", fn, (long long)a->heads, (long long)a->kv_heads);
  if (a->causal != 0 && a->causal != 1) return fail(FF_EINVAL, "%s: causal %d", fn, a->causal);
  if (a->scale != 0.f && !(std::fabs(a->scale) >= 0x1p-64f && std::fabs(a->scale) <= 0x1p64f))
    return fail(FF_EINVAL, "%s: scale %g (0, or a magnitude between 2^-64 and 2^64)", fn, a->scale);
  if (reinterpret_cast<uintptr_t>(a->kv_len) % 4) return fail(FF_EINVAL, "%s: kv_len must be 4-byte aligned", fn);
  const int unit = a->dtype == FF_BF16 ? 8 : 4;
  if (a->head_dim > 128 || a->head_dim % unit) return fail(FF_EUNSUPPORTED, "%s: head_dim %lld (a multiple of %d up to 128)", fn, (long long)a->head_dim, unit);
  constexpr int64_t most = int64_t(1) << 27;
  if (a->n_q > most || a->n_kv > most || a->heads > 65536 || a->B > most) return fail(FF_EUNSUPPORTED, "%s: n_q, n_kv or B above 2^27 or heads above 2^16", fn);
  const double tiles = static_cast<double>(a->B) * a->heads * (static_cast<double>(a->n_q + a->n_kv) / 32 + 2);
  if (tiles >= 16777216.0) return fail(FF_EUNSUPPORTED, "%s: too many workgroups", fn);
  return FF_OK;
}
// Alignment and strides; outputs have to have an element of their own at every index.
int check_heads(const char* fn, const char* name, const ff_attn_shape& a, const ff_heads* t, bool key_side, bool output) {
  const int64_t heads = key_side ? a.kv_heads : a.heads, n = key_side ? a.n_kv : a.n_q;
  if (!t) return fail(FF_EINVAL, "%s: null %s", fn, name);
  if (a.B == 0 || n == 0) return FF_OK;
  if (!t->data) return fail(FF_EINVAL, "%s: null %s", fn, name);
  if (!aligned16(t->data)) return fail(FF_EINVAL, "%s: %s must be 16-byte aligned", fn, name);
  const int unit = a.dtype == FF_BF16 ? 8 : 4;
  struct Axis { int64_t stride, extent; } dims[3] = {{t->batch, a.B}, {t->head, heads}, {t->token, n}};
  for (const Axis& x : dims) {
    if (x.extent == 1) continue;   // no stride that matters
    if (x.stride < 0 || x.stride % unit) return fail(FF_EINVAL, "%s: strides of %s must be non-negative multiples of %d", fn, name, unit);
    if (&x == &dims[2] && x.stride > int64_t(1) << 24) return fail(FF_EUNSUPPORTED, "%s: token stride of %s above 2^24", fn, name);
    if (x.stride >= int64_t(1) << 40) return fail(FF_EUNSUPPORTED, "%s: stride of %s above 2^40", fn, name);
  }
  if (output) {   // from the innermost axis out, each stride passes over all that lies within it
    std::sort(dims, dims + 3, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
    int64_t span = a.head_dim;
    for (const Axis& x : dims) {
      if (x.extent == 1) continue;
      if (x.stride < span) return fail(FF_EINVAL, "%s: rows of the output %s overlap", fn, name);
      span += x.stride * (x.extent - 1);
    }
  }
  return FF_OK;
}
// An output at the address of another operand shares its first element at least.  Other overlaps are not looked for: slices
// of one buffer lie between one another without touching.
struct Operand { const char* name; const void* p; bool empty; };
int check_apart(const char* fn, std::initializer_list<Operand> outputs, std::initializer_list<Operand> inputs) {
  for (const Operand* o = outputs.begin(); o != outputs.end(); ++o) {
    if (o->empty) continue;
    for (const Operand& x : inputs)
      if (!x.empty && x.p == o->p) return fail(FF_EINVAL, "%s: the output %s is the input %s", fn, o->name, x.name);
    for (const Operand* x = o + 1; x != outputs.end(); ++x)
      if (!x->empty && x->p == o->p) return fail(FF_EINVAL, "%s: the outputs %s and %s are the same", fn, o->name, x->name);
  }
  return FF_OK;
}
}  // namespace
}  // namespace ff

using namespace ff;

extern "C" {

int ff_attention_forward_workspace_size(const ff_attn_shape* shape, size_t* bytes) {
  const char* fn = "ff_attention_forward_workspace_size";
  FF_TRY(check_shape(fn, shape));
  if (!bytes) return fail(FF_EINVAL, "%s: null output", fn);
  *bytes = bytes_fwd(room_fwd(*shape, plan(*shape)));
  return FF_OK;
}

int ff_attention_backward_workspace_size(const ff_attn_shape* shape, size_t* bytes) {
  const char* fn = "ff_attention_backward_workspace_size";
  FF_TRY(check_shape(fn, shape));
  if (!bytes) return fail(FF_EINVAL, "%s: null output", fn);
  *bytes = bytes_bwd(room_bwd(*shape, plan(*shape)));
  return FF_OK;
}

int ff_attention_forward(const ff_attn_shape* shape, const ff_heads* Q, const ff_heads* K, const ff_heads* V,
                         const ff_heads* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "ff_attention_forward";
  FF_TRY(check_shape(fn, shape));
  const ff_attn_shape& a = *shape;
  FF_TRY(check_heads(fn, "Q", a, Q, false, false));
  FF_TRY(check_heads(fn, "K", a, K, true, false));
  FF_TRY(check_heads(fn, "V", a, V, true, false));
  FF_TRY(check_heads(fn, "out", a, out, false, true));
  if (a.B == 0 || a.n_q == 0) return FF_OK;
  if (!lse || reinterpret_cast<uintptr_t>(lse) % 4) return fail(FF_EINVAL, "%s: lse null or not 4-byte aligned", fn);
  const Plan pl = plan(a);
  const Room r = room_fwd(a, pl);
  const size_t need = bytes_fwd(r);
  if (need > 0 && (!workspace || ws_bytes < need)) return fail(FF_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
  if (!aligned16(workspace)) return fail(FF_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  const bool no_keys = a.n_kv == 0;
  FF_TRY(check_apart(fn, {{"out", out->data, false}, {"lse", lse, false}},
                     {{"Q", Q->data, false}, {"K", K->data, no_keys}, {"V", V->data, no_keys}}));
  if (pl.bf16) FF_TRY(attn_bf16_prepare());
  Carver c(workspace, ws_bytes);
  AttnGrad p = args(a, *Q, *K, *V);
  p.O = view(*out);
  p.lse = lse;
  p.splits = pl.fwd.splits;
  p.mix = together(a, pl.fwd);
  if (p.splits > 1) {
    p.part = static_cast<float*>(c.take(r.part));
    p.part_lse = static_cast<float*>(c.take(r.lse));
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double es = static_cast<double>(dtype_size(a.dtype));
  const double flops = 4.0 * seen_pairs(a) * a.head_dim;
  const double bytes = 2.0 * es * a.B * a.head_dim * (static_cast<double>(a.heads) * a.n_q + static_cast<double>(a.kv_heads) * a.n_kv);
  {
    const int64_t blocks = pl.fwd.blocks * p.splits;
    LaunchScope ls("attn_forward", s, flops, bytes);
    if (pl.bf16) attn_fwd_bf16(p, blocks, pl.narrow, s);
    else FF_WIDTHS(attn_fwd_f32math);
    FF_TRY(ls.status());
  }
  if (p.splits > 1) {
    const int64_t threads = a.B * a.heads * a.n_q * 64;
    LaunchScope ls("attn_forward_join", s, 0.0, static_cast<double>(r.part));
    if (a.dtype == FF_BF16) hipLaunchKernelGGL(attn_join_fwd<bf16_t>, dim3(join_blocks(threads)), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(attn_join_fwd<float>, dim3(join_blocks(threads)), dim3(256), 0, s, p);
    FF_TRY(ls.status());
  }
  return FF_OK;
}

int ff_attention_backward(const ff_attn_shape* shape, const ff_heads* dO, const ff_heads* Q, const ff_heads* K,
                          const ff_heads* V, const ff_heads* out, const float* lse, const ff_heads* dQ,
                          const ff_heads* dK, const ff_heads* dV, void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "ff_attention_backward";
  FF_TRY(check_shape(fn, shape));
  const ff_attn_shape& a = *shape;
  FF_TRY(check_heads(fn, "dO", a, dO, false, false));
  FF_TRY(check_heads(fn, "Q", a, Q, false, false));
  FF_TRY(check_heads(fn, "K", a, K, true, false));
  FF_TRY(check_heads(fn, "V", a, V, true, false));
  FF_TRY(check_heads(fn, "out", a, out, false, false));
  FF_TRY(check_heads(fn, "dQ", a, dQ, false, true));
  FF_TRY(check_heads(fn, "dK", a, dK, true, true));
  FF_TRY(check_heads(fn, "dV", a, dV, true, true));
  if (a.B == 0 || (a.n_q == 0 && a.n_kv == 0)) return FF_OK;
  if (a.n_q > 0 && (!lse || reinterpret_cast<uintptr_t>(lse) % 4)) return fail(FF_EINVAL, "%s: lse null or not 4-byte aligned", fn);
  const Plan pl = plan(a);
  const Room r = room_bwd(a, pl);
  const size_t need = bytes_bwd(r);
  if (need > 0 && (!workspace || ws_bytes < need)) return fail(FF_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
  if (!aligned16(workspace)) return fail(FF_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  const bool no_keys = a.n_kv == 0, no_rows = a.n_q == 0;
  FF_TRY(check_apart(fn, {{"dQ", dQ->data, no_rows}, {"dK", dK->data, no_keys}, {"dV", dV->data, no_keys}},
                     {{"dO", dO->data, no_rows}, {"Q", Q->data, no_rows}, {"K", K->data, no_keys}, {"V", V->data, no_keys},
                      {"out", out->data, no_rows}, {"lse", lse, no_rows}}));
  if (pl.bf16) FF_TRY(attn_bf16_prepare());
  Carver c(workspace, ws_bytes);
  AttnGrad p = args(a, *Q, *K, *V);
  p.O = view(*out);
  p.dO = view(*dO);
  p.dQ = view(*dQ); p.dK = view(*dK); p.dV = view(*dV);
  p.lse = const_cast<float*>(lse);
  p.delta = static_cast<float*>(c.take(r.delta));
  p.part = static_cast<float*>(c.take(r.part));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const double es = static_cast<double>(dtype_size(a.dtype));
  const double work = seen_pairs(a) * a.head_dim;
  const double rows_q = es * a.B * a.heads * a.n_q * a.head_dim, rows_k = es * a.B * a.kv_heads * a.n_kv * a.head_dim;
  if (a.n_q > 0) {
    p.splits = pl.dq.splits;
    p.mix = together(a, pl.dq);
    {
      const int64_t blocks = pl.dq.blocks * p.splits;
      LaunchScope ls("attn_backward_dq", s, 6.0 * work, 4.0 * rows_q + 2.0 * rows_k);
      if (pl.bf16) attn_dq_bf16(p, blocks, pl.narrow, s);
      else FF_WIDTHS(attn_dq_f32math);
      FF_TRY(ls.status());
    }
    if (p.splits > 1) {
      JoinSum j{p.part, p.splits, a.B, a.heads, a.n_q, a.head_dim, 1, {p.dQ, p.dQ}};
      const unsigned g = join_blocks(a.B * a.heads * a.n_q * (a.head_dim / 4));
      LaunchScope ls("attn_backward_join", s, 0.0, 4.0 * p.splits * a.B * a.heads * a.n_q * a.head_dim);
      if (a.dtype == FF_BF16) hipLaunchKernelGGL(attn_join_sum<bf16_t>, dim3(g), dim3(256), 0, s, j);
      else hipLaunchKernelGGL(attn_join_sum<float>, dim3(g), dim3(256), 0, s, j);
      FF_TRY(ls.status());
    }
  }
  if (a.n_kv > 0) {
    p.splits = pl.dkv.splits;
    p.mix = together(a, pl.dkv);
    {
      const int64_t blocks = pl.dkv.blocks * p.splits;
      LaunchScope ls("attn_backward_dkv", s, 8.0 * work, 2.0 * rows_q + 4.0 * rows_k);
      if (pl.bf16) attn_dkv_bf16(p, blocks, s);
      else FF_WIDTHS(attn_dkv_f32math);
      FF_TRY(ls.status());
    }
    if (p.splits > 1) {
      JoinSum j{p.part, p.splits, a.B, a.kv_heads, a.n_kv, a.head_dim, 2, {p.dK, p.dV}};
      const unsigned g = join_blocks(a.B * a.kv_heads * a.n_kv * 2 * (a.head_dim / 4));
      LaunchScope ls("attn_backward_join", s, 0.0, 8.0 * p.splits * a.B * a.kv_heads * a.n_kv * a.head_dim);
      if (a.dtype == FF_BF16) hipLaunchKernelGGL(attn_join_sum<bf16_t>, dim3(g), dim3(256), 0, s, j);
      else hipLaunchKernelGGL(attn_join_sum<float>, dim3(g), dim3(256), 0, s, j);
      FF_TRY(ls.status());
    }
  }
  return FF_OK;
}

}  // extern "C"
