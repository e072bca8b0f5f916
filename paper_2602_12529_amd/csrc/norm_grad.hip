// The affine norm and the gradients of the affine and the modulated norm.
//
//   xh = (x - mean) rstd (RMS norm: mean = 0), y = xh m + a
//   g = dy m,  dx = rstd (g - mean(g) - xh mean(g xh)) + add,  dm = sum_rows dy xh,  da = sum_rows dy
//
// Bound by memory: dy and x are read once, dx is written once.  A row is held in registers by TPR
// threads, 8 NI columns each, so that the statistics (recomputed: they cost two reductions of what is
// in registers, stored ones a forward pass that keeps them) and the gradient need no second read.  A
// workgroup walks every strips-th row of one sample with its columns' sums of dy xh and dy in registers,
// and leaves them as one partial row; a second kernel adds a sample's strips in order.  The workgroups of
// a sample thus read neighbouring rows at any time (9000 x 10000 bf16 with `add` 147 us, a run of rows to
// each workgroup 182).  No atomics: a launch gives the same bits every time.  Reached: 32760 x 1536 bf16
// with `add` 65 us, 6.2 TB/s of what is read and written once (78 with nothing in the caches); 32768 x 3072 without 104 us,
// 5.8 TB/s (122).
#include <cmath>
#include <initializer_list>
#include <utility>

#include "../../include/ff_grad.h"
#include "dev.h"
#include "ff_internal.h"
#include "norm_plan.h"

namespace ff {
namespace {

struct NormGrad {
  const void* dy; int64_t lddy;
  const void* x; int64_t ldx;
  const void* add; int64_t ldadd;
  void* dx; int64_t lddx;
  const void* w;                            // affine: [H] of dtype, or null
  const float* scale; int64_t mod_ld;       // modulated: m = 1 + scale[sample], or null
  float* dm; float* da; int64_t dmod_ld;    // outputs, or null: written here where a sample is one strip
  float* part;                              // else [samples][strips][part_ld]: H sums of dy xh, H sums of dy
  int64_t part_ld;
  int64_t rows, H, rows_per_sample;
  int64_t strips, strip_rows;
  int layer;
  float eps;
};

struct NormFwd {
  const void* x; int64_t ldx;
  const void* w; const void* bias;
  void* y; int64_t ldy;
  int64_t rows, H, block_rows;
  int layer;
  float eps;
};

// Sum over aligned groups of W lanes, in every lane: neighbours by DPP (a few cycles each, where a shuffle is a trip
// through LDS), rows of 16 and halves by the lane-swap instructions, which put the two sides' values side by side.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int W>
__device__ __forceinline__ float group_sum(float v) {
  v = dpp_add<0xB1>(v);                  // quad_perm [1, 0, 3, 2]
  v = dpp_add<0x4E>(v);                  // quad_perm [2, 3, 0, 1]
  v = dpp_add<0x141>(v);                 // row_half_mirror
  if constexpr (W >= 16) v = dpp_add<0x140>(v);   // row_mirror
  if constexpr (W >= 32) {
    const uint32_t u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (W >= 64) {
    const uint32_t u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}
// Sums of a and b over the TPR threads of a row; every thread gets them.  Above a wave, through LDS:
// two buffers in turn, so that one barrier a sum is enough (a thread that writes buffer p has passed the
// barrier behind which every thread read it two sums ago).
template <int TPR>
struct RowSum {
  float (*s)[2][TPR > 64 ? TPR / 64 : 1];
  int p = 0;
  __device__ __forceinline__ void operator()(float& a, float& b) {
    constexpr int W = TPR < 64 ? TPR : 64;
    a = group_sum<W>(a);
    b = group_sum<W>(b);
    if constexpr (TPR > 64) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0) { s[p][0][wave] = a; s[p][1][wave] = b; }
      __syncthreads();
      a = 0.f; b = 0.f;
#pragma unroll
      for (int i = 0; i < TPR / 64; ++i) { a += s[p][0][i]; b += s[p][1][i]; }
      p ^= 1;
    }
  }
  __device__ __forceinline__ float operator()(float a) {
    float b = 0.f;
    (*this)(a, b);
    return a;
  }
};

// Column of element k (0 .. 8 NI - 1) of thread t: VEC takes 8 neighbours at a time.
template <int TPR, bool VEC>
__device__ __forceinline__ int col_of(int k, int t) {
  return VEC ? ((k >> 3) * TPR + t) * 8 + (k & 7) : k * TPR + t;
}
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Threads of a workgroup, and rows it works on at once: four waves of rows of up to a wave, else one row.
constexpr int block_threads(int tpr) { return tpr <= 64 ? 256 : tpr; }

// A [*, H] matrix as a wave reads and writes it: through a buffer descriptor of the wave's own rows (one, or the
// neighbours of 64 / TPR), which ends with the last of them, so that columns past H and rows past the end load as 0 and
// are not stored, without a branch.  With a branch around each access the compiler waits for all of them, stores too, before
// the first use of what was loaded a row earlier, and one by one where elements are loaded singly (backward, layer norm
// with `add`: 32768 x 2048 branches 145 us, descriptors 103; 20000 x 1501 232 and 46).
template <bool BF16, int TPR, int NI, bool VEC>
struct Rows {
  static constexpr uint32_t ES = BF16 ? 2 : 4;
  static constexpr int PER = TPR < 64 ? 64 / TPR : 1, N = 8 * NI;
  static constexpr uint32_t NOWHERE = 0x80000000u;   // past the end of every descriptor
  char* p;
  int64_t ld;          // bytes; 0: the same row for all
  uint32_t lane, H;    // the lane's first byte within the wave's rows
  int t;
  __device__ __forceinline__ Rows(const void* base, int64_t stride, int t, int h)
      : p(static_cast<char*>(const_cast<void*>(base))), ld(stride * ES), H(h), t(t) {
    lane = (VEC ? 8 : 1) * ES * t;
    if constexpr (PER > 1) lane += (threadIdx.x & 63) / TPR * static_cast<uint32_t>(ld);
  }
  // Descriptor of row r (the wave's first) on, up to row `end`: below 2^27 bytes, for a row is below 2^24.
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(int64_t r, int64_t end) const {
    const int64_t left = p ? end - r : 0;
    uint32_t bytes = 0;
    if (left > 0) bytes = static_cast<uint32_t>((left < PER ? left : PER) - 1) * static_cast<uint32_t>(ld) + H * ES;
    return __builtin_amdgcn_make_buffer_rsrc(p + r * ld, 0, static_cast<int>(bytes), 0x00027000);
  }
  __device__ __forceinline__ uint32_t off(int k) const {   // of element k
    const uint32_t o = lane + (VEC ? (k >> 3) * TPR * 8 + (k & 7) : k * TPR) * ES;
    if constexpr (PER == 1) return o;   // the descriptor ends with the row
    return col_of<TPR, VEC>(VEC ? k & ~7 : k, t) < static_cast<int>(H) ? o : NOWHERE;
  }
  // Non-temporal (32760 x 1536 backward: 52 us, plain stores 55; 32768 x 3072 forward 61 and 81).
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t to, const float (&v)[N]) const {
    if constexpr (VEC) {
#pragma unroll
      for (int k = 0; k < N; k += BF16 ? 8 : 4) {
        u32x4 u;
        if constexpr (BF16) u = u32x4{f2bf2(v[k], v[k + 1]), f2bf2(v[k + 2], v[k + 3]), f2bf2(v[k + 4], v[k + 5]), f2bf2(v[k + 6], v[k + 7])};
        else u = u32x4{__float_as_uint(v[k]), __float_as_uint(v[k + 1]), __float_as_uint(v[k + 2]), __float_as_uint(v[k + 3])};
        __builtin_amdgcn_raw_buffer_store_b128(u, to, off(k), 0, 2);
      }
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if constexpr (BF16) __builtin_amdgcn_raw_buffer_store_b16(f2bf(v[k]), to, off(k), 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[k]), to, off(k), 0, 0);
      }
    }
  }
};
// A row as it lies in memory, so that the next one can be in flight in half the registers (bf16).
template <bool BF16, int TPR, int NI, bool VEC>
struct Raw {
  static constexpr int STEP = VEC && BF16 ? 2 : 1, W = 8 * NI / STEP;   // elements a word, words
  uint32_t w[W];
  // NT: non-temporal.  Plain loads use what an operator before has left in the caches (32768 x 3072 forward: 61 us,
  // non-temporal 75).
  template <bool NT = false>
  __device__ __forceinline__ void load(const Rows<BF16, TPR, NI, VEC>& m, __amdgpu_buffer_rsrc_t from) {
      if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < W; i += 4) {
        const u32x4 u = __builtin_amdgcn_raw_buffer_load_b128(from, m.off(i * STEP), 0, NT ? 2 : 0);
        w[i] = u.x; w[i + 1] = u.y; w[i + 2] = u.z; w[i + 3] = u.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k) {
        if constexpr (BF16) w[k] = __builtin_amdgcn_raw_buffer_load_b16(from, m.off(k), 0, 0);
        else w[k] = __builtin_amdgcn_raw_buffer_load_b32(from, m.off(k), 0, 0);
      }
    }
  }
  __device__ __forceinline__ void get(float (&v)[8 * NI]) const {
#pragma unroll
    for (int k = 0; k < 8 * NI; ++k) {
      if constexpr (VEC && BF16) v[k] = __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
      else v[k] = __uint_as_float(BF16 ? w[k] << 16 : w[k]);
    }
  }
};
// A vector of H elements, the same for every row.
template <bool BF16, int TPR, int NI, bool VEC>
__device__ __forceinline__ void ld_vec(const void* p, int t, int H, float (&v)[8 * NI]) {
  const Rows<BF16, TPR, NI, VEC> m(p, 0, t, H);
  Raw<BF16, TPR, NI, VEC> x;
  x.load(m, m.at(0, 64));
  x.get(v);
}
// The wave's first row among those that the workgroup works on at once.
template <int TPR>
__device__ __forceinline__ int wave_row() {
  return TPR > 64 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (64 / TPR);
}
// mean and 1 / sqrt(var + eps) of the row in v (zeros past H); the variance from the differences, for a
// mean far from zero leaves nothing of a difference of sums.
template <int TPR, int NI, bool VEC>
__device__ __forceinline__ void row_stats(RowSum<TPR>& sum, const float (&v)[8 * NI], int t, int H, float inv_h, int layer,
                                          float eps, float& mean, float& rstd) {
  mean = 0.f;
  if (layer) {
    float a = 0.f;
#pragma unroll
    for (int k = 0; k < 8 * NI; ++k) a += v[k];
    mean = sum(a) * inv_h;
  }
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < 8 * NI; ++k) {
    const float d = col_of<TPR, VEC>(k, t) < H ? v[k] - mean : 0.f;
    ss = fmaf(d, d, ss);
  }
  rstd = rsqrtf(sum(ss) * inv_h + eps);
}

template <bool BF16, int TPR, int NI, bool VEC>
__global__ __launch_bounds__(block_threads(TPR)) void norm_affine_kernel(NormFwd a) {
  constexpr int RPB = block_threads(TPR) / TPR;
  __shared__ float red[2][2][TPR > 64 ? TPR / 64 : 1];
  RowSum<TPR> sum{red};
  const int t = threadIdx.x % TPR, H = static_cast<int>(a.H);
  const float inv_h = 1.0f / static_cast<float>(H);
  float m[8 * NI], c[8 * NI];
#pragma unroll
  for (int k = 0; k < 8 * NI; ++k) { m[k] = 1.f; c[k] = 0.f; }
  if (a.w) ld_vec<BF16, TPR, NI, VEC>(a.w, t, H, m);
  if (a.bias) ld_vec<BF16, TPR, NI, VEC>(a.bias, t, H, c);
  const Rows<BF16, TPR, NI, VEC> x(a.x, a.ldx, t, H), y(a.y, a.ldy, t, H);
  const int64_t r0 = static_cast<int64_t>(blockIdx.x) * a.block_rows;
  const int64_t r1 = r0 + a.block_rows < a.rows ? r0 + a.block_rows : a.rows;
  int64_t r = r0 + wave_row<TPR>();
  Raw<BF16, TPR, NI, VEC> xa, xb;   // this row and the next, in turn
  auto row = [&](const Raw<BF16, TPR, NI, VEC>& now, Raw<BF16, TPR, NI, VEC>& next) __attribute__((always_inline)) {
    next.load(x, x.at(r + RPB, r1));
    float v[8 * NI], mean, rstd;
    now.get(v);
    row_stats<TPR, NI, VEC>(sum, v, t, H, inv_h, a.layer, a.eps, mean, rstd);
#pragma unroll
    for (int k = 0; k < 8 * NI; ++k) v[k] = fmaf((v[k] - mean) * rstd, m[k], c[k]);
    y.store(y.at(r, r1), v);
    r += RPB;
  };
  xa.load(x, x.at(r, r1));
  y.store(y.at(r, r), m);   // to nowhere: see the gradients' kernel
  while (r < r1) {
    row(xa, xb);
    if (r < r1) row(xb, xa);
  }
}

// Workgroup blockIdx.x takes strip blockIdx.x % strips of sample blockIdx.x / strips.
template <bool BF16, int TPR, int NI, bool VEC>
__global__ __launch_bounds__(block_threads(TPR)) void norm_grad_kernel(NormGrad a) {
  constexpr int RPB = block_threads(TPR) / TPR, N = 8 * NI;
  __shared__ float red[2][2][TPR > 64 ? TPR / 64 : 1];
  __shared__ float cols[RPB > 1 ? RPB : 1][RPB > 1 ? TPR : 1][9];
  RowSum<TPR> sum{red};
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR, H = static_cast<int>(a.H);
  const float inv_h = 1.0f / static_cast<float>(H);
  const int64_t b = blockIdx.x / a.strips, strip = blockIdx.x % a.strips;
  const int64_t s0 = b * a.rows_per_sample;
  const int64_t s1 = s0 + a.rows_per_sample < a.rows ? s0 + a.rows_per_sample : a.rows;
  const int64_t r1 = s1, step = a.strips * RPB;
  float m[N], dm[N], da[N];
#pragma unroll
  for (int k = 0; k < N; ++k) { m[k] = 1.f; dm[k] = 0.f; da[k] = 0.f; }
  if (a.w) ld_vec<BF16, TPR, NI, VEC>(a.w, t, H, m);
  if (a.scale) {
    ld_vec<false, TPR, NI, VEC>(a.scale + b * a.mod_ld, t, H, m);
#pragma unroll
    for (int k = 0; k < N; ++k) m[k] += 1.f;
  }
  typedef Rows<BF16, TPR, NI, VEC> Mat;
  typedef Raw<BF16, TPR, NI, VEC> Row;
  const Mat xm(a.x, a.ldx, t, H), gm(a.dy, a.lddy, t, H), am(a.add, a.ldadd, t, H), dxm(a.dx, a.lddx, t, H);
  int64_t r = s0 + strip * RPB + wave_row<TPR>();
  // This row and the next, in turn; three chunks that are not packed leave no registers for a second row.
  // x was kept since the forward pass and leaves the caches to the gradients, which an operator has just written
  // (non-temporal loads of x; 32768 x 3072 with dy partly there 103 us, plain 125; nothing there 120 and 126; where a row
  // is not loaded ahead they are slower: float32 9000 x 10000 291 and 277).
  constexpr bool ahead = NI < 3 || (VEC && (BF16 || TPR < 512));
  Row xa, ga, xb, gb;
  auto row = [&](Row& x, Row& dy, Row& xn, Row& gn) __attribute__((always_inline)) {
    Row ar;
    if constexpr (!ahead) {
      x.load(xm, xm.at(r, r1));
      dy.load(gm, gm.at(r, r1));
    }
    ar.load(am, am.at(r, r1));
    if constexpr (ahead) {
      xn.template load<true>(xm, xm.at(r + step, r1));
      gn.load(gm, gm.at(r + step, r1));
    }
    float v[N], g[N], mean, rstd;
    x.get(v);
    row_stats<TPR, NI, VEC>(sum, v, t, H, inv_h, a.layer, a.eps, mean, rstd);
    dy.get(g);
    // a row past the end adds 0 to the columns' sums
    if constexpr (TPR < 64) rstd = r + (threadIdx.x & 63) / TPR < r1 ? rstd : 0.f;
    float s1_ = 0.f, s2_ = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = (v[k] - mean) * rstd;
      dm[k] = fmaf(g[k], v[k], dm[k]);
      da[k] += g[k];
      g[k] *= m[k];
      s1_ += g[k];
      s2_ = fmaf(g[k], v[k], s2_);
    }
    sum(s1_, s2_);
    const float c1 = a.layer ? s1_ * inv_h : 0.f, c2 = s2_ * inv_h;
#pragma unroll
    for (int k = 0; k < N; ++k) g[k] = (g[k] - c1 - v[k] * c2) * rstd;
    ar.get(v);
#pragma unroll
    for (int k = 0; k < N; ++k) g[k] += v[k];
    dxm.store(dxm.at(r, r1), g);
    r += step;
  };
  if constexpr (ahead) {
    xa.template load<true>(xm, xm.at(r, r1));
    ga.load(gm, gm.at(r, r1));
    // stores to nowhere: with as many accesses behind the first row's loads as behind any other's, no wait for a row's
    // loads takes in the stores of the row before
    dxm.store(dxm.at(r, r), da);
  }
  while (r < r1) {
    row(xa, ga, xb, gb);
    if (ahead && r < r1) row(xb, gb, xa, ga);
  }
  if (!a.dm && !a.da) return;
  float* const outs[2] = {a.part ? a.part + blockIdx.x * a.part_ld : a.dm ? a.dm + b * a.dmod_ld : nullptr,
                          a.part ? a.part + blockIdx.x * a.part_ld + a.H : a.da ? a.da + b * a.dmod_ld : nullptr};
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    float* const out = outs[half];
    if (!out) continue;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      float (&acc)[N] = half ? da : dm;
      if constexpr (RPB > 1) {   // the rows that the workgroup worked on at once, added in order
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) cols[sub][t][j] = acc[8 * i + j];
        __syncthreads();
        for (int e = threadIdx.x; e < TPR * 8; e += 256) {
          const int tt = e >> 3, j = e & 7;
          float u = 0.f;
#pragma unroll
          for (int q = 0; q < RPB; ++q) u += cols[q][tt][j];
          const int c = col_of<TPR, VEC>(8 * i + j, tt);
          if (c < H) out[c] = u;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int c = col_of<TPR, VEC>(8 * i + j, t);
          if (c < H) out[c] = acc[8 * i + j];
        }
      }
    }
  }
}

// Adds each sample's strips in order.  A workgroup takes 32 columns of a sample's partial rows at a time, four of
// them a thread, 32 threads a column, which add every 32nd strip each.
__global__ __launch_bounds__(256) void strip_sum_kernel(const float* part, int64_t part_ld, int64_t samples, int64_t strips,
                                                        int64_t H, float* dm, float* da, int64_t ld) {
  __shared__ float4 s[32][9];
  const int lane = threadIdx.x & 7, q = threadIdx.x >> 3;
  const int64_t chunks = (2 * H + 31) / 32;
  for (int64_t w = blockIdx.x; w < samples * chunks; w += gridDim.x) {
    const int64_t b = w / chunks, c = w % chunks * 32 + lane * 4;
    const float* p = part + b * strips * part_ld + c;
    float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < part_ld) {
#pragma unroll 8
      for (int64_t i = q; i < strips; i += 32) {
        const float4 x = *reinterpret_cast<const float4*>(p + i * part_ld);
        u.x += x.x; u.y += x.y; u.z += x.z; u.w += x.w;
      }
    }
    s[q][lane] = u;
    __syncthreads();
    const int col = threadIdx.x;
    if (col < 32 && w % chunks * 32 + col < 2 * H) {
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) v += reinterpret_cast<const float*>(&s[i][col >> 2])[col & 3];
      const int64_t k = w % chunks * 32 + col;
      float* out = k < H ? dm : da;
      if (out) out[b * ld + (k < H ? k : k - H)] = v;
    }
    __syncthreads();
  }
}

// Rows too wide for registers: a workgroup a row, three passes over it (the second and third from the
// caches), and its statistics kept for the column sums.
template <bool BF16>
__global__ __launch_bounds__(256) void norm_affine_wide_kernel(NormFwd a) {
  __shared__ float red[2][2][4];
  RowSum<256> sum{red};
  const float inv_h = 1.0f / static_cast<float>(a.H);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    float mean = 0.f, u = 0.f;
    if (a.layer) {
      for (int64_t j = threadIdx.x; j < a.H; j += 256) u += ld1<BF16>(a.x, r * a.ldx + j);
      mean = sum(u) * inv_h;
    }
    u = 0.f;
    for (int64_t j = threadIdx.x; j < a.H; j += 256) {
      const float d = ld1<BF16>(a.x, r * a.ldx + j) - mean;
      u = fmaf(d, d, u);
    }
    const float rstd = rsqrtf(sum(u) * inv_h + a.eps);
    for (int64_t j = threadIdx.x; j < a.H; j += 256) {
      const float xh = (ld1<BF16>(a.x, r * a.ldx + j) - mean) * rstd;
      st1<BF16>(a.y, r * a.ldy + j, fmaf(xh, a.w ? ld1<BF16>(a.w, j) : 1.f, a.bias ? ld1<BF16>(a.bias, j) : 0.f));
    }
  }
}
template <bool BF16>
__device__ __forceinline__ float mul_at(const NormGrad& a, int64_t b, int64_t j) {
  return a.w ? ld1<BF16>(a.w, j) : a.scale ? 1.f + a.scale[b * a.mod_ld + j] : 1.f;
}
// stats[row] = (mean, rstd, mean(g), mean(g xh)).
template <bool BF16>
__global__ __launch_bounds__(256) void norm_wide_stats_kernel(NormGrad a, float4* stats) {
  __shared__ float red[2][2][4];
  RowSum<256> sum{red};
  const float inv_h = 1.0f / static_cast<float>(a.H);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int64_t b = r / a.rows_per_sample;
    float mean = 0.f, u = 0.f;
    if (a.layer) {
      for (int64_t j = threadIdx.x; j < a.H; j += 256) u += ld1<BF16>(a.x, r * a.ldx + j);
      mean = sum(u) * inv_h;
    }
    u = 0.f;
    for (int64_t j = threadIdx.x; j < a.H; j += 256) {
      const float d = ld1<BF16>(a.x, r * a.ldx + j) - mean;
      u = fmaf(d, d, u);
    }
    const float rstd = rsqrtf(sum(u) * inv_h + a.eps);
    float c1 = 0.f, c2 = 0.f;
    for (int64_t j = threadIdx.x; j < a.H; j += 256) {
      const float g = ld1<BF16>(a.dy, r * a.lddy + j) * mul_at<BF16>(a, b, j);
      c1 += g;
      c2 = fmaf(g, (ld1<BF16>(a.x, r * a.ldx + j) - mean) * rstd, c2);
    }
    sum(c1, c2);
    if (threadIdx.x == 0) stats[r] = make_float4(mean, rstd, a.layer ? c1 * inv_h : 0.f, c2 * inv_h);
  }
}
// The column sums and then dx of 256 columns of one strip: dx may be dy or x, whose element the same
// thread has read.
template <bool BF16>
__global__ __launch_bounds__(256) void norm_wide_grad_kernel(NormGrad a, const float4* stats, int64_t blocks) {
  const int64_t chunks = (a.H + 255) / 256;
  for (int64_t w = blockIdx.x; w < blocks * chunks; w += gridDim.x) {
    const int64_t j = (w % chunks) * 256 + threadIdx.x, bs = w / chunks;
    if (j >= a.H) continue;
    const int64_t b = bs / a.strips, strip = bs % a.strips;
    const int64_t s0 = b * a.rows_per_sample;
    const int64_t s1 = s0 + a.rows_per_sample < a.rows ? s0 + a.rows_per_sample : a.rows;
    const int64_t r0 = s0 + strip * a.strip_rows;
    const int64_t r1 = r0 + a.strip_rows < s1 ? r0 + a.strip_rows : s1;
    const float m = mul_at<BF16>(a, b, j);
    float dm = 0.f, da = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
      const float4 st = stats[r];
      const float g = ld1<BF16>(a.dy, r * a.lddy + j), xh = (ld1<BF16>(a.x, r * a.ldx + j) - st.x) * st.y;
      dm = fmaf(g, xh, dm);
      da += g;
      if (a.dx) {
        float d = (g * m - st.z - xh * st.w) * st.y;
        if (a.add) d += ld1<BF16>(a.add, r * a.ldadd + j);
        st1<BF16>(a.dx, r * a.lddx + j, d);
      }
    }
    if (a.part) {
      a.part[bs * a.part_ld + j] = dm;
      a.part[bs * a.part_ld + a.H + j] = da;
    }
  }
}

// Workgroups of a launch: as many to each of 256 compute units as make nine waves or less (8192 x 7000 of eight waves: one
// 91 us, two 107; 32768 x 3072 of three: three 126, four 127, five 138; all of them long strips, and not measured on short
// ones: five samples of 333 x 2560 come to 48 strips of seven rows each by it, 16 us).  And the fewest rows in turn that pay
// for a strip's partial row, where that limit leaves the choice (one sample of 333 x 2560: four 13.1 us, eight 16.9; 1000 x
// 1536: two 15.5, four 14.0), while up to eight are one strip, which needs no second launch (192 x 64: 9.4 us, two strips 12.0).
int64_t strip_blocks(int waves) { return waves <= 9 ? 256 * (9 / waves) : 256; }
constexpr int64_t kStripTurns = 4, kOneStrip = 8;
struct StripPlan { int64_t samples, strips, strip_rows; };
StripPlan strip_plan(int64_t rows, int64_t H, int64_t rps) {
  const RowPlanH p = row_plan_h(rows, H);
  const int64_t at_once = p.ni ? block_threads(p.tpr) / p.tpr : 1, blocks = strip_blocks(p.ni ? block_threads(p.tpr) / 64 : 2);
  StripPlan s{(rows + rps - 1) / rps, 1, rps};
  const int64_t len = rows < rps ? rows : rps;
  if (s.samples == 0) return s;
  const int64_t want = (blocks + s.samples - 1) / s.samples, turns = (len + at_once - 1) / at_once;
  s.strips = turns <= kOneStrip ? 1 : (turns + kStripTurns - 1) / kStripTurns;
  if (s.strips > want) s.strips = want;
  s.strip_rows = (turns + s.strips - 1) / s.strips * at_once;
  s.strips = (len + s.strip_rows - 1) / s.strip_rows;
  return s;
}
// Partial rows are needed where a sample is more than one strip; rows too wide for registers always take them.
bool strip_direct(const StripPlan& s, int64_t rows, int64_t H) { return s.strips == 1 && row_plan_h(rows, H).ni > 0; }
int64_t strip_ld(int64_t H) { return (2 * H + 3) / 4 * 4; }

// A plan outside its pass's list is an error of the library, and not a launch left out.
int no_kernel(const RowPlanH& p) { return fail(FF_EUNSUPPORTED, "norm: no kernel of %d threads a row and %d chunks", p.tpr, p.ni); }
template <bool BF16, bool VEC>
int fwd_dispatch(const NormFwd& a, unsigned blocks, const RowPlanH& p, hipStream_t s) {
  switch (p.tpr * 10 + p.ni) {
#define FF_CASE(T, N) \
  case T * 10 + N: hipLaunchKernelGGL((norm_affine_kernel<BF16, T, N, VEC>), dim3(blocks), dim3(block_threads(T)), 0, s, a); break;
    FF_NORM_FORWARD(FF_CASE)
#undef FF_CASE
    default: return no_kernel(p);
  }
  return FF_OK;
}
template <bool BF16, bool VEC>
int grad_dispatch(const NormGrad& a, unsigned blocks, const RowPlanH& p, hipStream_t s) {
  switch (p.tpr * 10 + p.ni) {
#define FF_CASE(T, N) \
  case T * 10 + N: hipLaunchKernelGGL((norm_grad_kernel<BF16, T, N, VEC>), dim3(blocks), dim3(block_threads(T)), 0, s, a); break;
    FF_NORM_BACKWARD(FF_CASE)
#undef FF_CASE
    default: return no_kernel(p);
  }
  return FF_OK;
}

bool vec_ok(const void* p, int64_t ld) { return !p || (aligned16(p) && ld % 8 == 0); }

int norm_backward(const char* fn, NormGrad a, float* dm, float* da, int64_t dmod_ld, int dtype, void* ws, size_t ws_bytes,
                  hipStream_t s) {
  const StripPlan sp = strip_plan(a.rows, a.H, a.rows_per_sample);
  size_t need = 0;
  FF_TRY(ff_norm_backward_workspace_size(a.rows, a.H, a.rows_per_sample, &need));
  if (need > 0 && (!ws || ws_bytes < need)) return fail(FF_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
  if (!aligned16(ws)) return fail(FF_EINVAL, "%s: workspace must be 16-byte aligned", fn);
  if (dm && dm == da) return fail(FF_EINVAL, "%s: the two column sums are the same output", fn);
  for (const void* o : {static_cast<const void*>(dm), static_cast<const void*>(da)})
    for (const void* in : {a.dy, a.x, a.add, static_cast<const void*>(a.dx), a.w, static_cast<const void*>(a.scale)})
      if (o && o == in) return fail(FF_EINVAL, "%s: a column sum is another operand", fn);
  if (a.dx && (a.dx == a.w || a.dx == a.scale)) return fail(FF_EINVAL, "%s: dx is the multiplier", fn);
  const RowPlanH p = row_plan_h(a.rows, a.H);
  a.strips = sp.strips;
  a.strip_rows = sp.strip_rows;
  Carver c(ws, ws_bytes);
  a.dm = dm; a.da = da; a.dmod_ld = dmod_ld;
  a.part_ld = strip_ld(a.H);
  const bool direct = a.rows > 0 && strip_direct(sp, a.rows, a.H);
  if (a.rows > 0 && !direct) a.part = static_cast<float*>(c.take(sp.samples * sp.strips * a.part_ld * sizeof(float)));
  const bool bf = dtype == FF_BF16;
  const bool vec = a.H % 8 == 0 && vec_ok(a.dy, a.lddy) && vec_ok(a.x, a.ldx) && vec_ok(a.add, a.ldadd) && vec_ok(a.dx, a.lddx) &&
                   vec_ok(a.w, 8);
  const double bytes = static_cast<double>(dtype_size(dtype)) * a.rows * a.H * (2 + (a.dx != nullptr) + (a.add != nullptr));
  const unsigned blocks = static_cast<unsigned>(sp.samples * sp.strips);
  if (a.rows > 0 && p.ni > 0) {
    LaunchScope ls("norm_grad", s, 0.0, bytes);
    if (bf) FF_TRY((vec ? grad_dispatch<true, true>(a, blocks, p, s) : grad_dispatch<true, false>(a, blocks, p, s)));
    else FF_TRY((vec ? grad_dispatch<false, true>(a, blocks, p, s) : grad_dispatch<false, false>(a, blocks, p, s)));
    FF_TRY(ls.status());
  } else if (a.rows > 0) {
    float4* stats = static_cast<float4*>(c.take(a.rows * sizeof(float4)));
    LaunchScope ls("norm_grad", s, 0.0, bytes);
    const unsigned g = static_cast<unsigned>(a.rows < 65536 ? a.rows : 65536);
    const int64_t all = blocks * ((a.H + 255) / 256);
    const unsigned g2 = static_cast<unsigned>(all < 65536 ? all : 65536);
    if (bf) {
      hipLaunchKernelGGL(norm_wide_stats_kernel<true>, dim3(g), dim3(256), 0, s, a, stats);
      hipLaunchKernelGGL(norm_wide_grad_kernel<true>, dim3(g2), dim3(256), 0, s, a, static_cast<const float4*>(stats), int64_t(blocks));
    } else {
      hipLaunchKernelGGL(norm_wide_stats_kernel<false>, dim3(g), dim3(256), 0, s, a, stats);
      hipLaunchKernelGGL(norm_wide_grad_kernel<false>, dim3(g2), dim3(256), 0, s, a, static_cast<const float4*>(stats), int64_t(blocks));
    }
    FF_TRY(ls.status());
  }
  if ((!dm && !da) || direct) return FF_OK;
  const int64_t samples = a.rows > 0 ? sp.samples : 1;   // no rows: an affine norm's sums are zero
  LaunchScope ls("norm_strip_sum", s, 0.0, 8.0 * samples * sp.strips * a.H);
  const int64_t all = samples * ((2 * a.H + 31) / 32);
  hipLaunchKernelGGL(strip_sum_kernel, dim3(static_cast<unsigned>(all < 65536 ? all : 65536)), dim3(256), 0, s,
                     a.part, a.part_ld, samples, a.rows > 0 ? sp.strips : 0, a.H, dm, da, dmod_ld);
  return ls.status();
}

constexpr int64_t kMaxRows = int64_t(1) << 27, kMaxWidth = int64_t(1) << 22, kMaxSamples = 65535;

// Checks shared by the entry points below (element alignment of the pointers included).
int check_norm(const char* fn, int64_t rows, int64_t H, int32_t kind, float eps, int32_t dtype,
               std::initializer_list<std::pair<const void*, int64_t>> mats) {
  if (dtype != FF_F32 && dtype != FF_BF16) return fail(FF_EINVAL, "%s: bad dtype %d", fn, dtype);
  if (rows < 0 || H < 1) return fail(FF_EINVAL, "%s: bad shape rows=%lld H=%lld", fn, (long long)rows, (long long)H);
  if (kind != FF_NORM_RMS && kind != FF_NORM_LN) return fail(FF_EINVAL, "%s: bad norm_kind %d", fn, kind);
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(FF_EINVAL, "%s: eps must be positive and finite", fn);
  if (rows > kMaxRows || H > kMaxWidth) return fail(FF_EUNSUPPORTED, "%s: rows above 2^27 or H above 2^22", fn);
  for (const auto& m : mats) {
    if (!m.first) continue;
    if (reinterpret_cast<uintptr_t>(m.first) % dtype_size(dtype)) return fail(FF_EINVAL, "%s: pointer not aligned to an element", fn);
    if (m.second < H) return fail(FF_EINVAL, "%s: row stride %lld below H", fn, (long long)m.second);
    if (m.second > kMaxWidth) return fail(FF_EUNSUPPORTED, "%s: row stride above 2^22", fn);
  }
  return FF_OK;
}
bool misaligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace
}  // namespace ff

using namespace ff;

extern "C" {

int ff_norm_affine(const void* x, int64_t ldx, const void* w, const void* bias, void* y, int64_t ldy, int64_t rows,
                   int64_t H, int32_t norm_kind, float eps, int32_t dtype, void* stream) {
  const char* fn = "ff_norm_affine";
  FF_TRY(check_norm(fn, rows, H, norm_kind, eps, dtype, {{x, ldx}, {y, ldy}, {w, H}, {bias, H}}));
  if (rows == 0) return FF_OK;
  if (!x || !y) return fail(FF_EINVAL, "%s: null x or y", fn);
  if (y == w || y == bias) return fail(FF_EINVAL, "%s: y is w or bias", fn);
  if (x == y && ldx != ldy) return fail(FF_EINVAL, "%s: y in place of x needs the same row stride", fn);
  hipStream_t s = static_cast<hipStream_t>(stream);
  NormFwd a{x, ldx, w, bias, y, ldy, rows, H, 0, norm_kind == FF_NORM_LN, eps};
  const RowPlanH p = row_plan_h(rows, H, true);
  LaunchScope ls("norm_affine", s, 0.0, 2.0 * dtype_size(dtype) * rows * H);
  const bool bf = dtype == FF_BF16;
  if (p.ni == 0) {
    const unsigned g = static_cast<unsigned>(rows < 65536 ? rows : 65536);
    if (bf) hipLaunchKernelGGL(norm_affine_wide_kernel<true>, dim3(g), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(norm_affine_wide_kernel<false>, dim3(g), dim3(256), 0, s, a);
    return ls.status();
  }
  const bool vec = H % 8 == 0 && vec_ok(x, ldx) && vec_ok(y, ldy) && vec_ok(w, 8) && vec_ok(bias, 8);
  const int64_t at_once = block_threads(p.tpr) / p.tpr;
  const int64_t want = 2 * strip_blocks(block_threads(p.tpr) / 64);
  a.block_rows = (rows + want * at_once - 1) / (want * at_once) * at_once;
  const unsigned blocks = static_cast<unsigned>((rows + a.block_rows - 1) / a.block_rows);
  if (bf) FF_TRY((vec ? fwd_dispatch<true, true>(a, blocks, p, s) : fwd_dispatch<true, false>(a, blocks, p, s)));
  else FF_TRY((vec ? fwd_dispatch<false, true>(a, blocks, p, s) : fwd_dispatch<false, false>(a, blocks, p, s)));
  return ls.status();
}

int ff_norm_backward_workspace_size(int64_t rows, int64_t H, int64_t rows_per_sample, size_t* bytes) {
  const char* fn = "ff_norm_backward_workspace_size";
  if (!bytes) return fail(FF_EINVAL, "%s: null output", fn);
  if (rows < 0 || H < 1 || (rows > 0 && rows_per_sample < 1)) return fail(FF_EINVAL, "%s: bad shape", fn);
  if (rows > kMaxRows || H > kMaxWidth || (rows > 0 && (rows - 1) / rows_per_sample + 1 > kMaxSamples))
    return fail(FF_EUNSUPPORTED, "%s: rows above 2^27, H above 2^22 or more than 65535 samples", fn);
  *bytes = 0;
  if (rows == 0) return FF_OK;
  const StripPlan sp = strip_plan(rows, H, rows_per_sample < rows ? rows_per_sample : rows);
  Carver c(nullptr, 0);
  if (!strip_direct(sp, rows, H)) c.take(sp.samples * sp.strips * strip_ld(H) * sizeof(float));
  if (row_plan_h(rows, H).ni == 0) c.take(rows * sizeof(float4));
  *bytes = c.off;
  return FF_OK;
}

int ff_norm_affine_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w, const void* add,
                            int64_t ldadd, void* dx, int64_t lddx, float* dw, float* dbias, int64_t rows, int64_t H,
                            int32_t norm_kind, float eps, int32_t dtype, void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "ff_norm_affine_backward";
  FF_TRY(check_norm(fn, rows, H, norm_kind, eps, dtype, {{dy, lddy}, {x, ldx}, {add, ldadd}, {dx, lddx}, {w, H}}));
  if (rows > 0 && (!dy || !x)) return fail(FF_EINVAL, "%s: null dy or x", fn);
  if (misaligned4(dw) || misaligned4(dbias)) return fail(FF_EINVAL, "%s: dw and dbias must be 4-byte aligned", fn);
  if ((dx && dx == dy && lddx != lddy) || (dx && dx == add && lddx != ldadd) || (dx && dx == x && lddx != ldx))
    return fail(FF_EINVAL, "%s: dx in place of an input needs its row stride", fn);
  NormGrad a{dy, lddy, x, ldx, dx ? add : nullptr, ldadd, dx, lddx, w, nullptr, 0, nullptr, nullptr, 0, nullptr, 0,
             rows, H, rows > 0 ? rows : 1, 0, 0, norm_kind == FF_NORM_LN, eps};
  return norm_backward(fn, a, dw, dbias, H, dtype, workspace, ws_bytes, static_cast<hipStream_t>(stream));
}

int ff_norm_modulate_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* scale,
                              int64_t mod_ld, int64_t rows_per_sample, const void* add, int64_t ldadd, void* dx,
                              int64_t lddx, float* dshift, float* dscale, int64_t dmod_ld, int64_t rows, int64_t H,
                              int32_t norm_kind, float eps, int32_t dtype, void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "ff_norm_modulate_backward";
  FF_TRY(check_norm(fn, rows, H, norm_kind, eps, dtype, {{dy, lddy}, {x, ldx}, {add, ldadd}, {dx, lddx}}));
  if (rows == 0) return FF_OK;
  if (!dy || !x) return fail(FF_EINVAL, "%s: null dy or x", fn);
  if (rows_per_sample < 1) return fail(FF_EINVAL, "%s: rows_per_sample %lld", fn, (long long)rows_per_sample);
  if ((rows - 1) / rows_per_sample + 1 > kMaxSamples) return fail(FF_EUNSUPPORTED, "%s: more than 65535 samples", fn);
  if ((scale && mod_ld < H) || ((dshift || dscale) && dmod_ld < H)) return fail(FF_EINVAL, "%s: mod_ld or dmod_ld below H", fn);
  if (misaligned4(scale) || misaligned4(dshift) || misaligned4(dscale)) return fail(FF_EINVAL, "%s: scale, dshift and dscale must be 4-byte aligned", fn);
  if ((dx && dx == dy && lddx != lddy) || (dx && dx == add && lddx != ldadd) || (dx && dx == x && lddx != ldx))
    return fail(FF_EINVAL, "%s: dx in place of an input needs its row stride", fn);
  NormGrad a{dy, lddy, x, ldx, dx ? add : nullptr, ldadd, dx, lddx, nullptr, scale, mod_ld, nullptr, nullptr, 0, nullptr, 0,
             rows, H, rows_per_sample < rows ? rows_per_sample : rows, 0, 0, norm_kind == FF_NORM_LN, eps};
  return norm_backward(fn, a, dscale, dshift, dmod_ld, dtype, workspace, ws_bytes, static_cast<hipStream_t>(stream));
}

}  // extern "C"
