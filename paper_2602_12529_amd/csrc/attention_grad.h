// Shared by the attention kernels of a training step (attention_grad.hip, attention_grad_bf16.hip): the
// launch's arguments and how its workgroups find their work.
#pragma once

#include "../../include/ff_grad.h"
#include "dev.h"
#include "ff_internal.h"

namespace ff {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// [B, heads, n, d] with strides in elements.
struct Heads { void* p; int64_t b, h, n; };

struct AttnGrad {
  int64_t B, heads, kv_heads, group, n_q, n_kv;
  int d, causal, splits;
  int mix;                     // key heads whose workgroups run together (place_of)
  float scale, scale_log2;
  const int32_t* kv_len;
  Heads Q, K, V, O, dO, dQ, dK, dV;
  float* lse;                  // [B, heads, n_q]
  float* delta;                // backward: row statistics that the dQ kernel leaves for the dK, dV kernel
  float* part;                 // partial results of splits (float32)
  float* part_lse;             // forward: their log-sum-exp
};

__device__ __forceinline__ int64_t sample_len(const AttnGrad& p, int64_t b) {
  if (!p.kv_len) return p.n_kv;
  const int64_t n = p.kv_len[b];
  return n < 0 ? 0 : n < p.n_kv ? n : p.n_kv;
}

// Workgroups go round the eight XCDs, each with an L2 of its own: the id to work with, so that one XCD's workgroups
// are neighbours and share the other side's tiles.
__device__ __forceinline__ uint32_t near_id() {
  const uint32_t id = blockIdx.x, full = gridDim.x / 8 * 8;
  return id < full ? (id % 8) * (full / 8) + id / 8 : id;
}
// Of `mix` key heads after another, first every head's workgroups of rank 0, then those of rank 1, ...: (sample and key
// head, rank, split) of this workgroup among `tiles` ranks a head.
// Everything that is counted here fits 32 bits (the host keeps heads x (n_q + n_kv) below 2^29), where a division takes a
// third of the instructions.
struct Place { uint32_t bh, rank, split; };
__device__ __forceinline__ Place place_of(const AttnGrad& p, uint32_t tiles) {
  const uint32_t id = near_id(), splits = p.splits, row = p.mix * splits, all = row * tiles;
  const uint32_t set = id / all, j = id - set * all, rank = j / row, within = j - rank * row, head = within / splits;
  return {set * p.mix + head, rank, within - head * splits};
}

// Query side: the rows of a workgroup are those of the group's query heads one after another (row =
// head-in-group * n_q + query), so that single tokens of shared heads fill a tile together and read the
// keys once.  A split takes keys [key0, key1).
struct QueryTile {
  int64_t b, kvh, row0, len, key0, key1, k_b, k_h;
  int split;
};
__device__ __forceinline__ QueryTile query_tile(const AttnGrad& p, int rows) {
  QueryTile t;
  const uint32_t all = static_cast<uint32_t>(p.group * p.n_q), n_q = static_cast<uint32_t>(p.n_q), group = static_cast<uint32_t>(p.group);
  const uint32_t tiles = (all + rows - 1) / rows;
  const Place at = place_of(p, tiles);
  t.split = static_cast<int>(at.split);
  uint32_t tile = at.rank;
  if (p.causal) {   // the longest rows first: what runs last is short.  The group's heads have `each` tiles, and what is over
    const uint32_t each = tiles / group, over = tiles - each * group, r = tile - over;
    tile = tile < over ? tiles - 1 - tile : r % group * each + (each - 1 - r / group);
  }
  t.row0 = static_cast<int64_t>(tile) * rows;
  t.b = at.bh / static_cast<uint32_t>(p.kv_heads);
  t.kvh = at.bh - t.b * p.kv_heads;
  t.len = sample_len(p, t.b);
  // the keys that the tile's last query sees
  int64_t end = t.len;
  if (p.causal) {
    const uint32_t row0 = tile * rows, last = row0 + rows - 1 < all ? row0 + rows - 1 : all - 1;
    const uint32_t head = last / n_q, query = row0 / n_q == head ? last - head * n_q : n_q - 1;
    const int64_t sees = query + int64_t(1) + t.len - p.n_q;
    end = sees < 0 ? 0 : sees < t.len ? sees : t.len;
  }
  const uint32_t tiles_k = static_cast<uint32_t>((end + 63) / 64);
  const int64_t per = static_cast<int64_t>((tiles_k + p.splits - 1) / static_cast<uint32_t>(p.splits)) * 64;
  t.key0 = t.split * per < end ? t.split * per : end;
  t.key1 = t.key0 + per < end ? t.key0 + per : end;
  return t;
}
struct OwnQuery {
  int64_t b, h, i, stat;
  int lim;      // keys it sees: 0 .. lim - 1
  bool ok;
  template <typename T>
  __device__ __forceinline__ T* at(const Heads& t) const {
    return static_cast<T*>(t.p) + b * t.b + h * t.h + i * t.n;
  }
};
// Row `row` of the key head's rows; past the last one: the last one, not ok.
__device__ __forceinline__ OwnQuery own_query(const AttnGrad& p, const QueryTile& t, int64_t row) {
  OwnQuery q;
  const int64_t all = p.group * p.n_q;
  q.ok = row < all;
  if (!q.ok) row = all - 1;
  q.b = t.b;
  const uint32_t n = static_cast<uint32_t>(p.n_q), h = static_cast<uint32_t>(row) / n;
  q.h = t.kvh * p.group + h;
  q.i = static_cast<uint32_t>(row) - h * n;
  q.stat = (t.b * p.heads + q.h) * p.n_q + q.i;
  int64_t lim = t.len;
  if (p.causal) {
    const int64_t sees = q.i + 1 + t.len - p.n_q;
    lim = sees < 0 ? 0 : sees < lim ? sees : lim;
  }
  q.lim = static_cast<int>(lim < t.key1 ? lim : t.key1);
  return q;
}
__device__ __forceinline__ int64_t split_row(const AttnGrad& p, const QueryTile& t, const OwnQuery& q) {
  return static_cast<int64_t>(t.split) * p.B * p.heads * p.n_q + q.stat;
}
// First element of (b, kv head) of a key-side tensor.
template <typename T, typename Tile>
__device__ __forceinline__ const T* key_base(const Heads& h, const Tile& t) {
  return static_cast<const T*>(h.p) + t.b * h.b + t.kvh * h.h;
}

// Key side: a workgroup owns `rows` keys of one key head and walks the ROWS-query tiles of the group's query
// heads, head by head; a split takes one part of them.
struct KeyTile {
  int64_t b, kvh, key0, len;
  int split;
};
__device__ __forceinline__ KeyTile key_tile(const AttnGrad& p, int rows) {
  KeyTile t;
  const Place at = place_of(p, static_cast<uint32_t>((p.n_kv + rows - 1) / rows));
  t.split = static_cast<int>(at.split);
  t.key0 = static_cast<int64_t>(at.rank) * rows;
  t.b = at.bh / static_cast<uint32_t>(p.kv_heads);
  t.kvh = at.bh - t.b * p.kv_heads;
  t.len = sample_len(p, t.b);
  return t;
}
template <int ROWS>
struct TileWalk {
  int64_t first, tiles, pos, end;   // per head: tiles first .. first + tiles - 1
  int64_t head, tile;
  __device__ __forceinline__ TileWalk(const AttnGrad& p, const KeyTile& t) {
    const int64_t all = (p.n_q + ROWS - 1) / ROWS;
    int64_t i0 = 0;
    if (p.causal) {   // the first query that sees key0
      i0 = t.key0 - (t.len - p.n_q);
      i0 = i0 < 0 ? 0 : i0 < p.n_q ? i0 : p.n_q;
    }
    first = t.key0 < t.len ? i0 / ROWS : all;
    if (i0 >= p.n_q) first = all;
    tiles = all - first;
    const uint32_t n = static_cast<uint32_t>(tiles * p.group), per = (n + p.splits - 1) / static_cast<uint32_t>(p.splits);
    pos = static_cast<uint32_t>(t.split) * per < n ? static_cast<uint32_t>(t.split) * per : n;
    end = pos + per < n ? pos + per : n;
    set();
  }
  __device__ __forceinline__ void set() {
    const uint32_t n = static_cast<uint32_t>(tiles), h = n > 0 ? static_cast<uint32_t>(pos) / n : 0;
    head = h;
    tile = first + (static_cast<uint32_t>(pos) - h * n);
  }
  __device__ __forceinline__ bool more() const { return pos < end; }
  __device__ __forceinline__ void next() {
    ++pos;
    if (++tile == first + tiles) { tile = first; ++head; }
  }
};

// Launchers of attention_grad_bf16.hip: bfloat16 with head dimension 64 or 128 (`blocks` workgroups; query side
// of kWideRows or kNarrowRows rows a workgroup, key side of kKeyRows keys).
constexpr int kWideRows = 128, kNarrowRows = 32, kKeyRows = 128;
// Their row statistics, a sample and head after another: for each 32 queries 32 values of -lse / scale and 32 of
// -D, with n_q rounded up to 64.
__host__ __device__ inline int64_t stat_rows(int64_t n_q) { return (n_q + 63) / 64 * 64; }
void attn_fwd_bf16(const AttnGrad& p, int64_t blocks, bool narrow, hipStream_t s);
void attn_dq_bf16(const AttnGrad& p, int64_t blocks, bool narrow, hipStream_t s);
void attn_dkv_bf16(const AttnGrad& p, int64_t blocks, hipStream_t s);
int attn_bf16_prepare();

}  // namespace ff
