// The work of a chunk call (attention of several new tokens per sequence over the graded cache) and how it is cut into CTAs.
// Host code without CUDA calls: it runs on a host alone as well.
//
// A tile is up to 128 or 256 rows of one stream: the query heads of `tile_tokens` consecutive new tokens.  It walks the stream's items: those of
// the cache, then the chunk's own rows in groups of `item_keys` as far as the tile's last token sees them.  All tiles' items are laid end to end and
// cut into equal ranges, one per CTA, so a CTA has the end of one tile, whole tiles, and the beginning of another.  A tile that was cut leaves
// partial results in slots; the slots of a tile follow one another.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace gkv {

constexpr int kChunkRows = 128;            // rows of a tile, or of half of one
constexpr int kChunkCtas = 148;            // one CTA per SM: all of its tensor memory, most of its shared memory
constexpr int kChunkParts = 2 * kChunkCtas;      // most slots of a call (a CTA has at most two), and most tiles to be merged
constexpr int kChunkSlotFloats = kChunkRows * (128 + 2);

constexpr int kChunkMaxBatch = 1024;       // sequences of a call with lengths of their own
constexpr int kChunkMaxNew = 1 << 30;      // new tokens of a sequence (far more than any memory holds): what is counted of them fits 32 bits

struct ChunkShape {
  int32_t batch, n_kv_heads, group, n_new;
  int32_t cache_items, item_keys;
  int32_t tile_tokens, row_tiles, tile_rows;      // tile_rows: of a slot
};

inline int chunk_len(const ChunkShape& s, const int32_t* len, int b) { return len ? len[b] : s.n_new; }
// items of row tile rt of a sequence with `len` new tokens
#if defined(__CUDACC__)
__host__ __device__
#endif
inline int chunk_items(const ChunkShape& s, int len, int rt) {
  if (rt * s.tile_tokens >= len) return 0;
  const int seen = (rt + 1) * s.tile_tokens < len ? (rt + 1) * s.tile_tokens : len;
  return s.cache_items + (seen + s.item_keys - 1) / s.item_keys;
}

struct ChunkCuts {
  int32_t n;                                 // CTAs
  int32_t tile[kChunkCtas + 1], item[kChunkCtas + 1];      // CTA c: from (tile, item) c to c + 1
  int32_t slot[kChunkCtas];                  // its first slot
};
struct ChunkMerge {
  int32_t n;                                 // tiles that left slots
  int32_t tile[kChunkParts], slot[kChunkParts + 1];
};

// Does the part [begin, end) of a tile with `items` items go through a slot?
#if defined(__CUDACC__)
__host__ __device__
#endif
inline bool chunk_needs_slot(int begin, int end, int items) { return begin > 0 || end < items; }

// Cuts `tiles` tiles, tile t of items(t) steps (asked for in order), into ranges of equal cost, one per CTA: a tile costs its steps and `start` more for its
// beginning, `total` in all.  A cut that would come within `snap` of a tile's beginning or end comes there: a tile that is not cut needs no slots.
// n_ctas: ranges, at most kChunkCtas.  Returns the number of slots; 0 with cuts->n = 0 where there is nothing to do.
template <class Items>
inline int cut_tiles(int tiles, int64_t total, int n_ctas, int start, int snap, Items items, ChunkCuts* cuts, ChunkMerge* merge) {
  cuts->n = 0;
  merge->n = 0;
  merge->slot[0] = 0;
  if (total == 0) return 0;
  // where CTAs begin: at the first tile that has steps, then at every n_ctas-th of the cost, places that fall together counted once
  int64_t at = 0;
  int c = 1, last_tile = -1, last_item = 0;
  bool to_next = false;                      // a cut was moved to the next tile's beginning
  auto begin = [&](int tile, int item) {
    if (last_tile > tile || (last_tile == tile && last_item >= item)) return;
    cuts->tile[cuts->n] = last_tile = tile;
    cuts->item[cuts->n++] = last_item = item;
  };
  for (int tile = 0; tile < tiles; ++tile) {
    const int n = items(tile);
    if (n == 0) continue;
    if (last_tile < 0 || to_next) begin(tile, 0);
    to_next = false;
    for (; c < n_ctas && total * c / n_ctas < at + start + n; ++c) {
      const int64_t cut = total * c / n_ctas - at - start;
      if (cut <= snap) begin(tile, 0);
      else if (cut < n - snap) begin(tile, static_cast<int>(cut));
      else to_next = true;
    }
    at += n + start;
  }
  cuts->tile[cuts->n] = tiles;
  cuts->item[cuts->n] = 0;
  // their slots
  int slots = 0;
  for (int i = 0; i < cuts->n; ++i) {
    cuts->slot[i] = slots;
    for (int tile = cuts->tile[i]; tile <= cuts->tile[i + 1] && tile < tiles; ++tile) {
      const int n = items(tile), from = tile == cuts->tile[i] ? cuts->item[i] : 0, to = tile == cuts->tile[i + 1] ? cuts->item[i + 1] : n;
      if (from >= to || !chunk_needs_slot(from, to, n)) continue;
      if (merge->n == 0 || merge->tile[merge->n - 1] != tile) merge->tile[merge->n++] = tile;
      merge->slot[merge->n] = ++slots;
    }
  }
  return slots;
}

// After a given-up wait: f(part) for every part of a CTA that some of its warps may not have begun (and perhaps for some that they have done).  A part is put
// over the one kRing before it once all warps have begun that one, so what they have not begun is in the ring (`published` went through it, one without a
// tile at the end), in hand (`hand`: `part` was taken, but not published), or still to come (next(part), with a part in hand only).
template <int kRing, class Part, class Next, class F>
#if defined(__CUDACC__)
__host__ __device__
#endif
inline void parts_left(const Part* ring, int published, bool hand, Part part, Next next, F f) {
  for (int k = published > kRing ? published - kRing : 0; k < published; ++k)
    if (ring[k % kRing].tile >= 0) f(ring[k % kRing]);
  if (!hand) return;
  do f(part);
  while (next(part));
}

// CTAs for so much work, where one is worth starting for min_items
inline int chunk_ctas(int64_t total, int min_items) { return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kChunkCtas, total / min_items))); }

// Tiles in the order (sequence, KV head, row tile).  second: what a CTA's second tile costs it, in items.  Where all tiles have the same number of items and it
// is cheaper, every tile gets the same number of CTAs and none has two.
inline int chunk_plan(const ChunkShape& s, const int32_t* len, int min_items, int start, int snap, int second, ChunkCuts* cuts, ChunkMerge* merge) {
  int64_t total = 0, filled = 0;
  int most = 0, least = INT32_MAX;
  for (int b = 0; b < s.batch; ++b) {
    const int n = chunk_len(s, len, b);
    for (int rt = 0; rt < s.row_tiles && rt * s.tile_tokens < n; ++rt) {
      const int items = chunk_items(s, n, rt);
      total += static_cast<int64_t>(s.n_kv_heads) * (items + start);
      filled += s.n_kv_heads;
      most = std::max(most, items);
      least = std::min(least, items);
    }
  }
  int n = chunk_ctas(total, min_items);
  if (most == least && filled <= n) {
    const int even = n - static_cast<int>(n % filled);
    if ((total + even - 1) / even <= total / n + second) n = even;
  }
  return cut_tiles(s.batch * s.n_kv_heads * s.row_tiles, total, n, start, snap,
                   [&](int tile) { return chunk_items(s, chunk_len(s, len, tile / s.row_tiles / s.n_kv_heads), tile % s.row_tiles); }, cuts, merge);
}

#if defined(__CUDACC__)
struct TableEntry;
struct ChunkCall {
  const uint8_t* arena;
  size_t arena_bytes;
  const TableEntry* table;
  const uint32_t* res_off256;
  const int32_t* res_count;
  const uint16_t *q, *k_new, *v_new;
  uint16_t* out;
  float *lse, *workspace;
  uint32_t* status;
  int32_t table_stride, n_closed, n_tail, res_rows;      // residual rows: of the stream that has most
  float scale;
  ChunkShape shape;
};
template <int N>
struct ChunkLens {                          // N = 1: every sequence has n_new rows
  int32_t len[N];
};
cudaError_t launch_verify(const ChunkCall& call, const ChunkCuts& cuts, const ChunkMerge& merge, const int32_t* len, cudaStream_t st);
cudaError_t launch_dense(const ChunkCall& call, int first, int seqs, const int32_t* len, cudaStream_t st);
cudaError_t launch_chunk_merge(const ChunkCall& call, const ChunkMerge& merge, const int32_t* len, cudaStream_t st);
#endif

// A step coprime to n, about 0.618 of it: multiplied by it, neighbouring places of a walk are blocks of different ages.
inline int chunk_walk(int n) {
  if (n <= 2) return 1;
  auto gcd = [](int a, int b) {
    while (b) {
      const int t = a % b;
      a = b;
      b = t;
    }
    return a;
  };
  int walk = static_cast<int>(n * 0.6180339887);
  while (gcd(walk, n) != 1) ++walk;
  return walk;
}

// ---- chunks of few rows (gkv_verify.cu): a tile is a stream, an item half a block, 32 keys ----
// Rows up to which a chunk counts as one of few.  64 rows here and 68 and 96 written out: 16 streams of 8,200 tokens 43, 68 and 62 us, 64 of 16,384 tokens
// 206, 339 and 324, two of 1,000 tokens 21, 32 and 24.  (Two tiles of up to 64 rows each would read the codes twice: 65 for 69, 255 for 339, but 82 for
// 64 and 378 for 327 at 128 rows.)
constexpr int kVerifyRows = 64;
inline void verify_shape(ChunkShape* s, int n_closed, int n_tail, int res_rows) {
  s->tile_tokens = s->n_new;
  s->tile_rows = kChunkRows;
  s->row_tiles = 1;
  s->item_keys = 32;
  s->cache_items = 2 * n_closed + (n_tail + 31) / 32 + (res_rows + 31) / 32;
}
constexpr int kVerifyWarps = 12;             // of a CTA; a team has one per 16 rows
inline int verify_teams(const ChunkShape& s) { return kVerifyWarps / ((s.n_new * s.group + 15) / 16); }
// (two streams of 33 items, 16 rows, twelve teams: 12.8 us with 12 CTAs, 13.4 with 6, 22 and 32, 19.4 with 11, of which one had two streams)
inline int verify_min_items(const ChunkShape& s) { return std::max(2, verify_teams(s) / 2 - 1); }
// A second stream costs a CTA about 9500 cycles (queries, the teams' merge, slots), an item 6000 of a team's (sixteen streams of 8,200 tokens, 64 rows: 45 us
// with nine CTAs each, 50 with 148 cut anywhere; 64 streams of 32,757 would lose an eighth of the CTAs)
inline int verify_second(const ChunkShape& s) { return 3 * verify_teams(s) / 2; }

// ---- chunks of many rows (gkv_dense.cu): a tile is 256 rows in two halves, an item 128 rows of keys; centroids have a row each ----
inline void dense_shape(ChunkShape* s, int rows) {      // rows: of the stream that has most
  s->tile_tokens = 2 * (kChunkRows / s->group);
  s->tile_rows = 2 * kChunkRows;
  s->row_tiles = (s->n_new + s->tile_tokens - 1) / s->tile_tokens;
  s->item_keys = 128;
  s->cache_items = (rows + 127) / 128;
}
struct DensePlaces {
  size_t k_hi, k_lo, v, q16, bias, flags, order, blocks, parts;
};
size_t dense_bytes(const ChunkShape& s, int n_closed, int seqs, DensePlaces* at);
constexpr size_t kDenseBytes = size_t(1) << 30;      // what a call's workspace stays below, unless one sequence needs more

}  // namespace gkv
