// Chunks of many rows (the next turn of a conversation, a document behind a cached context): the stored blocks are worth writing out once.
//
// order_kernel   puts a stream's blocks in the order of their rows: those with 64 rows, then the centroids, one row each; queries become fp16 rows
// expand_kernel  writes keys and values as fp16 rows: a quantised key as a pair hi + lo (22 bits: the log-sum-exp of a short context would
//                otherwise miss 32 bits by the rounding of a few heavy keys), a value rounded once (off by 2^-11 of itself at most, 2^-25 below 2^-14).
//                Exact rows and the chunk's own rows become fp16 too, exactly but for numbers below 2^-14 (off by up to 2^-25, lo included: 2^-24 is
//                fp16's last step) and beyond +-65504 (clamped)
// attend_kernel  (gkv_attend.cuh) with a second product Q K_lo where keys have one, a term per key where some are hidden or stand for many (log2 of
//                how many), and the chunk's own rows causally
//
// What bounds it: the matrix products, 4 * 128 flops per row and key and half as much again for K_lo.  Writing a block out costs 48 KB and reading it
// back once per 256 rows; a kernel that dequantised into shared memory for every 128 rows needed 700 issue cycles of an SM per 64 keys for that
// alone and took 2.1 times as long over 32,768 tokens.
//
// Work split.  gkv_chunk.h cuts all tiles' steps into equal ranges, one per CTA, whose parts of a tile are merged by attend_merge_kernel.
// The four launches overlap at their edges (programmatic dependent launch).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "gkv_attend.cuh"
#include "gkv_chunk.h"
#include "gkv_internal.h"
#include "gkv_tc.cuh"

namespace gkv {
namespace {

using namespace tc;

// ---- order ---------------------------------------------------------------------------------------
struct DenseParams {
  const uint8_t* arena;
  const TableEntry* table;
  const uint32_t* res_off256;
  const int32_t* res_count;
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  uint16_t* out;
  float* lse;
  float* part_o;
  float2* part_ml;
  uint32_t* status;
  // workspace: of stream s the rows [s * stream_rows, (s + 1) * stream_rows)
  uint16_t* k_hi;
  uint16_t* k_lo;
  uint16_t* v;
  uint16_t* q16;             // [batch * n_new][heads][128]
  float* bias;               // per row, in units of q . k
  int32_t* flags;            // per step of a stream
  TableEntry* order;         // [stream][n_closed]
  int32_t* blocks;           // per stream: blocks with 64 rows
  int32_t table_stride, n_closed, n_tail, steps, cache_steps, stream_rows, first_stream;
  float scale_log2;
  ChunkShape s;
};

__device__ __forceinline__ uint32_t sat_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 halves(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
__device__ __forceinline__ float half_of(uint32_t w, int i) { return __half2float(__ushort_as_half(static_cast<unsigned short>(i ? w >> 16 : w))); }

// CTAs [0, streams): a stream's blocks in order.  The others: queries as fp16 rows, and the steps' flags cleared.
__global__ void __launch_bounds__(256) order_kernel(const __grid_constant__ DenseParams p, int streams, size_t pieces, size_t first) {
  pdl_wait();
  pdl_launch();
  const int stream = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (stream >= streams) {
    const size_t i = static_cast<size_t>(blockIdx.x - streams) * 256 + tid;
    if (i < static_cast<size_t>(streams) * p.steps) p.flags[i] = 0;
    if (i >= pieces) return;
    const uint4 x = reinterpret_cast<const uint4*>(p.q)[first + i];
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t a[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = sat_pair(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    reinterpret_cast<uint4*>(p.q16)[i] = make_uint4(a[0], a[1], a[2], a[3]);
    return;
  }
  __shared__ int full[8], cent[8], base[2];
  const TableEntry* table = p.table + static_cast<size_t>(p.first_stream + stream) * p.table_stride;
  TableEntry* const order = p.order + static_cast<size_t>(stream) * p.n_closed;
  // centroids are counted from the end
  if (tid == 0) base[0] = 0, base[1] = p.n_closed;
  for (int i0 = 0; i0 < p.n_closed; i0 += 256) {
    const int i = i0 + tid;
    TableEntry e{};
    if (i < p.n_closed) e = table[i];
    const uint32_t f = __ballot_sync(0xffffffffu, e.level > 1), c = __ballot_sync(0xffffffffu, e.level == 1);
    __syncthreads();
    if (lane == 0) full[warp] = __popc(f), cent[warp] = __popc(c);
    __syncthreads();
    int at_f = base[0], at_c = base[1], all_f = 0, all_c = 0;
    for (int w = 0; w < 8; ++w) {
      if (w < warp) at_f += full[w], at_c -= cent[w];
      all_f += full[w], all_c += cent[w];
    }
    const uint32_t below = (1u << lane) - 1u;
    if (e.level > 1) order[at_f + __popc(f & below)] = e;
    if (e.level == 1) order[at_c - 1 - __popc(c & below)] = e;
    __syncthreads();
    if (tid == 0) base[0] += all_f, base[1] -= all_c;
  }
  __syncthreads();
  if (tid == 0) p.blocks[stream] = base[0];
}

// ---- rows ----------------------------------------------------------------------------------------
constexpr int kEThreads = 256;
// Where element c of a staged row lies: 16-byte pieces of neighbouring rows are swapped, so that a column's are in different banks
__device__ __forceinline__ int staged(int r, int c) { return r * kD + (((c >> 3) ^ (r & 7)) << 3) + (c & 7); }

// Four 8 x 8 tiles of 16-bit elements from the lanes' fragments: rows, or columns where the fragments hold the transposed tiles
template <bool kTrans>
__device__ __forceinline__ void store_tiles(uint32_t at, const uint32_t (&x)[4]) {
  if (kTrans) asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
  else asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
}

// A warp's tile of a quantised half block (16 tokens, 128 channels).  A lane's codes are 4, 2 or 1 pieces of 16 bytes; all of its loads are in flight
// at once.  A code is exact in 24 bits (the low bits of 2^23 + code), code * scale + zero is rounded once, and again to 16 bits.
template <int kBits, bool kV>
__device__ __forceinline__ void expand_tile(const uint8_t* raw, int tile, int lane, uint32_t hi, uint32_t lo) {
  const int c4 = lane & 3, m = lane >> 3, j8 = lane & 7;
  const uint8_t* codes = raw + (kV ? off_vc(kBits, tile & 1) : off_kc(kBits, tile & 1)) + lane * 16;
  constexpr int kQuads = kBits / 2;
  uint32_t w[4 * kQuads], q[4][4], z[4][4];            // scales and zeros by pairs of steps; keys: [2 * pair of channels + step], values: [pair of tokens]
#pragma unroll
  for (int i = 0; i < kQuads; ++i) {
    const uint4 x = *reinterpret_cast<const uint4*>(codes + i * 512);
    w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
  }
#pragma unroll
  for (int sp = 0; sp < 4; ++sp) {
    if (!kV) {
      const uint4* kp = reinterpret_cast<const uint4*>(raw + off_kp() + (sp * 4 + c4) * 32);
      const uint4 a = kp[0], b = kp[1];
      z[sp][0] = a.x, z[sp][1] = a.y, z[sp][2] = a.z, z[sp][3] = a.w;
      q[sp][0] = b.x, q[sp][1] = b.y, q[sp][2] = b.z, q[sp][3] = b.w;
    } else {
      const uint8_t* vp = raw + off_vp(kBits, tile & 1);
      const uint2 a = *reinterpret_cast<const uint2*>(vp + c4 * 32 + sp * 8), b = *reinterpret_cast<const uint2*>(vp + 128 + (sp * 4 + c4) * 8);
      q[sp][0] = a.x, q[sp][1] = a.y;
      z[sp][0] = b.x, z[sp][1] = b.y;
    }
  }
  // where lane's row of tile m of a step goes (the steps differ in the 16-byte piece)
  const uint32_t row = (tile * 16 + 8 * (kV ? m >> 1 : m & 1) + j8) * kRowBytes, piece = kV ? m & 1 : m >> 1;
  const uint64_t base = f2_pack(-8388608.f, -8388608.f);
  constexpr uint32_t kMask = (1u << kBits) - 1u;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    uint32_t x[4], d[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      int byte, bit;
      code_pos(kBits, kV, 0, s, a, 0, &byte, &bit);
      const uint32_t c = w[byte / 512 * 4 + byte % 512 / 4];
      const int p = kV ? a >> 1 : 2 * (a >> 1) + (s & 1);
      const float2 sc = halves(q[s >> 1][p]), ze = halves(z[s >> 1][p]);
      const uint64_t code = f2_add(f2_pack(__uint_as_float((c >> bit & kMask) | 0x4b000000u), __uint_as_float((c >> (bit + 16) & kMask) | 0x4b000000u)), base);
      float f0, f1;
      f2_unpack(f2_fma(code, f2_pack(sc.x, sc.y), f2_pack(ze.x, ze.y)), f0, f1);
      x[a] = sat_pair(f0, f1);
      if (!kV) {
        const float2 g = halves(x[a]);
        d[a] = sat_pair(f0 - g.x, f1 - g.y);
      }
    }
    const uint32_t at = row + (((2 * s + piece) ^ j8) << 4);
    store_tiles<kV>(hi + at, x);
    if (!kV) store_tiles<false>(lo + at, d);
  }
}

// A step's 64 rows: one CTA.  24 us for the 137,000 rows of two sequences of 8,191 tokens and 300 new ones, 105 MB written (18 us at 5.9 TB/s): issue of
// the conversions and the copy out of shared memory; with codes read in the loop and stored by 2 and 4 bytes it was 44.  blockIdx.x: half step, blockIdx.y: stream of the group.
template <int N>
__global__ void __launch_bounds__(kEThreads) expand_kernel(const __grid_constant__ DenseParams p, const __grid_constant__ ChunkLens<N> lens) {
  __shared__ __align__(16) uint16_t hi[kBlock * kD], lo[kBlock * kD], va[kBlock * kD];
  const ChunkShape& sh = p.s;
  const int unit = blockIdx.x, stream = blockIdx.y, real = p.first_stream + stream, b = real / sh.n_kv_heads, h = real % sh.n_kv_heads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t row0 = static_cast<size_t>(stream) * p.stream_rows + static_cast<size_t>(unit) * kBlock;
  const int len = lens.len[N == 1 ? 0 : b];
  pdl_wait();
  pdl_launch();
  const TableEntry* table = p.table + static_cast<size_t>(real) * p.table_stride;
  const TableEntry* order = p.order + static_cast<size_t>(stream) * p.n_closed;
  const int blocks = p.blocks[stream];
  bool low = false, term = false;
  if (unit < blocks) {
    const TableEntry e = order[unit];
    const uint8_t* slot = p.arena + static_cast<size_t>(e.off256) * 256;
    term = e.resmask != 0;
    if (tid < kBlock) p.bias[row0 + tid] = e.resmask >> tid & 1u ? -INFINITY : 0.f;
    if (e.level == 16) {
      low = true;                          // (below 2^-14 a bf16 value has bits that fp16 has not)
      constexpr int kPieces = kBlock * 16 / kEThreads;
      uint4 ks[kPieces], vs[kPieces];
#pragma unroll
      for (int n = 0; n < kPieces; ++n) {
        const uint4* at = reinterpret_cast<const uint4*>(slot) + n * kEThreads + tid;
        ks[n] = at[0];
        vs[n] = at[kBlock * 16];
      }
#pragma unroll
      for (int n = 0; n < kPieces; ++n) {
        const int i = n * kEThreads + tid, r = i >> 4, c = (i & 15) * 8;
        const uint4 k = ks[n], v = vs[n];
        const uint32_t kw[4] = {k.x, k.y, k.z, k.w}, vw[4] = {v.x, v.y, v.z, v.w};
        uint32_t a[4], d[4], x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float f0 = __uint_as_float(kw[j] << 16), f1 = __uint_as_float(kw[j] & 0xffff0000u);
          a[j] = sat_pair(f0, f1);
          const float2 g = halves(a[j]);
          d[j] = sat_pair(f0 - g.x, f1 - g.y);
          x[j] = sat_pair(__uint_as_float(vw[j] << 16), __uint_as_float(vw[j] & 0xffff0000u));
        }
        *reinterpret_cast<uint4*>(&hi[staged(r, c)]) = make_uint4(a[0], a[1], a[2], a[3]);
        *reinterpret_cast<uint4*>(&lo[staged(r, c)]) = make_uint4(d[0], d[1], d[2], d[3]);
        *reinterpret_cast<uint4*>(&va[staged(r, c)]) = make_uint4(x[0], x[1], x[2], x[3]);
      }
    } else {
      low = true;
      const bool is_v = warp >= 4;
      const int tile = warp & 3;
      const uint8_t* raw = slot + (tile >> 1) * half_bytes(static_cast<int>(e.level));
      const uint32_t to = smem_u32(is_v ? va : hi), to_lo = smem_u32(lo);
      if (e.level == 8) is_v ? expand_tile<8, true>(raw, tile, lane, to, to_lo) : expand_tile<8, false>(raw, tile, lane, to, to_lo);
      else if (e.level == 4) is_v ? expand_tile<4, true>(raw, tile, lane, to, to_lo) : expand_tile<4, false>(raw, tile, lane, to, to_lo);
      else is_v ? expand_tile<2, true>(raw, tile, lane, to, to_lo) : expand_tile<2, false>(raw, tile, lane, to, to_lo);
    }
  } else {
    // single rows: centroids, the partial block, residual rows; behind the cache's steps the chunk's own; nothing else
    const int rest = (unit - blocks) * kBlock, cents = p.n_closed - blocks, res = p.res_count[real];
    const bool fresh = unit >= 2 * p.cache_steps;
    low = true;
    for (int i = tid; i < kBlock * 16; i += kEThreads) {
      const int r = i >> 4, c = (i & 15) * 8;
      const uint8_t *k = nullptr, *v = nullptr;
      float t = -INFINITY;
      if (fresh) {
        const int tok = (unit - 2 * p.cache_steps) * kBlock + r;
        if (tok < len) {
          const size_t at = (static_cast<size_t>(b) * sh.n_new + tok) * sh.n_kv_heads + h;
          k = reinterpret_cast<const uint8_t*>(p.k_new + at * kD);
          v = reinterpret_cast<const uint8_t*>(p.v_new + at * kD);
          t = 0.f;
        }
      } else {
        const int j = rest + r;
        if (j < cents) {
          const TableEntry e = order[p.n_closed - 1 - j];
          k = p.arena + static_cast<size_t>(e.off256) * 256;
          v = k + kRowBytes;
          const int n = kBlock - __popcll(e.resmask);
          t = n > 0 ? lg2(static_cast<float>(n)) / p.scale_log2 : -INFINITY;
        } else if (j < cents + p.n_tail) {
          k = p.arena + static_cast<size_t>(table[p.n_closed].off256) * 256 + (j - cents) * kRowBytes;
          v = k + kBlock * kRowBytes;
          t = 0.f;
        } else if (j < cents + p.n_tail + res) {
          k = p.arena + static_cast<size_t>(p.res_off256[real]) * 256 + static_cast<size_t>(j - cents - p.n_tail) * 2 * kRowBytes;
          v = k + kRowBytes;
          t = 0.f;
        }
      }
      term = term || t != 0.f;
      uint4 x = make_uint4(0, 0, 0, 0), y = x;
      if (k) {
        x = *reinterpret_cast<const uint4*>(k + c * 2);
        y = *reinterpret_cast<const uint4*>(v + c * 2);
      }
      const uint32_t kw[4] = {x.x, x.y, x.z, x.w}, vw[4] = {y.x, y.y, y.z, y.w};
      uint32_t a[4], d[4], o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float f0 = __uint_as_float(kw[j] << 16), f1 = __uint_as_float(kw[j] & 0xffff0000u);
        a[j] = sat_pair(f0, f1);
        const float2 g = halves(a[j]);
        d[j] = sat_pair(f0 - g.x, f1 - g.y);
        o[j] = sat_pair(__uint_as_float(vw[j] << 16), __uint_as_float(vw[j] & 0xffff0000u));
      }
      *reinterpret_cast<uint4*>(&hi[staged(r, c)]) = make_uint4(a[0], a[1], a[2], a[3]);
      *reinterpret_cast<uint4*>(&lo[staged(r, c)]) = make_uint4(d[0], d[1], d[2], d[3]);
      *reinterpret_cast<uint4*>(&va[staged(r, c)]) = make_uint4(o[0], o[1], o[2], o[3]);
      if (c == 0) p.bias[row0 + r] = t;
    }
  }
  // (a chunk's own rows are masked causally: no term)
  term = __syncthreads_or(term && unit < 2 * p.cache_steps);
  bool any_low = false;
  for (int i = tid; i < kBlock * 16; i += kEThreads) {
    const int r = i >> 4, c = (i & 15) * 8;
    const size_t at = (row0 + r) * kD + c;
    const uint4 l = *reinterpret_cast<const uint4*>(&lo[staged(r, c)]);
    any_low = any_low || ((l.x | l.y | l.z | l.w) & 0x7fff7fffu) != 0;
    *reinterpret_cast<uint4*>(p.k_hi + at) = *reinterpret_cast<const uint4*>(&hi[staged(r, c)]);
    *reinterpret_cast<uint4*>(p.k_lo + at) = l;
    *reinterpret_cast<uint4*>(p.v + at) = *reinterpret_cast<const uint4*>(&va[staged(r, c)]);
  }
  low = __syncthreads_or(any_low);
  // (two CTAs have a step's halves: the flags were cleared in front of this)
  if (tid == 0 && (term || low)) atomicOr(p.flags + static_cast<size_t>(stream) * p.steps + (unit >> 1), (term ? attend::kHasTerm : 0) | (low ? attend::kHasLow : 0));
}

// ---- attention -----------------------------------------------------------------------------------
constexpr int kDRows = attend::kRows;
using attend::kHasLow;
using attend::kHasTerm;

template <int N>
struct DenseWork {
  static constexpr bool kBf16 = false, kPairs = true;
  static constexpr float ln2_rest = 0.f;
  uint16_t* out;
  float* lse;
  float* part_o;
  float2* part_ml;
  uint32_t* status;
  const float* bias;
  const int32_t* step_flags;
  int64_t out_stride;
  int32_t group, n_q_heads, half_tokens, first_seq, steps, cache_steps, stream_rows;
  float scale_log2;
  ChunkShape s;
  ChunkCuts cuts;
  ChunkLens<N> lens;
  __device__ __forceinline__ int first_slot() const { return cuts.slot[blockIdx.x]; }
  __device__ __forceinline__ bool whole_tiles() const { return false; }
  __device__ __forceinline__ void whole(int, attend::Part&) const {}
  __device__ __forceinline__ bool next(int& state, int& slot, attend::Part& x) const {
    const int t0 = cuts.tile[blockIdx.x], t1 = cuts.tile[blockIdx.x + 1];
    for (; t0 + state <= t1 && t0 + state < s.batch * s.n_kv_heads * s.row_tiles; ++state) {
      x.tile = t0 + state;
      const int rt = x.tile % s.row_tiles, stream = x.tile / s.row_tiles, b = stream / s.n_kv_heads;
      x.len = lens.len[N == 1 ? 0 : first_seq + b];
      x.items = chunk_items(s, x.len, rt);
      x.begin = state == 0 ? cuts.item[blockIdx.x] : 0;
      x.end = x.tile == t1 ? cuts.item[blockIdx.x + 1] : x.items;
      if (x.begin >= x.end) continue;
      x.tok0 = rt * s.tile_tokens;
      x.causal0 = cache_steps;
      x.row0 = static_cast<int64_t>(first_seq + b) * s.n_new;
      x.head0 = (stream % s.n_kv_heads) * s.group;
      x.kv = stream;
      x.q_row = b * s.n_new;
      x.slot = chunk_needs_slot(x.begin, x.end, x.items) ? slot++ : -1;
      x.two = x.tok0 + half_tokens < x.len;
      x.keep = kDRows;                       // (rows that are not there were written as zeros)
      ++state;
      return true;
    }
    return false;
  }
  __device__ __forceinline__ void load_q(const CUtensorMap* map, uint32_t dst, const attend::Part& x, int t, uint32_t bar) const {
    for (int k = 0; k < 2; ++k) tma_load_3d(dst + k * attend::kPanel, map, 64 * k, x.head0, x.q_row + x.tok0 + t * half_tokens, bar);
  }
  __device__ __forceinline__ void load_keys(const CUtensorMap* map, uint32_t dst, const attend::Part& x, int step, uint32_t bar) const {
    tma_load_3d(dst, map, 0, x.kv * stream_rows + step * kDRows, 0, bar);
  }
  __device__ __forceinline__ int flags(const attend::Part& x, int step) const { return __ldg(step_flags + static_cast<size_t>(x.kv) * steps + step); }
  __device__ __forceinline__ const float* term(const attend::Part& x, int step) const {
    return bias + static_cast<size_t>(x.kv) * stream_rows + static_cast<size_t>(step) * kDRows;
  }
  struct Where {
    int tok0, len, head0;
    int64_t row0;
  };
  __device__ __forceinline__ Where place(int tile) const {
    const int rt = tile % s.row_tiles, stream = tile / s.row_tiles, b = stream / s.n_kv_heads;
    return {rt * s.tile_tokens, lens.len[N == 1 ? 0 : first_seq + b], (stream % s.n_kv_heads) * s.group, static_cast<int64_t>(first_seq + b) * s.n_new};
  }
  __device__ __forceinline__ void fail() const { atomicOr(status, kStatusInternal); }
};

template <int N>
cudaError_t launch_attend(const DenseParams& p, const attend::Maps& maps, const ChunkCuts& cuts, const ChunkMerge& merge, const ChunkLens<N>& lens, cudaStream_t st) {
  DenseWork<N> w;
  w.out = p.out;
  w.lse = p.lse;
  w.part_o = p.part_o;
  w.part_ml = p.part_ml;
  w.status = p.status;
  w.bias = p.bias;
  w.step_flags = p.flags;
  w.group = p.s.group;
  w.n_q_heads = p.s.n_kv_heads * p.s.group;
  w.out_stride = static_cast<int64_t>(w.n_q_heads) * kD;
  w.half_tokens = p.s.tile_tokens / 2;
  w.first_seq = p.first_stream / p.s.n_kv_heads;
  w.steps = p.steps;
  w.cache_steps = p.cache_steps;
  w.stream_rows = p.stream_rows;
  w.scale_log2 = p.scale_log2;
  w.s = p.s;
  w.cuts = cuts;
  w.lens = lens;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = raise_smem_limit(attend::attend_kernel<DenseWork<N>>, attend::kSmem, done);
  if (e == cudaSuccess) e = attend::launch_behind(attend::attend_kernel<DenseWork<N>>, dim3(cuts.n), attend::kThreads, attend::kSmem, st, w, maps);
  if (e != cudaSuccess || merge.n == 0) return e;
  return attend::launch_behind(attend::attend_merge_kernel<DenseWork<N>>, dim3((p.s.tile_tokens * p.s.group + 31) / 32, merge.n), 128, 0, st, w, merge);
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

// Bytes of workspace of `seqs` sequences, and where its parts lie (offsets are filled in where `at` is given).
size_t dense_bytes(const ChunkShape& s, int n_closed, int seqs, DensePlaces* at) {
  const size_t streams = static_cast<size_t>(seqs) * s.n_kv_heads, steps = s.cache_items + (s.n_new + kDRows - 1) / kDRows, rows = streams * steps * kDRows;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += up256(bytes);
    return o;
  };
  DensePlaces d;
  d.k_hi = take(rows * kRowBytes);
  d.k_lo = take(rows * kRowBytes);
  d.v = take(rows * kRowBytes);
  d.q16 = take(static_cast<size_t>(seqs) * s.n_new * s.n_kv_heads * s.group * kRowBytes);
  d.bias = take(rows * sizeof(float));
  d.flags = take(streams * steps * sizeof(int32_t));
  d.order = take(streams * std::max(n_closed, 1) * sizeof(TableEntry));
  d.blocks = take(streams * sizeof(int32_t));
  d.parts = take(static_cast<size_t>(std::min<int64_t>(kChunkParts, static_cast<int64_t>(streams) * s.row_tiles + kChunkCtas - 1)) * s.tile_rows * (kD + 2) * sizeof(float));
  if (at) *at = d;
  return off;
}

// Sequences [first, first + seqs) of the call, in a workspace of dense_bytes.  len: HOST, of all sequences, or null.
cudaError_t launch_dense(const ChunkCall& call, int first, int seqs, const int32_t* len, cudaStream_t st) {
  ChunkShape s = call.shape;
  s.batch = seqs;
  ChunkCuts cuts;
  ChunkMerge merge;
  const int slots = chunk_plan(s, len ? len + first : nullptr, 4, attend::kStart, attend::kSnap, attend::kStart, &cuts, &merge);
  if (cuts.n == 0) return cudaSuccess;
  DensePlaces at;
  dense_bytes(s, call.n_closed, seqs, &at);
  uint8_t* const ws = reinterpret_cast<uint8_t*>(call.workspace);
  DenseParams p{};
  p.arena = call.arena;
  p.table = call.table;
  p.res_off256 = call.res_off256;
  p.res_count = call.res_count;
  p.q = call.q;
  p.k_new = call.k_new;
  p.v_new = call.v_new;
  p.out = call.out;
  p.lse = call.lse;
  p.part_o = reinterpret_cast<float*>(ws + at.parts);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + static_cast<size_t>(slots) * s.tile_rows * kD);
  p.status = call.status;
  p.k_hi = reinterpret_cast<uint16_t*>(ws + at.k_hi);
  p.k_lo = reinterpret_cast<uint16_t*>(ws + at.k_lo);
  p.v = reinterpret_cast<uint16_t*>(ws + at.v);
  p.q16 = reinterpret_cast<uint16_t*>(ws + at.q16);
  p.bias = reinterpret_cast<float*>(ws + at.bias);
  p.flags = reinterpret_cast<int32_t*>(ws + at.flags);
  p.order = reinterpret_cast<TableEntry*>(ws + at.order);
  p.blocks = reinterpret_cast<int32_t*>(ws + at.blocks);
  p.table_stride = call.table_stride;
  p.n_closed = call.n_closed;
  p.n_tail = call.n_tail;
  p.cache_steps = s.cache_items;
  p.steps = s.cache_items + (s.n_new + kDRows - 1) / kDRows;
  p.stream_rows = p.steps * kDRows;
  p.first_stream = first * s.n_kv_heads;
  p.scale_log2 = call.scale * kLog2e;
  p.s = s;
  const int streams = seqs * s.n_kv_heads;
  const uint64_t rows = static_cast<uint64_t>(streams) * p.stream_rows, heads = static_cast<uint64_t>(s.n_kv_heads) * s.group;
  attend::Maps maps;
  const uint64_t rd[3] = {64, rows, 2}, rs[2] = {kRowBytes, 128}, qd[3] = {kD, heads, static_cast<uint64_t>(seqs) * s.n_new}, qs[2] = {kRowBytes, heads * kRowBytes};
  const uint32_t rb[3] = {64, kDRows, 2}, qb[3] = {64, static_cast<uint32_t>(s.group), static_cast<uint32_t>(s.tile_tokens / 2)};
  if (!make_map(&maps.q, p.q16, 3, qd, qs, qb) || !make_map(&maps.k, p.k_hi, 3, rd, rs, rb) || !make_map(&maps.k_lo, p.k_lo, 3, rd, rs, rb) ||
      !make_map(&maps.v, p.v, 3, rd, rs, rb))
    return cudaErrorInvalidValue;
  const size_t per_seq = static_cast<size_t>(s.n_new) * heads * kD / 8, pieces = per_seq * seqs;
  const size_t threads = std::max(pieces, static_cast<size_t>(streams) * p.steps);
  cudaError_t e = attend::launch_behind(order_kernel, dim3(static_cast<unsigned>(streams + (threads + 255) / 256)), 256, 0, st, p, streams, pieces, per_seq * first);
  if (e != cudaSuccess) return e;
  const dim3 grid(2 * p.steps, streams);
  const bool one = !len || call.shape.batch == 1;
  ChunkLens<1> l1{{len ? len[0] : s.n_new}};
  ChunkLens<kChunkMaxBatch> ln;
  if (!one) std::copy(len, len + call.shape.batch, ln.len);
  e = one ? attend::launch_behind(expand_kernel<1>, grid, kEThreads, 0, st, p, l1) : attend::launch_behind(expand_kernel<kChunkMaxBatch>, grid, kEThreads, 0, st, p, ln);
  if (e != cudaSuccess) return e;
  return one ? launch_attend(p, maps, cuts, merge, l1, st) : launch_attend(p, maps, cuts, merge, ln, st);
}

}  // namespace gkv
