// Chunks of many rows (the next turn of a conversation, a document behind a cached context): the stored blocks are worth writing out once.
//
// order_kernel   puts a stream's blocks in the order of their rows: those with 64 rows, then the centroids, one row each
// expand_kernel  writes keys and values as fp16 rows: a quantised key as a pair hi + lo (22 bits: the log-sum-exp of a short context would
//                otherwise miss 32 bits by the rounding of a few heavy keys), a value rounded once (2^-12 of itself).  Exact rows and the chunk's own
//                rows become fp16 too, exactly but for values below 2^-14 (their last bits, kept in lo for keys) and beyond +-65504 (clamped)
// dense_kernel   attention of two tiles of 128 rows at a time over 128 rows of keys per step, as gkv_prompt.cu does it, with a second product
//                Q K_lo where keys have one, a term per key where some are hidden or stand for many (log2 of how many), and the chunk's own rows causally
//
// What bounds it: the matrix products, 4 * 128 flops per row and key and half as much again for K_lo.  Writing a block out costs 48 KB and reading it
// back once per 256 rows; a kernel that dequantised into shared memory for every 128 rows needed 700 issue cycles of an SM per 64 keys for that
// alone and took 2.1 times as long over 32,768 tokens.
//
// Work split.  gkv_chunk.h cuts all tiles' steps into equal ranges, one per CTA, whose parts of a tile are merged by chunk_merge_kernel.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

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
  int32_t* order;            // [stream][n_closed]
  int32_t* blocks;           // per stream: blocks with 64 rows
  int32_t table_stride, n_closed, n_tail, steps, cache_steps, stream_rows, first_stream;
  float scale_log2;
  ChunkShape s;
};
constexpr int kHasTerm = 1, kHasLow = 2;   // flags: rows need their term; keys are pairs

__global__ void __launch_bounds__(256) order_kernel(const __grid_constant__ DenseParams p) {
  __shared__ int full[8], cent[8], base[2];
  const int stream = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const TableEntry* table = p.table + static_cast<size_t>(p.first_stream + stream) * p.table_stride;
  int32_t* const order = p.order + static_cast<size_t>(stream) * p.n_closed;
  // centroids are counted from the end
  if (tid == 0) base[0] = 0, base[1] = p.n_closed;
  for (int i0 = 0; i0 < p.n_closed; i0 += 256) {
    const int i = i0 + tid;
    const uint32_t level = i < p.n_closed ? table[i].level : 0;
    const uint32_t f = __ballot_sync(0xffffffffu, level > 1), c = __ballot_sync(0xffffffffu, level == 1);
    __syncthreads();
    if (lane == 0) full[warp] = __popc(f), cent[warp] = __popc(c);
    __syncthreads();
    int at_f = base[0], at_c = base[1], all_f = 0, all_c = 0;
    for (int w = 0; w < 8; ++w) {
      if (w < warp) at_f += full[w], at_c -= cent[w];
      all_f += full[w], all_c += cent[w];
    }
    const uint32_t below = (1u << lane) - 1u;
    if (level > 1) order[at_f + __popc(f & below)] = i;
    if (level == 1) order[at_c - 1 - __popc(c & below)] = i;
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

__device__ __forceinline__ uint32_t sat_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 halves(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
__device__ __forceinline__ float half_of(uint32_t w, int i) { return __half2float(__ushort_as_half(static_cast<unsigned short>(i ? w >> 16 : w))); }

// A step's 64 rows: one CTA.  blockIdx.x: half step, blockIdx.y: stream of the group.
template <int N>
__global__ void __launch_bounds__(kEThreads) expand_kernel(const __grid_constant__ DenseParams p, const __grid_constant__ ChunkLens<N> lens) {
  __shared__ __align__(16) uint16_t hi[kBlock * kD], lo[kBlock * kD], va[kBlock * kD];
  const ChunkShape& sh = p.s;
  const int unit = blockIdx.x, stream = blockIdx.y, real = p.first_stream + stream, b = real / sh.n_kv_heads, h = real % sh.n_kv_heads;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t row0 = static_cast<size_t>(stream) * p.stream_rows + static_cast<size_t>(unit) * kBlock;
  const int len = lens.len[N == 1 ? 0 : b];
  pdl_wait();
  const TableEntry* table = p.table + static_cast<size_t>(real) * p.table_stride;
  const int32_t* order = p.order + static_cast<size_t>(stream) * p.n_closed;
  const int blocks = p.blocks[stream];
  bool low = false, term = false;
  if (unit < blocks) {
    const TableEntry e = table[order[unit]];
    const uint8_t* slot = p.arena + static_cast<size_t>(e.off256) * 256;
    term = e.resmask != 0;
    if (tid < kBlock) p.bias[row0 + tid] = e.resmask >> tid & 1u ? -INFINITY : 0.f;
    if (e.level == 16) {
      low = true;                          // (below 2^-14 a bf16 value has bits that fp16 has not)
      for (int i = tid; i < kBlock * 16; i += kEThreads) {
        const int r = i >> 4, c = (i & 15) * 8;
        const uint4 k = *reinterpret_cast<const uint4*>(slot + r * kRowBytes + c * 2), v = *reinterpret_cast<const uint4*>(slot + (kBlock + r) * kRowBytes + c * 2);
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
      const int bits = static_cast<int>(e.level), tile = warp & 3, half = tile >> 1, r = lane >> 2, c4 = lane & 3;
      const uint8_t* raw = slot + half * half_bytes(bits);
      const bool is_v = warp >= 4;
      const uint8_t* codes = raw + (is_v ? off_vc(bits, tile & 1) : off_kc(bits, tile & 1));
      const uint32_t mask = (1u << bits) - 1u;
#pragma unroll 1
      for (int s = 0; s < 8; ++s) {
        float sc[4], ze[4];                // keys: of channels c0, c0 + 1, c0 + 8, c0 + 9; values: of tokens t0, t0 + 1, t0 + 8, t0 + 9
        if (!is_v) {
          const uint32_t* kp = reinterpret_cast<const uint32_t*>(raw + ((s >> 1) * 4 + c4) * 32);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t z = kp[j * 2 + (s & 1)], q = kp[4 + j * 2 + (s & 1)];
            ze[2 * j] = half_of(z, 0);
            ze[2 * j + 1] = half_of(z, 1);
            sc[2 * j] = half_of(q, 0);
            sc[2 * j + 1] = half_of(q, 1);
          }
        } else {
          const uint8_t* vp = raw + off_vp(bits, tile & 1);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t q = *reinterpret_cast<const uint32_t*>(vp + c4 * 32 + (s >> 1) * 8 + j * 4);
            const uint32_t z = *reinterpret_cast<const uint32_t*>(vp + 128 + ((s >> 1) * 4 + c4) * 8 + j * 4);
            ze[2 * j] = half_of(z, 0);
            ze[2 * j + 1] = half_of(z, 1);
            sc[2 * j] = half_of(q, 0);
            sc[2 * j + 1] = half_of(q, 1);
          }
        }
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          int byte, bit;
          code_pos(bits, is_v, lane, s, a, 0, &byte, &bit);
          const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + byte) >> bit;
          const int j = (a >> 1) * 2;
          const float f0 = fmaf(static_cast<float>(w & mask), sc[j], ze[j]), f1 = fmaf(static_cast<float>(w >> 16 & mask), sc[j + 1], ze[j + 1]);
          const uint32_t x = sat_pair(f0, f1);
          if (!is_v) {
            const int at = staged(tile * 16 + r + 8 * (a & 1), 16 * s + 8 * (a >> 1) + 2 * c4);
            const float2 g = halves(x);
            *reinterpret_cast<uint32_t*>(&hi[at]) = x;
            *reinterpret_cast<uint32_t*>(&lo[at]) = sat_pair(f0 - g.x, f1 - g.y);
          } else {
            const int tok = tile * 16 + 8 * (a >> 1) + 2 * c4, ch = 16 * s + r + 8 * (a & 1);
            va[staged(tok, ch)] = static_cast<uint16_t>(x);
            va[staged(tok + 1, ch)] = static_cast<uint16_t>(x >> 16);
          }
        }
      }
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
          const TableEntry e = table[order[p.n_closed - 1 - j]];
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
  if (tid == 0 && (term || low)) atomicOr(p.flags + static_cast<size_t>(stream) * p.steps + (unit >> 1), (term ? kHasTerm : 0) | (low ? kHasLow : 0));
}

// Queries as fp16 rows, and the steps' flags cleared.
__global__ void __launch_bounds__(256) queries_kernel(const __grid_constant__ DenseParams p, size_t pieces, size_t first, int n_flags) {
  const size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i < static_cast<size_t>(n_flags)) p.flags[i] = 0;
  if (i >= pieces) return;
  const uint4 x = reinterpret_cast<const uint4*>(p.q)[first + i];
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t a[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = sat_pair(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
  reinterpret_cast<uint4*>(p.q16)[i] = make_uint4(a[0], a[1], a[2], a[3]);
}

// ---- attention -----------------------------------------------------------------------------------
constexpr int kDRows = 128;                // rows of a tile's half, keys of a step
constexpr int kDPanel = kDRows * 128;
constexpr int kDTile = 2 * kDPanel;
constexpr int kDThreads = 384;             // softmax of the halves (four warps each), loads, products, -, -
constexpr int kDStages = 5;
constexpr int kDOffStage = 2 * kDTile, kDOffBar = kDOffStage + kDStages * kDTile, kDSmem = kDOffBar + 256 + 1024;
constexpr int kDLaunchRegs = 168, kDSoftRegs = 216, kDOtherRegs = 72;
static_assert(2 * kDSoftRegs + kDOtherRegs <= 3 * kDLaunchRegs, "a split draws on the launch's registers");
constexpr float kDSlack = 8.f;

struct DenseMaps {
  CUtensorMap q, k_hi, k_lo, v;
};

template <int N>
__global__ void __launch_bounds__(kDThreads, 1)
    dense_kernel(const __grid_constant__ DenseParams p, const __grid_constant__ ChunkCuts cuts, const __grid_constant__ ChunkLens<N> lens,
                 const __grid_constant__ DenseMaps maps) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base = smem_raw + (smem - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bars = smem + kDOffBar;
  const uint32_t bar_q = bars, bar_qfree = bars + 8, bar_s = bars + 16, bar_p = bars + 32, bar_o = bars + 48, bar_drain_mma = bars + 64, bar_pa = bars + 72;
  const uint32_t bar_full = bars + 88, bar_empty = bar_full + 8 * kDStages;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(base + kDOffBar + 240);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base + kDOffBar + 244);
  static_assert(88 + 16 * kDStages <= 240, "room for the barriers");
  const ChunkShape& sh = p.s;

  if (threadIdx.x == 0) {
    bar_init(bar_q, 1);
    bar_init(bar_qfree, 1);
    for (int t = 0; t < 2; ++t) {
      bar_init(bar_s + 8 * t, 1);
      bar_init(bar_pa + 8 * t, 4);
      bar_init(bar_p + 8 * t, 4);
      bar_init(bar_o + 8 * t, 1);
    }
    bar_init(bar_drain_mma, 1);
    for (int i = 0; i < kDStages; ++i) {
      bar_init(bar_full + 8 * i, 1);
      bar_init(bar_empty + 8 * i, 1);
    }
    *abort = 0;
    bar_init_fence();
  }
  if (warp == 9) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *tmem_slot;
  pdl_launch();
  pdl_wait();

  const int cta = blockIdx.x, t0 = cuts.tile[cta], i0 = cuts.item[cta], t1 = cuts.tile[cta + 1], i1 = cuts.item[cta + 1];
  const int half_tokens = sh.tile_tokens / 2;
  // The CTA's parts of tiles, in order; everyone walks them.
  struct Part {
    int tile, rt, stream, b, h, len, items, begin, end, tok0;
    bool two;                              // the tile's second half has rows
  };
  auto next_part = [&](int from, Part& x) {
    for (x.tile = from; x.tile <= t1 && x.tile < sh.batch * sh.n_kv_heads * sh.row_tiles; ++x.tile) {
      x.rt = x.tile % sh.row_tiles;
      x.stream = x.tile / sh.row_tiles;
      x.b = x.stream / sh.n_kv_heads;
      x.h = x.stream % sh.n_kv_heads;
      x.len = lens.len[N == 1 ? 0 : p.first_stream / sh.n_kv_heads + x.b];
      x.items = chunk_items(sh, x.len, x.rt);
      x.begin = x.tile == t0 ? i0 : 0;
      x.end = x.tile == t1 ? i1 : x.items;
      x.tok0 = x.rt * sh.tile_tokens;
      x.two = x.tok0 + half_tokens < x.len;
      if (x.begin < x.end) return true;
    }
    return false;
  };
  Part x;

  if (warp < 8) {
    more_regs<kDSoftRegs>();
    const int t = warp >> 2;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp & 3) << 21);
    const uint32_t s_tm = lanes + t * kDRows, o_tm = lanes + 256 + t * kDRows;
    const int r = (warp & 3) * 32 + lane, tok_in = r / sh.group;
    const float c = p.scale_log2;
    int steps = 0, parts = 0, slot = cuts.slot[cta];
    bool ok = true;
    for (int from = t0; ok && next_part(from, x); from = x.tile + 1) {
      const int to = chunk_needs_slot(x.begin, x.end, x.items) ? slot++ : -1;
      if (t && !x.two) continue;
      const int tok = x.tok0 + t * half_tokens + tok_in;
      const bool real = tok_in < half_tokens && tok < x.len;
      const int first_tok = x.tok0 + t * half_tokens + (warp & 3) * 32 / sh.group;
      const int32_t* const flags = p.flags + static_cast<size_t>(x.stream) * p.steps;
      float m = -INFINITY, l = 0.f;
      for (int j = x.begin; j < x.end; ++j) {
        const int flag = __ldg(flags + j);
        if (!(ok = bar_wait(bar_s + 8 * t, steps & 1, abort))) break;
        ++steps;
        tmem_after();
        uint32_t v[kDRows];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld32(s_tm + 32 * i, v + 32 * i);
        tmem_wait_ld();
        if (flag & kHasTerm) {
          const float4* add = reinterpret_cast<const float4*>(p.bias + static_cast<size_t>(x.stream) * p.stream_rows + static_cast<size_t>(j) * kDRows);
#pragma unroll
          for (int i = 0; i < kDRows / 4; ++i) {
            const float4 a = __ldg(add + i);
            v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + a.x);
            v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + a.y);
            v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + a.z);
            v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + a.w);
          }
        }
        const int limit = tok - (j - p.cache_steps) * kDRows;              // last key of the step that the row sees
        if (j >= p.cache_steps && (j - p.cache_steps + 1) * kDRows - 1 > first_tok) {
#pragma unroll
          for (int i = 0; i < kDRows; ++i)
            if (i > limit) v[i] = 0xff800000u;
        }
        float mx[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) mx[k] = max3(__uint_as_float(v[3 * k]), __uint_as_float(v[3 * k + 1]), __uint_as_float(v[3 * k + 2]));
#pragma unroll
        for (int i = 12; i < kDRows; i += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + 2 * k < kDRows) mx[k] = max3(mx[k], __uint_as_float(v[i + 2 * k]), __uint_as_float(v[i + 2 * k + 1]));
        const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
        const bool first = m == -INFINITY;
        const bool move = first ? top > -INFINITY : (top - m) * c > kDSlack;
        if (__any_sync(0xffffffffu, move && !first)) {
          const float f = move && !first ? ex2((m - top) * c) : 1.f;
          l *= f;
          const uint64_t ff = f2_pack(f, f);
          for (int i = 0; i < 4; ++i) {
            uint32_t o[32];
            tmem_ld32(o_tm + 32 * i, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              float a, b;
              f2_unpack(f2_mul(f2_pack(__uint_as_float(o[k]), __uint_as_float(o[k + 1])), ff), a, b);
              o[k] = __float_as_uint(a);
              o[k + 1] = __float_as_uint(b);
            }
            tmem_st32(o_tm + 32 * i, o);
          }
        }
        if (move) m = top;
        const float at = m == -INFINITY ? 0.f : -m * c;
        const uint64_t cc = f2_pack(c, c), mm = f2_pack(at, at);
        uint64_t sum0 = 0, sum1 = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t pk[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float a, b;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(v[32 * i + 2 * k]), __uint_as_float(v[32 * i + 2 * k + 1])), cc, mm), a, b);
            a = ex2(a);
            b = ex2(b);
            if (k & 1) sum1 = f2_add(sum1, f2_pack(a, b));
            else sum0 = f2_add(sum0, f2_pack(a, b));
            pk[k] = f16_pair(a, b);
          }
          tmem_st16(s_tm + 16 * i, pk);
          if (i == 2) {                      // three quarters of the weights: their product starts while the rest are made
            tmem_wait_st();
            tmem_before();
            __syncwarp();
            if (lane == 0) bar_arrive(bar_pa + 8 * t);
          }
        }
        float a, b;
        f2_unpack(f2_add(sum0, sum1), a, b);
        l += a + b;
        tmem_wait_st();
        tmem_before();
        __syncwarp();
        if (lane == 0) bar_arrive(bar_p + 8 * t);
      }
      ok = ok && bar_wait(bar_o + 8 * t, parts & 1, abort);
      if (!ok) break;
      ++parts;
      tmem_after();
      const int hq = x.h * sh.group + r % sh.group;
      const size_t at = (static_cast<size_t>(p.first_stream / sh.n_kv_heads + x.b) * sh.n_new + tok) * (sh.n_kv_heads * sh.group) + hq;
      const float inv = to < 0 ? 1.f / l : 1.f;
      for (int i = 0; i < 4; ++i) {
        uint32_t o[32];
        tmem_ld32(o_tm + 32 * i, o);
        tmem_wait_ld();
        if (real) {
          if (to < 0) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint4 w;
              w.x = bf16_pair(__uint_as_float(o[8 * k]) * inv, __uint_as_float(o[8 * k + 1]) * inv);
              w.y = bf16_pair(__uint_as_float(o[8 * k + 2]) * inv, __uint_as_float(o[8 * k + 3]) * inv);
              w.z = bf16_pair(__uint_as_float(o[8 * k + 4]) * inv, __uint_as_float(o[8 * k + 5]) * inv);
              w.w = bf16_pair(__uint_as_float(o[8 * k + 6]) * inv, __uint_as_float(o[8 * k + 7]) * inv);
              *reinterpret_cast<uint4*>(p.out + at * kD + 32 * i + 8 * k) = w;
            }
          } else {
            uint4* dst = reinterpret_cast<uint4*>(p.part_o + (static_cast<size_t>(to) * sh.tile_rows + t * half_tokens * sh.group + r) * kD + 32 * i);
#pragma unroll
            for (int k = 0; k < 8; ++k) dst[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
          }
        }
      }
      if (real) {
        if (to < 0) {
          if (p.lse) p.lse[at] = (m * c + lg2(l)) * kLn2;
        } else {
          p.part_ml[static_cast<size_t>(to) * sh.tile_rows + t * half_tokens * sh.group + r] = make_float2(m * c, l);
        }
      }
      tmem_before();
    }
    if (!ok && lane == 0) atomicOr(p.status, kStatusInternal);
  } else {
    fewer_regs<kDOtherRegs>();
    if (warp == 8) {
      // ---- loads: per step K_hi, K_lo where keys are pairs, V ----
      if (elect()) {
        int i = 0, parts = 0;                // stages filled
        bool ok = true;
        const uint32_t q_bytes = 2u * half_tokens * sh.group * 128u;
        auto load = [&](const CUtensorMap* map, int row) {
          const int slot = i % kDStages, turn = i / kDStages;
          if (turn > 0 && !bar_wait(bar_empty + 8 * slot, (turn - 1) & 1, abort)) return false;
          bar_expect(bar_full + 8 * slot, kDTile);
          tma_load_3d(smem + kDOffStage + slot * kDTile, map, 0, row, 0, bar_full + 8 * slot);
          ++i;
          return true;
        };
        for (int from = t0; ok && next_part(from, x); from = x.tile + 1) {
          if (parts > 0 && !(ok = bar_wait(bar_qfree, (parts - 1) & 1, abort))) break;
          ++parts;
          bar_expect(bar_q, x.two ? 2 * q_bytes : q_bytes);
          for (int t = 0; t < (x.two ? 2 : 1); ++t)
            for (int k = 0; k < 2; ++k)
              tma_load_3d(smem + t * kDTile + k * kDPanel, &maps.q, 64 * k, x.h * sh.group, x.b * sh.n_new + x.tok0 + t * half_tokens, bar_q);
          const int32_t* const flags = p.flags + static_cast<size_t>(x.stream) * p.steps;
          int flag = __ldg(flags + x.begin);
          for (int j = x.begin; ok && j < x.end; ++j) {
            const int now = flag, row = x.stream * p.stream_rows + j * kDRows;
            if (j + 1 < x.end) flag = __ldg(flags + j + 1);
            ok = load(&maps.k_hi, row) && (!(now & kHasLow) || load(&maps.k_lo, row)) && load(&maps.v, row);
          }
        }
        if (*abort) {
          if (parts) bar_drain(bar_q, (parts - 1) & 1);
          for (int k = max(0, i - kDStages); k < i; ++k) bar_drain(bar_full + 8 * (k % kDStages), (k / kDStages) & 1);
        }
      }
    } else if (warp == 9) {
      // ---- products ----
      if (elect()) {
        constexpr uint32_t id_qk = instr_desc(false, false, kDRows, kDRows), id_pv = instr_desc(false, true, kDRows, kD);
        bool ok = true;
        int at = 0, parts = 0, weights[2] = {0, 0};      // the next stage; parts begun; steps whose weights were waited for
        auto wait_stage = [&](int i) { return bar_wait(bar_full + 8 * (i % kDStages), (i / kDStages) & 1, abort); };
        auto free_stage = [&](int i) { mma_commit(bar_empty + 8 * (i % kDStages)); };
        auto qk = [&](int t, int i, bool add) {
          const uint64_t a = smem_desc(smem + t * kDTile, 16), b = smem_desc(smem + kDOffStage + (i % kDStages) * kDTile, 16);
          for (int k = 0; k < kD / 16; ++k) {
            const uint32_t off = ((k >> 2) * kDPanel + (k & 3) * 32) >> 4;
            mma_ss(tmem + t * kDRows, a + off, b + off, id_qk, add || k > 0);
          }
        };
        auto pv = [&](int t, int i, bool first, int from, int to) {
          const uint64_t b = smem_desc(smem + kDOffStage + (i % kDStages) * kDTile, kDPanel);
          for (int k = from; k < to; ++k) mma_ts(tmem + 256 + t * kDRows, tmem + t * kDRows + 8 * k, b + ((k * 16 * 128) >> 4), id_pv, !first || k > 0);
        };
        for (int from = t0; ok && next_part(from, x); from = x.tile + 1) {
          const int halves = x.two ? 2 : 1;
          const int32_t* const flags = p.flags + static_cast<size_t>(x.stream) * p.steps;
          int flag = __ldg(flags + x.begin);
          ok = bar_wait(bar_q, parts & 1, abort);
          ++parts;
          // keys of the step at stage `at`: both halves' S (the second half's later, where `late` says so)
          bool low = flag & kHasLow;
          ok = ok && wait_stage(at) && (!low || wait_stage(at + 1));
          if (!ok) break;
          tmem_after();
          for (int t = 0; t < halves; ++t) {
            qk(t, at, false);
            if (low) qk(t, at + 1, true);
            mma_commit(bar_s + 8 * t);
          }
          free_stage(at);
          if (low) free_stage(at + 1);
          if (x.begin + 1 == x.end) mma_commit(bar_qfree);
          at += low ? 2 : 1;
          for (int j = x.begin; ok && j < x.end; ++j) {
            const int v = at, k = at + 1;
            const bool more = j + 1 < x.end;
            if (more) flag = __ldg(flags + j + 1);
            low = more && (flag & kHasLow);
            ok = wait_stage(v) && (!more || wait_stage(k)) && (!low || wait_stage(k + 1));
            for (int t = 0; t < halves && ok; ++t) {
              ok = bar_wait(bar_pa + 8 * t, weights[t] & 1, abort);
              if (!ok) break;
              tmem_after();
              pv(t, v, j == x.begin, 0, 6);
              ok = bar_wait(bar_p + 8 * t, weights[t] & 1, abort);
              if (!ok) break;
              ++weights[t];
              tmem_after();
              pv(t, v, j == x.begin, 6, 8);
              if (!more) {
                mma_commit(bar_o + 8 * t);
              } else {
                qk(t, k, false);
                if (low) qk(t, k + 1, true);
                mma_commit(bar_s + 8 * t);
              }
            }
            if (!ok) break;
            free_stage(v);
            if (more) {
              free_stage(k);
              if (low) free_stage(k + 1);
              if (j + 2 == x.end) mma_commit(bar_qfree);
            }
            at = more ? k + (low ? 2 : 1) : v + 1;
          }
        }
        if (!ok) {
          mma_commit(bar_drain_mma);
          bar_drain(bar_drain_mma, 0);
        }
      }
    }
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
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
  d.order = take(streams * std::max(n_closed, 1) * sizeof(int32_t));
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
  const int slots = chunk_plan(s, len ? len + first : nullptr, 6, &cuts, &merge);
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
  p.order = reinterpret_cast<int32_t*>(ws + at.order);
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
  DenseMaps maps;
  const uint64_t rd[3] = {64, rows, 2}, rs[2] = {kRowBytes, 128}, qd[3] = {kD, heads, static_cast<uint64_t>(seqs) * s.n_new}, qs[2] = {kRowBytes, heads * kRowBytes};
  const uint32_t rb[3] = {64, kDRows, 2}, qb[3] = {64, static_cast<uint32_t>(s.group), static_cast<uint32_t>(s.tile_tokens / 2)};
  if (!make_map(&maps.q, p.q16, 3, qd, qs, qb) || !make_map(&maps.k_hi, p.k_hi, 3, rd, rs, rb) || !make_map(&maps.k_lo, p.k_lo, 3, rd, rs, rb) ||
      !make_map(&maps.v, p.v, 3, rd, rs, rb))
    return cudaErrorInvalidValue;
  const size_t per_seq = static_cast<size_t>(s.n_new) * heads * kD / 8, pieces = per_seq * seqs;
  const size_t threads = std::max(pieces, static_cast<size_t>(streams) * p.steps);
  queries_kernel<<<static_cast<unsigned>((threads + 255) / 256), 256, 0, st>>>(p, pieces, per_seq * first, streams * p.steps);
  order_kernel<<<streams, 256, 0, st>>>(p);
  const dim3 grid(2 * p.steps, streams);
  const bool one = !len || call.shape.batch == 1;
  ChunkLens<1> l1{{len ? len[0] : s.n_new}};
  ChunkLens<kChunkMaxBatch> ln;
  if (!one) std::copy(len, len + call.shape.batch, ln.len);
  if (one) expand_kernel<1><<<grid, kEThreads, 0, st>>>(p, l1);
  else expand_kernel<kChunkMaxBatch><<<grid, kEThreads, 0, st>>>(p, ln);
  static std::atomic<uint64_t> done1{0}, done2{0};
  cudaError_t e = one ? raise_smem_limit(dense_kernel<1>, kDSmem, done1) : raise_smem_limit(dense_kernel<kChunkMaxBatch>, kDSmem, done2);
  if (e != cudaSuccess) return e;
  if (one) dense_kernel<1><<<cuts.n, kDThreads, kDSmem, st>>>(p, cuts, l1, maps);
  else dense_kernel<kChunkMaxBatch><<<cuts.n, kDThreads, kDSmem, st>>>(p, cuts, ln, maps);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  // the merge sees the group as a call of its own
  ChunkCall part = call;
  part.shape = s;
  part.workspace = p.part_o;
  part.out = call.out + static_cast<size_t>(first) * s.n_new * heads * kD;
  part.lse = call.lse ? call.lse + static_cast<size_t>(first) * s.n_new * heads : nullptr;
  return launch_chunk_merge(part, merge, len ? len + first : nullptr, st);
}

}  // namespace gkv
