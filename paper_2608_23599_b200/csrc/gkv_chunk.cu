// Attention of a chunk of new tokens over the graded cache and, causally, over one another (the multi-query form of the read path
// of Sec. 3.7): verification of drafted tokens, and the next turn of a conversation.
//
// Mathematics.  As gkv_decode.cu reads a block, with 128 rows instead of eight columns per stream: a step is 64 keys,
//   S = Q K~^T, P = exp2(c S - c m), O += P V~
// on the fifth-generation tensor cores, Q and P in tensor memory, keys and values in shared memory.  With this many rows a
// block is worth dequantising once: a quantised value becomes fp16(code s + z), one rounding of 2^-12 (Q and P enter those steps as
// fp16, Q exactly); exact rows, the partial block, residual rows, centroids and the chunk's own rows stay the bf16 that they are (P then is
// bf16, a rounding of 2^-9 of a weight).  A centroid is one key whose logit gets log2 of the tokens that it stands for; up to 64 of them share a step.
//
// Work split.  gkv_chunk.h cuts all tiles' items into equal ranges, one per CTA; a block's place in its stream's walk is a golden-ratio
// permutation of its age, so that a range holds every rung in its proportion.  Inside a CTA (one per SM: all 512 columns of tensor memory)
//   warps 0-3, 4-7  softmax of even and odd steps: each four warps have an accumulator O of their own, merged where a tile ends
//   warps 8-19      fill the key and value slots, four warps per step, three steps at once: a warp each for half of the keys or values
//   warps 20, 23    issue O += P V and S = Q K^T.  S, keys, values and raw blocks lie in rings of three steps: a step's logits are there
//                   when the four warps that take it have finished the step before.  (One thread for both was busy for 1150 cycles a step:
//                   code that runs once a step comes from the instruction caches line by line.)
//   warp 21         walks the items, publishes what each step is, and asks L2 for its bytes ahead of use
//   warp 22         issues the bulk copies of quantised blocks as they are stored
// Keys lie as [token][channel] rows.  Codes are stored in the order of warp-level fragments (gkv_layout.cuh), in which a lane's pairs run along
// channels for keys and along tokens for values: dequantised values are written as [channel][token] rows, value rows of the other kinds as
// [token][channel]; the product reads either (one bit of its descriptor).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "gkv_chunk.h"
#include "gkv_internal.h"
#include "gkv_tc.cuh"

namespace gkv {
namespace {

using namespace tc;

constexpr int kCThreads = 768;
constexpr int kCRing = 3;                  // steps that are filled at once, slots of keys and of values, buffers of S, raw blocks
constexpr int kCEntries = 12;              // steps published ahead; a multiple of the ring and of the softmax halves
constexpr int kCHalf = 16384;              // 64 keys or values
constexpr int kCPanel = 8192;              // 64 channels of 64 rows
constexpr int kCRawBytes = 18432;          // a block as it is stored, up to 8 bits
constexpr int kCLaunchRegs = 80, kCSoftRegs = 120, kCFillRegs = 64, kCOtherRegs = 48;
static_assert(2 * kCSoftRegs + kCRing * kCFillRegs + kCOtherRegs <= 6 * kCLaunchRegs, "a split draws on the launch's registers");
// tensor memory: the fp16 query, an accumulator per softmax half, the buffers of S
constexpr uint32_t kCColQh = 0, kCColO = 64, kCColS = 320;
static_assert(kCEntries % kCRing == 0 && kCEntries % 2 == 0 && kCColS + 64 * kCRing <= 512, "");

enum : int32_t { kNone = 0, kCodes = 1, kRowsOf = 2, kCentroids = 3, kTileEnd = 4, kEnd = 5 };

struct alignas(16) Entry {
  uint64_t hide;             // keys that are served from elsewhere
  uint64_t k, v;             // row kinds: address of the first row
  uint32_t stride;           // bytes from row to row
  int32_t kind, level;
  int32_t rows;              // keys of the step
  int32_t causal;            // the chunk token of its first key, -1 = all rows see all of it
  int32_t tile, slot;        // kTileEnd: where the result goes (slot -1: the output)
  uint32_t block;            // kCodes: offset of the slot in 256-byte units
  uint32_t off[kChunkKeys];  // kCentroids: offsets
  alignas(16) float bias[kChunkKeys];      // and what their logits get
};

constexpr int kCOffK = 0, kCOffV = kCRing * kCHalf, kCOffQ = 2 * kCRing * kCHalf;      // (the bf16 query: two panels of 128 rows)
constexpr int kCOffRaw = kCOffQ + kChunkRows * kD * 2;
constexpr int kCOffEntry = kCOffRaw + kCRing * kCRawBytes;
constexpr int kCOffMl = kCOffEntry + kCEntries * static_cast<int>(sizeof(Entry));
constexpr int kCOffPend = kCOffMl + 2 * kChunkRows * 8;
constexpr int kCOffBar = kCOffPend + 96 * 8;
constexpr int kCBars = 6 * kCRing + 2 * kCEntries + 5;
constexpr int kCSmem = kCOffBar + kCBars * 8 + 16 + 1024;
static_assert(kCSmem <= 232448, "shared memory of a CTA");

struct ChunkParams {
  const uint8_t* arena;
  const TableEntry* table;
  const uint32_t* res_off256;
  const int32_t* res_count;
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  uint16_t* out;
  float* lse;
  float* part_o;             // [slot][128][128]
  float2* part_ml;           // [slot][128]: reference (log2), sum
  uint32_t* status;
  int32_t table_stride, walk;      // walk: the permutation's step, coprime to the closed blocks
  int32_t n_closed, n_tail, res_groups;
  float scale_log2;
  ChunkShape s;
};

// ---- dequantisation ------------------------------------------------------------------------------
__device__ __forceinline__ uint4 ldg128(const uint8_t* p) {
  uint4 v;
  asm("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ __half2 h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ uint32_t u32(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
// 1 / 2^p and -1024 / 2^p as fp16 pairs
__device__ __forceinline__ constexpr uint32_t inv_pow2(int p) { return static_cast<uint32_t>(0x3c00 - (p << 10)) * 0x10001u; }
__device__ __forceinline__ constexpr uint32_t neg_bias(int p) { return static_cast<uint32_t>(0xe400 - (p << 10)) * 0x10001u; }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(v) : "r"(a));
  return v;
}
// A lane's words of the MMA indices s = 2 j, 2 j + 1 of a 16-token tile: word 2 i + (a >> 1) at 8 bits, i at 4 bits, 0 (both) at 2 bits
template <int BITS>
__device__ __forceinline__ void lane_words(uint32_t tile, int j, int lane, uint32_t (&w)[4]) {
  if constexpr (BITS == 8) {
    const uint4 v = lds128(tile + (j * 32 + lane) * 16);
    w[0] = v.x;
    w[1] = v.y;
    w[2] = v.z;
    w[3] = v.w;
  } else if constexpr (BITS == 4) {
    const uint2 v = lds64(tile + ((j >> 1) * 32 + lane) * 16 + (j & 1) * 8);
    w[0] = v.x;
    w[1] = v.y;
  } else {
    w[0] = lds32(tile + lane * 16 + j * 4);
  }
}
// The codes of fields (i = s & 1, register a) as an fp16 pair, exactly: or-ed into the mantissa of 1024 they are 1024 + code 2^p.
template <int BITS, bool V>
__device__ __forceinline__ __half2 code_pair(const uint32_t (&w)[4], int i, int a) {
  const int f = V ? ((a >> 1) | ((a & 1) << 1)) : a;
  const int at = BITS == 8 ? 2 * i + (a >> 1) : BITS == 4 ? i : 0;
  int p = BITS == 8 ? 8 * (a & 1) : BITS == 4 ? 4 * f : 4 * i + 2 * (f & 1) + 8 * (f >> 1);
  uint32_t word = w[at];
  if (p + BITS > 10) {
    word >>= 8;
    p -= 8;
  }
  const uint32_t mask = ((1u << BITS) - 1u) << p;
  const uint32_t x = (word & (mask * 0x10001u)) | 0x64006400u;
  return __hfma2(h2(x), h2(inv_pow2(p)), h2(neg_bias(p)));
}
__device__ __forceinline__ uint32_t pick(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Half of a block's keys (32 tokens) from the raw block in shared memory: rows of the key tile.  (The loop over the channels is not
// unrolled further: three bit widths of keys and values unrolled whole are 60 KB of instructions, and a mixed context then waits for instructions
// ten times as long as it issues them.)
template <int BITS>
__device__ __forceinline__ void write_keys(uint32_t raw, int half, uint32_t dst, int lane) {
  const int r = lane >> 2, c4 = lane & 3;
  const uint32_t row = dst + (half * 32 + r) * 128 + 4 * c4;
#pragma unroll 1
  for (int j = 0; j < 4; ++j) {          // a slab of 32 channels: s = 2 j, 2 j + 1
    const uint4 z = lds128(raw + (j * 4 + c4) * 32), sc = lds128(raw + (j * 4 + c4) * 32 + 16);
    const uint32_t panel = row + (j >> 1) * kCPanel;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t w[4];
      lane_words<BITS>(raw + off_kc(BITS, t), j, lane, w);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t at = panel + ((((j & 1) * 4 + 2 * i) ^ r) << 4);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int f = (a >> 1) * 2 + i;
          const __half2 v = __hfma2(code_pair<BITS, false>(w, i, a), h2(pick(sc, f)), h2(pick(z, f)));
          sts32((a >> 1 ? at ^ 16u : at) + (16 * t + 8 * (a & 1)) * 128, u32(v));
        }
      }
    }
  }
}
// Half of a block's values (32 tokens): columns of the value tile, whose rows are channels.
template <int BITS>
__device__ __forceinline__ void write_values(uint32_t raw, int half, uint32_t dst, int lane) {
  const int r = lane >> 2, c4 = lane & 3;
  const uint32_t row = dst + r * 128 + 4 * c4;
#pragma unroll 1
  for (int j = 0; j < 4; ++j) {          // a group of 32 channels
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint2 sc = lds64(raw + off_vp(BITS, t) + c4 * 32 + j * 8), z = lds64(raw + off_vp(BITS, t) + 128 + (j * 4 + c4) * 8);
      uint32_t w[4];
      lane_words<BITS>(raw + off_vc(BITS, t), j, lane, w);
      const uint32_t at = row + (((4 * half + 2 * t) ^ r) << 4) + j * 32 * 128;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const __half2 v = __hfma2(code_pair<BITS, true>(w, i, a), h2(a >> 1 ? sc.y : sc.x), h2(a >> 1 ? z.y : z.x));
          sts32((a >> 1 ? at ^ 16u : at) + (16 * i + 8 * (a & 1)) * 128, u32(v));
        }
    }
  }
}
// A quarter of a step's rows, bf16, as they are; rows that are not there are zeros.
__device__ __forceinline__ void fetch_rows(uint4 (&x)[8], const uint8_t* base, uint32_t stride, const uint32_t* off, int rows, int row0, int lane) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = row0 + 2 * i + (lane >> 4);
    x[i] = make_uint4(0, 0, 0, 0);
    if (row < rows) x[i] = ldg128(base + (off ? static_cast<size_t>(off[row]) * 256 : static_cast<size_t>(row) * stride) + (lane & 15) * 16);
  }
}
__device__ __forceinline__ void write_rows(const uint4 (&x)[8], int row0, uint32_t dst, int lane) {
  const int c = lane & 15;
  const uint32_t panel = dst + (c >> 3) * kCPanel;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = row0 + 2 * i + (lane >> 4);
    sts128(panel + row * 128 + (((c & 7) ^ (row & 7)) << 4), x[i]);
  }
}

__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(p), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
                 "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// ---- the kernel ----------------------------------------------------------------------------------
template <int COPIES, int N>
__global__ void __launch_bounds__(kCThreads, 1)
    chunk_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ ChunkCuts cuts, const __grid_constant__ ChunkLens<N> lens) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base = smem_raw + (smem - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  Entry* const entries = reinterpret_cast<Entry*>(base + kCOffEntry);
  const uint32_t bars = smem + kCOffBar;
  // of a step, by place in the ring: keys are there; S is done (and its keys are free); weights and values are there; O is done (and its
  // values and S are free); the raw block is there, is free
  const uint32_t bar_k = bars, bar_s = bar_k + 8 * kCRing, bar_pv = bar_s + 8 * kCRing, bar_o = bar_pv + 8 * kCRing, bar_raw = bar_o + 8 * kCRing;
  const uint32_t bar_rawfree = bar_raw + 8 * kCRing, bar_put = bar_rawfree + 8 * kCRing, bar_got = bar_put + 8 * kCEntries;
  // of a tile: its queries are there; the halves' sums are there; all products are done
  const uint32_t bar_q = bar_got + 8 * kCEntries, bar_ml = bar_q + 8, bar_tile = bar_ml + 8, bar_drain = bar_tile + 8;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(base + kCOffBar + kCBars * 8);
  volatile uint32_t* const tmem_slot = abort + 1;
  const ChunkShape& sh = p.s;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kCRing; ++i) {
      bar_init(bar_k + 8 * i, 2);
      bar_init(bar_s + 8 * i, 1);
      bar_init(bar_pv + 8 * i, 6);         // four warps of the softmax, two that fill the values
      bar_init(bar_o + 8 * i, 1);
      bar_init(bar_raw + 8 * i, 1);
      bar_init(bar_rawfree + 8 * i, 4);
    }
    for (int i = 0; i < kCEntries; ++i) {
      bar_init(bar_put + 8 * i, 1);
      bar_init(bar_got + 8 * i, 10);       // four warps that fill, four of the softmax, the O products', the raw blocks'
    }
    bar_init(bar_q, 8);
    bar_init(bar_ml, 8);
    bar_init(bar_tile, 1);
    for (int i = 0; i < 2; ++i) bar_init(bar_drain + 8 * i, 1);
    *abort = 0;
    bar_init_fence();
  }
  pdl_launch();
  if (warp == 20) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *tmem_slot;
  // Step k's turn of its place in a ring of n barriers.  (The softmax halves wait for every other step only; no turn that they leave out is
  // unfinished then, and none that they wait for is overtaken: S(k) and S(k + 3) are issued in order, the second after O(k).)
  auto wait_turn = [&](uint32_t bar, int n, int k) { return bar_wait(bar + 8 * (k % n), (k / n) & 1, abort); };
  auto wait_put = [&](int k) { return wait_turn(bar_put, kCEntries, k); };

  if (warp < 8) {
    // ---- softmax ----
    more_regs<kCSoftRegs>();
    constexpr int kCols = kChunkKeys / COPIES;           // columns of a step that a row of this copy takes
    const int w = warp >> 2, quarter = warp & 3;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quarter) << 21);
    const int vrow = quarter * 32 + lane;                // row of the tile, copies included
    const int row = vrow % (kChunkRows / COPIES), copy = vrow / (kChunkRows / COPIES);
    const int tok_in = row / sh.group, head_in = row % sh.group;
    const float c = p.scale_log2;
    float2* const ml = reinterpret_cast<float2*>(base + kCOffMl);
    int seg = 0;
    bool ok = true, fresh = true, real = false, any_real = false;
    int tok = 0;
    float m = -INFINITY, l = 0.f;
    for (int k = w; ok; k += 2) {
      if (!(ok = wait_put(k))) break;
      const Entry& e = entries[k % kCEntries];
      const int kind = e.kind;
      if (kind == kEnd) {
        if (lane == 0) bar_arrive(bar_pv + 8 * (k % kCRing));
        break;
      }
      if (fresh) {                                       // a tile begins: its rows go to shared memory as bf16 (warps 0-3), to tensor memory as fp16
        const int tile = e.tile, rt = tile % sh.row_tiles, stream = tile / sh.row_tiles, b = stream / sh.n_kv_heads, h = stream % sh.n_kv_heads;
        tok = rt * sh.tile_tokens + tok_in;
        real = tok_in < sh.tile_tokens && tok < lens.len[N == 1 ? 0 : b];
        any_real = __any_sync(0xffffffffu, real);
        const uint4* src = reinterpret_cast<const uint4*>(
            p.q + ((static_cast<size_t>(b) * sh.n_new + tok) * (sh.n_kv_heads * sh.group) + h * sh.group + head_in) * kD);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint4 v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = real ? src[4 * i + j] : make_uint4(0, 0, 0, 0);
          if (w == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              sts128(smem + kCOffQ + (i >> 1) * (kChunkRows * 128) + vrow * 128 + ((((i & 1) * 4 + j) ^ (vrow & 7)) << 4), v[j]);
          } else {
            uint32_t x[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const uint32_t u = pick(v[j >> 2], j & 3);
              x[j] = f16_pair(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
            }
            tmem_st16(lanes + kCColQh + 16 * i, x);
          }
        }
        fence_async();
        tmem_wait_st();
        tmem_before();
        __syncwarp();
        if (lane == 0) bar_arrive(bar_q);
        fresh = false;
        m = -INFINITY;
        l = 0.f;
      }
      if (!(ok = wait_turn(bar_s, kCRing, k))) break;
      const uint32_t s_tm = lanes + kCColS + 64 * (k % kCRing);
      if (kind == kTileEnd) {
        __syncwarp();
        if (lane == 0) bar_arrive(bar_pv + 8 * (k % kCRing));      // (no weights)
        // ---- the two halves of the tile's steps are merged; these warps take channels 64 w .. + 63 ----
        ok = bar_wait(bar_q, seg & 1, abort);            // (everyone is past the previous tile's merge)
        ml[w * kChunkRows + vrow] = make_float2(m * c, l);
        __syncwarp();
        if (lane == 0) bar_arrive(bar_ml);
        ok = ok && bar_wait(bar_ml, seg & 1, abort) && bar_wait(bar_tile, seg & 1, abort);
        if (!ok) break;
        tmem_after();
        const float2 a = ml[vrow], b2 = ml[kChunkRows + vrow];
        const float top = fmaxf(a.y > 0.f ? a.x : -INFINITY, b2.y > 0.f ? b2.x : -INFINITY);
        const float fa = a.y > 0.f ? ex2(a.x - top) : 0.f, fb = b2.y > 0.f ? ex2(b2.x - top) : 0.f;
        const float sum = fa * a.y + fb * b2.y;
        const int tile = e.tile, slot = e.slot, stream = tile / sh.row_tiles, b = stream / sh.n_kv_heads, h = stream % sh.n_kv_heads;
        const size_t at = (static_cast<size_t>(b) * sh.n_new + tok) * (sh.n_kv_heads * sh.group) + h * sh.group + head_in;
        const float inv = slot < 0 ? 1.f / sum : 1.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t x[16], y[16];
          tmem_ld16(lanes + kCColO + 64 * w + 16 * i, x);
          tmem_ld16(lanes + kCColO + 128 + 64 * w + 16 * i, y);
          tmem_wait_ld();
          float o[16];
#pragma unroll
          for (int j = 0; j < 16; ++j)                   // (an O that no step wrote is not looked at)
            o[j] = ((a.y > 0.f ? fa * __uint_as_float(x[j]) : 0.f) + (b2.y > 0.f ? fb * __uint_as_float(y[j]) : 0.f)) * inv;
          if (real) {
            if (slot < 0) {
              uint4* dst = reinterpret_cast<uint4*>(p.out + at * kD + 64 * w + 16 * i);
              dst[0] = make_uint4(bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3]), bf16_pair(o[4], o[5]), bf16_pair(o[6], o[7]));
              dst[1] = make_uint4(bf16_pair(o[8], o[9]), bf16_pair(o[10], o[11]), bf16_pair(o[12], o[13]), bf16_pair(o[14], o[15]));
            } else {
              float4* dst = reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(slot) * kChunkRows + vrow) * kD + 64 * w + 16 * i);
#pragma unroll
              for (int j = 0; j < 4; ++j) dst[j] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
            }
          }
        }
        if (real && w == 0) {
          if (slot < 0) {
            if (p.lse) p.lse[at] = (top + lg2(sum)) * kLn2;
          } else {
            p.part_ml[static_cast<size_t>(slot) * kChunkRows + vrow] = make_float2(top, sum);
          }
        }
        tmem_before();
        fresh = true;
        ++seg;
      } else {
        if (kind != kNone && any_real) {
          tmem_after();
          uint32_t x[kCols];
          if constexpr (COPIES == 4) {
            tmem_ld16(s_tm + kCols * copy, x);
          } else {
#pragma unroll
            for (int i = 0; i < kCols / 32; ++i) tmem_ld32(s_tm + kCols * copy + 32 * i, x + 32 * i);
          }
          tmem_wait_ld();
          if (kind == kCentroids) {
#pragma unroll
            for (int i = 0; i < kCols; i += 4) {
              const float4 add = *reinterpret_cast<const float4*>(e.bias + kCols * copy + i);
              x[i] = __float_as_uint(__uint_as_float(x[i]) + add.x);
              x[i + 1] = __float_as_uint(__uint_as_float(x[i + 1]) + add.y);
              x[i + 2] = __float_as_uint(__uint_as_float(x[i + 2]) + add.z);
              x[i + 3] = __float_as_uint(__uint_as_float(x[i + 3]) + add.w);
            }
          }
          uint64_t see = (e.rows >= kChunkKeys ? ~uint64_t{0} : (uint64_t{1} << e.rows) - 1) & ~e.hide;
          if (e.causal >= 0) {
            const int d = tok - e.causal;                // keys 0 .. d
            see &= d < 0 ? 0 : d >= kChunkKeys - 1 ? ~uint64_t{0} : (uint64_t{2} << d) - 1;
          }
          see >>= kCols * copy;
          constexpr uint64_t kAll = kCols == 64 ? ~uint64_t{0} : (uint64_t{1} << (kCols & 63)) - 1;
          if (__any_sync(0xffffffffu, (see & kAll) != kAll)) {
            const uint32_t lo = static_cast<uint32_t>(see), hi = static_cast<uint32_t>(see >> 32);
#pragma unroll
            for (int i = 0; i < kCols; ++i)
              if (!((i < 32 ? lo : hi) >> (i & 31) & 1u)) x[i] = 0xff800000u;
          }
          float mx[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) mx[j] = __uint_as_float(x[j]);
#pragma unroll
          for (int i = 4; i + 8 <= kCols; i += 8)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx[j] = max3(mx[j], __uint_as_float(x[i + 2 * j]), __uint_as_float(x[i + 2 * j + 1]));
#pragma unroll
          for (int j = 0; j < 4; ++j) mx[j] = fmaxf(mx[j], __uint_as_float(x[kCols - 4 + j]));
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          const bool first = m == -INFINITY;
          const bool move = first ? top > -INFINITY : (top - m) * c > 8.f;
          if (__any_sync(0xffffffffu, move && !first)) {
            // (S of this step was issued ahead of the O of the four warps' step before, which has to be complete now)
            if (!(ok = wait_turn(bar_o, kCRing, k - 2))) break;
            tmem_after();
            const float f = move && !first ? ex2((m - top) * c) : 1.f;
            l *= f;
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
              uint32_t o[16];
              tmem_ld16(lanes + kCColO + 128 * w + 16 * i, o);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              tmem_st16(lanes + kCColO + 128 * w + 16 * i, o);
            }
          }
          if (move) m = top;
          const float at = m == -INFINITY ? 0.f : -m * c;
          const uint64_t cc = f2_pack(c, c), mm = f2_pack(at, at);
          uint64_t sum0 = 0, sum1 = 0;
          uint32_t pk[kCols / 2];
#pragma unroll
          for (int i = 0; i < kCols / 2; ++i) {
            float a, b;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), cc, mm), a, b);
            a = ex2(a);
            b = ex2(b);
            if (i & 1) sum1 = f2_add(sum1, f2_pack(a, b));
            else sum0 = f2_add(sum0, f2_pack(a, b));
            x[2 * i] = __float_as_uint(a);
            x[2 * i + 1] = __float_as_uint(b);
          }
          if (kind == kCodes) {
#pragma unroll
            for (int i = 0; i < kCols / 2; ++i) pk[i] = f16_pair(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1]));
          } else {
#pragma unroll
            for (int i = 0; i < kCols / 2; ++i) pk[i] = bf16_pair(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1]));
          }
          float a, b;
          f2_unpack(f2_add(sum0, sum1), a, b);
          l += a + b;
          // the weights lie over the logits, 32 columns of pairs; another copy's keys have weight zero here
          if constexpr (COPIES == 1) {
            tmem_st32(s_tm, pk);
          } else if constexpr (COPIES == 2) {
            uint32_t z[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0;
            tmem_st16(s_tm + 16 * copy, pk);
            tmem_st16(s_tm + 16 * (copy ^ 1), z);
          } else {
            uint32_t z[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = 0;
            tmem_st8(s_tm + 8 * copy, pk);
#pragma unroll
            for (int i = 1; i < 4; ++i) tmem_st8(s_tm + 8 * (copy ^ i), z);
          }
          tmem_wait_st();
          tmem_before();
        }
        __syncwarp();
        if (lane == 0) bar_arrive(bar_pv + 8 * (k % kCRing));
      }
      __syncwarp();
      if (lane == 0) bar_arrive(bar_got + 8 * (k % kCEntries));
    }
  } else if (warp < 8 + 4 * kCRing) {
    // ---- key and value slots ----
    fewer_regs<kCFillRegs>();
    const int half = warp & 1, is_v = (warp >> 1) & 1, place = (warp - 8) >> 2;
    const uint32_t bar_full = (is_v ? bar_pv : bar_k) + 8 * place, bar_free = is_v ? bar_o : bar_s;
    const uint32_t dst = smem + (is_v ? kCOffV : kCOffK) + place * kCHalf;
    for (int k = place;; k += kCRing) {
      if (!wait_put(k)) break;
      const Entry& e = entries[k % kCEntries];
      const int kind = e.kind;
      auto slot_free = [&]() { return k < kCRing || wait_turn(bar_free, kCRing, k - kCRing); };
      if (kind == kEnd) {
        if (slot_free() && lane == 0) bar_arrive(bar_full);
        break;
      }
      bool ok;
      if (kind == kRowsOf || kind == kCentroids) {
        const bool gather = kind == kCentroids;
        const uint8_t* src = gather ? p.arena + is_v * kRowBytes : reinterpret_cast<const uint8_t*>(is_v ? e.v : e.k);
        uint4 x[8];
        fetch_rows(x, src, e.stride, gather ? e.off : nullptr, e.rows, half * 32, lane);
        if ((ok = slot_free())) {
          write_rows(x, half * 32, dst, lane);
          fetch_rows(x, src, e.stride, gather ? e.off : nullptr, e.rows, half * 32 + 16, lane);
          write_rows(x, half * 32 + 16, dst, lane);
        }
        ok = ok && wait_turn(bar_raw, kCRing, k);
      } else {
        ok = wait_turn(bar_raw, kCRing, k) && slot_free();
        if (ok && kind == kCodes) {
          const int level = e.level;
          const uint32_t src = smem + kCOffRaw + place * kCRawBytes + half * half_bytes(level);
          if (is_v) {
            if (level == 4) write_values<4>(src, half, dst, lane);
            else if (level == 8) write_values<8>(src, half, dst, lane);
            else write_values<2>(src, half, dst, lane);
          } else {
            if (level == 4) write_keys<4>(src, half, dst, lane);
            else if (level == 8) write_keys<8>(src, half, dst, lane);
            else write_keys<2>(src, half, dst, lane);
          }
        }
      }
      if (!ok) break;
      fence_async();
      __syncwarp();
      if (lane == 0) {
        bar_arrive(bar_full);
        bar_arrive(bar_rawfree + 8 * place);
        bar_arrive(bar_got + 8 * (k % kCEntries));
      }
    }
  } else {
    fewer_regs<kCOtherRegs>();
    if (warp == 23) {
      // ---- S = Q K^T ----  (whole warps walk, one lane issues: addresses stay in uniform registers)
      constexpr uint32_t id_h = instr_desc(false, false, kChunkRows, kChunkKeys), id_b = instr_desc(true, false, kChunkRows, kChunkKeys);
      const bool leader = elect();
      const uint64_t q = smem_desc(smem + kCOffQ, 16);
      int seg = 0;
      bool ok = true, begin = true;
      for (int k = 0;; ++k) {
        const int place = k % kCRing;
        ok = wait_turn(bar_k, kCRing, k) && (k < kCRing || wait_turn(bar_o, kCRing, k - kCRing));
        if (!ok) break;
        const int kind = entries[k % kCEntries].kind;
        if (kind == kEnd) break;
        if (begin) {
          if (!(ok = bar_wait(bar_q, seg & 1, abort))) break;
          ++seg;
        }
        begin = kind == kTileEnd && (k & 1);
        tmem_after();
        if (leader) {
          const uint64_t b = smem_desc(smem + kCOffK + place * kCHalf, 16);
          const uint32_t d = tmem + kCColS + 64 * place;
          if (kind == kCodes) {
#pragma unroll
            for (int i = 0; i < kD / 16; ++i) mma_ts(d, tmem + kCColQh + 8 * i, b + (((i >> 2) * kCPanel + (i & 3) * 32) >> 4), id_h, i > 0);
          } else if (kind == kRowsOf || kind == kCentroids) {
#pragma unroll
            for (int i = 0; i < kD / 16; ++i)
              mma_ss(d, q + (((i >> 2) * (kChunkRows * 128) + (i & 3) * 32) >> 4), b + (((i >> 2) * kCPanel + (i & 3) * 32) >> 4), id_b, i > 0);
          }
          mma_commit(bar_s + 8 * place);
        }
        __syncwarp();
      }
      if (leader) {
        mma_commit(bar_drain);                           // products in flight end before tensor memory is given back
        tc::bar_drain(bar_drain, 0);
        if (!ok) atomicOr(p.status, kStatusInternal);
      }
    } else if (warp == 20) {
      // ---- O += P V ----
      constexpr uint32_t id_h = instr_desc(false, false, kChunkRows, kD), id_b = instr_desc(true, true, kChunkRows, kD);
      const bool leader = elect();
      bool ok = true, some[2] = {false, false};          // the halves' O hold something
      for (int k = 0;; ++k) {
        const int place = k % kCRing;
        if (!(ok = wait_turn(bar_pv, kCRing, k))) break;
        const int kind = entries[k % kCEntries].kind;
        if (kind == kEnd) break;
        tmem_after();
        const bool real = kind == kCodes || kind == kRowsOf || kind == kCentroids;
        if (leader) {
          const uint32_t v = smem + kCOffV + place * kCHalf, d = tmem + kCColO + 128 * (k & 1), a = tmem + kCColS + 64 * place;
          if (kind == kCodes) {
            const uint64_t b = smem_desc(v, 16);
#pragma unroll
            for (int i = 0; i < kChunkKeys / 16; ++i) mma_ts(d, a + 8 * i, b + i * (32 >> 4), id_h, i > 0 || some[k & 1]);
          } else if (real) {
            const uint64_t b = smem_desc(v, kCPanel);
#pragma unroll
            for (int i = 0; i < kChunkKeys / 16; ++i) mma_ts(d, a + 8 * i, b + i * (16 * 128 >> 4), id_b, i > 0 || some[k & 1]);
          } else if (kind == kTileEnd && (k & 1)) {
            mma_commit(bar_tile);
          }
          mma_commit(bar_o + 8 * place);
          bar_arrive(bar_got + 8 * (k % kCEntries));
        }
        __syncwarp();
        if (real) some[k & 1] = true;
        if (kind == kTileEnd) some[k & 1] = false;
      }
      if (leader) {
        mma_commit(bar_drain + 8);
        tc::bar_drain(bar_drain + 8, 0);
        if (!ok) atomicOr(p.status, kStatusInternal);
      }
    } else if (warp == 22) {
      // ---- raw blocks, a few steps ahead of the stages ----
      if (elect()) {
        int k = 0;
        for (;; ++k) {
          if (!wait_put(k)) break;
          const Entry& e = entries[k % kCEntries];
          if (e.kind == kEnd) break;
          const int slot = k % kCRing;
          if (k >= kCRing && !wait_turn(bar_rawfree, kCRing, k - kCRing)) break;
          if (e.kind == kCodes) {
            const uint32_t bytes = slot_bytes(e.level);
            bar_expect(bar_raw + 8 * slot, bytes);
            bulk_load(smem + kCOffRaw + slot * kCRawBytes, p.arena + static_cast<size_t>(e.block) * 256, bytes, bar_raw + 8 * slot);
          } else {
            bar_arrive(bar_raw + 8 * slot);
          }
          bar_arrive(bar_got + 8 * (k % kCEntries));
        }
        if (*abort)                              // what is on its way arrives before the CTA leaves
          for (int i = max(0, k - kCRing); i < k; ++i) tc::bar_drain(bar_raw + 8 * (i % kCRing), (i / kCRing) & 1);
      }
    } else if (warp == 21) {
      // ---- walk ----
      uint32_t* const pend_off = reinterpret_cast<uint32_t*>(base + kCOffPend);
      float* const pend_bias = reinterpret_cast<float*>(pend_off + 96);
      int k = 0, pend = 0;
      bool ok = true;
      // the next step's entry, once its place is free; everyone's lane sees the same arguments
      auto put = [&](const Entry& head, bool centroids) {
        if (!ok) return;
        if (k >= kCEntries) ok = wait_turn(bar_got, kCEntries, k - kCEntries);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        Entry& e = entries[k % kCEntries];
        if (lane == 0) {
          e.hide = head.hide;
          e.k = head.k;
          e.v = head.v;
          e.stride = head.stride;
          e.kind = head.kind;
          e.level = head.level;
          e.rows = head.rows;
          e.causal = head.causal;
          e.tile = head.tile;
          e.slot = head.slot;
          e.block = head.block;
        }
        if (centroids)
          for (int i = lane; i < kChunkKeys; i += 32) {
            e.off[i] = pend_off[i];
            e.bias[i] = i < head.rows ? pend_bias[i] : 0.f;
          }
        __syncwarp();
        if (lane == 0) bar_arrive(bar_put + 8 * (k % kCEntries));
        ++k;
      };
      const int cta = blockIdx.x;
      const int t0 = cuts.tile[cta], i0 = cuts.item[cta], t1 = cuts.tile[cta + 1], i1 = cuts.item[cta + 1];
      int slot = cuts.slot[cta];
      const float to_raw = 1.f / p.scale_log2;
      for (int tile = t0; ok && tile <= t1; ++tile) {
        if (tile >= sh.batch * sh.n_kv_heads * sh.row_tiles) break;
        const int rt = tile % sh.row_tiles, stream = tile / sh.row_tiles, b = stream / sh.n_kv_heads, h = stream % sh.n_kv_heads;
        const int len = lens.len[N == 1 ? 0 : b];
        const int items = chunk_items(sh, len, rt);
        const int begin = tile == t0 ? i0 : 0, end = tile == t1 ? i1 : items;
        if (begin >= end) continue;
        Entry head{};
        head.tile = tile;
        head.causal = -1;
        const TableEntry* table = p.table + static_cast<size_t>(stream) * p.table_stride;
        const int last_block = min(end, p.n_closed);
        auto centroid_step = [&]() {
          Entry x = head;
          x.kind = kCentroids;
          x.rows = min(pend, kChunkKeys);
          put(x, true);
          pend -= x.rows;
          __syncwarp();
          if (lane < pend) {                             // what is left moves down (fewer than 32)
            pend_off[lane] = pend_off[kChunkKeys + lane];
            pend_bias[lane] = pend_bias[kChunkKeys + lane];
          }
          __syncwarp();
        };
        for (int i = begin; ok && i < last_block; i += 32) {
          TableEntry t{};
          if (i + lane < last_block) t = table[static_cast<uint64_t>(i + lane) * static_cast<uint32_t>(p.walk) % static_cast<uint32_t>(p.n_closed)];
          const bool cent = t.level == 1;
          const uint32_t cents = __ballot_sync(0xffffffffu, cent);
          if (cent) {
            const int at = pend + __popc(cents & ((1u << lane) - 1u));
            const int n = kBlock - __popcll(t.resmask);
            pend_off[at] = t.off256;
            pend_bias[at] = n > 0 ? lg2(static_cast<float>(n)) * to_raw : -INFINITY;
            prefetch_l2(p.arena + static_cast<size_t>(t.off256) * 256, 2 * kRowBytes);
          }
          __syncwarp();
          pend += __popc(cents);
          if (pend >= kChunkKeys) centroid_step();
          const int n = min(32, last_block - i);
          for (int j = 0; ok && j < n; ++j) {
            if (cents >> j & 1u) continue;
            Entry x = head;
            const uint32_t off = __shfl_sync(0xffffffffu, t.off256, j);
            const int level = static_cast<int>(__shfl_sync(0xffffffffu, t.level, j));
            x.hide = __shfl_sync(0xffffffffu, t.resmask, j);
            x.rows = kBlock;
            const uint8_t* at = p.arena + static_cast<size_t>(off) * 256;
            if (level == 16) {
              x.kind = kRowsOf;
              x.k = reinterpret_cast<uint64_t>(at);
              x.v = reinterpret_cast<uint64_t>(at + kBlock * kRowBytes);
              x.stride = kRowBytes;
            } else {
              x.kind = kCodes;
              x.level = level;
              x.block = off;
            }
            if (lane == 0) prefetch_l2(at, slot_bytes(level));
            put(x, false);
          }
        }
        if (ok && pend > 0) centroid_step();
        int i = max(begin, p.n_closed);
        if (ok && p.n_tail > 0 && i == p.n_closed && i < end) {
          Entry x = head;
          const uint8_t* at = p.arena + static_cast<size_t>(table[p.n_closed].off256) * 256;
          x.kind = kRowsOf;
          x.rows = p.n_tail;
          x.k = reinterpret_cast<uint64_t>(at);
          x.v = reinterpret_cast<uint64_t>(at + kBlock * kRowBytes);
          x.stride = kRowBytes;
          put(x, false);
          ++i;
        }
        const int res0 = p.n_closed + (p.n_tail > 0), new0 = res0 + p.res_groups;
        for (; ok && i < min(end, new0); ++i) {
          const int row0 = (i - res0) * kChunkKeys, n = min(kChunkKeys, p.res_count[stream] - row0);
          if (n <= 0) continue;
          Entry x = head;
          const uint8_t* at = p.arena + static_cast<size_t>(p.res_off256[stream]) * 256 + static_cast<size_t>(row0) * 2 * kRowBytes;
          x.kind = kRowsOf;
          x.rows = n;
          x.k = reinterpret_cast<uint64_t>(at);
          x.v = reinterpret_cast<uint64_t>(at + kRowBytes);
          x.stride = 2 * kRowBytes;
          put(x, false);
        }
        for (; ok && i < end; ++i) {
          const int tok0 = (i - new0) * kChunkKeys;
          Entry x = head;
          const size_t at = (static_cast<size_t>(b) * sh.n_new + tok0) * sh.n_kv_heads + h;
          x.kind = kRowsOf;
          x.rows = min(kChunkKeys, len - tok0);
          x.causal = tok0;
          x.k = reinterpret_cast<uint64_t>(p.k_new + at * kD);
          x.v = reinterpret_cast<uint64_t>(p.v_new + at * kD);
          x.stride = static_cast<uint32_t>(sh.n_kv_heads) * kRowBytes;
          put(x, false);
        }
        if (k & 1) put(head, false);                     // even and odd steps come in pairs
        Entry x = head;
        x.kind = kTileEnd;
        x.slot = chunk_needs_slot(sh, begin, end, items) ? slot++ : -1;
        put(x, false);
        put(x, false);
      }
      Entry x{};
      x.kind = kEnd;
      for (int i = 0; i < kCRing; ++i) put(x, false);      // everyone who walks the steps meets one
    }
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  if (warp == 20) tmem_dealloc(tmem, 512);
}

// Merges the slots of tiles that were cut (or hold copies of their rows): a warp per row, four channels per lane, slots in order.
template <int N>
__global__ void __launch_bounds__(128) chunk_merge_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ ChunkMerge merge,
                                                          const __grid_constant__ ChunkLens<N> lens) {
  const ChunkShape& sh = p.s;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31, rows = kChunkRows / sh.copies;
  const int tile = merge.tile[blockIdx.y], first = merge.slot[blockIdx.y], n = (merge.slot[blockIdx.y + 1] - first) * sh.copies;
  const int rt = tile % sh.row_tiles, stream = tile / sh.row_tiles, b = stream / sh.n_kv_heads, h = stream % sh.n_kv_heads;
  const int tok = rt * sh.tile_tokens + row / sh.group;
  if (row >= sh.tile_tokens * sh.group || tok >= lens.len[N == 1 ? 0 : b]) return;
  // part i: copy i % copies of slot first + i / copies
  auto index = [&](int i) { return static_cast<size_t>(first + i / sh.copies) * kChunkRows + (i % sh.copies) * rows + row; };
  pdl_wait();
  float top = -INFINITY;
  for (int i = lane; i < n; i += 32) {
    const float2 v = p.part_ml[index(i)];
    if (v.y > 0.f) top = fmaxf(top, v.x);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  float sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0; i0 < n; i0 += 8) {      // (eight parts' loads in flight)
    float2 v[8];
    float4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const size_t at = index(min(i0 + k, n - 1));
      v[k] = p.part_ml[at];
      x[k] = reinterpret_cast<const float4*>(p.part_o + at * kD)[lane];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (i0 + k >= n || !(v[k].y > 0.f)) continue;
      const float f = ex2(v[k].x - top);
      sum += f * v[k].y;
      o.x += f * x[k].x;
      o.y += f * x[k].y;
      o.z += f * x[k].z;
      o.w += f * x[k].w;
    }
  }
  const float inv = 1.f / sum;
  const size_t at = (static_cast<size_t>(b) * sh.n_new + tok) * (sh.n_kv_heads * sh.group) + h * sh.group + row % sh.group;
  reinterpret_cast<uint2*>(p.out + at * kD)[lane] = make_uint2(bf16_pair(o.x * inv, o.y * inv), bf16_pair(o.z * inv, o.w * inv));
  if (p.lse && lane == 0) p.lse[at] = (top + lg2(sum)) * kLn2;
}

ChunkParams params_of(const ChunkCall& call, int slots) {
  ChunkParams p{};
  p.arena = call.arena;
  p.table = call.table;
  p.res_off256 = call.res_off256;
  p.res_count = call.res_count;
  p.q = call.q;
  p.k_new = call.k_new;
  p.v_new = call.v_new;
  p.out = call.out;
  p.lse = call.lse;
  p.part_o = call.workspace;
  p.part_ml = reinterpret_cast<float2*>(call.workspace + static_cast<size_t>(slots) * kChunkRows * kD);
  p.status = call.status;
  p.table_stride = call.table_stride;
  p.walk = chunk_walk(call.n_closed);
  p.n_closed = call.n_closed;
  p.n_tail = call.n_tail;
  p.res_groups = (call.res_rows + kChunkKeys - 1) / kChunkKeys;
  p.scale_log2 = call.scale * kLog2e;
  p.s = call.shape;
  return p;
}
template <int N>
ChunkLens<N> lens_of(const ChunkCall& call, const int32_t* len) {
  ChunkLens<N> lens;
  for (int b = 0; b < (N == 1 ? 1 : call.shape.batch); ++b) lens.len[b] = len ? len[b] : call.shape.n_new;
  return lens;
}

template <int COPIES, int N>
cudaError_t launch_as(const ChunkParams& p, const ChunkCuts& cuts, const ChunkLens<N>& lens, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = raise_smem_limit(chunk_kernel<COPIES, N>, kCSmem, done);
  if (e != cudaSuccess) return e;
  chunk_kernel<COPIES, N><<<cuts.n, kCThreads, kCSmem, st>>>(p, cuts, lens);
  return cudaGetLastError();
}
template <int N>
cudaError_t launch_lens(const ChunkParams& p, const ChunkCuts& cuts, const ChunkLens<N>& lens, cudaStream_t st) {
  if (p.s.copies == 4) return launch_as<4, N>(p, cuts, lens, st);
  if (p.s.copies == 2) return launch_as<2, N>(p, cuts, lens, st);
  return launch_as<1, N>(p, cuts, lens, st);
}
bool one_len(const ChunkCall& call, const int32_t* len) { return !len || call.shape.batch == 1; }

}  // namespace

// len: HOST [batch], or null where every sequence has n_new rows.
cudaError_t launch_chunk(const ChunkCall& call, const ChunkCuts& cuts, const ChunkMerge& merge, const int32_t* len, cudaStream_t st) {
  if (cuts.n == 0) return cudaSuccess;
  const ChunkParams p = params_of(call, merge.slot[merge.n]);
  const cudaError_t e = one_len(call, len) ? launch_lens<1>(p, cuts, lens_of<1>(call, len), st) : launch_lens<kChunkMaxBatch>(p, cuts, lens_of<kChunkMaxBatch>(call, len), st);
  return e != cudaSuccess ? e : launch_chunk_merge(call, merge, len, st);
}

cudaError_t launch_chunk_merge(const ChunkCall& call, const ChunkMerge& merge, const int32_t* len, cudaStream_t st) {
  if (merge.n == 0) return cudaSuccess;
  const ChunkParams p = params_of(call, merge.slot[merge.n]);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((std::min(p.s.tile_tokens * p.s.group, kChunkRows / p.s.copies) + 3) / 4, merge.n);
  cfg.blockDim = dim3(128);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return one_len(call, len) ? cudaLaunchKernelEx(&cfg, chunk_merge_kernel<1>, p, merge, lens_of<1>(call, len))
                            : cudaLaunchKernelEx(&cfg, chunk_merge_kernel<kChunkMaxBatch>, p, merge, lens_of<kChunkMaxBatch>(call, len));
}

}  // namespace gkv
