// Chunks of few rows (drafted tokens that are verified): every warp reads the stored codes themselves.
//
// Mathematics.  A warp has 16 rows (new token x query head of a KV head) as the A operand of warp-level MMAs (m16n8k16) and the keys of
// its step as columns.  A quantised key is k~[c] = s[c] code + z[c] with one (s, z) per channel and 32 tokens, so
//   q . k~ = (q s) . code + q . z
// exactly as gkv_decode.cu reads it: codes are used as they lie (a code in the mantissa of an fp16 with a zero exponent field is code 2^(p - 24)),
// the scaled query is an fp16 pair hi + lo formed once per half block, and q . z starts the accumulators.  Values the same way with
// the scales in the weights: O += (P s) code, and sum_j p_j z_j in four more accumulators, one per group of 32 channels.  Nothing about the logits is
// rounded to fewer than 22 bits; weights are fp16 (2^-12 of themselves) over codes, bf16 (2^-9) over exact rows, as the bf16 output allows.
//
// What bounds it: at 4 bits a block of 64 tokens is 10 KB, 420 cycles of an SM's share of the copy bandwidth; its products are 212 MMAs per 16 rows,
// 424 cycles of the SM's warp-level tensor pipes.  Tiles of 128 rows on the fifth-generation tensor cores would need the same 512 cycles for
// any number of rows and every value written to shared memory first: with up to 64 rows a kernel of that kind took 1.9 times as long.
//
// Work split.  gkv_chunk.h cuts the streams' items (half blocks: 32 tokens) into equal ranges, one per CTA.  The CTA's warps form teams of
// one warp per 16 rows; a team takes every n-th item of the range and streams it through a ring of its own, filled by its first warp with bulk copies.
// The teams' results are merged in shared memory in team order, the CTAs' by chunk_merge_kernel.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "gkv_chunk.h"
#include "gkv_internal.h"
#include "gkv_tc.cuh"

namespace gkv {
namespace {

using namespace tc;

constexpr int kVWarps = 12;                // 168 registers a thread
constexpr int kVThreads = kVWarps * 32;
constexpr int kVStage = 5120;              // a 4-bit half block, the keys or the values of an 8-bit one, or of 16 exact rows
constexpr int kVPitch = kRowBytes + 16;    // exact rows (conflict-free ldmatrix)
constexpr int kVMeta = 96;                 // a stage's description
constexpr int kVPend = 64;                 // centroids that a team has collected
constexpr int kVMaxRing = 6;
constexpr int kVOPitch = kD + 4;           // floats of a row in the merge
constexpr float kVUp = 1048576.f;          // 2^20: what the value accumulators lack (codes are code 2^(p - 24), weights carry 2^(4 - p))

struct VMeta {
  int32_t kind;              // 0 = no more, 1 = codes, 2 = rows, 3 = centroids
  int32_t level, n;          // rows of a row step
  int32_t causal;            // chunk token of its first key, or -1
  uint32_t hide;             // keys that are served from elsewhere
  int32_t pad[3];
  float bias[16];            // kind 3: what the logits get (in units of q . k)
};
static_assert(sizeof(VMeta) == kVMeta, "");

// shared memory of a CTA
struct VLayout {
  int teams, ring, stages, q, meta, pend, bars, bytes;
};
__host__ __device__ inline VLayout verify_layout(int groups) {
  VLayout l;
  l.teams = kVWarps / groups;
  l.ring = 200000 / (l.teams * kVStage);
  if (l.ring > kVMaxRing) l.ring = kVMaxRing;
  l.stages = 0;
  l.q = l.stages + l.teams * l.ring * kVStage;
  l.meta = l.q + groups * 4096;
  l.pend = l.meta + l.teams * l.ring * kVMeta;
  l.bars = l.pend + l.teams * kVPend * 8;
  l.bytes = l.bars + l.teams * l.ring * 16 + 16;
  // the merge: every warp's rows, their references and sums
  const int merge = kVWarps * 16 * (kVOPitch + 2) * 4;
  if (l.q < merge) l.q = merge, l.meta = l.q + groups * 4096, l.pend = l.meta + l.teams * l.ring * kVMeta, l.bars = l.pend + l.teams * kVPend * 8,
                   l.bytes = l.bars + l.teams * l.ring * 16 + 16;
  return l;
}

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ __half2 h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ uint32_t u32(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ uint32_t pick(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
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
template <bool TRANS>
__device__ __forceinline__ void ldmatrix4(uint32_t (&x)[4], uint32_t addr) {
  if (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr));
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr));
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
// The codes of (i = s & 1, register a) where they lie, as an fp16 pair code 2^(p - 24): p depends on a & 1 only for keys (the 8-token column
// group) and on a >> 1 only for values (the half of the contraction); see code_exp.
template <int BITS, bool V>
__device__ __forceinline__ uint32_t code_bits(const uint32_t (&w)[4], int i, int a) {
  const int x = V ? a & 1 : a >> 1, y = V ? a >> 1 : a & 1;
  if constexpr (BITS == 8) {
    return __byte_perm(w[2 * i + (a >> 1)], 0u, a & 1 ? 0x4341 : 0x4240);
  } else if constexpr (BITS == 4) {
    return (x ? w[i] >> 8 : w[i]) & (y ? 0x00f000f0u : 0x000f000fu);
  } else {
    return (w[0] >> (4 * i + 8 * x)) & (y ? 0x000c000cu : 0x00030003u);
  }
}
__device__ __forceinline__ constexpr int code_exp(int bits, int y) { return y == 0 || bits == 8 ? 0 : bits == 4 ? 4 : 2; }

struct VState {
  float o[16][4], oz[4];     // channels 8 n + 2 c4, + 1 of rows r (0, 1) and r + 8 (2, 3); groups 2 c4, + 1
  float m0, m1, l0, l1;      // references of the two rows (units of q . k), this lane's part of their sums
};

// The reference moves to the maximum (weights stay at most 1: a weight times a value scale of up to 4094 and 2^4 has to fit fp16); x becomes the weights.
template <int NT>
__device__ __forceinline__ void weigh(VState& st, float (&x)[NT][4], float c) {
  float t0 = fmaxf(x[0][0], x[0][1]), t1 = fmaxf(x[0][2], x[0][3]);
#pragma unroll
  for (int n = 1; n < NT; ++n) {
    t0 = max3(t0, x[n][0], x[n][1]);
    t1 = max3(t1, x[n][2], x[n][3]);
  }
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, d));
    t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, d));
  }
  if (__any_sync(0xffffffffu, t0 > st.m0 || t1 > st.m1)) {
    const float n0 = fmaxf(st.m0, t0), n1 = fmaxf(st.m1, t1);
    const float f0 = st.m0 == -INFINITY ? 0.f : ex2((st.m0 - n0) * c), f1 = st.m1 == -INFINITY ? 0.f : ex2((st.m1 - n1) * c);
    st.m0 = n0;
    st.m1 = n1;
    st.l0 *= f0;
    st.l1 *= f1;
#pragma unroll
    for (int n = 0; n < 16; ++n) {
      st.o[n][0] *= f0;
      st.o[n][1] *= f0;
      st.o[n][2] *= f1;
      st.o[n][3] *= f1;
    }
    st.oz[0] *= f0;
    st.oz[1] *= f0;
    st.oz[2] *= f1;
    st.oz[3] *= f1;
  }
  const float a0 = st.m0 == -INFINITY ? 0.f : -st.m0 * c, a1 = st.m1 == -INFINITY ? 0.f : -st.m1 * c;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    x[n][0] = ex2(fmaf(x[n][0], c, a0));
    x[n][1] = ex2(fmaf(x[n][1], c, a0));
    x[n][2] = ex2(fmaf(x[n][2], c, a1));
    x[n][3] = ex2(fmaf(x[n][3], c, a1));
    st.l0 += x[n][0] + x[n][1];
    st.l1 += x[n][2] + x[n][3];
  }
}

// Logits of a half block's 32 tokens: columns 8 n + 2 c4, + 1 of rows r, r + 8.  raw: parameters and codes of the keys; q: the rows' fragments (fp16).
template <int BITS>
__device__ __forceinline__ void code_logits(float (&x)[4][4], uint32_t raw, uint32_t q, int lane) {
  const int c4 = lane & 3;
  float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int n = 0; n < 4; ++n) x[n][0] = x[n][1] = x[n][2] = x[n][3] = 0.f;
#pragma unroll 1
  for (int j = 0; j < 4; ++j) {
    const uint4 zr = lds128(raw + (j * 4 + c4) * 32), sr = lds128(raw + (j * 4 + c4) * 32 + 16);
    uint32_t w[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) lane_words<BITS>(raw + off_kc(BITS, t), j, lane, w[t]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 qv = lds128(q + ((2 * j + i) * 32 + lane) * 16);
      const uint32_t a[4] = {qv.x, qv.y, qv.z, qv.w};
      mma_f16(z, a, pick(zr, i), pick(zr, 2 + i));
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const __half2 s = h2(pick(sr, (k >> 1) * 2 + i)), h = __hmul2(h2(a[k]), s);
        hi[k] = u32(h);
        lo[k] = u32(__hfma2(h2(a[k]), s, __hneg2(h)));
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t b0 = code_bits<BITS, false>(w[t], i, y), b1 = code_bits<BITS, false>(w[t], i, y + 2);
          mma_f16(x[2 * t + y], hi, b0, b1);
          mma_f16(x[2 * t + y], lo, b0, b1);
        }
    }
  }
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const float up = static_cast<float>(1 << (24 - code_exp(BITS, n & 1)));
#pragma unroll
    for (int k = 0; k < 4; ++k) x[n][k] = fmaf(x[n][k], up, z[k]);
  }
}
// O += P V of a half block; `raw`: where its value parameters would lie behind the keys (off_vp, off_vc).
template <int BITS>
__device__ __forceinline__ void code_values(VState& st, const float (&x)[4][4], uint32_t raw, int lane) {
  const int r = lane >> 2, c4 = lane & 3;
  const __half2 up0 = __float2half2_rn(16.f), up1 = __float2half2_rn(static_cast<float>(1 << (4 - code_exp(BITS, 1))));
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint32_t a[4] = {f16_pair(x[2 * t][0], x[2 * t][1]), f16_pair(x[2 * t][2], x[2 * t][3]), f16_pair(x[2 * t + 1][0], x[2 * t + 1][1]),
                           f16_pair(x[2 * t + 1][2], x[2 * t + 1][3])};
    const uint32_t vp = raw + off_vp(BITS, t);
    uint2 z = lds64(vp + 128 + ((r & 3) * 4 + c4) * 8);      // column r: group r
    if (r >= 4) z.x = z.y = 0u;
    mma_f16(st.oz, a, z.x, z.y);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint2 s = lds64(vp + c4 * 32 + j * 8);
      const __half2 s0 = __hmul2(h2(s.x), up0), s1 = __hmul2(h2(s.y), up1);
      const uint32_t ps[4] = {u32(__hmul2(h2(a[0]), s0)), u32(__hmul2(h2(a[1]), s0)), u32(__hmul2(h2(a[2]), s1)), u32(__hmul2(h2(a[3]), s1))};
      uint32_t w[4];
      lane_words<BITS>(raw + off_vc(BITS, t), j, lane, w);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) mma_f16(st.o[4 * j + 2 * i + k], ps, code_bits<BITS, true>(w, i, k), code_bits<BITS, true>(w, i, k + 2));
    }
  }
}

struct VerifyParams {
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
  int32_t table_stride, walk, n_closed, n_tail, res_items, groups;      // groups: of 16 rows
  float scale_log2;
  ChunkShape s;
};

// A team's walk over its items, in the lanes of its first warp.
struct VWalk {
  int it, end, step;         // items
  int base;                  // first item of the window
  uint32_t off, level;       // this lane's entry: item base + lane * step
  uint64_t res;
  int pend;                  // centroids collected
  // the rest of a row item
  uint64_t k, v;
  uint32_t stride, hide;
  int rows, causal;
};

template <int N>
__global__ void __launch_bounds__(kVThreads, 1)
    verify_kernel(const __grid_constant__ VerifyParams p, const __grid_constant__ ChunkCuts cuts, const __grid_constant__ ChunkLens<N> lens) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  const uint32_t smem = smem_u32(smem_raw);
  const VLayout lay = verify_layout(p.groups);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, c4 = lane & 3;
  const int team = warp / p.groups, grp = warp % p.groups;
  const bool in_team = team < lay.teams;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(smem_raw + lay.bars + lay.teams * lay.ring * 16);
  const ChunkShape& sh = p.s;
  const float c = p.scale_log2;
  const uint32_t ring = smem + lay.stages + (in_team ? team : 0) * lay.ring * kVStage;
  const uint32_t bar_full = smem + lay.bars + (in_team ? team : 0) * lay.ring * 16, bar_free = bar_full + 8 * lay.ring;
  VMeta* const meta = reinterpret_cast<VMeta*>(smem_raw + lay.meta) + (in_team ? team : 0) * lay.ring;
  uint32_t* const pend_off = reinterpret_cast<uint32_t*>(smem_raw + lay.pend) + (in_team ? team : 0) * kVPend * 2;
  float* const pend_bias = reinterpret_cast<float*>(pend_off + kVPend);
  if (threadIdx.x == 0) *abort = 0;
  if (in_team && grp == 0 && lane == 0) {
    for (int i = 0; i < lay.ring; ++i) {
      bar_init(bar_full + 8 * i, 1);
      bar_init(bar_free + 8 * i, p.groups);
    }
    bar_init_fence();
  }
  const int cta = blockIdx.x, t0 = cuts.tile[cta], i0 = cuts.item[cta], t1 = cuts.tile[cta + 1], i1 = cuts.item[cta + 1];
  int slot = cuts.slot[cta];
  int put = 0, got = 0;                    // parts of the ring that the team's first warp has filled, that this warp has used
  bool ok = true;

  for (int tile = t0; tile <= t1 && tile < sh.batch * sh.n_kv_heads; ++tile) {
    const int b = tile / sh.n_kv_heads, h = tile % sh.n_kv_heads;
    const int len = lens.len[N == 1 ? 0 : b];
    const int items = chunk_items(sh, len, 0);
    const int begin = tile == t0 ? i0 : 0, end = tile == t1 ? i1 : items;
    if (begin >= end) continue;
    const int rows = len * sh.group;
    __syncthreads();                       // (barriers are initialised; the previous stream's merge has been read)
    // the rows' fragments: lane (r, c4) of MMA index s holds channels 16 s + 2 c4, + 1 of rows r and r + 8, then the channels eight further
    for (int i = threadIdx.x; i < p.groups * 8 * 32; i += kVThreads) {
      const int s = i >> 5 & 7, g16 = i >> 8, ln = i & 31;
      uint32_t x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int row = g16 * 16 + (ln >> 2) + 8 * (k & 1), ch = 16 * s + 2 * (ln & 3) + 8 * (k >> 1);
        uint32_t u = 0;
        if (row < rows)
          u = *reinterpret_cast<const uint32_t*>(
              p.q + ((static_cast<size_t>(b) * sh.n_new + row / sh.group) * (sh.n_kv_heads * sh.group) + h * sh.group + row % sh.group) * kD + ch);
        x[k] = f16_pair(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
      }
      sts128(smem + lay.q + i * 16, make_uint4(x[0], x[1], x[2], x[3]));
    }
    fence_async();                         // (the merge wrote where copies land next)
    __syncthreads();

    VState st;
#pragma unroll
    for (int n = 0; n < 16; ++n) st.o[n][0] = st.o[n][1] = st.o[n][2] = st.o[n][3] = 0.f;
    st.oz[0] = st.oz[1] = st.oz[2] = st.oz[3] = 0.f;
    st.m0 = st.m1 = -INFINITY;
    st.l0 = st.l1 = 0.f;

    if (in_team) {
      const TableEntry* table = p.table + static_cast<size_t>(tile) * p.table_stride;
      const int blocks_end = 2 * p.n_closed, tail_end = blocks_end + (p.n_tail + 31) / 32, res_end = tail_end + p.res_items;
      VWalk wk{};
      wk.it = begin + team;
      wk.end = end;
      wk.step = lay.teams;
      wk.base = -1;
      bool more = true;                    // the walk has not ended

      // Fills a part of the ring; whole first warps.  Row parts: lane i < 16 copies row i (rows that are not there: row 0 again, their keys are masked)
      auto part = [&](const VMeta& m, uint64_t src, uint32_t bytes, uint64_t row, bool by_row) {
        const int at = put % lay.ring;
        if (put >= lay.ring) ok = ok && bar_wait(bar_free + 8 * at, (put / lay.ring - 1) & 1, abort);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        VMeta& e = meta[at];
        if (lane == 0) {
          e.kind = m.kind;
          e.level = m.level;
          e.n = m.n;
          e.causal = m.causal;
          e.hide = m.hide;
        }
        if (m.kind == 3 && lane < 16) e.bias[lane] = m.bias[0];
        __syncwarp();
        const uint32_t dst = ring + at * kVStage, bar = bar_full + 8 * at;
        if (lane == 0) {
          if (bytes) bar_expect(bar, by_row ? 16 * kRowBytes : bytes);
          else bar_arrive(bar);
        }
        __syncwarp();
        if (by_row) {
          if (lane < 16) bulk_load(dst + lane * kVPitch, reinterpret_cast<const void*>(row), kRowBytes, bar);
        } else if (bytes && lane == 0) {
          bulk_load(dst, reinterpret_cast<const void*>(src), bytes, bar);
        }
        ++put;
      };
      // The next step of the walk goes into the ring (one part or two); false at its end.
      auto produce = [&]() {
        VMeta m{};
        m.causal = -1;
        for (;;) {
          if (wk.rows > 0) {               // 16 rows of a row item
            m.kind = 2;
            m.n = min(wk.rows, 16);
            m.hide = wk.hide & 0xffffu;
            m.causal = wk.causal;
            const int i = lane < m.n ? lane : 0;
            part(m, 0, 1, wk.k + static_cast<uint64_t>(i) * wk.stride, true);
            part(m, 0, 1, wk.v + static_cast<uint64_t>(i) * wk.stride, true);
            wk.rows -= m.n;
            wk.hide >>= 16;
            wk.k += static_cast<uint64_t>(16) * wk.stride;
            wk.v += static_cast<uint64_t>(16) * wk.stride;
            if (wk.causal >= 0) wk.causal += 16;
            return;
          }
          if (wk.pend >= 16 || (wk.it >= wk.end && wk.pend > 0)) {
            m.kind = 3;
            m.n = min(wk.pend, 16);
            const int i = lane < m.n ? lane : 0;
            const uint64_t row = reinterpret_cast<uint64_t>(p.arena) + static_cast<uint64_t>(pend_off[i]) * 256;
            m.bias[0] = pend_bias[i];
            part(m, 0, 1, row, true);
            part(m, 0, 1, row + kRowBytes, true);
            __syncwarp();
            uint32_t o = 0;
            float f = 0.f;
            const int left = wk.pend - m.n;      // at most 47
            for (int k = 0; k < left; k += 32) {
              if (k + lane < left) {
                o = pend_off[16 + k + lane];
                f = pend_bias[16 + k + lane];
              }
              __syncwarp();
              if (k + lane < left) {
                pend_off[k + lane] = o;
                pend_bias[k + lane] = f;
              }
              __syncwarp();
            }
            wk.pend = left;
            return;
          }
          if (wk.it >= wk.end) {
            more = false;
            part(m, 0, 0, 0, false);       // "no more"
            return;
          }
          const int it = wk.it;
          if (it < blocks_end) {
            if (wk.base < 0 || it >= wk.base + 32 * wk.step) {
              const int mine = it + lane * wk.step;
              wk.base = it;
              uint4 e = make_uint4(0, 0, 0, 0);
              if (mine < min(wk.end, blocks_end))
                e = *reinterpret_cast<const uint4*>(table + static_cast<uint64_t>(mine >> 1) * static_cast<uint32_t>(p.walk) % static_cast<uint32_t>(p.n_closed));
              wk.off = e.x;
              wk.level = e.y;
              wk.res = static_cast<uint64_t>(e.w) << 32 | e.z;
              const bool cent = wk.level == 1 && !(mine & 1);
              const uint32_t cents = __ballot_sync(0xffffffffu, cent);
              if (cent) {
                const int at = wk.pend + __popc(cents & ((1u << lane) - 1u)), n = kBlock - __popcll(wk.res);
                pend_off[at] = wk.off;
                pend_bias[at] = n > 0 ? lg2(static_cast<float>(n)) / c : -INFINITY;
              }
              __syncwarp();
              wk.pend += __popc(cents);
              if (wk.pend >= 16) continue;
            }
            const int from = (it - wk.base) / wk.step;
            const uint32_t off = __shfl_sync(0xffffffffu, wk.off, from);
            const int level = static_cast<int>(__shfl_sync(0xffffffffu, wk.level, from));
            const uint64_t res = __shfl_sync(0xffffffffu, wk.res, from);
            wk.it += wk.step;
            if (level == 1) continue;
            const int half = it & 1;
            const uint64_t at = reinterpret_cast<uint64_t>(p.arena) + static_cast<uint64_t>(off) * 256;
            const uint32_t hide = static_cast<uint32_t>(half ? res >> 32 : res);
            if (level == 16) {
              wk.rows = 32;
              wk.hide = hide;
              wk.causal = -1;
              wk.stride = kRowBytes;
              wk.k = at + half * 32 * kRowBytes;
              wk.v = wk.k + kBlock * kRowBytes;
              continue;
            }
            m.kind = 1;
            m.level = level;
            m.hide = hide;
            const uint32_t bytes = half_bytes(level);
            if (level == 8) {
              part(m, at + half * bytes, bytes / 2, 0, false);
              part(m, at + half * bytes + bytes / 2, bytes / 2, 0, false);
            } else {
              part(m, at + half * bytes, bytes, 0, false);
            }
            return;
          }
          wk.it += wk.step;
          wk.hide = 0;
          wk.causal = -1;
          if (it < tail_end) {
            const int row0 = (it - blocks_end) * 32;
            wk.rows = min(32, p.n_tail - row0);
            wk.stride = kRowBytes;
            wk.k = reinterpret_cast<uint64_t>(p.arena) + static_cast<uint64_t>(table[p.n_closed].off256) * 256 + row0 * kRowBytes;
            wk.v = wk.k + kBlock * kRowBytes;
          } else if (it < res_end) {
            const int row0 = (it - tail_end) * 32;
            wk.rows = max(0, min(32, p.res_count[tile] - row0));
            wk.stride = 2 * kRowBytes;
            wk.k = reinterpret_cast<uint64_t>(p.arena) + static_cast<uint64_t>(p.res_off256[tile]) * 256 + static_cast<uint64_t>(row0) * 2 * kRowBytes;
            wk.v = wk.k + kRowBytes;
          } else {
            const int tok0 = (it - res_end) * 32;
            const size_t at = (static_cast<size_t>(b) * sh.n_new + tok0) * sh.n_kv_heads + h;
            wk.rows = min(32, len - tok0);
            wk.causal = tok0;
            wk.stride = static_cast<uint32_t>(sh.n_kv_heads) * kRowBytes;
            wk.k = reinterpret_cast<uint64_t>(p.k_new + at * kD);
            wk.v = reinterpret_cast<uint64_t>(p.v_new + at * kD);
          }
        }
      };
      auto wait_part = [&]() { return bar_wait(bar_full + 8 * (got % lay.ring), (got / lay.ring) & 1, abort); };
      auto free_part = [&]() {
        __syncwarp();
        if (lane == 0) bar_arrive(bar_free + 8 * (got % lay.ring));
        ++got;
      };

      const int row0 = grp * 16 + r, tok_a = row0 / sh.group, tok_b = (row0 + 8) / sh.group;      // of the lane's two rows
      const uint32_t q = smem + lay.q + grp * 4096;
      for (;;) {
        // as many steps ahead as the ring holds for certain (a step has one part or two)
        if (grp == 0)
          while (ok && more && put - got + 2 <= lay.ring) produce();
        if (!ok || !(ok = wait_part())) break;
        const VMeta& e = meta[got % lay.ring];
        const int kind = e.kind, level = e.level;
        const uint32_t raw = ring + (got % lay.ring) * kVStage;
        if (kind == 0) {
          free_part();
          break;
        }
        if (kind == 1) {
          float x[4][4];
          if (level == 4) code_logits<4>(x, raw, q, lane);
          else if (level == 8) code_logits<8>(x, raw, q, lane);
          else code_logits<2>(x, raw, q, lane);
          const uint32_t hide = e.hide;
          if (hide) {
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (hide >> (8 * n + 2 * c4 + (k & 1)) & 1u) x[n][k] = -INFINITY;
          }
          weigh<4>(st, x, c);
          if (level == 8) {
            free_part();
            if (!(ok = wait_part())) break;
            code_values<8>(st, x, ring + (got % lay.ring) * kVStage - half_bytes(8) / 2, lane);
          } else if (level == 4) {
            code_values<4>(st, x, raw, lane);
          } else {
            code_values<2>(st, x, raw, lane);
          }
          free_part();
        } else {
          // 16 rows of bf16: keys [token][channel] are B fragments as they are, values with the transposing load
          float x[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
          const uint32_t km = raw + ((lane & 7) + (lane >> 4) * 8) * kVPitch + (lane >> 3 & 1) * 16;
#pragma unroll 2
          for (int s = 0; s < 8; ++s) {
            const uint4 qv = lds128(q + (s * 32 + lane) * 16);
            uint32_t a[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float2 f = __half22float2(h2(pick(qv, k)));      // (the rows are bf16 by origin: exact)
              a[k] = bf16_pair(f.x, f.y);
            }
            uint32_t kb[4];
            ldmatrix4<false>(kb, km + s * 32);
            mma_bf16(x[0], a, kb[0], kb[1]);
            mma_bf16(x[1], a, kb[2], kb[3]);
          }
          const int n = e.n, causal = e.causal;
          const uint32_t hide = e.hide;
          if (kind == 3) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int k = 0; k < 4; ++k) x[t][k] += e.bias[8 * t + 2 * c4 + (k & 1)];
          }
          if (n < 16 || hide || causal >= 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int j = 8 * t + 2 * c4 + (k & 1);
                if (j >= n || (hide >> j & 1u) || (causal >= 0 && causal + j > (k < 2 ? tok_a : tok_b))) x[t][k] = -INFINITY;
              }
          }
          weigh<2>(st, x, c);
          free_part();
          if (!(ok = wait_part())) break;
          const float down = 1.f / kVUp;
          const uint32_t a[4] = {bf16_pair(x[0][0] * down, x[0][1] * down), bf16_pair(x[0][2] * down, x[0][3] * down), bf16_pair(x[1][0] * down, x[1][1] * down),
                                 bf16_pair(x[1][2] * down, x[1][3] * down)};
          const uint32_t vm = ring + (got % lay.ring) * kVStage + (lane & 15) * kVPitch + (lane >> 4) * 16;
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            uint32_t vb[4];
            ldmatrix4<true>(vb, vm + g * 32);
            mma_bf16(st.o[2 * g], a, vb[0], vb[1]);
            mma_bf16(st.o[2 * g + 1], a, vb[2], vb[3]);
          }
          free_part();
        }
      }
      if (!ok && grp == 0) {                 // what is on its way arrives before the memory is used otherwise
        for (int i = max(0, put - lay.ring); i < put; ++i) bar_drain(bar_full + 8 * (i % lay.ring), (i / lay.ring) & 1);
      }
      // the four lanes of a row hold its sum in parts; zero points of group n / 4 come from the lane that has its column
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        st.l0 += __shfl_xor_sync(0xffffffffu, st.l0, d);
        st.l1 += __shfl_xor_sync(0xffffffffu, st.l1, d);
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int from = (lane & ~3) | (g >> 1);
        const float z0 = __shfl_sync(0xffffffffu, st.oz[g & 1], from), z1 = __shfl_sync(0xffffffffu, st.oz[2 + (g & 1)], from);
#pragma unroll
        for (int n = 4 * g; n < 4 * g + 4; ++n) {
          st.o[n][0] = fmaf(st.o[n][0], kVUp, z0);
          st.o[n][1] = fmaf(st.o[n][1], kVUp, z0);
          st.o[n][2] = fmaf(st.o[n][2], kVUp, z1);
          st.o[n][3] = fmaf(st.o[n][3], kVUp, z1);
        }
      }
    }
    // ---- merge of the teams, in shared memory that the rings do not need now ----
    __syncthreads();
    float* const mo = reinterpret_cast<float*>(smem_raw);
    float2* const mml = reinterpret_cast<float2*>(mo + kVWarps * 16 * kVOPitch);
    if (in_team) {
      float* const d0 = mo + (warp * 16 + r) * kVOPitch + 2 * c4;
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        *reinterpret_cast<float2*>(d0 + 8 * n) = make_float2(st.o[n][0], st.o[n][1]);
        *reinterpret_cast<float2*>(d0 + 8 * kVOPitch + 8 * n) = make_float2(st.o[n][2], st.o[n][3]);
      }
      if (c4 == 0) {
        mml[warp * 16 + r] = make_float2(st.m0 * c, st.l0);
        mml[warp * 16 + r + 8] = make_float2(st.m1 * c, st.l1);
      }
    }
    __syncthreads();
    const int to = chunk_needs_slot(sh, begin, end, items) ? slot++ : -1;
    for (int i = warp; i < rows; i += kVWarps) {           // a warp per row, four channels per lane
      const int g16 = i >> 4, in = i & 15;
      float top = -INFINITY;
      for (int t = 0; t < lay.teams; ++t) {
        const float2 v = mml[(t * p.groups + g16) * 16 + in];
        if (v.y > 0.f) top = fmaxf(top, v.x);
      }
      float sum = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int t = 0; t < lay.teams; ++t) {
        const int at = (t * p.groups + g16) * 16 + in;
        const float2 v = mml[at];
        if (!(v.y > 0.f)) continue;
        const float f = ex2(v.x - top);
        const float4 x = *reinterpret_cast<const float4*>(mo + at * kVOPitch + 4 * lane);
        sum += f * v.y;
        o.x += f * x.x;
        o.y += f * x.y;
        o.z += f * x.z;
        o.w += f * x.w;
      }
      if (to >= 0) {
        const size_t at = static_cast<size_t>(to) * kChunkRows + i;
        reinterpret_cast<float4*>(p.part_o + at * kD)[lane] = o;
        if (lane == 0) p.part_ml[at] = make_float2(top, sum);
      } else {
        const size_t at = (static_cast<size_t>(b) * sh.n_new + i / sh.group) * (sh.n_kv_heads * sh.group) + h * sh.group + i % sh.group;
        const float inv = 1.f / sum;
        reinterpret_cast<uint2*>(p.out + at * kD)[lane] = make_uint2(bf16_pair(o.x * inv, o.y * inv), bf16_pair(o.z * inv, o.w * inv));
        if (p.lse && lane == 0) p.lse[at] = (top + lg2(sum)) * kLn2;
      }
    }
    if (!ok) atomicOr(p.status, kStatusInternal);
    if (*abort) break;                       // (set by whoever gave up: everyone has passed the barrier behind its waits)
  }
}

template <int N>
cudaError_t launch_as(const VerifyParams& p, const ChunkCuts& cuts, const ChunkCall& call, const int32_t* len, cudaStream_t st) {
  ChunkLens<N> lens;
  for (int b = 0; b < (N == 1 ? 1 : p.s.batch); ++b) lens.len[b] = len ? len[b] : p.s.n_new;
  static std::atomic<uint64_t> done{0};
  size_t most = 0;
  for (int g = 1; g <= kVerifyRows / 16; ++g) most = std::max(most, static_cast<size_t>(verify_layout(g).bytes));
  const cudaError_t e = raise_smem_limit(verify_kernel<N>, most, done);
  if (e != cudaSuccess) return e;
  verify_kernel<N><<<cuts.n, kVThreads, verify_layout(p.groups).bytes, st>>>(p, cuts, lens);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_verify(const ChunkCall& call, const ChunkCuts& cuts, const ChunkMerge& merge, const int32_t* len, cudaStream_t st) {
  if (cuts.n == 0) return cudaSuccess;
  VerifyParams p{};
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
  p.part_ml = reinterpret_cast<float2*>(call.workspace + static_cast<size_t>(merge.slot[merge.n]) * kChunkRows * kD);
  p.status = call.status;
  p.table_stride = call.table_stride;
  p.walk = chunk_walk(call.n_closed);
  p.n_closed = call.n_closed;
  p.n_tail = call.n_tail;
  p.res_items = (call.res_rows + 31) / 32;
  p.groups = (call.shape.n_new * call.shape.group + 15) / 16;
  p.scale_log2 = call.scale * kLog2e;
  p.s = call.shape;
  const cudaError_t e = len && p.s.batch > 1 ? launch_as<kChunkMaxBatch>(p, cuts, call, len, st) : launch_as<1>(p, cuts, call, len, st);
  return e != cudaSuccess ? e : launch_chunk_merge(call, merge, len, st);
}

}  // namespace gkv
