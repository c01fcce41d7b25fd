// Chunks of few rows (drafted tokens that are verified): every warp reads the stored codes themselves.
//
// Mathematics.  A warp has 16 rows (new token x query head of a KV head) as the A operand of warp-level MMAs (m16n8k16) and the keys of
// its step as columns.  A quantised key is k~[c] = s[c] code + z[c] with one (s, z) per channel and 32 tokens, so
//   q . k~ = (q s) . code + q . z
// exactly as gkv_decode.cu reads it: codes are used as they lie (a code in the mantissa of an fp16 with a zero exponent field is code 2^(p - 24)),
// the scaled query is an fp16 pair hi + lo formed once per half block, and q . z starts the accumulators.  Values the same way with
// the scales in the weights: O += (P s) code, and sum_j p_j z_j in four more accumulators, one per group of 32 channels.  A scaled query is off by 2^-22 of
// itself or 2^-25, a logit by what the tensor cores keep of products with codes (see code_exp): 2^-20 of a large one at 8 bits.  Weights are single numbers, as the bf16 output allows: bf16 (off by 2^-8 at most) over exact rows, relative to the row's reference; fp16
// (2^-11) over codes, relative to the item's own maximum (weigh_codes, code_values), since fp16 has no room for those of a row whose keys lie far apart.
//
// What bounds it: at 4 bits a block of 64 tokens is 10 KB, 420 cycles of an SM's share of the copy bandwidth; its products are 212 MMAs per 16 rows,
// 424 cycles of the SM's warp-level tensor pipes.  Tiles of 128 rows on the fifth-generation tensor cores would need the same 512 cycles for
// any number of rows and every value written to shared memory first: with up to 64 rows a kernel of that kind took 1.9 times as long.
//
// What it measured: 64 streams of 32,757 tokens on mixed rungs, 20 rows, 220 us, 0.23 of the copy bandwidth.  With weights relative to the row's
// reference (199 us) a warp's item of 106 MMAs and 830 other instructions took 6000 cycles, of which 25% were waits of dependent instructions on one another
// with three warps a scheduler, 42% issue slots used, tensor pipes 30%.  More warps have no registers (68 accumulators, 16 of an item and 16 logits each); unrolling the logits' loop by 2 and 4 took 1.06 and 1.10 times as
// long (instruction cache), a rolled value loop the same.
//
// Work split.  gkv_chunk.h cuts the streams' items (half blocks: 32 tokens) into equal ranges, one per CTA, or every stream into the same number.  The CTA's warps form teams of
// one warp per 16 rows; a team takes every n-th item of the range and streams it through a ring of its own.  The rings are filled with bulk copies by
// one warp more, in which a lane walks the items of each team.  (The team's first warp needed 1400 cycles of 6100 per half block for that.)  Exact
// rows come 16 at a time by tensor map, two panels of 64 channels with the 128-byte swizzle: copies row by row took 80 cycles each to issue.
// The teams' results are merged in shared memory in team order, the CTAs' by chunk_merge_kernel, whose launch overlaps.
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

constexpr int kVWarps = kVerifyWarps;      // that compute
constexpr int kVThreads = kVWarps * 32 + 128;
constexpr int kVLaunchRegs = 128, kVWarpRegs = 152, kVFillRegs = 56;
static_assert(kVWarps / 4 * kVWarpRegs + kVFillRegs <= (kVWarps / 4 + 1) * kVLaunchRegs, "a split draws on the launch's registers");
constexpr int kVStage = 5120;              // a 4-bit half block, the keys or the values of an 8-bit one, or of 16 exact rows
constexpr int kVPitch = kRowBytes + 16;    // centroid rows, copied one by one (conflict-free ldmatrix)
constexpr int kVPanel = 16 * 128;          // 64 channels of 16 rows that came by tensor map
constexpr int kVMeta = 80;                 // a stage's description
constexpr int kVPend = 64;                 // centroids that a team has collected
constexpr int kVMaxRing = 6;
constexpr float kVAbove = 4.f;             // log2
constexpr float kVTop = 11.f;              // log2 of an item's heaviest weight over codes: see code_values
constexpr int kVIdle = 1 << 22;            // fruitless looks for room after which the walk gives up
constexpr int kVOPitch = kD + 4;           // floats of a row in the merge

struct alignas(16) VMeta {
  uint32_t what;             // kind (0 = no more, 1 = codes, 2 = rows, 3 = centroids) | level << 8 | rows << 16
  int32_t causal;            // chunk token of the first key, or -1
  uint32_t hide, pad;        // keys that are served from elsewhere
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
  l.bytes = l.bars + l.teams * l.ring * 16 + 16 + 1024;
  // the merge: every warp's rows, their references and sums
  const int merge = kVWarps * 16 * (kVOPitch + 2) * 4;
  if (l.q < merge) l.q = merge, l.meta = l.q + groups * 4096, l.pend = l.meta + l.teams * l.ring * kVMeta, l.bars = l.pend + l.teams * kVPend * 8,
                   l.bytes = l.bars + l.teams * l.ring * 16 + 16 + 1024;
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
    if constexpr (V) return (x ? w[i] >> 8 : w[i]) & (y ? 0x00f000f0u : 0x000f000fu);
    else return (x ? w[i] >> 6 : w[i] << 2) & (y ? 0x03c003c0u : 0x003c003cu);
  } else if constexpr (V) {
    return (w[0] >> (4 * i + 8 * x)) & (y ? 0x000c000cu : 0x00030003u);
  } else {
    const int up = 6 - 4 * i - 8 * x;
    return (up > 0 ? w[0] << up : w[0] >> -up) & (y ? 0x03000300u : 0x00c000c0u);
  }
}
// Keys' codes are moved up in the mantissa (to bits 6 and 8, or 2 and 6): a product with a number that begins with n zeros is added with n bits fewer.  Two bits
// at 0 and 2 left 15 of a logit's bits (off by 1.4e-3 at 60), four at 0 and 4 left 17.
template <bool V>
__device__ __forceinline__ constexpr int code_exp(int bits, int y) {
  return bits == 8 ? 0 : bits == 4 ? 4 * y + (V ? 0 : 2) : 2 * y + (V ? 0 : 6);
}

// q s as an fp16 pair: the rounded product and what is left of it (exact)
__device__ __forceinline__ void split(uint32_t q, uint32_t s, uint32_t& hi, uint32_t& lo) {
  asm("{\n"
      ".reg .b32 n;\n"
      "mul.rn.f16x2 %0, %2, %3;\n"
      "neg.f16x2 n, %0;\n"
      "fma.rn.f16x2 %1, %2, %3, n;\n"
      "}\n"
      : "=&r"(hi), "=r"(lo)
      : "r"(q), "r"(s));
}

struct VState {
  float o[16][4], oz[4];     // channels 8 n + 2 c4, + 1 of rows r (0, 1) and r + 8 (2, 3); groups 2 c4, + 1
  float m0, m1, l0, l1;      // references of the two rows (log2), this lane's part of their sums
};

// t0, t1: the largest logits of the two rows (log2).  The references stay at or above them; where a maximum passes its reference, that goes kVAbove beyond
// it, so that it does not move again for the next small step (16 rows' accumulators are rescaled for it: without that in four of five steps of a team).
template <int NT>
__device__ __forceinline__ void raise(VState& st, const float (&x)[NT][4], float c, float& t0, float& t1) {
  t0 = fmaxf(x[0][0], x[0][1]), t1 = fmaxf(x[0][2], x[0][3]);
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
  t0 *= c;
  t1 *= c;
  if (__any_sync(0xffffffffu, t0 > st.m0 || t1 > st.m1)) {
    const float n0 = t0 > st.m0 ? t0 + kVAbove : st.m0, n1 = t1 > st.m1 ? t1 + kVAbove : st.m1;
    const float f0 = st.m0 == -INFINITY ? 0.f : ex2(st.m0 - n0), f1 = st.m1 == -INFINITY ? 0.f : ex2(st.m1 - n1);
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
}
// Exact rows: x becomes the weights exp2(c x - m).  bf16 has room for any of them.
__device__ __forceinline__ void weigh_rows(VState& st, float (&x)[2][4], float c) {
  float t0, t1;
  raise(st, x, c, t0, t1);
  const float a0 = st.m0 == -INFINITY ? 0.f : -st.m0, a1 = st.m1 == -INFINITY ? 0.f : -st.m1;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    x[n][0] = ex2(fmaf(x[n][0], c, a0));
    x[n][1] = ex2(fmaf(x[n][1], c, a0));
    x[n][2] = ex2(fmaf(x[n][2], c, a1));
    x[n][3] = ex2(fmaf(x[n][3], c, a1));
    st.l0 += x[n][0] + x[n][1];
    st.l1 += x[n][2] + x[n][3];
  }
}
// Codes: x becomes the weights relative to the item's own maximum, 2^kVTop for the heaviest, and g what they have to be multiplied by (in 32 bits) to be
// exp2(c x - m).  fp16 has no room for weights relative to a row's maximum: behind a key that leads by 11 nats all others would be below 2^-16, and a weight
// times a value scale of 2^-8 a handful of steps of 2^-24.
__device__ __forceinline__ void weigh_codes(VState& st, float (&x)[4][4], float c, float& g0, float& g1) {
  float t0, t1;
  raise(st, x, c, t0, t1);
  const float a0 = t0 == -INFINITY ? 0.f : kVTop - t0, a1 = t1 == -INFINITY ? 0.f : kVTop - t1;
  g0 = t0 == -INFINITY ? 0.f : ex2(-a0 - st.m0);
  g1 = t1 == -INFINITY ? 0.f : ex2(-a1 - st.m1);
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    x[n][0] = ex2(fmaf(x[n][0], c, a0));
    x[n][1] = ex2(fmaf(x[n][1], c, a0));
    x[n][2] = ex2(fmaf(x[n][2], c, a1));
    x[n][3] = ex2(fmaf(x[n][3], c, a1));
    s0 += x[n][0] + x[n][1];
    s1 += x[n][2] + x[n][3];
  }
  st.l0 = fmaf(s0, g0, st.l0);
  st.l1 = fmaf(s1, g1, st.l1);
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
      uint32_t hi[4], lo[4], b[4][2];
#pragma unroll
      for (int k = 0; k < 4; ++k) split(a[k], pick(sr, (k >> 1) * 2 + i), hi[k], lo[k]);
#pragma unroll
      for (int n = 0; n < 4; ++n) {          // (a tile's two products are apart: the second waits for the first's sum)
        b[n][0] = code_bits<BITS, false>(w[n >> 1], i, n & 1);
        b[n][1] = code_bits<BITS, false>(w[n >> 1], i, (n & 1) + 2);
        mma_f16(x[n], hi, b[n][0], b[n][1]);
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) mma_f16(x[n], lo, b[n][0], b[n][1]);
    }
  }
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    const float up = static_cast<float>(1 << (24 - code_exp<false>(BITS, n & 1)));
#pragma unroll
    for (int k = 0; k < 4; ++k) x[n][k] = fmaf(x[n][k], up, z[k]);
  }
}
// The largest of a half block's value scales, as an fp16 pattern (they are not negative)
template <int BITS>
__device__ __forceinline__ uint32_t largest_scale(uint32_t raw, int lane) {
  uint32_t top = 0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint32_t at = raw + off_vp(BITS, t) + (lane & 3) * 32;
    const uint4 x = lds128(at), y = lds128(at + 16);
    top = __vmaxu2(top, __vmaxu2(__vmaxu2(__vmaxu2(x.x, x.y), __vmaxu2(x.z, x.w)), __vmaxu2(__vmaxu2(y.x, y.y), __vmaxu2(y.z, y.w))));
  }
  return __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

// O += P V of a half block; `raw`: where its value parameters would lie behind the keys (off_vp, off_vc); g: see weigh_codes.
// The products P s are single fp16 numbers, in the middle of their range whatever the values' size: with the largest scale below 2^-b the
// scales are multiplied by 2^b (exactly; where b < 0, the weights are), and the item's sum leaves by one multiplication in 32 bits.  So
// a product is off by 2^-11 of itself or by 2^-36 of the item's heaviest key's.  Items without that, weights relative to the row's reference and
// scales times 16: 199 us for 64 streams of 32,757 tokens, 20 rows, but outputs off by tenths of their norm behind a leading key.
template <int BITS>
__device__ __forceinline__ void code_values(VState& st, const float (&x)[4][4], uint32_t raw, int lane, float g0, float g1) {
  const int r = lane >> 2, c4 = lane & 3;
  const uint32_t top = largest_scale<BITS>(raw, lane);
  const int b = min(11, 14 - static_cast<int>(top >> 10)), up = max(b, 0) + 4;
  // 2^up and, for the tokens whose codes lie higher, 2^(up - p)
  const __half2 up0 = h2(static_cast<uint32_t>(up + 15) * 0x04000400u), up1 = h2(static_cast<uint32_t>(up + 15 - code_exp<true>(BITS, 1)) * 0x04000400u);
  uint32_t a[2][4];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    a[t][0] = f16_pair(x[2 * t][0], x[2 * t][1]);
    a[t][1] = f16_pair(x[2 * t][2], x[2 * t][3]);
    a[t][2] = f16_pair(x[2 * t + 1][0], x[2 * t + 1][1]);
    a[t][3] = f16_pair(x[2 * t + 1][2], x[2 * t + 1][3]);
  }
  float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    uint2 z = lds64(raw + off_vp(BITS, t) + 128 + ((r & 3) * 4 + c4) * 8);      // column r: group r
    if (r >= 4) z.x = z.y = 0u;
    mma_f16(zero, a[t], z.x, z.y);
  }
  st.oz[0] = fmaf(zero[0], g0, st.oz[0]);
  st.oz[1] = fmaf(zero[1], g0, st.oz[1]);
  st.oz[2] = fmaf(zero[2], g1, st.oz[2]);
  st.oz[3] = fmaf(zero[3], g1, st.oz[3]);
  if (b < 0) {
    const float down = exp2i(b);
    const __half2 d = __float2half2_rn(down);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) a[t][k] = u32(__hmul2(h2(a[t][k]), d));
  }
  const float out = exp2i(20 - b);             // codes are code 2^(p - 24)
  const uint64_t f0 = f2_pack(g0 * out, g0 * out), f1 = f2_pack(g1 * out, g1 * out);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float o[4][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint2 s = lds64(raw + off_vp(BITS, t) + c4 * 32 + j * 8);
      const __half2 s0 = __hmul2(h2(s.x), up0), s1 = __hmul2(h2(s.y), up1);
      const uint32_t ps[4] = {u32(__hmul2(h2(a[t][0]), s0)), u32(__hmul2(h2(a[t][1]), s0)), u32(__hmul2(h2(a[t][2]), s1)), u32(__hmul2(h2(a[t][3]), s1))};
      uint32_t w[4];
      lane_words<BITS>(raw + off_vc(BITS, t), j, lane, w);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) mma_f16(o[2 * i + k], ps, code_bits<BITS, true>(w, i, k), code_bits<BITS, true>(w, i, k + 2));
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      float (&to)[4] = st.o[4 * j + n];
      f2_unpack(f2_fma(f2_pack(o[n][0], o[n][1]), f0, f2_pack(to[0], to[1])), to[0], to[1]);
      f2_unpack(f2_fma(f2_pack(o[n][2], o[n][3]), f1, f2_pack(to[2], to[3])), to[2], to[3]);
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
  VLayout lay;
};

// Rows of 64 channels, two panels each: the arena's (rows of 256 bytes; pairs of such rows, of which one is read), the chunk's keys and values
struct VerifyMaps {
  CUtensorMap rows, pairs, k, v;
};

// A barrier's state, without waiting
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// The next step of a team.  kNone: the walk has to find it; kDone: there is none
enum : int { kNone = 0, kPiece = 1, kTwoPieces = 2, kSixteenRows = 3, kSixteenCentroids = 4, kNoMore = 5, kDone = 6 };

template <int N>
__global__ void __launch_bounds__(kVThreads, 1)
    verify_kernel(const __grid_constant__ VerifyParams p, const __grid_constant__ ChunkCuts cuts, const __grid_constant__ ChunkLens<N> lens,
                  const __grid_constant__ VerifyMaps maps) {
  extern __shared__ uint8_t smem_all[];
  uint8_t* const smem_raw = smem_all + (1023u & (0u - smem_u32(smem_all)));
  const uint32_t smem = smem_u32(smem_raw);
  const VLayout& lay = p.lay;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, c4 = lane & 3;
  const bool fills = warp == kVWarps && lane < lay.teams;                 // (the other warps of its four have nothing to do)
  const int team = warp < kVWarps ? warp / p.groups : lane, grp = warp < kVWarps ? warp % p.groups : 0;
  const bool in_team = warp < kVWarps && team < lay.teams;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(smem_raw + lay.bars + lay.teams * lay.ring * 16);
  const ChunkShape& sh = p.s;
  const float c = p.scale_log2;
  const int mine = in_team || fills ? team : 0;
  const uint32_t ring = smem + lay.stages + mine * lay.ring * kVStage;
  const uint32_t bar_full = smem + lay.bars + mine * lay.ring * 16, bar_free = bar_full + 8 * lay.ring;
  VMeta* const meta = reinterpret_cast<VMeta*>(smem_raw + lay.meta) + mine * lay.ring;
  if (threadIdx.x == 0) *abort = 0;
  if (threadIdx.x == kVThreads - 1) {
    prefetch_map(&maps.rows);
    prefetch_map(&maps.k);
    prefetch_map(&maps.v);
  }
  if (fills) {
    for (int i = 0; i < lay.ring; ++i) {
      bar_init(bar_full + 8 * i, 1);
      bar_init(bar_free + 8 * i, p.groups);
    }
    bar_init_fence();
  }
  const int cta = blockIdx.x, t0 = cuts.tile[cta], i0 = cuts.item[cta], t1 = cuts.tile[cta + 1], i1 = cuts.item[cta + 1];
  int slot = cuts.slot[cta];
  int got_at = 0;                          // place of the ring, and its turn's parity
  uint32_t got_turn = 0;
  bool ok = true;
  // Both branches walk the same streams of the CTA's range and meet at the same barriers.
  struct Part {
    int tile, b, h, len, items, begin, end;
  };
  auto next_part = [&](int from, Part& x) {
    for (x.tile = from; x.tile <= t1 && x.tile < sh.batch * sh.n_kv_heads; ++x.tile) {
      x.b = x.tile / sh.n_kv_heads;
      x.h = x.tile % sh.n_kv_heads;
      x.len = lens.len[N == 1 ? 0 : x.b];
      x.items = chunk_items(sh, x.len, 0);
      x.begin = x.tile == t0 ? i0 : 0;
      x.end = x.tile == t1 ? i1 : x.items;
      if (x.begin < x.end) return true;
    }
    return false;
  };
  Part x;
  pdl_wait();                              // (nothing but parameters was read so far)
  pdl_launch();                            // (the merge waits for the whole grid; its blocks may take their places)

  if (warp >= kVWarps) {
    fewer_regs<kVFillRegs>();
    int put_at = 0;                        // the ring's next place, and the parity of its last turn (places not used yet count as freed)
    uint32_t put_turn = 1;
    for (int from = t0; next_part(from, x); from = x.tile + 1) {
    const int tile = x.tile, b = x.b, h = x.h, len = x.len, begin = x.begin, end = x.end;
    __syncthreads();                       // (barriers are initialised; the previous stream's merge has been read)
    if (warp == kVWarps) {
      // ---- the walks, a lane per team ----
      const TableEntry* table = p.table + static_cast<size_t>(tile) * p.table_stride;
      const int blocks_end = 2 * p.n_closed, tail_end = blocks_end + (p.n_tail + 31) / 32, res_end = tail_end + p.res_items;
      uint32_t* const pend_off = reinterpret_cast<uint32_t*>(smem_raw + lay.pend) + (fills ? team : 0) * kVPend * 2;
      float* const pend_bias = reinterpret_cast<float*>(pend_off + kVPend);
      int pend = 0, it = begin + team;
      // of an item's block, loaded an item ahead
      auto entry = [&](int i) {
        return fills && i < min(end, blocks_end) ? *reinterpret_cast<const uint4*>(
                                                       table + static_cast<uint64_t>(i >> 1) * static_cast<uint32_t>(p.walk) % static_cast<uint32_t>(p.n_closed))
                                                 : make_uint4(0, 0, 0, 0);
      };
      uint4 e = entry(it);
      const uint8_t* k = nullptr;                    // the step's codes
      uint32_t row = 0, hide = 0;                    // first row of what is left of a row item: of the arena, or new token
      int left = 0, causal = -1, level = 0, source = 0, step = fills ? kNone : kDone;      // source: 0 a block, 1 residual rows, 2 new rows
      int idle = 0;
      for (;;) {
        while (step == kNone) {
          if (left > 0) {
            step = kSixteenRows;
          } else if (pend == 16 || (it >= end && pend > 0)) {
            step = kSixteenCentroids;
          } else if (it >= end) {
            step = kNoMore;
          } else if (it < blocks_end) {
            const uint4 now = e;
            const int half = it & 1;
            it += lay.teams;
            e = entry(it);
            level = static_cast<int>(now.y);
            hide = half ? now.w : now.z;
            k = p.arena + static_cast<size_t>(now.x) * 256;
            if (level == 1) {
              if (half) continue;
              const int n = kBlock - __popc(now.z) - __popc(now.w);
              pend_off[pend] = now.x;
              pend_bias[pend] = n > 0 ? lg2(static_cast<float>(n)) / c : -INFINITY;
              ++pend;
            } else if (level == 16) {
              row = now.x + half * 32;
              source = 0;
              left = 32;
              causal = -1;
            } else {
              k += half * half_bytes(level);
              step = level == 8 ? kTwoPieces : kPiece;
            }
          } else {
            hide = 0;
            causal = -1;
            if (it < tail_end) {
              const int row0 = (it - blocks_end) * 32;
              row = table[p.n_closed].off256 + row0;
              source = 0;
              left = min(32, p.n_tail - row0);
            } else if (it < res_end) {
              const int row0 = (it - tail_end) * 32;
              row = p.res_off256[tile] + 2 * row0;
              source = 1;
              left = max(0, min(32, p.res_count[tile] - row0));
            } else {
              const int tok0 = (it - res_end) * 32;
              row = b * sh.n_new + tok0;
              source = 2;
              left = min(32, len - tok0);
              causal = tok0;
            }
            it += lay.teams;
          }
        }
        __syncwarp();
        // is there room for the step's one or two parts?
        const bool two = step == kTwoPieces || step == kSixteenRows || step == kSixteenCentroids;
        const int at2 = put_at + 1 == lay.ring ? 0 : put_at + 1;
        const uint32_t turn2 = put_at + 1 == lay.ring ? put_turn ^ 1u : put_turn;
        const bool ready = step != kDone && bar_test(bar_free + 8 * put_at, put_turn) && (!two || bar_test(bar_free + 8 * at2, turn2));
        if (__ballot_sync(0xffffffffu, ready) == 0) {
          if (__all_sync(0xffffffffu, step == kDone)) break;
          if (++idle > kVIdle) *abort = 1;
          if (__any_sync(0xffffffffu, *abort != 0)) break;
          continue;
        }
        idle = 0;
        const uint32_t dst = ring + put_at * kVStage, bar = bar_full + 8 * put_at, dst2 = ring + at2 * kVStage, bar2 = bar_full + 8 * at2;
        const int n = step == kSixteenCentroids ? pend : min(left, 16);
        if (ready) {
          VMeta& m = meta[put_at];
          const uint32_t kind = step == kNoMore ? 0 : step == kSixteenRows ? 2 : step == kSixteenCentroids ? 3 : 1;
          *reinterpret_cast<uint4*>(&m) = make_uint4(kind | level << 8 | n << 16, step == kSixteenRows ? causal : -1, step == kSixteenCentroids ? 0u : hide, 0u);
          if (step == kNoMore) {
            bar_arrive(bar);
          } else if (step == kPiece || step == kTwoPieces) {
            const uint32_t bytes = step == kPiece ? half_bytes(level) : half_bytes(8) / 2;
            bar_expect(bar, bytes);
            bulk_load(dst, k, bytes, bar);
            if (step == kTwoPieces) {
              bar_expect(bar2, bytes);
              bulk_load(dst2, k + bytes, bytes, bar2);
            }
          } else if (step == kSixteenRows) {
            bar_expect(bar, 16 * kRowBytes);
            bar_expect(bar2, 16 * kRowBytes);
            if (source == 0) {
              tma_load_3d(dst, &maps.rows, 0, static_cast<int>(row), 0, bar);
              tma_load_3d(dst2, &maps.rows, 0, static_cast<int>(row) + kBlock, 0, bar2);
            } else if (source == 1) {
              tma_load_4d(dst, &maps.pairs, 0, static_cast<int>(row & 1u), static_cast<int>(row >> 1), 0, bar);
              tma_load_4d(dst2, &maps.pairs, 0, static_cast<int>((row + 1) & 1u), static_cast<int>((row + 1) >> 1), 0, bar2);
            } else {
              tma_load_4d(dst, &maps.k, 0, h, static_cast<int>(row), 0, bar);
              tma_load_4d(dst2, &maps.v, 0, h, static_cast<int>(row), 0, bar2);
            }
          }
        }
        // centroids: lane i copies key row i, lane 16 + i value row i (rows that are not there: the first again, their keys are masked)
        for (uint32_t m = __ballot_sync(0xffffffffu, ready && step == kSixteenCentroids); m; m &= m - 1) {
          const int t = __ffs(m) - 1, i = lane & 15;
          const int rows = __shfl_sync(0xffffffffu, n, t);
          const uint32_t d1 = __shfl_sync(0xffffffffu, dst, t), d2 = __shfl_sync(0xffffffffu, dst2, t);
          const uint32_t b1 = __shfl_sync(0xffffffffu, bar, t), b2 = __shfl_sync(0xffffffffu, bar2, t);
          const int place = __shfl_sync(0xffffffffu, put_at, t);
          const int from = i < rows ? i : 0;
          const uint32_t* const off = reinterpret_cast<const uint32_t*>(smem_raw + lay.pend) + t * kVPend * 2;
          const uint8_t* src = p.arena + static_cast<size_t>(off[from]) * 256 + (lane >> 4) * kRowBytes;
          if (lane < 16) (reinterpret_cast<VMeta*>(smem_raw + lay.meta) + t * lay.ring + place)->bias[i] = reinterpret_cast<const float*>(off + kVPend)[from];
          __syncwarp();
          if (lane == t) {
            bar_expect(b1, 16 * kRowBytes);
            bar_expect(b2, 16 * kRowBytes);
          }
          __syncwarp();
          bulk_load((lane < 16 ? d1 : d2) + i * kVPitch, src, kRowBytes, lane < 16 ? b1 : b2);
        }
        __syncwarp();
        if (ready) {
          if (step == kSixteenRows) {
            left -= n;
            hide >>= 16;
            row += source == 1 ? 32 : 16;
            if (causal >= 0) causal += 16;
          } else if (step == kSixteenCentroids) {
            pend = 0;
          }
          for (int i = 0; i < (two ? 2 : 1); ++i)
            if (++put_at == lay.ring) {
              put_at = 0;
              put_turn ^= 1u;
            }
          step = step == kNoMore ? kDone : kNone;
        }
      }
      if (fills && *abort)                   // what is on its way arrives before the memory is used otherwise
        for (int i = 0; i < lay.ring; ++i) bar_drain(bar_full + 8 * i, i < put_at ? put_turn ^ 1u : put_turn);
    }
    __syncwarp();
    __syncthreads();
    __syncthreads();
    if (*abort) break;
    }
  } else {
    more_regs<kVWarpRegs>();
    for (int from = t0; next_part(from, x); from = x.tile + 1) {
    const int b = x.b, h = x.h, len = x.len, items = x.items, begin = x.begin, end = x.end;
    const int rows = len * sh.group;
    __syncthreads();
    // the rows' fragments: lane (r, c4) of MMA index s holds channels 16 s + 2 c4, + 1 of rows r and r + 8, then the channels eight further
      for (int i = threadIdx.x; i < p.groups * 8 * 32; i += kVWarps * 32) {
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
    asm volatile("bar.sync 1, %0;\n" ::"n"(kVWarps * 32) : "memory");

    VState st;
#pragma unroll
    for (int n = 0; n < 16; ++n) st.o[n][0] = st.o[n][1] = st.o[n][2] = st.o[n][3] = 0.f;
    st.oz[0] = st.oz[1] = st.oz[2] = st.oz[3] = 0.f;
    st.m0 = st.m1 = -INFINITY;
    st.l0 = st.l1 = 0.f;

    if (in_team) {
      auto wait_part = [&]() { return bar_wait(bar_full + 8 * got_at, got_turn, abort); };
      auto free_part = [&]() {
        __syncwarp();
        if (lane == 0) bar_arrive(bar_free + 8 * got_at);
        if (++got_at == lay.ring) {
          got_at = 0;
          got_turn ^= 1u;
        }
      };

      const int row0 = grp * 16 + r, tok_a = row0 / sh.group, tok_b = (row0 + 8) / sh.group;      // of the lane's two rows
      const uint32_t q = smem + lay.q + grp * 4096;
      for (;;) {
        if (!(ok = wait_part())) break;
        const VMeta& e = meta[got_at];
        const uint4 m = *reinterpret_cast<const uint4*>(&e);
        const int kind = m.x & 255u, level = m.x >> 8 & 255u;
        const uint32_t raw = ring + got_at * kVStage;
        if (kind == 0) {
          free_part();
          break;
        }
        if (kind == 1) {
          float x[4][4];
          if (level == 4) code_logits<4>(x, raw, q, lane);
          else if (level == 8) code_logits<8>(x, raw, q, lane);
          else code_logits<2>(x, raw, q, lane);
          const uint32_t hide = m.z;
          if (hide) {
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (hide >> (8 * n + 2 * c4 + (k & 1)) & 1u) x[n][k] = -INFINITY;
          }
          float g0, g1;
          weigh_codes(st, x, c, g0, g1);
          if (level == 8) {
            free_part();
            if (!(ok = wait_part())) break;
            code_values<8>(st, x, ring + got_at * kVStage - half_bytes(8) / 2, lane, g0, g1);
          } else if (level == 4) {
            code_values<4>(st, x, raw, lane, g0, g1);
          } else {
            code_values<2>(st, x, raw, lane, g0, g1);
          }
          free_part();
        } else {
          // 16 rows of bf16: keys [token][channel] are B fragments as they are, values with the transposing load.  Chunk i of a row lies in
          // panel i / 8; where the rows came by tensor map the chunks of a panel are swizzled
          const bool swizzled = kind == 2;
          const int panel = swizzled ? kVPanel : 128, pitch = swizzled ? 128 : kVPitch;
          float x[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
          {
            const int row = (lane & 7) + (lane >> 4) * 8;
            const uint32_t at = raw + row * pitch, flip = swizzled ? (row & 7) << 4 : 0, hi = (lane >> 3 & 1) << 4;
#pragma unroll 4
            for (int s = 0; s < 8; ++s) {
              const uint4 qv = lds128(q + (s * 32 + lane) * 16);
              uint32_t a[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 f = __half22float2(h2(pick(qv, k)));      // (the rows are bf16 by origin: exact)
                a[k] = bf16_pair(f.x, f.y);
              }
              uint32_t kb[4];
              ldmatrix4<false>(kb, at + (s >> 2) * panel + (((s & 3) * 32 + hi) ^ flip));
              mma_bf16(x[0], a, kb[0], kb[1]);
              mma_bf16(x[1], a, kb[2], kb[3]);
            }
          }
          const int n = m.x >> 16, causal = static_cast<int>(m.y);
          const uint32_t hide = m.z;
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
          weigh_rows(st, x, c);
          free_part();
          if (!(ok = wait_part())) break;
          const uint32_t a[4] = {bf16_pair(x[0][0], x[0][1]), bf16_pair(x[0][2], x[0][3]), bf16_pair(x[1][0], x[1][1]), bf16_pair(x[1][2], x[1][3])};
          const uint32_t vraw = ring + got_at * kVStage;
          if (swizzled && n < 16) {          // rows that are not there may hold anything: zeros (every warp of the team writes the same ones)
            for (int i = n * 8 + lane; i < 128; i += 32) {
              sts128(vraw + i * 16, make_uint4(0, 0, 0, 0));
              sts128(vraw + kVPanel + i * 16, make_uint4(0, 0, 0, 0));
            }
            __syncwarp();
          }
          const int vrow = lane & 15;
          const uint32_t at = vraw + vrow * pitch, flip = swizzled ? (vrow & 7) << 4 : 0, hi = (lane >> 4) << 4;
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            uint32_t vb[4];
            ldmatrix4<true>(vb, at + (g >> 2) * panel + (((g & 3) * 32 + hi) ^ flip));
            mma_bf16(st.o[2 * g], a, vb[0], vb[1]);
            mma_bf16(st.o[2 * g + 1], a, vb[2], vb[3]);
          }
          if (swizzled && n < 16) fence_async();      // (copies land there next)
          free_part();
        }
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
          st.o[n][0] += z0;
          st.o[n][1] += z0;
          st.o[n][2] += z1;
          st.o[n][3] += z1;
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
        mml[warp * 16 + r] = make_float2(st.m0, st.l0);
        mml[warp * 16 + r + 8] = make_float2(st.m1, st.l1);
      }
    }
    fence_async();                         // (copies land there next)
    __syncthreads();
    const int to = chunk_needs_slot(begin, end, items) ? slot++ : -1;
    auto write_row = [&](int i, const float4& o, float top, float sum) {
      const size_t at = (static_cast<size_t>(b) * sh.n_new + i / sh.group) * (sh.n_kv_heads * sh.group) + h * sh.group + i % sh.group;
      const float inv = 1.f / sum;
      reinterpret_cast<uint2*>(p.out + at * kD)[lane] = make_uint2(bf16_pair(o.x * inv, o.y * inv), bf16_pair(o.z * inv, o.w * inv));
      if (p.lse && lane == 0) p.lse[at] = (top + lg2(sum)) * kLn2;
    };
    for (int i = warp; i < rows; i += kVWarps) {           // a warp per row, four channels per lane; lane t has team t's factor
      const int at0 = (i >> 4) * 16 + (i & 15), step = p.groups * 16;
      const float2 v = lane < lay.teams ? mml[at0 + lane * step] : make_float2(0.f, 0.f);
      float top = v.y != 0.f ? v.x : -INFINITY;      // (NaN counts: it has to come through)
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));      // (at most 12 teams)
      const float f = v.y != 0.f ? ex2(v.x - top) : 0.f;
      float sum = f * v.y;
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      top = __shfl_sync(0xffffffffu, top, 0);
      sum = __shfl_sync(0xffffffffu, sum, 0);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int t = 0; t < lay.teams; ++t) {
        const float g = __shfl_sync(0xffffffffu, f, t);
        const float4 x = *reinterpret_cast<const float4*>(mo + (at0 + t * step) * kVOPitch + 4 * lane);
        o.x += g * x.x;
        o.y += g * x.y;
        o.z += g * x.z;
        o.w += g * x.w;
      }
      if (to >= 0) {
        const size_t at = static_cast<size_t>(to) * kChunkRows + i;
        reinterpret_cast<float4*>(p.part_o + at * kD)[lane] = o;
        if (lane == 0) p.part_ml[at] = make_float2(top, sum);
      } else {
        write_row(i, o, top, sum);
      }
    }
    if (!ok) atomicOr(p.status, kStatusInternal);
    if (*abort) break;                       // (set by whoever gave up: everyone has passed the barrier behind its waits)
    }
  }
}

template <int N>
cudaError_t launch_as(const VerifyParams& p, const VerifyMaps& maps, const ChunkCuts& cuts, const int32_t* len, cudaStream_t st) {
  ChunkLens<N> lens;
  for (int b = 0; b < (N == 1 ? 1 : p.s.batch); ++b) lens.len[b] = len ? len[b] : p.s.n_new;
  static std::atomic<uint64_t> done{0};
  size_t most = 0;
  for (int g = 1; g <= kVerifyRows / 16; ++g) most = std::max(most, static_cast<size_t>(verify_layout(g).bytes));
  const cudaError_t e = raise_smem_limit(verify_kernel<N>, most, done);
  if (e != cudaSuccess) return e;
  return attend::launch_behind(verify_kernel<N>, dim3(cuts.n), kVThreads, p.lay.bytes, st, p, cuts, lens, maps);
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
  p.lay = verify_layout(p.groups);
  VerifyMaps maps;
  const uint64_t units = call.arena_bytes / 256, kv = static_cast<uint64_t>(p.s.n_kv_heads), tokens = static_cast<uint64_t>(p.s.batch) * p.s.n_new;
  const uint64_t rows[3] = {64, units, 2}, rows_step[2] = {256, 128}, pairs[4] = {64, 2, units / 2, 2}, pairs_step[3] = {256, 512, 128};
  const uint64_t fresh[4] = {64, kv, tokens, 2}, fresh_step[3] = {256, kv * 256, 128};
  const uint32_t rows_box[3] = {64, 16, 2}, box[4] = {64, 1, 16, 2};
  if (!make_map(&maps.rows, p.arena, 3, rows, rows_step, rows_box) || !make_map(&maps.pairs, p.arena, 4, pairs, pairs_step, box) ||
      !make_map(&maps.k, p.k_new, 4, fresh, fresh_step, box) || !make_map(&maps.v, p.v_new, 4, fresh, fresh_step, box))
    return cudaErrorInvalidValue;
  const cudaError_t e = len && p.s.batch > 1 ? launch_as<kChunkMaxBatch>(p, maps, cuts, len, st) : launch_as<1>(p, maps, cuts, len, st);
  return e != cudaSuccess ? e : launch_chunk_merge(call, merge, len, st);
}

}  // namespace gkv
