// Attention of whole prompts over their own exact rows, and the attention mass that their tokens get from the newest queries
// (Sec. 3.1, Eq. 2): what a serving program runs before it hands a prompt's rows to the bulk ingest.
//
// prompt_kernel.  Causal softmax attention of packed sequences, grouped heads.  A CTA has two row tiles of up to 128 rows; the
// rows of a tile are the g query heads of 128 / g consecutive tokens, so that all of them read one KV head and the diagonal is
// 128 / g tokens wide.  Per step of 128 keys and row tile:
//   S = Q K^T            tcgen05, both operands in shared memory, fp32 accumulator in tensor memory
//   m' = max(m, row max) the reference m moves only when the maximum has grown by more than 2^8: P then stays below 2^8, and the
//                        accumulator is rescaled a handful of times per row, not once per step
//   P = exp2(c S - c m)  bf16 (a rounding of at most 2^-9 of each weight; its sum l is taken before it), over S in tensor memory
//   O += P V             tcgen05, P from tensor memory, V as it lies ([token][channel], MN-major)
// While four warps work on one tile's S, the tensor cores work for the other tile: the four products of a step are issued by one
// thread in the order P0 V, Q0 K, P1 V, Q1 K.  K and V tiles come by TMA through a ring of 32 KB stages.
//
// mass_kernel.  S^T = K Q^T for the observing rows: a thread owns a token, so the sum over rows of exp2(c S - lse) needs no
// exchange, and every sum has a fixed order.  K is read once.
//
// Values of a sequence have to be finite; what lies behind a sequence's end may hold anything: its logits are masked by
// selection and its value rows are zeroed in shared memory before they are used.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <numeric>
#include <vector>

#include "../../include/gkv.h"
#include "gkv_internal.h"
#include "gkv_tc.cuh"

namespace gkv {
namespace {

using namespace tc;

constexpr int kRows = 128;                 // rows of a tile, keys of a step
constexpr int kPanel = kRows * 128;        // bytes of 64 channels of 128 rows
constexpr int kTileBytes = 2 * kPanel;
constexpr int kMaxSeqs = 1024;             // sequences of one launch
constexpr int kFewSeqs = 32;               // the same where the parameters are to stay short

// Sequences in the order in which their work is dealt out (longest first).  Work items of sequence i: [first[i], first[i + 1]).
template <int N>
struct Seqs {
  int32_t n;
  int32_t row[N], len[N], first[N + 1];
};
template <int N>
__device__ __forceinline__ int find_seq(const Seqs<N>& s, int item) {
  int lo = 0, hi = s.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.first[mid] <= item) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// ---- prompt attention ----------------------------------------------------------------------------
constexpr int kPThreads = 384;             // softmax of tile 0, of tile 1 (four warps each), loads, products, value rows' end, -
constexpr int kPStages = 5;
constexpr int kPOffStage = 2 * kTileBytes;
constexpr int kPOffBar = kPOffStage + kPStages * kTileBytes;
constexpr int kPSmem = kPOffBar + 256 + 1024;
constexpr int kPLaunchRegs = 168, kPSoftRegs = 216, kPOtherRegs = 72;
static_assert(2 * kPSoftRegs + kPOtherRegs <= 3 * kPLaunchRegs, "a split draws on the launch's registers");
constexpr float kSlack = 8.f;              // log2 of what a weight may exceed 1 by before the reference moves

struct PromptParams {
  uint16_t* out;
  float* lse;
  int64_t out_stride;
  int32_t n_q_heads, n_kv_heads, group, tile_tokens;
  float scale_log2;
};

template <int N>
__global__ void __launch_bounds__(kPThreads, 1)
    prompt_kernel(const __grid_constant__ PromptParams p, const __grid_constant__ Seqs<N> seqs, const __grid_constant__ CUtensorMap map_q,
                  const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base = smem_raw + (smem - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bars = smem + kPOffBar;
  const uint32_t bar_q = bars, bar_s = bars + 16, bar_p = bars + 32, bar_o = bars + 48, bar_fix = bars + 64, bar_last = bars + 72, bar_drain_mma = bars + 80, bar_pa = bars + 88;
  const uint32_t bar_full = bars + 104, bar_empty = bar_full + 8 * kPStages;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(base + kPOffBar + 240);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base + kPOffBar + 244);
  static_assert(104 + 16 * kPStages <= 240, "room for the barriers");

  const int head = blockIdx.x % p.n_kv_heads, item = blockIdx.x / p.n_kv_heads;
  const int si = find_seq(seqs, item);
  const int len = seqs.len[si], row0 = seqs.row[si];
  const int span = 2 * p.tile_tokens;
  // the last tiles of a sequence, the ones with most keys, first
  const int tok0 = ((len + span - 1) / span - 1 - (item - seqs.first[si])) * span;
  // keys that tile t needs, in steps of 128; 0 = no rows
  const int end0 = min(tok0 + p.tile_tokens, len), end1 = min(tok0 + span, len);
  const int n0 = (end0 + kRows - 1) / kRows;
  const int n1 = end1 > tok0 + p.tile_tokens ? (end1 + kRows - 1) / kRows : 0;
  const int nmax = max(n0, n1);
  const bool fix = nmax * kRows > len;       // the last step reaches behind the sequence

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      bar_init(bar_q + 8 * t, 1);
      bar_init(bar_s + 8 * t, 1);
      bar_init(bar_pa + 8 * t, 4);
      bar_init(bar_p + 8 * t, 4);
      bar_init(bar_o + 8 * t, 1);
    }
    bar_init(bar_fix, 1);
    bar_init(bar_last, 1);
    bar_init(bar_drain_mma, 1);
    for (int i = 0; i < kPStages; ++i) {
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

  if (warp < 8) {
    more_regs<kPSoftRegs>();
    const int t = warp >> 2;
    const int n_t = t ? n1 : n0;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp & 3) << 21);
    const uint32_t s_tm = lanes + t * kRows, o_tm = lanes + 256 + t * kRows;
    const int r = (warp & 3) * 32 + lane;
    const int tok_in = r / p.group;
    const int pos = tok0 + t * p.tile_tokens + tok_in;
    const bool real = tok_in < p.tile_tokens && pos < len;
    const int first_pos = tok0 + t * p.tile_tokens + (warp & 3) * 32 / p.group;      // of the warp's rows
    const float c = p.scale_log2;
    float m = 0.f, l = 0.f;
    bool ok = true;
    for (int j = 0; j < n_t; ++j) {
      if (!bar_wait(bar_s + 8 * t, j & 1, abort)) {
        ok = false;
        break;
      }
      tmem_after();
      uint32_t x[kRows];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32(s_tm + 32 * i, x + 32 * i);
      tmem_wait_ld();
      if ((j + 1) * kRows - 1 > first_pos) {
        const int limit = pos - j * kRows;
#pragma unroll
        for (int i = 0; i < kRows; ++i)
          if (i > limit) x[i] = 0xff800000u;
      }
      float mx[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) mx[k] = max3(__uint_as_float(x[3 * k]), __uint_as_float(x[3 * k + 1]), __uint_as_float(x[3 * k + 2]));
#pragma unroll
      for (int i = 12; i < kRows; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + 2 * k < kRows) mx[k] = max3(mx[k], __uint_as_float(x[i + 2 * k]), __uint_as_float(x[i + 2 * k + 1]));
      const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
      if (j == 0) {
        m = top == -INFINITY ? 0.f : top;
      } else {
        const bool move = (top - m) * c > kSlack;
        if (__any_sync(0xffffffffu, move)) {
          const float f = move ? ex2((m - top) * c) : 1.f;
          m = move ? top : m;
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
      }
      const uint64_t cc = f2_pack(c, c), mm = f2_pack(-m * c, -m * c);
      uint64_t sum0 = 0, sum1 = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t pk[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          float a, b;
          f2_unpack(f2_fma(f2_pack(__uint_as_float(x[32 * i + 2 * k]), __uint_as_float(x[32 * i + 2 * k + 1])), cc, mm), a, b);
          a = ex2(a);
          b = ex2(b);
          if (k & 1) sum1 = f2_add(sum1, f2_pack(a, b));
          else sum0 = f2_add(sum0, f2_pack(a, b));
          pk[k] = bf16_pair(a, b);
        }
        tmem_st16(s_tm + 16 * i, pk);
        if (i == 2) {                        // three quarters of the weights: their product starts while the rest are made
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
    if (n_t > 0) {
      ok = ok && bar_wait(bar_o + 8 * t, 0, abort);
      tmem_after();
      const float inv = ok ? 1.f / l : NAN;
      const int hq = head * p.group + r % p.group;
      uint16_t* dst = p.out + static_cast<int64_t>(row0 + pos) * p.out_stride + hq * kD;
      for (int i = 0; i < 4; ++i) {
        uint32_t o[32];
        tmem_ld32(o_tm + 32 * i, o);
        tmem_wait_ld();
        if (real) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint4 v;
            v.x = bf16_pair(__uint_as_float(o[8 * k]) * inv, __uint_as_float(o[8 * k + 1]) * inv);
            v.y = bf16_pair(__uint_as_float(o[8 * k + 2]) * inv, __uint_as_float(o[8 * k + 3]) * inv);
            v.z = bf16_pair(__uint_as_float(o[8 * k + 4]) * inv, __uint_as_float(o[8 * k + 5]) * inv);
            v.w = bf16_pair(__uint_as_float(o[8 * k + 6]) * inv, __uint_as_float(o[8 * k + 7]) * inv);
            *reinterpret_cast<uint4*>(dst + 32 * i + 8 * k) = v;
          }
        }
      }
      if (real && p.lse) p.lse[static_cast<int64_t>(row0 + pos) * p.n_q_heads + hq] = ok ? (m * c + lg2(l)) * kLn2 : NAN;
    }
  } else {
    fewer_regs<kPOtherRegs>();
    if (warp == 8) {
      if (elect()) {
        const uint32_t q_bytes = 2u * p.tile_tokens * p.group * 128u;
        for (int t = 0; t < (n1 ? 2 : 1); ++t) {
          bar_expect(bar_q + 8 * t, q_bytes);
          for (int h = 0; h < 2; ++h)
            tma_load_3d(smem + t * kTileBytes + h * kPanel, &map_q, 64 * h, head * p.group, row0 + tok0 + t * p.tile_tokens, bar_q + 8 * t);
        }
        int i = 0;
        for (; i < 2 * nmax; ++i) {
          const int slot = i % kPStages, turn = i / kPStages;
          if (turn > 0 && !bar_wait(bar_empty + 8 * slot, (turn - 1) & 1, abort)) break;
          bar_expect(bar_full + 8 * slot, kTileBytes);
          const uint32_t dst = smem + kPOffStage + slot * kTileBytes;
          for (int h = 0; h < 2; ++h)
            tma_load_3d(dst + h * kPanel, i & 1 ? &map_v : &map_k, 64 * h, head, row0 + (i >> 1) * kRows, bar_full + 8 * slot);
        }
        if (*abort) {                        // what is on its way arrives before the CTA leaves
          for (int t = 0; t < (n1 ? 2 : 1); ++t) bar_drain(bar_q + 8 * t, 0);
          for (int k = max(0, i - kPStages); k < i; ++k) bar_drain(bar_full + 8 * (k % kPStages), (k / kPStages) & 1);
        }
      }
    } else if (warp == 9) {
      if (elect()) {
        constexpr uint32_t id_qk = instr_desc(true, false, kRows, kRows), id_pv = instr_desc(true, true, kRows, kD);
        auto wait_stage = [&](int i) { return bar_wait(bar_full + 8 * (i % kPStages), (i / kPStages) & 1, abort); };
        auto free_stage = [&](int i) { mma_commit(bar_empty + 8 * (i % kPStages)); };
        auto qk = [&](int t, int i) {
          const uint64_t a = smem_desc(smem + t * kTileBytes, 16), b = smem_desc(smem + kPOffStage + (i % kPStages) * kTileBytes, 16);
          for (int k = 0; k < kD / 16; ++k) {
            const uint32_t off = ((k >> 2) * kPanel + (k & 3) * 32) >> 4;
            mma_ss(tmem + t * kRows, a + off, b + off, id_qk, k > 0);
          }
          mma_commit(bar_s + 8 * t);
        };
        auto pv = [&](int t, int i, bool first, int from, int to) {
          const uint64_t b = smem_desc(smem + kPOffStage + (i % kPStages) * kTileBytes, kPanel);
          for (int k = from; k < to; ++k) mma_ts(tmem + 256 + t * kRows, tmem + t * kRows + 8 * k, b + ((k * 16 * 128) >> 4), id_pv, !first || k > 0);
        };
        bool ok = bar_wait(bar_q, 0, abort) && wait_stage(0);
        if (ok) {
          tmem_after();
          qk(0, 0);
          if (n1) {
            ok = bar_wait(bar_q + 8, 0, abort);
            if (ok) qk(1, 0);
          }
          free_stage(0);
        }
        for (int j = 0; ok && j < nmax; ++j) {
          const int v = 2 * j + 1, k = 2 * j + 2;
          ok = wait_stage(v) && (j + 1 == nmax || wait_stage(k));
          if (ok && fix && j + 1 == nmax) {      // the last values are there: warp 10 zeroes the rows behind the sequence
            bar_arrive(bar_last);
            ok = bar_wait(bar_fix, 0, abort);
          }
          if (!ok) break;
          for (int t = 0; t < 2 && ok; ++t) {
            const int n_t = t ? n1 : n0;
            if (j < n_t) {
              ok = bar_wait(bar_pa + 8 * t, j & 1, abort);
              if (!ok) break;
              tmem_after();
              pv(t, v, j == 0, 0, 6);
              ok = bar_wait(bar_p + 8 * t, j & 1, abort);
              if (!ok) break;
              tmem_after();
              pv(t, v, j == 0, 6, 8);
              if (j + 1 == n_t) mma_commit(bar_o + 8 * t);
              else qk(t, k);
            }
          }
          free_stage(v);
          if (j + 1 < nmax) free_stage(k);
        }
        if (!ok) {                           // products in flight end before tensor memory is given back
          mma_commit(bar_drain_mma);
          bar_drain(bar_drain_mma, 0);
        }
      }
    } else if (warp == 10 && fix) {
      if (bar_wait(bar_last, 0, abort)) {
        const uint32_t v = smem + kPOffStage + (2 * nmax - 1) % kPStages * kTileBytes;
        for (int k = (len - (nmax - 1) * kRows) * 8 + lane; k < kRows * 8; k += 32) {
          sts128(v + k * 16, make_uint4(0, 0, 0, 0));
          sts128(v + kPanel + k * 16, make_uint4(0, 0, 0, 0));
        }
        fence_async();
        __syncwarp();
        if (lane == 0) bar_arrive(bar_fix);
      }
    }
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// ---- masses of prompt tokens ---------------------------------------------------------------------
constexpr int kMThreads = 192;             // four warps of tokens, loads, products
constexpr int kMStages = 2;
constexpr int kMOffLse = kMStages * kTileBytes;
constexpr int kMOffBar = kMOffLse + 256 * 4;
constexpr int kMOffQ = kMOffBar + 1024;
constexpr int kMaxObsRows = 256;           // rows of one product: its n dimension

struct MassParams {
  const float* lse;
  float* mass;
  int32_t row_base;                          // first row of the first sequence: where `mass` begins
  int32_t n_q_heads, n_kv_heads, group;
  int32_t n_obs, group_tokens;               // observing tokens of a sequence; of one product
  int32_t n_pad;                             // columns of a product, a multiple of 16
  int32_t pitch, tmem_cols;                  // the same rounded up to what one load reads; two of them
  int32_t chunk;                             // tiles of 128 tokens per CTA
  float scale_log2;
};

template <int N>
__global__ void __launch_bounds__(kMThreads)
    mass_kernel(const __grid_constant__ MassParams p, const __grid_constant__ Seqs<N> seqs, const __grid_constant__ CUtensorMap map_q,
                const __grid_constant__ CUtensorMap map_k) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base = smem_raw + (smem - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bars = smem + kMOffBar;
  const uint32_t bar_q = bars, bar_qfree = bars + 8, bar_s = bars + 16, bar_sfree = bars + 32, bar_full = bars + 48, bar_empty = bars + 64, bar_drain_mma = bars + 80;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(base + kMOffBar + 240);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base + kMOffBar + 244);
  float* const lse_s = reinterpret_cast<float*>(base + kMOffLse);

  const int head = blockIdx.x % p.n_kv_heads, item = blockIdx.x / p.n_kv_heads;
  const int si = find_seq(seqs, item);
  const int len = seqs.len[si], row0 = seqs.row[si];
  const int tile0 = (item - seqs.first[si]) * p.chunk;
  const int n_tiles = min(p.chunk, (len + kRows - 1) / kRows - tile0);
  const int obs = min(p.n_obs, len), obs0 = len - obs;         // observing tokens, the first of them
  const int n_groups = (obs + p.group_tokens - 1) / p.group_tokens;
  const int steps = n_tiles * n_groups;

  if (threadIdx.x == 0) {
    bar_init(bar_q, 1);
    bar_init(bar_qfree, 1);
    for (int i = 0; i < 2; ++i) {
      bar_init(bar_s + 8 * i, 1);
      bar_init(bar_sfree + 8 * i, 4);
      bar_init(bar_full + 8 * i, 1);
      bar_init(bar_empty + 8 * i, 1);
    }
    bar_init(bar_drain_mma, 1);
    *abort = 0;
    bar_init_fence();
  }
  if (warp == 5) tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), p.tmem_cols);
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *tmem_slot;

  if (warp < 4) {
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp) << 21);
    const int r = warp * 32 + lane;
    float sum = 0.f;
    bool ok = true;
    for (int i = 0; i < steps; ++i) {
      const int grp = i % n_groups, tok = (tile0 + i / n_groups) * kRows + r;
      const int q0 = obs0 + grp * p.group_tokens;                                  // first observing token of the product
      const int cols = min(p.group_tokens, obs - grp * p.group_tokens) * p.group;
      if (i == 0 || n_groups > 1) {
        asm volatile("bar.sync 1, 128;\n" ::: "memory");
        for (int k = r; k < cols; k += 128)
          lse_s[k] = -kLog2e * p.lse[static_cast<int64_t>(row0 + q0 + k / p.group) * p.n_q_heads + head * p.group + k % p.group];
        asm volatile("bar.sync 1, 128;\n" ::: "memory");
      }
      // (after an abort the loop goes on without products: its barriers need all four warps)
      ok = ok && bar_wait(bar_s + 8 * (i & 1), (i >> 1) & 1, abort);
      if (!ok) continue;
      tmem_after();
      const int from = max(0, (tok - q0) * p.group);           // rows before the token do not see it
      float part0 = 0.f, part1 = 0.f;
      for (int c0 = 0; c0 < cols; c0 += 32) {
        uint32_t x[32];
        tmem_ld32(lanes + (i & 1) * p.pitch + c0, x);
        tmem_wait_ld();
        if (c0 + 32 <= cols && __all_sync(0xffffffffu, from <= c0)) {
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            const float4 e = *reinterpret_cast<const float4*>(lse_s + c0 + k);
            part0 += ex2(fmaf(__uint_as_float(x[k]), p.scale_log2, e.x)) + ex2(fmaf(__uint_as_float(x[k + 1]), p.scale_log2, e.y));
            part1 += ex2(fmaf(__uint_as_float(x[k + 2]), p.scale_log2, e.z)) + ex2(fmaf(__uint_as_float(x[k + 3]), p.scale_log2, e.w));
          }
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            const float w = ex2(fmaf(__uint_as_float(x[k]), p.scale_log2, lse_s[c0 + k]));
            part0 += c0 + k >= from && c0 + k < cols ? w : 0.f;
          }
        }
      }
      sum += part0 + part1;
      tmem_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bar_sfree + 8 * (i & 1));
      if (grp + 1 == n_groups) {
        if (tok < len)
          p.mass[static_cast<int64_t>(row0 - p.row_base) * p.n_kv_heads + static_cast<int64_t>(head) * len + tok] = sum / static_cast<float>(obs * p.group);
        sum = 0.f;
      }
    }
    if (!ok)
      for (int i = 0; i < n_tiles; ++i) {
        const int tok = (tile0 + i) * kRows + r;
        if (tok < len) p.mass[static_cast<int64_t>(row0 - p.row_base) * p.n_kv_heads + static_cast<int64_t>(head) * len + tok] = NAN;
      }
  } else if (warp == 4) {
    if (elect()) {
      const int box_tokens = min(p.n_obs, p.group_tokens);
      const uint32_t q_bytes = 2u * box_tokens * p.group * 128u;
      bool ok = true;
      int i = 0, q_loads = 0, k_loads = 0;
      for (; ok && i < steps; ++i) {
        const int grp = i % n_groups, tile = i / n_groups;
        if (grp == 0) {
          const int slot = tile % kMStages, turn = tile / kMStages;
          ok = turn == 0 || bar_wait(bar_empty + 8 * slot, (turn - 1) & 1, abort);
          if (!ok) break;
          bar_expect(bar_full + 8 * slot, kTileBytes);
          for (int h = 0; h < 2; ++h)
            tma_load_3d(smem + slot * kTileBytes + h * kPanel, &map_k, 64 * h, head, row0 + (tile0 + tile) * kRows, bar_full + 8 * slot);
          ++k_loads;
        }
        if (i == 0 || n_groups > 1) {
          ok = i == 0 || bar_wait(bar_qfree, (i - 1) & 1, abort);
          if (!ok) break;
          bar_expect(bar_q, q_bytes);
          for (int h = 0; h < 2; ++h)
            tma_load_3d(smem + kMOffQ + h * p.n_pad * 128, &map_q, 64 * h, head * p.group, row0 + obs0 + grp * p.group_tokens, bar_q);
          ++q_loads;
        }
      }
      if (*abort) {
        if (q_loads) bar_drain(bar_q, (q_loads - 1) & 1);
        for (int k = max(0, k_loads - kMStages); k < k_loads; ++k) bar_drain(bar_full + 8 * (k % kMStages), (k / kMStages) & 1);
      }
    }
  } else {
    if (elect()) {
      const uint32_t idesc = instr_desc(true, false, kRows, p.n_pad);
      bool ok = true;
      for (int i = 0; i < steps; ++i) {
        const int grp = i % n_groups, tile = i / n_groups, slot = tile % kMStages;
        ok = (grp > 0 || bar_wait(bar_full + 8 * slot, (tile / kMStages) & 1, abort)) &&
             ((i > 0 && n_groups == 1) || bar_wait(bar_q, i & 1, abort)) && (i < 2 || bar_wait(bar_sfree + 8 * (i & 1), ((i >> 1) - 1) & 1, abort));
        if (!ok) break;
        tmem_after();
        const uint64_t a = smem_desc(smem + slot * kTileBytes, 16), b = smem_desc(smem + kMOffQ, 16);
        for (int k = 0; k < kD / 16; ++k)
          mma_ss(tmem + (i & 1) * p.pitch, a + (((k >> 2) * kPanel + (k & 3) * 32) >> 4), b + (((k >> 2) * p.n_pad * 128 + (k & 3) * 32) >> 4), idesc, k > 0);
        mma_commit(bar_s + 8 * (i & 1));
        if (n_groups > 1) mma_commit(bar_qfree);
        if (grp + 1 == n_groups) mma_commit(bar_empty + 8 * slot);
      }
      if (!ok) {
        mma_commit(bar_drain_mma);
        bar_drain(bar_drain_mma, 0);
      }
    }
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  if (warp == 5) tmem_dealloc(tmem, p.tmem_cols);
}

// ---- host ----------------------------------------------------------------------------------------
std::atomic<uint64_t> g_prompt_few{0}, g_prompt_many{0}, g_mass_few{0}, g_mass_many{0};

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Bounds, layout and place of the call's rows.  `rows`: rows up to the end of the last sequence.
int check_prompt(const gkv_prompt* d, int* rows) {
  if (!d || d->struct_size != sizeof(gkv_prompt) || d->abi_version != GKV_ABI_VERSION) return GKV_ERR_INVALID_ARG;
  if (d->n_seqs < 0 || d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->n_q_heads % d->n_kv_heads != 0) return GKV_ERR_INVALID_ARG;
  if (d->head_dim != kD || d->n_q_heads / d->n_kv_heads > kMaxHeadsPerKv) return GKV_ERR_UNSUPPORTED;
  if (!d->offsets || d->offsets[0] < 0) return GKV_ERR_INVALID_ARG;
  for (int i = 0; i < d->n_seqs; ++i)
    if (d->offsets[i + 1] < d->offsets[i]) return GKV_ERR_INVALID_ARG;
  const int64_t nq = static_cast<int64_t>(d->n_q_heads) * kD, nkv = static_cast<int64_t>(d->n_kv_heads) * kD;
  const int64_t strides[4] = {d->q_stride, d->k_stride, d->v_stride, d->out_stride};
  for (int i = 0; i < 4; ++i)      // (2^36 elements: what a tensor map takes as a stride in bytes)
    if (strides[i] != 0 && (strides[i] < (i == 0 || i == 3 ? nq : nkv) || strides[i] % 8 != 0 || strides[i] >= int64_t{1} << 36)) return GKV_ERR_INVALID_ARG;
  *rows = d->offsets[d->n_seqs];
  return GKV_OK;
}

// A map of [rows][heads][128] 16-bit elements: boxes of 64 channels x `heads_box` heads x `rows_box` rows.  Rows are `stride` elements apart.
bool make_rows_map(CUtensorMap* map, const void* base, int64_t rows, int heads, int64_t stride, int heads_box, int rows_box) {
  const uint64_t dims[3] = {kD, static_cast<uint64_t>(heads), static_cast<uint64_t>(rows)}, strides[2] = {kD * 2, static_cast<uint64_t>(stride) * 2};
  const uint32_t box[3] = {64, static_cast<uint32_t>(heads_box), static_cast<uint32_t>(rows_box)};
  return make_map(map, base, 3, dims, strides, box);
}

// Sequences [begin, end) with rows, longest first, `per` tokens to a work item.
template <int N>
int deal(Seqs<N>& s, const int32_t* offsets, const std::vector<int>& order, int begin, int end, int per) {
  s.n = end - begin;
  s.first[0] = 0;
  for (int i = 0; i < s.n; ++i) {
    const int q = order[begin + i];
    s.row[i] = offsets[q];
    s.len[i] = offsets[q + 1] - offsets[q];
    s.first[i + 1] = s.first[i] + (s.len[i] + per - 1) / per;
  }
  return s.first[s.n];
}
std::vector<int> longest_first(const gkv_prompt* d) {
  std::vector<int> order;
  for (int i = 0; i < d->n_seqs; ++i)
    if (d->offsets[i + 1] > d->offsets[i]) order.push_back(i);
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return d->offsets[a + 1] - d->offsets[a] > d->offsets[b + 1] - d->offsets[b]; });
  return order;
}

template <int N>
cudaError_t launch_prompt(PromptParams& p, const gkv_prompt* d, const std::vector<int>& order, int begin, int end, const CUtensorMap* maps, std::atomic<uint64_t>& done,
                          cudaStream_t st) {
  Seqs<N> s;
  const int items = deal(s, d->offsets, order, begin, end, 2 * p.tile_tokens);
  cudaError_t e = raise_smem_limit(prompt_kernel<N>, kPSmem, done);
  if (e != cudaSuccess) return e;
  prompt_kernel<N><<<items * p.n_kv_heads, kPThreads, kPSmem, st>>>(p, s, maps[0], maps[1], maps[2]);
  return cudaGetLastError();
}
template <int N>
cudaError_t launch_mass(MassParams& p, const gkv_prompt* d, const std::vector<int>& order, int begin, int end, const CUtensorMap* maps, size_t smem,
                        std::atomic<uint64_t>& done, cudaStream_t st) {
  Seqs<N> s;
  const int tiles = deal(s, d->offsets, order, begin, end, kRows);
  // a few CTAs per SM; beyond that a CTA takes more tiles and loads its queries once
  p.chunk = std::max(1, std::min(8, tiles * p.n_kv_heads / (3 * 148)));
  const int items = deal(s, d->offsets, order, begin, end, kRows * p.chunk);
  cudaError_t e = raise_smem_limit(mass_kernel<N>, kMOffQ + kMaxObsRows * 256 + 1024, done);
  if (e != cudaSuccess) return e;
  mass_kernel<N><<<items * p.n_kv_heads, kMThreads, smem, st>>>(p, s, maps[0], maps[1]);
  return cudaGetLastError();
}

float scale_of(const gkv_prompt* d) { return (d->softmax_scale > 0.f ? d->softmax_scale : static_cast<float>(1.0 / std::sqrt(static_cast<double>(kD)))) * kLog2e; }

}  // namespace

// Device memory of the current device (or memory that every device reaches): the kernels must not be given another GPU's.
bool on_current_device(std::initializer_list<const void*> ptrs) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  for (const void* p : ptrs) {
    if (!p) continue;
    cudaPointerAttributes a{};
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
      cudaGetLastError();
      return false;
    }
    if (a.type != cudaMemoryTypeManaged && (a.type != cudaMemoryTypeDevice || a.device != dev)) return false;
  }
  return true;
}

// A map of 16-bit elements with the 128-byte swizzle; strides of all dimensions but the first, in bytes.
bool make_map(CUtensorMap* map, const void* base, int n, const uint64_t* dims, const uint64_t* strides, const uint32_t* box) {
  using Encode = decltype(&cuTensorMapEncodeTiled);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found{};
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return false;
  cuuint64_t d[5], s[4];
  cuuint32_t b[5], step[5];
  for (int i = 0; i < n; ++i) {
    d[i] = dims[i];
    b[i] = box[i];
    step[i] = 1;
    if (i) s[i - 1] = strides[i - 1];
  }
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, n, const_cast<void*>(base), d, s, b, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace gkv

using namespace gkv;

int gkv_prompt_attn(const gkv_prompt* d, const void* q, const void* k, const void* v, void* out, float* lse, void* stream) {
  int rows = 0;
  const int rc = check_prompt(d, &rows);
  if (rc != GKV_OK) return rc;
  const std::vector<int> order = longest_first(d);
  if (order.empty()) return GKV_OK;
  if (!q || !k || !v || !out || misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16) || misaligned(lse, 4)) return GKV_ERR_INVALID_ARG;
  if (!on_current_device({q, k, v, out, lse})) return GKV_ERR_INVALID_ARG;
  const int64_t nq = static_cast<int64_t>(d->n_q_heads) * kD, nkv = static_cast<int64_t>(d->n_kv_heads) * kD;
  PromptParams p{};
  p.out = static_cast<uint16_t*>(out);
  p.lse = lse;
  p.out_stride = d->out_stride ? d->out_stride : nq;
  p.n_q_heads = d->n_q_heads;
  p.n_kv_heads = d->n_kv_heads;
  p.group = d->n_q_heads / d->n_kv_heads;
  p.tile_tokens = kRows / p.group;
  p.scale_log2 = scale_of(d);
  CUtensorMap maps[3];
  if (!make_rows_map(&maps[0], q, rows, d->n_q_heads, d->q_stride ? d->q_stride : nq, p.group, p.tile_tokens) ||
      !make_rows_map(&maps[1], k, rows, d->n_kv_heads, d->k_stride ? d->k_stride : nkv, 1, kRows) ||
      !make_rows_map(&maps[2], v, rows, d->n_kv_heads, d->v_stride ? d->v_stride : nkv, 1, kRows))
    return GKV_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int n = static_cast<int>(order.size());
  for (int at = 0; at < n; at += kMaxSeqs) {
    const int end = std::min(n, at + kMaxSeqs);
    const cudaError_t e = end - at <= kFewSeqs ? launch_prompt<kFewSeqs>(p, d, order, at, end, maps, g_prompt_few, st)
                                               : launch_prompt<kMaxSeqs>(p, d, order, at, end, maps, g_prompt_many, st);
    if (e != cudaSuccess) return GKV_ERR_CUDA;
  }
  return GKV_OK;
}

int gkv_prompt_mass(const gkv_prompt* d, const void* q, const void* k, const float* lse, int32_t n_obs, float* mass, void* stream) {
  int rows = 0;
  const int rc = check_prompt(d, &rows);
  if (rc != GKV_OK) return rc;
  if (n_obs <= 0) return GKV_ERR_INVALID_ARG;
  const std::vector<int> order = longest_first(d);
  if (order.empty()) return GKV_OK;
  if (!q || !k || !lse || !mass || misaligned(q, 16) || misaligned(k, 16) || misaligned(lse, 4) || misaligned(mass, 4)) return GKV_ERR_INVALID_ARG;
  if (!on_current_device({q, k, lse, mass})) return GKV_ERR_INVALID_ARG;
  const int64_t nq = static_cast<int64_t>(d->n_q_heads) * kD, nkv = static_cast<int64_t>(d->n_kv_heads) * kD;
  MassParams p{};
  p.lse = lse;
  p.mass = mass;
  p.row_base = d->offsets[0];
  p.n_q_heads = d->n_q_heads;
  p.n_kv_heads = d->n_kv_heads;
  p.group = d->n_q_heads / d->n_kv_heads;
  p.n_obs = n_obs;
  p.group_tokens = std::min(n_obs, kMaxObsRows / p.group);
  p.n_pad = (p.group_tokens * p.group + 15) / 16 * 16;
  p.pitch = (p.n_pad + 31) / 32 * 32;
  p.tmem_cols = 64;
  while (p.tmem_cols < 2 * p.pitch) p.tmem_cols *= 2;
  p.scale_log2 = scale_of(d);
  CUtensorMap maps[2];
  if (!make_rows_map(&maps[0], q, rows, d->n_q_heads, d->q_stride ? d->q_stride : nq, p.group, p.group_tokens) ||
      !make_rows_map(&maps[1], k, rows, d->n_kv_heads, d->k_stride ? d->k_stride : nkv, 1, kRows))
    return GKV_ERR_CUDA;
  const size_t smem = kMOffQ + static_cast<size_t>(p.n_pad) * 256 + 1024;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int n = static_cast<int>(order.size());
  for (int at = 0; at < n; at += kMaxSeqs) {
    const int end = std::min(n, at + kMaxSeqs);
    const cudaError_t e = end - at <= kFewSeqs ? launch_mass<kFewSeqs>(p, d, order, at, end, maps, smem, g_mass_few, st)
                                               : launch_mass<kMaxSeqs>(p, d, order, at, end, maps, smem, g_mass_many, st);
    if (e != cudaSuccess) return GKV_ERR_CUDA;
  }
  return GKV_OK;
}
