// Causal attention of row tiles over key steps on the fifth-generation tensor cores: what prompts (gkv_prompt.cu) and chunks of many rows (gkv_dense.cu)
// have in common.
//
// A CTA works on tiles of 256 rows in two halves; the rows of a half are the g query heads of 128 / g consecutive tokens, so that all of them read one KV
// head and the diagonal is 128 / g tokens wide.  Per step of 128 keys and half:
//   S = Q K^T            both operands in shared memory, fp32 accumulator in tensor memory (where keys are pairs, + Q K_lo^T)
//   m' = max(m, row max) the reference m moves only when the maximum has grown by more than 2^8: P then stays below 2^8 (2^15 as fp16: kUp), and the
//                        accumulator is rescaled a handful of times per row, not once per step
//   P = exp2(c S - c m)  16 bits, over S in tensor memory; its sum l is taken before it is rounded
//   O += P V             P from tensor memory, V as it lies ([token][channel], MN-major); it starts on three quarters of P
// While four warps work on one half's S, the tensor cores work for the other half: the products are issued by one thread in the order P0 V, Q0 K,
// P1 V, Q1 K.  Queries, keys and values come by TMA, keys and values through a ring of 32 KB stages.
//
// What bounds it: a half's chain of a step is 216 cycles to the maximum, 1490 for 128 exponentials a thread (1024 of the special-function unit), 400 until the
// product is issued and 1160 for the rest of P V and Q K, 3010 in all for 2048 cycles of matrix products of both halves; 16,384 tokens of 16
// query heads take 815 us, 1.35 PFLOP/s, ten times in a row, and 957 over seconds under the power limit (0.83 of what cuBLAS sustains there).  Evaluating a share of the exponentials by a polynomial on
// the FMA pipe gained nothing (1/8 and 1/4 of them: 0.99 and 0.97 of the rate): the clock falls by what the pipes gain.
//
// Work split.  One CTA per SM.  Either all tiles' steps are laid end to end and cut into equal ranges, one per CTA (gkv_chunk.h), and a tile that was cut
// leaves partial results in slots; or, where no tile is long enough for that to pay, a CTA has a whole tile and goes on
// with those of CTAs that have not been launched yet (cluster launch control), heaviest first.  A warp works out the
// CTA's parts ahead of the others (1250 cycles each, as much for constant memory as for arithmetic), and the next part's queries and keys are on
// their way while the results of this one are written.  A part costs 8,000 to 10,000 cycles beside its steps: its halves begin together and share the
// exponentials (the first step takes 5400), the last products end (2500), the rows leave (2600).
#pragma once
#include <cuda_runtime.h>

#include <cstring>

#include "gkv_chunk.h"
#include "gkv_internal.h"
#include "gkv_tc.cuh"

namespace gkv {
namespace attend {

using namespace tc;

constexpr int kRows = 128;                 // rows of a half, keys of a step
constexpr int kPanel = kRows * 128;        // bytes of 64 channels of 128 rows
constexpr int kTileBytes = 2 * kPanel;
constexpr int kThreads = 384;              // softmax of the halves (four warps each), loads, products, value rows behind a sequence, parts
constexpr int kStages = 5;
constexpr int kOffStage = 2 * kTileBytes, kOffBar = kOffStage + kStages * kTileBytes;
constexpr int kParts = 3, kOffParts = kOffBar + 336, kOffLeft = kOffParts + kParts * 64, kSmem = kOffLeft + 80 + 1024;
constexpr int kLaunchRegs = 168, kSoftRegs = 216, kOtherRegs = 72;
static_assert(2 * kSoftRegs + kOtherRegs <= 3 * kLaunchRegs, "a split draws on the launch's registers");
constexpr int kStart = 2, kSnap = 1;        // steps that a part's beginning and end cost (chunk_plan); how near to a tile's end a cut is not worth slots
constexpr float kSlack = 8.f;              // log2 of what a weight may exceed 1 by before the reference moves
// log2 of what all weights are multiplied by.  As fp16 they then reach from 2^15 (a row's maximum kSlack above its reference) down to 2^-14 with all their
// bits: 2^-21 of the reference's, where 2^-14 was off by a hundredth of the norm behind a key that leads the others by 14.5 nats.
template <class Work>
constexpr float kUp = Work::kBf16 ? 0.f : 7.f;
constexpr int kEarly = 6;                  // k-steps of P V that start early, of eight

// A CTA's part of a tile, as `Work::next` describes it.
struct alignas(16) Part {
  int64_t row0;                            // output row of token 0
  int tile, items, begin, end;             // steps [begin, end) of the tile's `items`; tile -1: no more
  int tok0, len, causal0;                  // first token of the tile, tokens of the sequence; step whose first key is token 0
  int head0, kv, q_row;                    // first query head; what the loads of keys and queries go by
  int slot;                                // where a part of a cut tile goes, -1 = the tile is whole
  bool two;                                // the second half has rows
  uint8_t keep;                            // value rows of the last step that count, 128 = all
};
static_assert(sizeof(Part) == 64, "");
// What the warp that works out the parts leaves: how many it published, and after a given-up wait the part that it had in hand, with the walk's state.
struct Left {
  Part part;
  int published, hand, state, slot;
};
static_assert(sizeof(Left) == 80 && kSmem <= 227 * 1024, "");
struct Maps {
  CUtensorMap q, k, k_lo, v;
};

// Work: kBf16 (else fp16), kPairs (steps may have K_lo and a term per key); group, n_q_heads, half_tokens, scale_log2, out, out_stride, lse, part_o,
// part_ml (slots: [128 channels][256 rows], [256 rows]), and on the device
//   next(state, slot, part)              the CTA's next part; state (at first 0) and slot (at first first_slot()) are the walk's
//   whole_tiles(), whole(tile, part)     CTAs have whole tiles, a CTA per tile launched; the tile of that number
//   ln2_rest                             see lse_of
//   load_q(map, dst, part, t, bar)       half t's queries (two panels of half_tokens * group rows)
//   load_keys(map, dst, part, step, bar) a step's 128 rows (two panels)
//   flags(part, step), term(part, step)  kPairs only
//   place(tile)                          where a tile lies (tok0, len, row0, head0)
//   fail()                               a wait was given up (the rows of the CTA's parts that are not done are NaN)
constexpr int kHasTerm = 1, kHasLow = 2;

// The log-sum-exp of weights 2^(x - top) that sum to `sum`; ln2_rest: what a logit is more of itself than its 32 bits say
template <class Work>
__device__ __forceinline__ float lse_of(const Work& work, float top, float sum) {
  return fmaf(top, kLn2, fmaf(top, work.ln2_rest, lg2(sum) * kLn2));
}

// NaN for the rows of a part, or into its slot, from which the merge takes it on
template <class Work>
__device__ __forceinline__ void spoil(const Work& work, const Part& x) {
  for (int i = threadIdx.x; i < 2 * work.half_tokens * work.group; i += kThreads) {
    const int tok = x.tok0 + i / work.group;
    if (tok >= x.len) continue;
    if (x.slot >= 0) {
      work.part_ml[static_cast<size_t>(x.slot) * 2 * kRows + i] = make_float2(NAN, NAN);
      continue;
    }
    const int64_t row = x.row0 + tok;
    const int head = x.head0 + i % work.group;
    uint4* const to = reinterpret_cast<uint4*>(work.out + row * work.out_stride + head * kD);
#pragma unroll 1
    for (int k = 0; k < kD / 8; ++k) to[k] = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    if (work.lse) work.lse[row * work.n_q_heads + head] = NAN;
  }
}
// (a function of its own: inside the kernel it cost others their registers, 84 -> 85.5 us of a batch of prompts)
template <class Work>
__device__ __noinline__ void spoil_left(const Work& work, const Part* ring, const Left* left) {
  int state = left->state, slot = left->slot;
  parts_left<kParts>(
      ring, left->published, left->hand != 0, left->part, [&](Part& x) { return !work.whole_tiles() && work.next(state, slot, x); },
      [&](const Part& x) { spoil(work, x); });
  if (threadIdx.x == 0) work.fail();
}

template <class Work>
__global__ void __launch_bounds__(kThreads, 1) attend_kernel(const __grid_constant__ Work work, const __grid_constant__ Maps maps) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base = smem_raw + (smem - smem_u32(smem_raw));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bars = smem + kOffBar;
  const uint32_t bar_q = bars, bar_qfree = bars + 8, bar_s = bars + 16, bar_pa = bars + 32, bar_p = bars + 48, bar_o = bars + 64, bar_last = bars + 80, bar_fix = bars + 88;
  const uint32_t bar_done = bars + 96, bar_full = bars + 104, bar_empty = bar_full + 8 * kStages;
  const uint32_t bar_put = bar_empty + 8 * kStages, bar_got = bar_put + 8 * kParts, bar_call = bar_got + 8 * kParts, bar_more = bar_call + 8, answer = bars + 320;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(base + kOffBar + 304);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base + kOffBar + 308);
  static_assert(120 + 16 * kStages + 16 * kParts <= 304, "room for the barriers");
  Part* const ring = reinterpret_cast<Part*>(base + kOffParts);
  Left* const left = reinterpret_cast<Left*>(base + kOffLeft);

  if (threadIdx.x == 0) {
    bar_init(bar_q, 1);
    bar_init(bar_qfree, 1);
    for (int t = 0; t < 2; ++t) {
      bar_init(bar_s + 8 * t, 1);
      bar_init(bar_pa + 8 * t, 4);
      bar_init(bar_p + 8 * t, 4);
      bar_init(bar_o + 8 * t, 1);
    }
    bar_init(bar_last, 1);
    bar_init(bar_fix, 1);
    bar_init(bar_done, 1);
    bar_init(bar_call, 1);
    bar_init(bar_more, 1);
    for (int i = 0; i < kStages; ++i) {
      bar_init(bar_full + 8 * i, 1);
      bar_init(bar_empty + 8 * i, 1);
    }
    for (int i = 0; i < kParts; ++i) {
      bar_init(bar_put + 8 * i, 1);
      bar_init(bar_got + 8 * i, 11);         // eight warps of the softmax, loads, products, zeroed rows
    }
    *abort = 0;
    bar_init_fence();
  }
  if (threadIdx.x == 256) {
    prefetch_map(&maps.q);
    prefetch_map(&maps.k);
    prefetch_map(&maps.v);
  }
  if (warp == 9) {                         // (no tensor memory is held while the kernel in front, which may still want some, is waited for)
    pdl_wait();
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
  }
  // the CTA's first part is worked out while tensor memory is allocated: it comes of the parameters alone
  Part x;
  int state = 0, slot = 0;
  bool more = false;
  if (warp == 11) {
    slot = work.first_slot();
    more = work.whole_tiles();
    if (more) work.whole(blockIdx.x, x);
    else more = work.next(state, slot, x);
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_launch();
  // The n-th part: false at the end, or after an abort.  Whoever has read it says so.
  auto part = [&](int n, Part& x) {
    if (!bar_wait(bar_put + 8 * (n % kParts), (n / kParts) & 1, abort)) return false;
    const uint4* from = reinterpret_cast<const uint4*>(&ring[n % kParts]);
    uint4 w[4];
    for (int i = 0; i < 4; ++i) w[i] = from[i];
    memcpy(&x, w, sizeof(x));
    return x.tile >= 0;
  };
  auto part_read = [&](int n) { bar_arrive(bar_got + 8 * (n % kParts)); };

  if (warp < 8) {
    more_regs<kSoftRegs>();
    const int t = warp >> 2;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp & 3) << 21);
    const uint32_t s_tm = lanes + t * kRows, o_tm = lanes + 256 + t * kRows;
    const int r = (warp & 3) * 32 + lane, tok_in = r / work.group, slot_row = t * work.half_tokens * work.group + r;
    const float c = work.scale_log2;
    int steps = 0, done = 0;
    bool ok = true;
    for (int n = 0; ok && part(n, x); ++n) {
      __syncwarp();
      if (lane == 0) part_read(n);
      const int to = x.slot;
      if (t && !x.two) continue;
      const int tok = x.tok0 + t * work.half_tokens + tok_in;
      const bool real = tok_in < work.half_tokens && tok < x.len;
      const int first_tok = x.tok0 + t * work.half_tokens + (warp & 3) * 32 / work.group;      // of the warp's rows
      float m = -INFINITY, l = 0.f;
      for (int j = x.begin; j < x.end; ++j) {
        const int flag = Work::kPairs ? work.flags(x, j) : 0;
        if (!(ok = bar_wait(bar_s + 8 * t, steps & 1, abort))) break;
        ++steps;
        tmem_after();
        uint32_t v[kRows];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld32(s_tm + 32 * i, v + 32 * i);
        tmem_wait_ld();
        if (Work::kPairs && (flag & kHasTerm)) {
          const float4* add = reinterpret_cast<const float4*>(work.term(x, j));
#pragma unroll
          for (int i = 0; i < kRows / 4; ++i) {
            const float4 a = __ldg(add + i);
            v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + a.x);
            v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + a.y);
            v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + a.z);
            v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + a.w);
          }
        }
        if (j >= x.causal0 && (j - x.causal0 + 1) * kRows - 1 > first_tok) {
          const int limit = tok - (j - x.causal0) * kRows;         // last key of the step that the row sees
#pragma unroll
          for (int i = 0; i < kRows; ++i)
            if (i > limit) v[i] = 0xff800000u;
        }
        float mx[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) mx[k] = max3(__uint_as_float(v[3 * k]), __uint_as_float(v[3 * k + 1]), __uint_as_float(v[3 * k + 2]));
#pragma unroll
        for (int i = 12; i < kRows; i += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (i + 2 * k < kRows) mx[k] = max3(mx[k], __uint_as_float(v[i + 2 * k]), __uint_as_float(v[i + 2 * k + 1]));
        const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
        const bool first = m == -INFINITY;
        const bool move = first ? top > -INFINITY : (top - m) * c > kSlack;
        // (S of this step was issued behind O of the one before: a row's accumulator is complete when its logits are there)
        if (__any_sync(0xffffffffu, move && !first)) {
          const float f = move && !first ? ex2((m - top) * c) : 1.f;
          l *= f;
          const uint64_t ff = f2_pack(f, f);
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            uint32_t o[16];
            tmem_ld16(o_tm + 16 * i, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
              float a, b;
              f2_unpack(f2_mul(f2_pack(__uint_as_float(o[k]), __uint_as_float(o[k + 1])), ff), a, b);
              o[k] = __float_as_uint(a);
              o[k + 1] = __float_as_uint(b);
            }
            tmem_st16(o_tm + 16 * i, o);
          }
        }
        if (move) m = top;
        const float at = m == -INFINITY ? 0.f : fmaf(-m, c, kUp<Work>);
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
            pk[k] = Work::kBf16 ? bf16_pair(a, b) : f16_pair(a, b);
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
      ok = ok && bar_wait(bar_o + 8 * t, done & 1, abort);
      ++done;
      tmem_after();
      // (a row that a given-up wait leaves without its result gets NaN)
      const int hq = x.head0 + r % work.group;
      const int64_t row = x.row0 + tok;
      const float inv = !ok ? NAN : to < 0 ? 1.f / l : 1.f;
      uint32_t o[kD];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32(o_tm + 32 * i, o + 32 * i);
      tmem_wait_ld();
#pragma unroll
      for (int k = 0; k < kD; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * inv);
      if (to >= 0) {                           // channel after channel: a warp's 32 rows are 128 bytes
        if (real) {
          float* dst = work.part_o + static_cast<size_t>(to) * kD * 2 * kRows + slot_row;
#pragma unroll
          for (int k = 0; k < kD; ++k) dst[k * 2 * kRows] = __uint_as_float(o[k]);
        }
      } else {
        // Four lanes exchange their rows' 16-byte pieces, so that 64 bytes of a row are stored at a time.  (Rows stored by a lane each kept the
        // load and store unit busy for 4096 cycles, and the barriers of the other warps waited behind them.)
        uint16_t* const mine = real ? work.out + row * work.out_stride + hq * kD : nullptr;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          uint32_t w[4][4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) w[j][k] = bf16_pair(__uint_as_float(o[32 * n + 8 * j + 2 * k]), __uint_as_float(o[32 * n + 8 * j + 2 * k + 1]));
#pragma unroll
          for (int d = 1; d < 4; d <<= 1)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (!(j & d))
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const uint32_t got = __shfl_xor_sync(0xffffffffu, lane & d ? w[j][k] : w[j | d][k], d);
                  if (lane & d) w[j][k] = got;
                  else w[j | d][k] = got;
                }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint4* const dst = reinterpret_cast<uint4*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), (lane & 28) | j));
            if (dst) dst[4 * n + (lane & 3)] = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
          }
        }
      }
      if (real) {
        if (to >= 0) work.part_ml[static_cast<size_t>(to) * 2 * kRows + slot_row] = make_float2(fmaf(m, c, -kUp<Work>), ok ? l : NAN);
        else if (work.lse) work.lse[row * work.n_q_heads + hq] = ok ? lse_of(work, fmaf(m, c, -kUp<Work>), l) : NAN;
      }
      tmem_before();
    }
  } else {
    fewer_regs<kOtherRegs>();
    if (warp == 8) {
      // ---- loads: per step keys, K_lo where they are pairs, values ----
      if (elect()) {
        int i = 0, n = 0;                      // stages filled, parts begun
        bool ok = true;
        const uint32_t q_bytes = 2u * work.half_tokens * work.group * 128u;
        auto load = [&](const CUtensorMap* map, int step) {
          const int slot = i % kStages, turn = i / kStages;
          if (turn > 0 && !bar_wait(bar_empty + 8 * slot, (turn - 1) & 1, abort)) return false;
          bar_expect(bar_full + 8 * slot, kTileBytes);
          work.load_keys(map, smem + kOffStage + slot * kTileBytes, x, step, bar_full + 8 * slot);
          ++i;
          return true;
        };
        for (; ok && part(n, x); ++n) {
          part_read(n);
          if (n > 0 && !(ok = bar_wait(bar_qfree, (n - 1) & 1, abort))) break;
          bar_expect(bar_q, x.two ? 2 * q_bytes : q_bytes);
          for (int t = 0; t < (x.two ? 2 : 1); ++t) work.load_q(&maps.q, smem + t * kTileBytes, x, t, bar_q);
          int flag = Work::kPairs ? work.flags(x, x.begin) : 0;
          for (int j = x.begin; ok && j < x.end; ++j) {
            if (j == x.end - 1) bar_arrive(bar_more);
            const int now = flag;
            if (Work::kPairs && j + 1 < x.end) flag = work.flags(x, j + 1);
            ok = load(&maps.k, j) && (!(now & kHasLow) || load(&maps.k_lo, j)) && load(&maps.v, j);
          }
        }
        if (*abort) {                          // what is on its way arrives before the CTA leaves
          for (int k = max(0, n - 1); k <= n; ++k) bar_drain(bar_q, k & 1);
          for (int k = max(0, i - kStages); k < i; ++k) bar_drain(bar_full + 8 * (k % kStages), (k / kStages) & 1);
        }
      }
    } else if (warp == 9) {
      // ---- products ----
      if (elect()) {
        constexpr uint32_t id_qk = instr_desc(Work::kBf16, false, kRows, kRows), id_pv = instr_desc(Work::kBf16, true, kRows, kD);
        bool ok = true;
        int at = 0, fixes = 0, weights[2] = {0, 0};      // the next stage; value steps with rows zeroed; steps whose weights were waited for
        auto wait_stage = [&](int i) { return bar_wait(bar_full + 8 * (i % kStages), (i / kStages) & 1, abort); };
        auto free_stage = [&](int i) { mma_commit(bar_empty + 8 * (i % kStages)); };
        auto qk = [&](int t, int i, bool add) {
          const uint64_t a = smem_desc(smem + t * kTileBytes, 16), b = smem_desc(smem + kOffStage + (i % kStages) * kTileBytes, 16);
          for (int k = 0; k < kD / 16; ++k) {
            const uint32_t off = ((k >> 2) * kPanel + (k & 3) * 32) >> 4;
            mma_ss(tmem + t * kRows, a + off, b + off, id_qk, add || k > 0);
          }
        };
        auto pv = [&](int t, int i, bool first, int from, int to) {
          const uint64_t b = smem_desc(smem + kOffStage + (i % kStages) * kTileBytes, kPanel);
          for (int k = from; k < to; ++k) mma_ts(tmem + 256 + t * kRows, tmem + t * kRows + 8 * k, b + ((k * 16 * 128) >> 4), id_pv, !first || k > 0);
        };
        for (int n = 0; ok && part(n, x); ++n) {
          part_read(n);
          const int halves = x.two ? 2 : 1;
          bool low = Work::kPairs && (work.flags(x, x.begin) & kHasLow);
          ok = bar_wait(bar_q, n & 1, abort) && wait_stage(at) && (!low || wait_stage(at + 1));
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
            low = Work::kPairs && more && (work.flags(x, j + 1) & kHasLow);
            ok = wait_stage(v) && (!more || wait_stage(k)) && (!low || wait_stage(k + 1));
            if (ok && x.keep < kRows && j + 1 == x.items) {      // warp 10 zeroes the rows behind the sequence
              bar_arrive(bar_last);
              ok = bar_wait(bar_fix, fixes & 1, abort);
              ++fixes;
            }
            for (int t = 0; t < halves && ok; ++t) {
              ok = bar_wait(bar_pa + 8 * t, weights[t] & 1, abort);
              if (!ok) break;
              tmem_after();
              pv(t, v, j == x.begin, 0, kEarly);
              ok = bar_wait(bar_p + 8 * t, weights[t] & 1, abort);
              if (!ok) break;
              ++weights[t];
              tmem_after();
              pv(t, v, j == x.begin, kEarly, kRows / 16);
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
        if (!ok) {                             // products in flight end before tensor memory is given back
          mma_commit(bar_done);
          bar_drain(bar_done, 0);
        }
      }
    } else if (warp == 10) {
      // ---- value rows behind a sequence may hold anything: zeros (their weights are zero) ----
      int at = 0, fixes = 0;
      for (int n = 0; part(n, x); ++n) {
        __syncwarp();
        if (lane == 0) part_read(n);
        if (Work::kPairs) continue;            // (such rows were written as zeros)
        at += 2 * (x.end - x.begin);
        if (x.keep == kRows || x.end < x.items) continue;
        if (!bar_wait(bar_last, fixes & 1, abort)) break;
        ++fixes;
        const uint32_t v = smem + kOffStage + (at - 1) % kStages * kTileBytes;
        for (int k = x.keep * 8 + lane; k < kRows * 8; k += 32) {
          sts128(v + k * 16, make_uint4(0, 0, 0, 0));
          sts128(v + kPanel + k * 16, make_uint4(0, 0, 0, 0));
        }
        fence_async();
        __syncwarp();
        if (lane == 0) bar_arrive(bar_fix);
      }
    } else if (elect()) {
      // ---- the CTA's parts ----
      // Whole tiles: the CTA's own, then those of CTAs that have not been launched yet and are called off here (heaviest first, as they come)
      const bool whole = work.whole_tiles();
      uint32_t tile = blockIdx.x;
      bool hand = false;
      int n = 0;
      for (;; ++n) {
        if (n > 0 && whole) {
          // not before the last step of the tile before is being loaded: a tile called off early is one that no idle CTA can have
          if (!bar_wait(bar_more, (n - 1) & 1, abort)) break;
          fence_async();
          bar_expect(bar_call, 16);
          call_off(answer, bar_call);
          if (!bar_wait(bar_call, (n - 1) & 1, abort)) {
            bar_drain(bar_call, (n - 1) & 1);
            hand = bar_poll(bar_call, (n - 1) & 1) && called_off(answer, tile);
            if (hand) work.whole(tile, x);
            break;
          }
          more = called_off(answer, tile);
          if (more) work.whole(tile, x);
        } else if (n > 0) {
          more = work.next(state, slot, x);
        }
        if (!more) x.tile = -1;
        hand = more;
        if (n >= kParts && !bar_wait(bar_got + 8 * (n % kParts), (n / kParts - 1) & 1, abort)) break;
        ring[n % kParts] = x;
        bar_arrive(bar_put + 8 * (n % kParts));
        hand = false;
        if (!more) {
          ++n;
          break;
        }
      }
      left->published = n;
      left->hand = hand;
      if (hand) {
        left->part = x;
        left->state = state;
        left->slot = slot;
      }
    }
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
  if (*abort) spoil_left(work, ring, left);      // (whoever was inside a part has written NaN itself)
}

// Merges the slots of tiles that were cut, in their order: 32 rows of a tile per CTA, a lane per row, 32 channels per warp.
template <class Work>
__global__ void __launch_bounds__(128) attend_merge_kernel(const __grid_constant__ Work work, const __grid_constant__ ChunkMerge merge) {
  __shared__ uint32_t turn[32 * 65];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = merge.slot[blockIdx.y], n = merge.slot[blockIdx.y + 1] - first;
  const auto at = work.place(merge.tile[blockIdx.y]);
  const int row = blockIdx.x * 32 + lane, rows = min(2 * work.half_tokens, at.len - at.tok0) * work.group;
  if (blockIdx.x * 32 >= rows) return;
  pdl_wait();
  pdl_launch();
  const float* const o0 = work.part_o + (static_cast<size_t>(first) * kD + 32 * warp) * 2 * kRows + row;
  const float2* const ml = work.part_ml + static_cast<size_t>(first) * 2 * kRows + row;
  float top = -INFINITY, sum = 0.f, o[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) o[k] = 0.f;
  if (row < rows) {
    for (int i = 0; i < n; ++i) {
      const float2 v = ml[static_cast<size_t>(i) * 2 * kRows];
      if (v.y != 0.f) top = fmaxf(top, v.x);
    }
    for (int i = 0; i < n; ++i) {
      const float2 v = ml[static_cast<size_t>(i) * 2 * kRows];
      float y[32];
#pragma unroll
      for (int k = 0; k < 32; ++k) y[k] = o0[(static_cast<size_t>(i) * kD + k) * 2 * kRows];
      const float f = v.y != 0.f ? ex2(v.x - top) : 0.f;
      sum += f * v.y;
#pragma unroll
      for (int k = 0; k < 32; ++k) o[k] = fmaf(f, y[k], o[k]);
    }
  }
  const float inv = 1.f / sum;
#pragma unroll
  for (int k = 0; k < 16; ++k) turn[lane * 65 + 16 * warp + k] = bf16_pair(o[2 * k] * inv, o[2 * k + 1] * inv);
  __syncthreads();
  for (int i = warp; i < 32 && blockIdx.x * 32 + i < rows; i += 4) {
    const int r = blockIdx.x * 32 + i, head = at.head0 + r % work.group;
    const int64_t line = at.row0 + at.tok0 + r / work.group;
    reinterpret_cast<uint2*>(work.out + line * work.out_stride + head * kD)[lane] = make_uint2(turn[i * 65 + 2 * lane], turn[i * 65 + 2 * lane + 1]);
  }
  if (warp == 0 && row < rows && work.lse) work.lse[(at.row0 + at.tok0 + row / work.group) * work.n_q_heads + at.head0 + row % work.group] = lse_of(work, top, sum);
}

// Launched while the kernel in front is still running, which lets it in (pdl_launch) and which it waits for (pdl_wait)
template <typename... Params, typename... Args>
cudaError_t launch_behind(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

}  // namespace attend
}  // namespace gkv
