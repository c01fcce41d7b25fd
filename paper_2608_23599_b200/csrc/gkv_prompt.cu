// Attention of whole prompts over their own exact rows, and the attention mass that their tokens get from the newest queries
// (Sec. 3.1, Eq. 2): what a serving program runs before it hands a prompt's rows to the bulk ingest.
//
// Attention: attend_kernel (gkv_attend.cuh) over tiles of the packed sequences, bf16 operands as they lie.
//
// mass_kernel.  S^T = K Q^T for the observing rows: a thread owns a token, so the sum over rows of exp2(c S - lse) needs no
// exchange, and every sum has a fixed order.  K is read once.  Few rows: K's bytes (57,000 tokens of 8 heads with 64 rows: 24.9 us for 116 MB,
// 0.71 of the copy's rate); many: 16 exponentials a cycle and SM (16,384 tokens of 2 heads with 512 rows: 12.8 us, 4 of them exponentials).
//
// Values of a sequence have to be finite; what lies behind a sequence's end may hold anything: its logits are masked by
// selection and its value rows are zeroed in shared memory before they are used.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <new>
#include <numeric>
#include <vector>

#include "../../include/gkv.h"
#include "gkv_attend.cuh"
#include "gkv_chunk.h"
#include "gkv_internal.h"
#include "gkv_tc.cuh"

namespace gkv {
namespace {

using namespace tc;

using attend::kPanel;
using attend::kRows;
using attend::kTileBytes;
constexpr int kMaxSeqs = 1024;             // sequences of one launch
constexpr int kFewSeqs = 32;               // the same where the parameters are short: 14 KB instead of 3 cost the host 5 us a call, of masses 2

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
// Tiles of a launch in the order (sequence, row tile from the last one on, KV head): those with most keys first.
template <int N>
struct Tiles {
  Seqs<N> seqs;                              // work items: row tiles
  int32_t n_kv_heads, span;                  // tokens of a tile
  __host__ __device__ int count() const { return seqs.first[seqs.n] * n_kv_heads; }
  struct Place {
    int seq, head, tok0, len;
  };
  __device__ __forceinline__ Place place(int tile) const {
    Place p;
    p.head = tile % n_kv_heads;
    const int item = tile / n_kv_heads;
    p.seq = find_seq(seqs, item);
    p.len = seqs.len[p.seq];
    p.tok0 = (seqs.first[p.seq + 1] - 1 - item) * span;
    return p;
  }
};
__host__ __device__ inline int steps_of(int tok0, int span, int len) { return ((tok0 + span < len ? tok0 + span : len) + kRows - 1) / kRows; }

template <int N>
struct PromptWork {
  static constexpr bool kBf16 = true, kPairs = false;
  uint16_t* out;
  float* lse;
  float* part_o;
  float2* part_ml;
  int64_t out_stride;
  int32_t group, n_q_heads, half_tokens;
  float scale_log2, ln2_rest;
  Tiles<N> tiles;
  ChunkCuts cuts;                            // n = 0: CTAs have whole tiles
  __device__ __forceinline__ int first_slot() const { return cuts.n ? cuts.slot[blockIdx.x] : 0; }
  __device__ __forceinline__ bool whole_tiles() const { return cuts.n == 0; }
  __device__ __forceinline__ void whole(int tile, attend::Part& x) const {
    const auto at = tiles.place(tile);
    x.tile = tile;
    x.len = at.len;
    x.tok0 = at.tok0;
    x.begin = 0;
    x.items = x.end = steps_of(x.tok0, tiles.span, x.len);
    x.causal0 = 0;
    x.row0 = x.q_row = tiles.seqs.row[at.seq];
    x.head0 = at.head * group;
    x.kv = at.head;
    x.slot = -1;
    x.two = x.tok0 + half_tokens < x.len;
    x.keep = static_cast<uint8_t>(min(kRows, x.len - (x.items - 1) * kRows));
  }
  __device__ __forceinline__ bool next(int& state, int& slot, attend::Part& x) const {
    const int tile = cuts.tile[blockIdx.x] + state, t1 = cuts.tile[blockIdx.x + 1], i1 = cuts.item[blockIdx.x + 1];
    if (tile >= tiles.count() || tile > t1 || (tile == t1 && i1 == 0)) return false;
    whole(tile, x);
    if (state == 0) x.begin = cuts.item[blockIdx.x];
    if (tile == t1) x.end = i1;
    if (chunk_needs_slot(x.begin, x.end, x.items)) x.slot = slot++;
    ++state;
    return true;
  }
  __device__ __forceinline__ void load_q(const CUtensorMap* map, uint32_t dst, const attend::Part& x, int t, uint32_t bar) const {
    for (int k = 0; k < 2; ++k) tma_load_3d(dst + k * kPanel, map, 64 * k, x.head0, x.q_row + x.tok0 + t * half_tokens, bar);
  }
  __device__ __forceinline__ void load_keys(const CUtensorMap* map, uint32_t dst, const attend::Part& x, int step, uint32_t bar) const {
    tma_load_4d(dst, map, 0, x.kv, x.q_row + step * kRows, 0, bar);
  }
  __device__ __forceinline__ int flags(const attend::Part&, int) const { return 0; }
  __device__ __forceinline__ const float* term(const attend::Part&, int) const { return nullptr; }
  struct Where {
    int tok0, len, head0;
    int64_t row0;
  };
  __device__ __forceinline__ Where place(int tile) const {
    const auto at = tiles.place(tile);
    return {at.tok0, at.len, at.head * group, tiles.seqs.row[at.seq]};
  }
  __device__ __forceinline__ void fail() const {}      // (a prompt has no status word: its NaN rows say it)
};

// ---- masses of prompt tokens ---------------------------------------------------------------------
constexpr int kMThreads = 192;             // four warps of tokens, loads, products
constexpr int kMaxObsRows = 128;           // rows of one product: its n dimension
constexpr int kMOffLse = 0, kMOffBar = kMaxObsRows * 8, kMOffTiles = 2048;
constexpr int kMCtas = 2;                  // resident on an SM
// One product per tile: two tiles of keys, the rows once.  Several: one tile of keys, the rows twice.  Either way 97 KB at most.
__host__ __device__ constexpr int mass_k_stages(bool one) { return one ? 2 : 1; }
__host__ __device__ constexpr int mass_q_stages(bool one) { return one ? 1 : 2; }
constexpr int mass_smem(bool one, int n_pad) { return kMOffTiles + mass_k_stages(one) * kTileBytes + mass_q_stages(one) * n_pad * 256 + 1024; }
static_assert(kMCtas * (std::max(mass_smem(true, kMaxObsRows), mass_smem(false, kMaxObsRows)) + 1024) <= 227 * 1024, "two CTAs on an SM");

struct MassParams {
  const float* lse;
  float* mass;
  int32_t row_base;                          // first row of the first sequence: where `mass` begins
  int32_t n_q_heads, n_kv_heads, group;
  int32_t n_obs, group_tokens;               // observing tokens of a sequence; of one product
  int32_t n_pad;                             // columns of a product, a multiple of 16
  int32_t pitch, tmem_cols;                  // the same rounded up to what one load reads; two of them
  int32_t chunk;                             // tiles of 128 tokens per CTA
  float scale_log2, scale_rest;              // what a logit is multiplied by, in two parts (see logit_of)
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
  const uint32_t bar_q = bars, bar_qfree = bars + 16, bar_s = bars + 32, bar_sfree = bars + 48, bar_full = bars + 64, bar_empty = bars + 80, bar_drain_mma = bars + 96;
  volatile uint32_t* const abort = reinterpret_cast<volatile uint32_t*>(base + kMOffBar + 240);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(base + kMOffBar + 244);
  float* const lse_s = reinterpret_cast<float*>(base + kMOffLse);      // what a row's logits get,
  float* const by_s = lse_s + kMaxObsRows;                             // and what its weights are multiplied by

  const int head = blockIdx.x % p.n_kv_heads, item = blockIdx.x / p.n_kv_heads;
  const int si = find_seq(seqs, item);
  const int len = seqs.len[si], row0 = seqs.row[si];
  const int tile0 = (item - seqs.first[si]) * p.chunk;
  const int n_tiles = min(p.chunk, (len + kRows - 1) / kRows - tile0);
  const int obs = min(p.n_obs, len), obs0 = len - obs;         // observing tokens, the first of them
  const int n_groups = (obs + p.group_tokens - 1) / p.group_tokens;
  const int steps = n_tiles * n_groups;
  const bool one = p.n_obs <= p.group_tokens;                  // the launch's layout: a product holds all rows
  const int k_stages = mass_k_stages(one), q_stages = mass_q_stages(one);
  const uint32_t tiles = smem + kMOffTiles, q_smem = tiles + k_stages * kTileBytes;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      bar_init(bar_q + 8 * i, 1);
      bar_init(bar_qfree + 8 * i, 1);
      bar_init(bar_s + 8 * i, 1);
      bar_init(bar_sfree + 8 * i, 4);
      bar_init(bar_full + 8 * i, 1);
      bar_init(bar_empty + 8 * i, 1);
    }
    bar_init(bar_drain_mma, 1);
    *abort = 0;
    bar_init_fence();
  }
  if (warp == 5) {                         // (no tensor memory is held while the kernel in front, which may still want some, is waited for)
    pdl_wait();
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), p.tmem_cols);
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();                              // (nothing but parameters was read so far)
  pdl_launch();

  if (warp < 4) {
    const uint32_t lanes = tmem + (static_cast<uint32_t>(warp) << 21);
    const int r = warp * 32 + lane;
    float sum = 0.f;
    bool ok = true;
    // a row's log-sum-exp, a thread per row, loaded a product ahead
    auto row_lse = [&](int grp) {
      const int q0 = obs0 + grp * p.group_tokens, cols = min(p.group_tokens, obs - grp * p.group_tokens) * p.group;
      return r < cols ? p.lse[static_cast<int64_t>(row0 + q0 + r / p.group) * p.n_q_heads + head * p.group + r % p.group] : 0.f;
    };
    const uint64_t scale2 = f2_pack(p.scale_log2, p.scale_log2), rest2 = f2_pack(p.scale_rest, p.scale_rest);
    auto weights = [&](uint32_t s0, uint32_t s1, float e0, float e1) {      // of two rows
      const uint64_t s = f2_pack(__uint_as_float(s0), __uint_as_float(s1));
      float a, b;
      f2_unpack(f2_fma(s, rest2, f2_fma(s, scale2, f2_pack(e0, e1))), a, b);
      return f2_pack(ex2(a), ex2(b));
    };
    float next = row_lse(0);
    for (int i = 0; i < steps; ++i) {
      const int grp = i % n_groups, tok = (tile0 + i / n_groups) * kRows + r;
      const int q0 = obs0 + grp * p.group_tokens;                                  // first observing token of the product
      const int cols = min(p.group_tokens, obs - grp * p.group_tokens) * p.group;
      if (i == 0 || n_groups > 1) {
        asm volatile("bar.sync 1, 128;\n" ::: "memory");
        // Its multiple of 32 bits would be off by up to 2^-20, as much as all else together: what is cut off goes into a factor.  (With the second part of
        // the scale 1.4 us of 16,384 tokens' 16; errors of given log-sum-exps' masses 1.8e-6 -> 1.0e-6 and 2.2e-6 -> 1.6e-6 at logits of 12 and 25.)
        constexpr float kRest = static_cast<float>(1.4426950408889634 - kLog2e);
        const float e = -next * kLog2e;
        lse_s[r] = e;
        by_s[r] = fmaf(fmaf(-next, kLog2e, -e) - next * kRest, kLn2, 1.f);
        asm volatile("bar.sync 1, 128;\n" ::: "memory");
        next = row_lse((grp + 1) % n_groups);
      }
      // (after an abort the loop goes on without products: its barriers need all four warps)
      ok = ok && bar_wait(bar_s + 8 * (i & 1), (i >> 1) & 1, abort);
      if (!ok) continue;
      tmem_after();
      const int from = max(0, (tok - q0) * p.group);           // rows before the token do not see it
      uint64_t sum0 = 0, sum1 = 0;
      for (int c0 = 0; c0 < cols; c0 += 32) {
        uint32_t x[32];
        tmem_ld32(lanes + (i & 1) * p.pitch + c0, x);
        tmem_wait_ld();
        if (c0 + 32 <= cols && __all_sync(0xffffffffu, from <= c0)) {
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            const float4 e = *reinterpret_cast<const float4*>(lse_s + c0 + k), f = *reinterpret_cast<const float4*>(by_s + c0 + k);
            sum0 = f2_fma(weights(x[k], x[k + 1], e.x, e.y), f2_pack(f.x, f.y), sum0);
            sum1 = f2_fma(weights(x[k + 2], x[k + 3], e.z, e.w), f2_pack(f.z, f.w), sum1);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            float a, b;
            f2_unpack(f2_mul(weights(x[k], x[k + 1], lse_s[c0 + k], lse_s[c0 + k + 1]), f2_pack(by_s[c0 + k], by_s[c0 + k + 1])), a, b);
            a = c0 + k >= from && c0 + k < cols ? a : 0.f;
            b = c0 + k + 1 >= from && c0 + k + 1 < cols ? b : 0.f;
            sum0 = f2_add(sum0, f2_pack(a, b));
          }
        }
      }
      float part0, part1;
      f2_unpack(f2_add(sum0, sum1), part0, part1);
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
          const int slot = tile % k_stages, turn = tile / k_stages;
          ok = turn == 0 || bar_wait(bar_empty + 8 * slot, (turn - 1) & 1, abort);
          if (!ok) break;
          bar_expect(bar_full + 8 * slot, kTileBytes);
          for (int h = 0; h < 2; ++h)
            tma_load_3d(tiles + slot * kTileBytes + h * kPanel, &map_k, 64 * h, head, row0 + (tile0 + tile) * kRows, bar_full + 8 * slot);
          ++k_loads;
        }
        if (i == 0 || n_groups > 1) {
          const int slot = i % q_stages, turn = i / q_stages;
          ok = turn == 0 || bar_wait(bar_qfree + 8 * slot, (turn - 1) & 1, abort);
          if (!ok) break;
          bar_expect(bar_q + 8 * slot, q_bytes);
          for (int h = 0; h < 2; ++h)
            tma_load_3d(q_smem + slot * p.n_pad * 256 + h * p.n_pad * 128, &map_q, 64 * h, head * p.group, row0 + obs0 + grp * p.group_tokens, bar_q + 8 * slot);
          ++q_loads;
        }
      }
      if (*abort) {
        for (int k = max(0, q_loads - q_stages); k < q_loads; ++k) bar_drain(bar_q + 8 * (k % q_stages), (k / q_stages) & 1);
        for (int k = max(0, k_loads - k_stages); k < k_loads; ++k) bar_drain(bar_full + 8 * (k % k_stages), (k / k_stages) & 1);
      }
    }
  } else {
    if (elect()) {
      const uint32_t idesc = instr_desc(true, false, kRows, p.n_pad);
      bool ok = true;
      for (int i = 0; i < steps; ++i) {
        const int grp = i % n_groups, tile = i / n_groups, slot = tile % k_stages, q_slot = n_groups == 1 ? 0 : i % q_stages;
        ok = (grp > 0 || bar_wait(bar_full + 8 * slot, (tile / k_stages) & 1, abort)) &&
             ((i > 0 && n_groups == 1) || bar_wait(bar_q + 8 * q_slot, (i / q_stages) & 1, abort)) && (i < 2 || bar_wait(bar_sfree + 8 * (i & 1), ((i >> 1) - 1) & 1, abort));
        if (!ok) break;
        tmem_after();
        const uint64_t a = smem_desc(tiles + slot * kTileBytes, 16), b = smem_desc(q_smem + q_slot * p.n_pad * 256, 16);
        for (int k = 0; k < kD / 16; ++k)
          mma_ss(tmem + (i & 1) * p.pitch, a + (((k >> 2) * kPanel + (k & 3) * 32) >> 4), b + (((k >> 2) * p.n_pad * 128 + (k & 3) * 32) >> 4), idesc, k > 0);
        mma_commit(bar_s + 8 * (i & 1));
        if (n_groups > 1) mma_commit(bar_qfree + 8 * q_slot);
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
std::atomic<uint64_t> g_mass_few{0}, g_mass_many{0};
constexpr int kCutGain = 8, kCutSteps = 3;      // steps: see cut_prompt; what a CTA is worth starting for

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Bounds, layout and place of the call's rows.  `rows`: rows up to the end of the last sequence.
int check_prompt(const gkv_prompt* d, int* rows) {
  if (!d || d->struct_size != sizeof(gkv_prompt) || d->abi_version != GKV_ABI_VERSION) return GKV_ERR_INVALID_ARG;
  if (d->n_seqs < 0 || d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->n_q_heads % d->n_kv_heads != 0) return GKV_ERR_INVALID_ARG;
  if (d->head_dim != kD || d->n_q_heads / d->n_kv_heads > kMaxHeadsPerKv) return GKV_ERR_UNSUPPORTED;
  if (d->softmax_scale != 0.f && !(std::isnormal(d->softmax_scale) && d->softmax_scale > 0.f)) return GKV_ERR_INVALID_ARG;
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

// Cuts the launch's tiles into equal ranges where the longest one would outlast the rest by more than the parts' merge costs (about the
// time of eight steps: one sequence of 4,097 tokens, 8 heads: 65 us whole, 33 steps for the last tile and 16.5 on average, 54 cut).  Returns the slots, 0 = whole tiles.
template <int N>
int cut_prompt(const Tiles<N>& t, ChunkCuts* cuts, ChunkMerge* merge) {
  int64_t total = 0;
  int longest = 0;
  for (int i = 0; i < t.seqs.n; ++i)
    for (int k = t.seqs.first[i]; k < t.seqs.first[i + 1]; ++k) {
      const int n = steps_of((t.seqs.first[i + 1] - 1 - k) * t.span, t.span, t.seqs.len[i]);
      total += static_cast<int64_t>(n + attend::kStart) * t.n_kv_heads;
      longest = std::max(longest, n + attend::kStart);
    }
  cuts->n = 0;
  merge->n = 0;
  merge->slot[0] = 0;
  if (longest <= total / kChunkCtas + kCutGain) return 0;
  int seq = 0;
  return cut_tiles(t.count(), total, chunk_ctas(total, kCutSteps), attend::kStart, attend::kSnap, [&](int tile) {
    const int item = tile / t.n_kv_heads;
    if (item < t.seqs.first[seq]) seq = 0;
    while (item >= t.seqs.first[seq + 1]) ++seq;
    return steps_of((t.seqs.first[seq + 1] - 1 - item) * t.span, t.span, t.seqs.len[seq]);
  }, cuts, merge);
}
constexpr size_t slot_bytes_of_prompt(int slots) { return static_cast<size_t>(slots) * 2 * kRows * (kD + 2) * sizeof(float); }

template <int N>
void set_tiles(Tiles<N>& t, const gkv_prompt* d, const std::vector<int>& order, int begin, int end) {
  t.n_kv_heads = d->n_kv_heads;
  t.span = 2 * (kRows / (d->n_q_heads / d->n_kv_heads));
  deal(t.seqs, d->offsets, order, begin, end, t.span);
}

template <int N>
cudaError_t launch_prompt(PromptWork<N>& w, const gkv_prompt* d, const std::vector<int>& order, int begin, int end, const attend::Maps& maps, void* workspace,
                          size_t bytes, cudaStream_t st) {
  set_tiles(w.tiles, d, order, begin, end);
  ChunkMerge merge;
  const int slots = cut_prompt(w.tiles, &w.cuts, &merge);
  if (slot_bytes_of_prompt(slots) > bytes || (slots && !workspace)) w.cuts.n = merge.n = 0;      // whole tiles then
  w.part_o = static_cast<float*>(workspace);
  w.part_ml = reinterpret_cast<float2*>(w.part_o + static_cast<size_t>(slots) * 2 * kRows * kD);
  static std::atomic<uint64_t> done{0};
  cudaError_t e = raise_smem_limit(attend::attend_kernel<PromptWork<N>>, attend::kSmem, done);
  if (e != cudaSuccess) return e;
  e = attend::launch_behind(attend::attend_kernel<PromptWork<N>>, dim3(w.cuts.n ? w.cuts.n : w.tiles.count()), attend::kThreads, attend::kSmem, st, w, maps);
  if (e != cudaSuccess || merge.n == 0) return e;
  return attend::launch_behind(attend::attend_merge_kernel<PromptWork<N>>, dim3((w.tiles.span * w.group + 31) / 32, merge.n), 128, 0, st, w, merge);
}
template <int N>
cudaError_t launch_mass(MassParams& p, const gkv_prompt* d, const std::vector<int>& order, int begin, int end, const CUtensorMap* maps, size_t smem,
                        std::atomic<uint64_t>& done, cudaStream_t st) {
  Seqs<N> s;
  const int tiles = deal(s, d->offsets, order, begin, end, kRows);
  // One CTA per place on the GPU with a stretch of tiles each (its rows are loaded once); where sequences are too many for that, several waves.  (Three
  // sequences of 57,000 tokens, 8 heads: 446 CTAs of eight tiles, 1.5 waves, took 28.8 us.)
  constexpr int kPlaces = 148 * kMCtas;
  const int all = tiles * p.n_kv_heads, even = (all + kPlaces - 1) / kPlaces;
  p.chunk = even;
  while (p.chunk <= even + even / 4 && deal(s, d->offsets, order, begin, end, kRows * p.chunk) * p.n_kv_heads > kPlaces) ++p.chunk;
  if (p.chunk > even + even / 4) p.chunk = std::max(1, all / (4 * kPlaces));
  const int items = deal(s, d->offsets, order, begin, end, kRows * p.chunk);
  cudaError_t e = raise_smem_limit(mass_kernel<N>, std::max(mass_smem(true, kMaxObsRows), mass_smem(false, kMaxObsRows)), done);
  if (e != cudaSuccess) return e;
  return attend::launch_behind(mass_kernel<N>, dim3(items * p.n_kv_heads), kMThreads, smem, st, p, s, maps[0], maps[1]);
}

double scale_of(const gkv_prompt* d) { return d->softmax_scale > 0.f ? d->softmax_scale : 1.0 / std::sqrt(static_cast<double>(kD)); }
float scale_log2_of(const gkv_prompt* d) { return static_cast<float>(scale_of(d)) * kLog2e; }
// What a logit is, in units of its multiple of scale_log2: ln 2, the rounding of scale_log2 taken out, and some of what tcgen05 loses.  It cuts sums instead
// of rounding them, so that a logit comes out too small, and by how much depends on the running sums: 0.9e-7 of itself on average for noise of any size,
// 1.6e-7 and 1.7e-7 where all products have one sign, 1.7e-7 for keys like the query, 2.6e-7 where one channel leads, 6.9e-7 where halves
// cancel.  No kind of data lost less than 7e-8, so that much is given back: root mean square errors 1.2e-7 -> 0.8e-7 for noise, 1.7e-7 -> 1.1e-7
// for one sign, 9.0e-7 -> 8.4e-7 where halves cancel (32-bit sums that round: 0.5e-7 to 1.0e-7).
double logit_of(const gkv_prompt* d) { return scale_of(d) / scale_log2_of(d) * (1.0 + 7e-8); }

}  // namespace
}  // namespace gkv

using namespace gkv;

namespace {
// No exception leaves a C entry point: the sequences' order is the only memory that the calls take from the host.
template <class F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return GKV_ERR_INVALID_ARG;
  }
}

int workspace_bytes_of(const gkv_prompt* d, size_t* bytes) {
  int rows = 0;
  const int rc = check_prompt(d, &rows);
  if (rc != GKV_OK) return rc;
  if (!bytes) return GKV_ERR_INVALID_ARG;
  *bytes = 0;
  const std::vector<int> order = longest_first(d);
  const int n = static_cast<int>(order.size());
  for (int at = 0; at < n; at += kMaxSeqs) {
    const int end = std::min(n, at + kMaxSeqs);
    ChunkCuts cuts;
    ChunkMerge merge;
    int slots;
    if (end - at <= kFewSeqs) {
      Tiles<kFewSeqs> t;
      set_tiles(t, d, order, at, end);
      slots = cut_prompt(t, &cuts, &merge);
    } else {
      Tiles<kMaxSeqs> t;
      set_tiles(t, d, order, at, end);
      slots = cut_prompt(t, &cuts, &merge);
    }
    *bytes = std::max(*bytes, slot_bytes_of_prompt(slots));
  }
  return GKV_OK;
}

int attn(const gkv_prompt* d, const void* q, const void* k, const void* v, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int rows = 0;
  const int rc = check_prompt(d, &rows);
  if (rc != GKV_OK) return rc;
  const std::vector<int> order = longest_first(d);
  if (order.empty()) return GKV_OK;
  if (!q || !k || !v || !out || misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16) || misaligned(lse, 4) || misaligned(workspace, 16))
    return GKV_ERR_INVALID_ARG;
  if (!on_current_device({q, k, v, out, lse, workspace})) return GKV_ERR_INVALID_ARG;
  const int64_t nq = static_cast<int64_t>(d->n_q_heads) * kD, nkv = static_cast<int64_t>(d->n_kv_heads) * kD;
  const int group = d->n_q_heads / d->n_kv_heads, half_tokens = kRows / group;
  attend::Maps maps;
  // keys and values: [rows][heads][two panels][64 channels], 128 rows of a head at a time
  const uint64_t dims[4] = {64, static_cast<uint64_t>(d->n_kv_heads), static_cast<uint64_t>(rows), 2};
  const uint64_t ks[3] = {kRowBytes, static_cast<uint64_t>(d->k_stride ? d->k_stride : nkv) * 2, 128}, vs[3] = {kRowBytes, static_cast<uint64_t>(d->v_stride ? d->v_stride : nkv) * 2, 128};
  const uint32_t box[4] = {64, 1, kRows, 2};
  if (!make_rows_map(&maps.q, q, rows, d->n_q_heads, d->q_stride ? d->q_stride : nq, group, half_tokens) || !make_map(&maps.k, k, 4, dims, ks, box) ||
      !make_map(&maps.v, v, 4, dims, vs, box))
    return GKV_ERR_CUDA;
  maps.k_lo = maps.k;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto launch = [&](auto& w, int at, int end) {
    w.out = static_cast<uint16_t*>(out);
    w.lse = lse;
    w.out_stride = d->out_stride ? d->out_stride : nq;
    w.group = group;
    w.n_q_heads = d->n_q_heads;
    w.half_tokens = half_tokens;
    w.scale_log2 = scale_log2_of(d);
    w.ln2_rest = static_cast<float>(logit_of(d) - kLn2);
    return launch_prompt(w, d, order, at, end, maps, workspace, workspace_bytes, st);
  };
  std::unique_lock<std::mutex> lock;
  if (workspace) lock = std::unique_lock<std::mutex>(launching(workspace));
  const int n = static_cast<int>(order.size());
  for (int at = 0; at < n; at += kMaxSeqs) {
    const int end = std::min(n, at + kMaxSeqs);
    PromptWork<kFewSeqs> few;
    PromptWork<kMaxSeqs> many;
    if ((end - at <= kFewSeqs ? launch(few, at, end) : launch(many, at, end)) != cudaSuccess) return GKV_ERR_CUDA;
  }
  return GKV_OK;
}

int mass_of(const gkv_prompt* d, const void* q, const void* k, const float* lse, int32_t n_obs, float* mass, void* stream) {
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
  p.scale_log2 = scale_log2_of(d);
  p.scale_rest = static_cast<float>(p.scale_log2 * (logit_of(d) * 1.4426950408889634 - 1.0));
  CUtensorMap maps[2];
  if (!make_rows_map(&maps[0], q, rows, d->n_q_heads, d->q_stride ? d->q_stride : nq, p.group, p.group_tokens) ||
      !make_rows_map(&maps[1], k, rows, d->n_kv_heads, d->k_stride ? d->k_stride : nkv, 1, kRows))
    return GKV_ERR_CUDA;
  const size_t smem = mass_smem(n_obs <= p.group_tokens, p.n_pad);
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
}  // namespace

int gkv_prompt_workspace_bytes(const gkv_prompt* d, size_t* bytes) {
  return guarded([&] { return workspace_bytes_of(d, bytes); });
}
int gkv_prompt_attn(const gkv_prompt* d, const void* q, const void* k, const void* v, void* out, float* lse, void* workspace, size_t workspace_bytes,
                    void* stream) {
  return guarded([&] { return attn(d, q, k, v, out, lse, workspace, workspace_bytes, stream); });
}
int gkv_prompt_mass(const gkv_prompt* d, const void* q, const void* k, const float* lse, int32_t n_obs, float* mass, void* stream) {
  return guarded([&] { return mass_of(d, q, k, lse, n_obs, mass, stream); });
}
