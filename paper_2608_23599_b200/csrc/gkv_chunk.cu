// Merges the parts of tiles that several CTAs of a chunk call worked on (gkv_chunk.h), in the order of their slots.
#include <cuda_runtime.h>

#include "gkv_attend.cuh"
#include "gkv_chunk.h"
#include "gkv_internal.h"
#include "gkv_tc.cuh"

namespace gkv {
namespace {

using namespace tc;

struct MergeParams {
  const float* part_o;       // [slot][tile rows][128], not normalised
  const float2* part_ml;     // [slot][tile rows]: reference (log2), sum
  uint16_t* out;
  float* lse;
  ChunkShape s;
};

// A warp per row, four channels per lane.  Launched while the parts are still being made (its blocks need little room), so that their last
// store is all it waits for.
template <int N>
__global__ void __launch_bounds__(128) chunk_merge_kernel(const __grid_constant__ MergeParams p, const __grid_constant__ ChunkMerge merge,
                                                          const __grid_constant__ ChunkLens<N> lens) {
  const ChunkShape& sh = p.s;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int tile = merge.tile[blockIdx.y], first = merge.slot[blockIdx.y], n = merge.slot[blockIdx.y + 1] - first;
  const int rt = tile % sh.row_tiles, stream = tile / sh.row_tiles, b = stream / sh.n_kv_heads, h = stream % sh.n_kv_heads;
  const int tok = rt * sh.tile_tokens + row / sh.group;
  if (row >= sh.tile_tokens * sh.group || tok >= lens.len[N == 1 ? 0 : b]) return;
  pdl_wait();
  pdl_launch();
  auto index = [&](int i) { return static_cast<size_t>(first + i) * sh.tile_rows + row; };
  float top = -INFINITY;
  for (int i = lane; i < n; i += 32) {
    const float2 v = p.part_ml[index(i)];
    if (v.y != 0.f) top = fmaxf(top, v.x);      // (NaN counts: it has to come through)
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
      if (i0 + k >= n || v[k].y == 0.f) continue;
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

template <int N>
cudaError_t launch_as(const MergeParams& p, const ChunkMerge& merge, const int32_t* len, cudaStream_t st) {
  ChunkLens<N> lens;
  for (int b = 0; b < (N == 1 ? 1 : p.s.batch); ++b) lens.len[b] = len ? len[b] : p.s.n_new;
  return attend::launch_behind(chunk_merge_kernel<N>, dim3((p.s.tile_tokens * p.s.group + 3) / 4, merge.n), 128, 0, st, p, merge, lens);
}

}  // namespace

// call.workspace: the slots, their sums behind them.  len: HOST [batch], or null where every sequence has n_new rows.
cudaError_t launch_chunk_merge(const ChunkCall& call, const ChunkMerge& merge, const int32_t* len, cudaStream_t st) {
  if (merge.n == 0) return cudaSuccess;
  const float* const ml = call.workspace + static_cast<size_t>(merge.slot[merge.n]) * call.shape.tile_rows * kD;
  const MergeParams p{call.workspace, reinterpret_cast<const float2*>(ml), call.out, call.lse, call.shape};
  return len && p.s.batch > 1 ? launch_as<kChunkMaxBatch>(p, merge, len, st) : launch_as<1>(p, merge, len, st);
}

}  // namespace gkv
