"""How a chunk call's work is cut into CTAs, run on the host from the kernel's own header: every item of every tile is in exactly one
range, ranges are equal to within one item (or what a tile's beginning counts for and cuts are moved by), a tile's slots follow one another, and a call never needs more of them than its workspace holds."""
import os
import shutil
import subprocess

import pytest

from paper_2608_23599_b200 import build as _build

HARNESS = r"""
#include <cstdio>
#include <numeric>
#include <random>
#include <vector>
#include "gkv_chunk.h"
using namespace gkv;

static int check(const ChunkShape& s, const int32_t* len, int min_items, int start, int snap, int second) {
  ChunkCuts cuts;
  ChunkMerge merge;
  const int slots = chunk_plan(s, len, min_items, start, snap, second, &cuts, &merge);
  const int tiles = s.batch * s.n_kv_heads * s.row_tiles;
  if (s.tile_tokens * s.group > s.tile_rows || s.tile_tokens < 1 || s.row_tiles * s.tile_tokens < s.n_new) return 1;
  long total = 0;
  for (int t = 0; t < tiles; ++t) total += chunk_items(s, chunk_len(s, len, t / s.row_tiles / s.n_kv_heads), t % s.row_tiles);
  if (total == 0) return slots || cuts.n || merge.n ? 2 : 0;
  if (cuts.n < 1 || cuts.n > kChunkCtas || cuts.tile[cuts.n] != tiles || cuts.item[cuts.n] != 0) return 3;
  // the kernel's own walk over its segments
  std::vector<std::vector<int>> of(tiles);
  long seen = 0, most = 0, least = 1L << 60, cost_all = 0;
  for (int t = 0; t < tiles; ++t) {
    const int n = chunk_items(s, chunk_len(s, len, t / s.row_tiles / s.n_kv_heads), t % s.row_tiles);
    cost_all += n ? n + start : 0;
  }
  int next_tile = 0, next_item = 0, slot_end = 0;
  for (int c = 0; c < cuts.n; ++c) {
    int slot = cuts.slot[c];
    if (slot != slot_end) return 4;
    long mine = 0, cost = 0;
    for (int t = cuts.tile[c]; t <= cuts.tile[c + 1] && t < tiles; ++t) {
      const int items = chunk_items(s, chunk_len(s, len, t / s.row_tiles / s.n_kv_heads), t % s.row_tiles);
      const int begin = t == cuts.tile[c] ? cuts.item[c] : 0, end = t == cuts.tile[c + 1] ? cuts.item[c + 1] : items;
      if (begin >= end) continue;
      if (end > items) return 5;
      while (next_item == chunk_items(s, chunk_len(s, len, next_tile / s.row_tiles / s.n_kv_heads), next_tile % s.row_tiles)) ++next_tile, next_item = 0;
      if (t != next_tile || begin != next_item) return 6;
      next_item = end;
      mine += end - begin;
      cost += end - begin + start;
      if (chunk_needs_slot(begin, end, items)) of[t].push_back(slot++);
    }
    slot_end = slot;
    seen += mine;
    if (mine == 0) return 12;
    // equal to within the beginning of a part, a step, and what cuts were moved by
    if (cost > cost_all / std::min<long>(kChunkCtas, std::max(1L, cost_all / min_items)) + start + 1 + 2 * snap + second) return 13;
    most = std::max(most, mine);
    least = std::min(least, mine);
  }
  if (seen != total || (start == 0 && snap == 0 && most - least > 1)) return 7;
  if (slot_end != slots || slots > kChunkParts || slots > tiles + kChunkCtas - 1) return 8;
  int m = 0;
  for (int t = 0; t < tiles; ++t) {
    if (of[t].empty()) continue;
    if (m >= merge.n || merge.tile[m] != t || merge.slot[m] != of[t].front() || merge.slot[m + 1] != of[t].back() + 1) return 9;
    ++m;
  }
  return m == merge.n && merge.slot[0] == 0 && (merge.n == 0 || merge.slot[m] == slots) ? 0 : 10;
}

int main() {
  std::mt19937 g(1);
  auto upto = [&](int n) { return static_cast<int>(g() % (n + 1)); };
  for (int i = 0; i < 20000; ++i) {
    ChunkShape s{};
    s.batch = 1 + upto(i % 7 == 0 ? 200 : 9);
    s.n_kv_heads = 1 + upto(8);
    s.group = 1 + upto(7);
    s.n_new = 1 + upto(i % 3 == 0 ? 700 : 20);
    const int n_closed = upto(i % 5 == 0 ? 600 : 12), n_tail = upto(63), res_rows = upto(3) * 50;
    if (s.n_new * s.group <= kVerifyRows && upto(3)) verify_shape(&s, n_closed, n_tail, res_rows);
    else dense_shape(&s, 64 * upto(n_closed) + n_tail + res_rows);
    if (std::gcd(chunk_walk(n_closed + 1), n_closed + 1) != 1) return 2;
    std::vector<int32_t> len(s.batch);
    for (auto& n : len) n = upto(3) ? upto(s.n_new) : 0;
    for (const int32_t* l : {static_cast<const int32_t*>(nullptr), static_cast<const int32_t*>(len.data())})
      if (const int rc = check(s, l, 1 + upto(8), upto(1) * 2, upto(1), upto(1) * upto(12))) {
        std::printf("case %d: %d (batch %d kv %d group %d new %d closed %d)\n", i, rc, s.batch, s.n_kv_heads, s.group, s.n_new, n_closed);
        return 1;
      }
  }
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_item_once_and_slots_in_order(tmp_path):
    src = tmp_path / "plan.cpp"
    src.write_text(HARNESS)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-O1", "-g", "-fsanitize=address,undefined", "-std=c++17", f"-I{_build.CSRC}", str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0, r.stdout + r.stderr
