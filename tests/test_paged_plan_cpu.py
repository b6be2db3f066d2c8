"""What the paged launches take for granted about their plan, on the CPU (``csrc/pbb_paged_index.h``
compiled with g++): skipped sequences are never cut, no call needs more states than the workspace that
any call of its descriptor is given, and the summary of many sequences fits its part of it."""
from __future__ import annotations

import os
import subprocess

import paper_2606_02680_amd as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHECK = r"""
#include <cstdio>
#include <random>
#include "pbb_paged_index.h"
using namespace pbb;
int main() {
  std::mt19937 rng(5);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < 300000; ++i) {
    const int group = pick(1, 16), hkv = i % 9 == 0 ? pick(1, 2000) : pick(1, 16);
    const PagedShape s = PagedShape::make(16 * pick(1, 16), 100, pick(1, i % 5 ? 300 : 20000),
                                          i % 4 == 1 ? 2 * pick(1, 2000) : 0, i % 4 == 2 ? pick(1, 5000) : 0);
    // the kinds of kernels there are: cols, step, round, few_least, pieces, many_least
    static const PagedKind kinds[2][2][3] = {
        {{{128, 32, 512, 8, 1024, 32}}, {{16, 32, 512, 8, 2048, 64}, {16, 32, 256, 8, 2048, 64}}},
        {{{64, 16, 512, 8, 2048, 32}}, {{16, 16, 512, 8, 2048, 32}}}};
    const int f32 = i & 1, batch = pick(1, i % 3 ? 10 : 4000);
    const bool ragged = (i >> 1) & 1;
    const int n = ragged ? pick(1, 20000) : batch * pick(1, i % 7 ? 20 : 400);
    const bool narrow = PagedPlan::is_narrow(batch, group, n, ragged);
    const PagedKind& k = kinds[f32][narrow][narrow && !f32 ? (i >> 3) & 1 : 0];
    const PagedPlan p = PagedPlan::make(s, k, batch, hkv, group, n, ragged);
    const PagedPlan most = narrow ? PagedPlan::make(s, k, batch, hkv, group, batch, false)
                                  : PagedPlan::make(s, k, batch, hkv, group, 1, true);
    if (p.slots > most.slots || p.cols != most.cols) return std::printf("slots %d\n", i), 1;
    const Chunk skipped{0, pick(1, 5000), -1};
    const float total = (float)pick(1, 1 << 30);
    if (p.steps_of(s, skipped) != 1 || p.pieces_of(1, 1.0f / p.share_of(total)) != 1)
      return std::printf("skipped %d\n", i), 1;
    // a summary only where the workspace has room for one; no search of the first kind in a large batch
    if (p.planned && batch <= (most.slots > 0 ? kPagedScan : kPagedScanUncut))
      return std::printf("planned %d\n", i), 1;
    if (!p.planned && batch > kPagedScanUncut && (ragged || p.pieces > 0)) return std::printf("search %d\n", i), 1;
  }
  for (int batch : {1, 128, 129, 192, 193, 1 << 24}) {
    const uint64_t bytes = paged_rounds_bytes(batch), rounds = (uint64_t)paged_rounds(batch);
    if (bytes < 4 * (8 + 6 * rounds) || bytes % 16 != 0)
      return std::printf("rounds %d\n", batch), 1;
  }
  return 0;
}
"""


def test_plan(tmp_path):
    src, exe = tmp_path / "check.cpp", str(tmp_path / "check")
    src.write_text(CHECK)
    inc = os.path.join(ROOT, "paper_2606_02680_amd", "csrc")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", inc, str(src), "-o", exe], check=True)
    p = subprocess.run([exe], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout


def test_workspace_depends_on_the_descriptor_alone():
    for batch, width in ((2, 4), (2, 1000), (500, 4), (500, 1000)):
        d = P.make_paged_desc(batch, 8, 2, 64, page_size=16, n_pages=9, table_width=width)
        sizes = {P.paged_workspace_bytes(d, n) for n in (0, 1, batch, 7 * batch, 100 * batch, 1 << 30)}
        assert len(sizes) == 1 and (sizes == {0}) == (batch == 2 and width == 4)
