"""The 8-bit attention's plan keeps its partials in the workspace: for random configurations and
lengths, at most `blocks` shares (so slots up to blocks + lists, the kernels' last), all of it below
the checked tables, a grid that covers every share, and shares of whole steps (no GPU)."""
import os
import shutil
import subprocess

import pytest

from paper_2607_24555_amd import build_lib
from paper_2607_24555_amd import locks as B

PROGRAM = r"""
#include "cache_api.hip"
#include <cstdio>
#include <random>
int main() {
  std::mt19937_64 g(7);
  auto spread = [&](double lo, double hi) {
    std::uniform_real_distribution<double> u(std::log(lo), std::log(hi));
    return (long)std::exp(u(g));
  };
  long split = 0, whole = 0, tight = 0;
  for (int i = 0; i < 300000; ++i) {
    locks_cfg_t c{};
    c.num_seqs = (int)spread(1, 6000);
    c.num_kv_heads = 1 << (g() % 5);
    c.num_q_heads = c.num_kv_heads * (1 + (int)(g() % 16));
    c.head_dim = 128;
    c.page_size = 16 << (g() % 3);
    c.rank = 1 + (int)(g() % 15);
    c.max_pages_per_seq = (int)spread(1, 1e5);
    c.budget_tokens = (int)spread(2 * c.page_size, 5e4);
    c.num_blocks = 1000;
    if (locks::validate(&c, false)) continue;
    const bool listed = g() % 2;
    const long width = listed ? locks::page_budget(c) : c.max_pages_per_seq;
    const long table = width << locks::sub_page_log2(c);
    const long lists = (long)c.num_seqs * c.num_kv_heads;
    if ((table + 7) * lists > 0x7fffffffL) continue;  // (refused by the calls)
    const locks::Q8Plan p = locks::q8_plan(c, table, listed);
    if (!p.blocks) {
      ++whole;
      if (p.grid != lists) return std::printf("grid %d of %ld lists\n", p.grid, lists), 1;
      continue;
    }
    ++split;
    const size_t slot = (size_t)(c.num_q_heads / c.num_kv_heads) * 130 * sizeof(float);
    const size_t room = locks::plan_workspace(c).chk_pt_off;
    if ((size_t)(p.blocks + lists) * slot > room || p.few > p.blocks || p.few < 1 || p.blocks < 1)
      return std::printf("%d blocks, few %d, %ld lists of %zu bytes in %zu\n", p.blocks, p.few, lists, slot, room), 1;
    tight += (size_t)(p.blocks + lists + 1) * slot > room;
    // units that the lengths may add up to: lists count as multiples of 8
    const long padded = (table + 7) / 8 * 8 * lists;
    for (int k = 0; k < 4; ++k) {
      const unsigned units = (unsigned)(k == 0 || listed ? padded : spread(8, padded + 1) / 8 * 8);
      const unsigned share = locks::q8_share(units, p.blocks, p.few);
      const unsigned n = (units + share - 1) / share;
      if (share % 8 || share == 0 || n > (unsigned)p.blocks || n > (unsigned)p.grid)
        return std::printf("%u units, %d blocks, few %d, grid %d: share %u\n", units, p.blocks, p.few, p.grid, share), 1;
    }
  }
  std::printf("%ld split, %ld whole, %ld tight\n", split, whole, tight);
  return 0;
}
"""


@pytest.mark.skipif(not shutil.which(build_lib.HIPCC), reason="needs hipcc")
def test_partials_stay_in_the_workspace(tmp_path):
    if not os.path.exists(B.LIB_PATH):
        build_lib.build()
    src, exe = tmp_path / "plan.hip", tmp_path / "plan"
    src.write_text(PROGRAM)
    lib = os.path.dirname(B.LIB_PATH)
    subprocess.run([build_lib.HIPCC, "-std=c++17", "-O1", "--offload-host-only", "-I", build_lib.CSRC, str(src), "-o",
                    str(exe), "-L", lib, "-llocks", f"-Wl,-rpath,{lib}"], check=True, capture_output=True, timeout=120)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
    split, whole, _ = (int(x.split()[0]) for x in r.stdout.split(", "))
    assert split > 10000 and whole > 10000, r.stdout
