"""The 8-bit fill's plan, built for the host: every item of every sequence is taken
once, and no wave has many of them, whatever the batch's mean length and however much
longer than it a history is."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_09200_amd", "csrc")
PROG = r"""
#include <cstdio>
#include <vector>
#define __host__
#define __device__
#include "seq_fill8.h"
using namespace lat;

// lengths, ring, items of a block, bound of the lengths: largest number of items of a wave
// (-1: an item is taken twice or not at all)
static long most_items(const std::vector<int>& len, int64_t cap, int sides, int64_t max_len, long* waves) {
  std::vector<int> off(1, 0);
  for (int n : len) off.push_back(off.back() + n);
  const int S = (int)len.size(), rows = off.back() + 5;          // rows behind the last sequence
  auto items = [&](int s) { return ((len[s] < cap ? len[s] : cap) + CACHE8_BLOCK - 1) / CACHE8_BLOCK * sides; };
  std::vector<std::vector<char>> seen(S);
  for (int s = 0; s < S; ++s) seen[s].assign(items(s), 0);
  const Fill8Plan p = fill8_plan(rows, S, max_len, cap, sides);
  *waves = p.waves;
  long most = 0;
  for (int wave = 0; wave < (p.waves + 3) / 4 * 4; ++wave) {
    Fill8Share w;
    if (!fill8_share(p, wave, rows, S, [&](int i) { return off[i]; }, &w)) continue;
    long n = 0;
    for (int64_t s = w.s; s < S; s += w.ds) {
      if (len[s] == 0 || (len[s] >= p.large) != w.behind) continue;
      for (int64_t it = w.it0; it < items(s); it += w.dit, ++n)
        if (seen[s][it]++) return -1;
    }
    if (n > most) most = n;
  }
  for (int s = 0; s < S; ++s)
    for (char c : seen[s])
      if (!c) return -1;
  return most;
}

int main() {
  struct { int n, mean, extra, len; int64_t cap; } mix[] = {
      {1000, 500, 1, 8000, 8192},   {100, 1000, 1, 100000, 100004}, {100, 4000, 1, 60000, 60000},
      {1000, 30, 1, 2000, 2048},    {3000, 20, 1, 32000, 4100},     {64, 2000, 3, 30000, 4000},
      {300, 1000, 2, 20000, 20004}, {50000, 8, 1, 32000, 1000},     {9, 100, 1, 100000, 1 << 20},
      {3, 10, 1, 100000, 100000},   {500, 100, 5, 1151, 3000},      {2000, 1, 1, 127, 500},
      {2000, 1, 3, 128, 500},       {8000, 20, 0, 0, 104},          {1, 300000, 0, 0, 4000},
      {700, 0, 1, 190, 400},        {40, 7000, 1, 70000, 1 << 20}};
  for (auto& m : mix)
    for (int sides : {1, 2, 6})
      for (int bound : {0, 1}) {
        std::vector<int> len;
        for (int i = 0; i < m.n; ++i) {
          len.push_back(m.mean ? m.mean * (3 + i % 5) / 5 : i % 2);
          if (m.extra && (i + 1) % (m.n / m.extra) == 0) len.push_back(m.len);
        }
        int longest = 0;
        for (int n : len) longest = n > longest ? n : longest;
        long waves = 0, r = most_items(len, m.cap, sides, bound ? longest : 0, &waves);
        std::printf("%d x %d, %d of %d, ring %ld, %d a block, bound %d: %ld, %ld waves\n", m.n, m.mean, m.extra, m.len,
                    (long)m.cap, sides, bound, r, waves);
      }
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_no_wave_has_many_items_and_none_is_missed(tmp_path):
    src = tmp_path / "prog.cpp"
    src.write_text(PROG)
    exe = str(tmp_path / "prog")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", exe], check=True)
    lines = subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout.splitlines()
    assert len(lines) == 17 * 3 * 2
    for line in lines:
        n = int(line.split(": ")[1].split(",")[0])
        # eight times a mean sequence's blocks, and one for a last part of a block
        assert 0 < n <= 9, line
