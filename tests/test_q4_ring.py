"""The attention's ring of stages (csrc/q4_ring.h) on the host: a warp whose
wait runs out waits for exactly the copies that are still under way, whichever
tile it stopped at."""
import shutil
import subprocess

import pytest

from paper_2606_24467_gb300 import _build

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "q4_ring.h"

// A barrier that each copy completes once, as the hardware's parity wait sees it.
struct Barrier {
  unsigned completed = 0;
  bool test(unsigned parity) const { return ((completed - 1u) & 1u) == parity; }
};

template <int kStages>
int run(int tiles, int stop) {
  ckv::TileRing<kStages> ring;
  std::vector<Barrier> bars(kStages);
  std::vector<int> tile_in(kStages, -1);
  int issued = 0, left = tiles;
  auto issue = [&](int stage) { tile_in[stage] = issued++; };
  for (int i = 0; i < kStages && issued < tiles; ++i) issue(i);
  for (int t = 0; t < stop; ++t, --left) {
    if (tile_in[ring.stage] != t) return 1;
    if (bars[ring.stage].test(ring.phase)) return 2;  // not before the copy lands
    ++bars[ring.stage].completed;
    if (!bars[ring.stage].test(ring.phase)) return 3;
    if (issued < tiles) issue(ring.stage);
    ring.advance();
  }
  // the wait for tile `stop` has run out; nothing that is under way has landed
  const int n = ring.in_flight(left);
  if (n != issued - stop) return 4;
  for (int k = 0; k < n; ++k) {
    if (tile_in[ring.stage_of(k)] != stop + k) return 5;
    if (bars[ring.stage_of(k)].test(ring.phase_of(k))) return 6;  // would not wait for it
  }
  for (int k = 0; k < n; ++k) {
    ++bars[ring.stage_of(k)].completed;
    if (!bars[ring.stage_of(k)].test(ring.phase_of(k))) return 7;  // would wait on
  }
  return 0;
}

int main() {
  for (int tiles = 1; tiles < 12; ++tiles)
    for (int stop = 0; stop < tiles; ++stop) {
      const int r = run<1>(tiles, stop) * 100 + run<2>(tiles, stop) * 10 + run<3>(tiles, stop);
      if (r) return std::printf("%d tiles, stopped at %d: %d\n", tiles, stop, r), 1;
    }
  return 0;
}
"""


def test_copies_in_flight_are_waited_for(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "ring.cpp", tmp_path / "ring"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-I", _build.CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
