"""CPU: context splits of the exact attention's row blocks and the staging of their
page ids, replayed on the host with the functions that the kernels call."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Every split of contexts of up to 2100 tiles, in the order in which the kernel
# locates tiles and stages runs of page ids (two places, run r in place r % 2).  What
# is staged in a period counts from the next one on; what it replaces is gone at once.
REPLAY = r"""
#include <cstdio>
#include "exact.h"
using namespace pkv;

int main() {
  long long wrong = 0, across = 0;
  for (int most = 1; most <= EX_MAX_SPLITS; ++most) {
    for (int tiles = 0; tiles <= 2100; ++tiles) {
      int per = 0, at = 0;
      const int n = ex_splits(most, tiles, per);
      if (n < 1 || n > most || (n > 1 && tiles < 2 * EX_MIN_TILES)) ++wrong;
      for (int s = 0; s < n; ++s) {
        const int t0 = s * per, t1 = t0 + per < tiles ? t0 + per : tiles;
        if (t0 != at || (tiles > 0 && t1 <= t0)) ++wrong;  // splits follow each other, none is empty
        at = t1;
        for (int shift = 0; shift <= 6 && t0 < t1; ++shift) {
          const int run = ex_run_tiles(shift);
          int held[2] = {-1, -1}, before = -1;
          auto stage = [&](int t) { held[(t / run) & 1] = t / run; };
          auto locate = [&](int t) {
            if (t >= t1) return;
            if (before >= 0 && t / run != before / run) ++across;
            before = t;
            if (held[(t / run) & 1] == t / run) return;
            if (wrong++ < 5) std::printf("unstaged: %d splits of %d tiles, [%d, %d), runs of %d, tile %d\n", n, tiles, t0, t1, run, t);
          };
          stage(t0);
          const int last = ex_ids_last(t0, t1);
          if (last / run != t0 / run) stage(last);
          for (int t = t0; t < t0 + 3; ++t) locate(t);
          for (int t = t0; t <= t1; ++t) {
            const bool due = ex_ids_due(t, t1, run);
            if (due) held[((t + 4) / run) & 1] = -1;
            locate(t + 3);
            if (due) stage(t + 4);
          }
        }
      }
      if (at != tiles) ++wrong;
    }
  }
  std::printf("%lld wrong, %lld runs entered\n", wrong, across);
  return wrong != 0 || across == 0;
}
"""


def test_page_ids_of_every_tile_are_staged_before_it_is_located(tmp_path):
    if not (shutil.which("g++") and os.path.exists("/opt/rocm/include/hip/hip_runtime.h")):
        pytest.skip("no compiler or headers")
    src, exe = tmp_path / "replay.cpp", tmp_path / "replay"
    src.write_text(REPLAY)
    subprocess.run(["g++", "-std=c++17", "-O2", "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2606_26762_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout
