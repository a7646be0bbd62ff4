"""Attention's parts: whatever an unfinished item's place in the workspace holds, the launch that joins parts stays inside it."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_05330_b200", "csrc")

MAIN = r"""
#include "attend_plan.h"
#include <climits>
#include <cstdio>
int main() {
  const int some[] = {INT_MIN, INT_MIN + 1, -1000000, -149, -148, -2, -1, 0, 1, 2, 73, 146, 147, 148, 149, 255, 1000000, 0x3f800000, 0x7fc00000, INT_MAX - 1, INT_MAX};
  for (int x : some)
    for (int y : some) {
      const sdms::PartRun r = sdms::part_run(x, y);
      std::printf("%d %d %d %d %d\n", x, y, r.first, r.count, sdms::kCtas);
    }
}
"""


def test_runs_of_parts(tmp_path):
    (tmp_path / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")],
                   check=True)
    lines = subprocess.run([str(tmp_path / "main")], check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(lines) == 21 * 21
    for line in lines:
        x, y, first, count, ctas = map(int, line.split())
        if 0 <= x <= y < ctas:
            assert (first, count) == (x, y - x + 1)
        else:
            assert 0 <= first < ctas and count == 0


def test_the_join_goes_by_them():
    """Every use of a range that comes from the workspace passes through the check."""
    with open(os.path.join(CSRC, "attend.cu")) as f:
        join = f.read().split("attend_join_kernel(const AttendDev a) {", 1)[1].split("// ---- host", 1)[0]
    uses = [line for line in join.splitlines() if "parts.range" in line]
    assert len(uses) == 1                                    # read once, into two pairs
    for name in ("c_pre", "c_own"):
        rest = join.replace(f"{name} = parts.range", "").replace(f"part_run({name}.x, {name}.y)", "")
        assert f"{name}.x" not in rest and f"{name}.y" not in rest


def test_who_gives_up_waits_for_what_is_under_way():
    """Where any warp has given up, all wait between the CTA's last barrier and its end, so that no tile is written to shared memory that is another's by then."""
    with open(os.path.join(CSRC, "attend.cu")) as f:
        kernel = f.read().split("\nattend_kernel(", 1)[1].split("attend_join_kernel(const AttendDev a) {", 1)[0]
    end = kernel.rsplit("__syncthreads();", 1)[1]
    wait, rest = end.split("tcgen05.dealloc", 1)
    assert "if (dead)" in wait and "clock64() - begin <" in wait
    assert "clock64()" not in rest
