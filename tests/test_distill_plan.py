"""Host-side rules of the distillation kernels, compiled without HIP: the column of a listed class, and the work splits."""
import os
import shutil
import subprocess

import pytest

from paper_2211_12858_amd import build as sb_build


def program(tmp_path, body):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ is not available")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text("#include <cstdio>\n#include <initializer_list>\n#include \"sb_distill_plan.h\"\n" + body)
    subprocess.run([cxx, "-std=c++17", "-I" + os.path.abspath(sb_build.CSRC), str(src), "-o", str(exe)], check=True)
    return str(exe)


def test_column_of_a_listed_class(tmp_path):
    """Lists may hold any int32; a constant expression allows no overflow."""
    exe = program(tmp_path, """
static_assert(sb::column_from(INT32_MIN, 65534) >= 65535u && sb::column_from(INT32_MAX, 1) >= 65535u, "");
static_assert(sb::column_from(-1, 640) >= 65535u && sb::column_from(639, 640) >= 65535u && sb::column_from(641, 640) == 1u, "");
int main() {
  const int32_t ids[] = {INT32_MIN, INT32_MIN + 1, -65536, -1, 0, 1, 639, 640, 767, 768, 65534, 65535, INT32_MAX};
  for (int32_t id : ids)
    for (int32_t j0 : {0, 128, 640, 65408})
      for (int32_t cols : {1, 128, 640}) {
        const bool in = sb::column_from(id, j0) < (uint32_t)cols;
        if (in != ((int64_t)id >= j0 && (int64_t)id < (int64_t)j0 + cols)) return 1;
      }
}
""")
    subprocess.run([exe], check=True)


def test_plans(tmp_path):
    exe = program(tmp_path, """
int main() {
  long long n; int d, k;
  while (std::scanf("%lld %d %d", &n, &d, &k) == 3) {
    if (d <= sb::DISTILL_REGS_MAX_D) {
      for (bool loss : {false, true}) {
        const sb::DistillPlan p = sb::distill_plan(n, d, k, loss);
        std::printf("%d %d %d %d %d %d %d\\n", p.rows, p.c, p.waves, p.groups, p.tiles, p.grid, p.lds);
      }
    } else {
      const sb::DistillWidePlan p = sb::distill_wide_plan(n, d);
      std::printf("%d %d %d %d\\n", p.ranges, p.cols, p.tiles, p.slots);
    }
  }
}
""")
    regs = [(n, d, k) for n in (1, 63, 65, 300, 65_537, 300_007, 2_000_000, 2**31 - 1) for k in (1, 10, 64)
            for d in (1, 8, 9, 64, 65, 100, 128, 129, 500, 512, 513, 600, 1000, 1024)]
    wide = [(n, d, 5) for n in (1, 64, 1000, 20_001, 100_003) for d in (1025, 1100, 5003, 9001, 65_535)]

    def run(shapes):
        text = "\n".join("%d %d %d" % s for s in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        return [tuple(map(int, line.split())) for line in out]

    lines = run(regs)
    assert len(lines) == 2 * len(regs)
    for (n, d, k), (rows, c, waves, groups, tiles, grid, lds) in zip([s for s in regs for _ in range(2)], lines):
        cols = c * (64 // rows)
        assert (waves - 1) * cols < d <= waves * cols and 1 <= waves * groups <= 16, "a wave without columns, or none for some"
        assert lds <= 160 * 1024, "more LDS than a CU has"
        assert tiles == -(-n // (rows * groups)) and 1 <= grid <= tiles
        per = -(-tiles // grid)
        assert (grid - 1) * per < tiles, "a block without tiles"
    for (n, d, k), (ranges, cols, tiles, slots) in zip(wide, run(wide)):
        assert cols % 64 == 0 and (ranges - 1) * cols < d <= ranges * cols
        assert tiles == -(-n // 64) and slots == min(tiles, 512)
        assert ranges * tiles < 2**31
