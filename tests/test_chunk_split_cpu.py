"""CPU: how the attention of a chunk is cut into pieces.  Either every unit has a fixed number of places
or a plan has a budget of pieces, never both, whatever the buffers' length; their records fit the
workspace.  The rule is compiled from the library's own header by the host compiler."""
import itertools
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include "dmc_internal.h"
int main() {
  int cu, rows, hkv, group, slots, total, chunk, shift, wide;
  while (std::scanf("%d %d %d %d %d %d %d %d %d", &cu, &rows, &hkv, &group, &slots, &total, &chunk, &shift, &wide) == 9) {
    const dmc::ChunkSplit x = dmc::chunk_split(cu, rows, hkv, group, slots, total, chunk, shift, wide != 0);
    std::printf("%d %d\n", x.fixed_parts, x.piece_budget);
  }
}
"""


def test_split_rule(tmp_path):
    cxx = shutil.which("g++")
    hip = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
    if cxx is None or not os.path.isdir(hip):
        pytest.skip("no host compiler")
    (tmp_path / "split.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", hip, "-I",
                    os.path.join(ROOT, "paper_2403_09636_amd", "csrc"), "-o", str(tmp_path / "split"),
                    str(tmp_path / "split.cpp")], check=True)
    cases = []
    for rows, hkv, group, slots, chunk, fp32 in itertools.product(
            (1, 4, 8, 24, 300), (1, 2, 8, 32), (1, 2, 4, 8), (100, 2000, 1 << 16, 1 << 24),
            (1, 4, 8, 32, 33, 500, 2 ** 31 - 1), (False, True)):
        wide = not fp32 and chunk * group > (32 if rows * hkv * slots >= 1 << 16 else 128)
        shift = (7 if wide else 5) - group.bit_length() + 1
        for total in (min(rows * chunk, 1 << 24), 1 << 24):   # as long as the rows can be, or far longer
            cases.append((256, rows, hkv, group, slots, total, chunk, shift, int(wide)))
    res = subprocess.run([str(tmp_path / "split")], input="\n".join(" ".join(map(str, c)) for c in cases),
                         capture_output=True, text=True, check=True)
    got = [tuple(map(int, line.split())) for line in res.stdout.strip().split("\n")]
    assert len(got) == len(cases)
    for i, ((cu, rows, hkv, group, slots, total, chunk, shift, wide), (fixed, budget)) in enumerate(zip(cases, got)):
        assert fixed >= 0 and budget >= 0 and fixed * budget == 0, cases[i]
        assert (fixed > 0) == (chunk * group <= 32 and rows * hkv <= 64), cases[i]
        assert fixed * rows * hkv <= 4 * cu and budget <= 4 * cu, cases[i]   # records in the workspace
        if i % 2:
            assert got[i] == got[i - 1], cases[i]   # rows of the buffer that no chunk can fill count for nothing
    assert len({g for g in got}) > 4
