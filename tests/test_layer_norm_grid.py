"""The layer norm's backward pass (csrc/layer_norm.hip, host side): its workgroups."""
import os
import subprocess

from test_head_routes import HIPCC, ROOT

PROGRAM = r"""
#include <cstdio>
#include "layer_norm.hip"
namespace tppo { int device_compute_units() { return 256; } }
using namespace tppo;
int main() {
    int wrong = 0;
    for (int at_once : {1, 4}) for (int resident : {1, 2, 4, 8})
        for (int64_t M = 1; M <= 200000; M += M < 9000 ? 1 : 997) {
            const int64_t groups = backward_groups(M, at_once, resident), tasks = (M + at_once - 1) / at_once, turns = (tasks + groups - 1) / groups;
            bool good = groups >= 1 && groups <= tasks && groups <= 1024 && groups <= 256 * resident;
            good = good && tasks > (turns - 1) * groups;                       // all of them in the last turn but for what is left over
            // as many as the next multiple of four rows has, which all workgroups share alike
            if (M > 1024) good = good && groups >= backward_groups((M + 3) / 4 * 4, at_once, resident) - 3;
            if (!good && ++wrong < 10) printf("M %ld at once %d resident %d: %ld\n", (long)M, at_once, resident, (long)groups);
        }
    printf("%d\n", wrong);
}
"""


def test_neighbouring_sizes_have_as_many_workgroups(tmp_path):
    (tmp_path / "grid.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O0", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2506_15050_amd", "csrc"), str(tmp_path / "grid.hip"),
                    "-o", str(tmp_path / "grid")], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    assert subprocess.run([str(tmp_path / "grid")], check=True, stdout=subprocess.PIPE, text=True).stdout.split("\n") == ["0", ""]
