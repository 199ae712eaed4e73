"""How the status words of blocks and portions become a call's, on the CPU."""
import itertools
import os
import subprocess

from paper_2608_26523_b200 import build

VPP_H = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


def test_the_worst_of_several_status_words(tmp_path):
    """A portion that timed out shows, whatever portions before and after it report."""
    src, exe = tmp_path / "status.cc", tmp_path / "status"
    src.write_text("""#include <cstdio>
#include "vpp.h"
#include "device_status.h"
int main() {
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) std::printf("%d %d %d %d\\n", VPP_DEV_BAD_LENGTHS, VPP_DEV_BAD_BLOCK, VPP_DEV_TIMEOUT, vpp::worse_status(a, b));
}
""")
    subprocess.check_call(["g++", "-I", VPP_H, "-I", build.CSRC, "-o", str(exe), str(src)])
    rows = [[int(x) for x in line.split()] for line in subprocess.check_output([str(exe)]).decode().splitlines()]
    for (a, b), (lengths, page, timeout, got) in zip(itertools.product(range(4), repeat=2), rows):
        assert got == next((s for s in (timeout, page, lengths) if s in (a, b)), 0)
