"""Offsets into the scales of matrices with more columns than 32-bit arithmetic allows for, on the CPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r'''
#include <cstdio>
#include "%s/paper_2101_10761_b200/csrc/sidco_mx4.cuh"
int main() {
    const int octs[] = {0, 1, 3, 4, 15, 16, 17, 1000, (1 << 26) - 1, 1 << 26, (1 << 26) + 21, (1 << 28) - 8193};
    for (int o : octs) std::printf("%%d %%lld\n", o, (long long)sidco_mx4::scale_of_oct(o));
    return 0;
}
'''


def test_scale_of_every_eight_columns(tmp_path):
    """The layout of the header: block j of a row lies at (j / 4) * 512 + j % 4 from the row's first scale."""
    from paper_2101_10761_b200 import build
    src, exe = tmp_path / "offsets.cu", tmp_path / "offsets"
    src.write_text(PROGRAM % ROOT)
    subprocess.run([build.nvcc_path(), "-std=c++17", "-o", str(exe), str(src)], check=True, timeout=300)
    lines = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout.split("\n")
    seen = [tuple(int(v) for v in line.split()) for line in lines if line]
    assert len(seen) == 12
    for oct_, offset in seen:
        block = oct_ * 8 // 32
        assert offset == block // 4 * 512 + block % 4, (oct_, offset)
