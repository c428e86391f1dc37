"""What the attention kernels over a cache of codes lay out in LDS, for every shape, without a GPU: sums and tables fit what is asked for, and where wide loads and stores
go is a multiple of their size."""
import os
import subprocess

from paper_1509_05194_amd import build

LAYOUT = r'''
#include "attend.hpp"
#include <stdio.h>
using namespace hclae;
int main()
{
    for (int R = 1; R <= 5; ++R)
        for (int M = 1; M <= 40; ++M)
            for (int K = 1; K <= 256; ++K)
                for (int wide = 0; wide < 2; ++wide) {
                    const CodesPlan p = codes_plan(R, M, K, wide);
                    if (!p.RB) continue;
                    const int MW = M <= 8 ? 2 : M <= 16 ? 4 : 8, threads = codes_threads(p.RB, p.wide, MW);
                    const int sums = M * K * (p.wide ? p.RB : p.RB / 2) * 8, tables = M * K * p.RB * 4, at = codes_lut(M * K * (p.wide ? p.RB : p.RB / 2));
                    if (at % 16 || at < sums || at + tables > p.lds || p.lds > kCodesLds) return printf("place: R %d M %d K %d wide %d\n", R, M, K, wide), 1;
                    if (codes_words(p.RB, p.wide, MW) * threads < sums / 8 || codes_words(p.RB, p.wide, MW) > 32) return printf("words: R %d M %d K %d wide %d\n", R, M, K, wide), 2;
                    if (threads == 512 && p.lds > 80 * 1024 - 2048) return printf("two blocks: R %d M %d K %d wide %d\n", R, M, K, wide), 3;
                }
    return 0;
}
'''


def test_sums_and_tables(tmp_path):
    src = tmp_path / "layout.hip"
    src.write_text(LAYOUT)
    exe = tmp_path / "layout"
    p = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-std=c++17", "-O1", "--offload-arch=gfx950", "-I", build.CSRC, "-o", str(exe), str(src)],
                       capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr
    p = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert p.returncode == 0, p.stdout
