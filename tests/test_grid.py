"""The rows that one launch takes at most, compiled for the host (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(__file__)), "paper_1905_09598_amd", "csrc")

# Rows of up to 4,000,000 values in 8 bits are up to 7813 units of four blocks, four of them
# to a workgroup of 256 threads; a grid counts 2^32 - 1 threads.
SOURCE = """
#include "som_grid.h"
#include <initializer_list>
#include <cstdio>
int main() {
    for (int64_t units = 1; units <= 7813; ++units)
        for (const int64_t per : {1, 4})
            for (const int64_t threads : {64, 256, 1024}) {
                const int64_t rows = som::rows_at_once(units, per, threads);
                const auto groups = [&](int64_t r) { return (r * units + per - 1) / per; };
                const bool fits = rows >= 1 && groups(rows) * threads <= 4294967295ll &&
                                  som::grid_holds(groups(rows), threads);
                // no fewer than fit, to a row
                const bool most = groups(rows + 1) * threads > 4294967295ll;
                if (!fits || !most) {
                    std::printf("%lld units, %lld to a group of %lld: %lld rows\\n", (long long)units,
                                (long long)per, (long long)threads, (long long)rows);
                    return 1;
                }
            }
    return 0;
}
"""


def test_rows_of_a_launch(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    src, exe = tmp_path / "rows.cpp", tmp_path / "rows"
    src.write_text(SOURCE)
    subprocess.run([cxx, "-std=c++17", "-O1", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
