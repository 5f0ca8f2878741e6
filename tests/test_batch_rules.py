"""The batch operators' host-checkable arithmetic (csrc/batch_rules.hpp), compiled and run on the CPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run_cpp(tmp_path, body, *args, stdin=None):
    """Output of a small program around batch_rules.hpp; overflow of a signed sum ends it (-ftrapv)."""
    cc = shutil.which("g++")
    if not cc:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "rules.cpp", tmp_path / "rules"
    src.write_text('#include <cstdio>\n#include <initializer_list>\n#include "batch_rules.hpp"\nusing namespace dllm;\n' + body)
    subprocess.check_call([cc, "-std=c++17", "-O0", "-ftrapv", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-I",
                           os.path.join(ROOT, "paper_2606_13740_amd", "csrc"), str(src), "-o", str(exe)])
    return subprocess.run([str(exe), *args], input=stdin, capture_output=True, text=True, check=True).stdout


def test_row_range_stays_inside_the_call(tmp_path):
    """Whatever row bounds device memory holds, and for a bound of 2^31 - 1 rows a sequence: [begin, end) inside [0, n_rows), at
    most the bound, and the plain range wherever that is valid."""
    out = run_cpp(tmp_path, r"""
int main() {
    const int lo = -2147483647 - 1, hi = 2147483647;
    const int v[] = {lo, lo + 1, -5, -1, 0, 1, 2, 31, 63, 64, 65, 70, 1 << 24, hi - 64, hi - 1, hi};
    const int most[] = {0, 1, 32, 64, 70, 1 << 24, hi - 64, hi};
    long n = 0;
    for (int T : {1, 64, 70, 1 << 24})
        for (int a : v)
            for (int b : v)
                for (int m : most) {
                    const RowRange r = row_range(a, b, m, T);
                    if (r.begin < 0 || r.begin > T || r.end < r.begin || r.end > T || r.end - r.begin > m) return 1;
                    if (a >= 0 && b >= a && b <= T && (r.begin != a || r.end - a != (b - a < m ? b - a : m))) return 2;
                    if (b <= a && r.end != r.begin) return 3;
                    ++n;
                }
    printf("%ld\n", n);
}
""")
    assert int(out) == 4 * 16 * 16 * 8
