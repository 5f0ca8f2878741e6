"""The batch operators' host-checkable arithmetic (csrc/batch_rules.hpp), compiled and run on the CPU."""
import os
import shutil
import subprocess

import pytest

import batch_large

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


def test_large_calls_get_the_launch_that_they_are_there_for(tmp_path):
    """Tiles, shared part, workgroup rows and heads a lane group of batch_large's cases, from the rules themselves."""
    body = r"""
int main(int argc, char** argv) {
    char kind;
    while (scanf(" %c", &kind) == 1) {
        if (kind == 'a') {
            dllm_attn_args g{};
            if (scanf("%d %d %d %d %d %d %d %d %d %d %d", &g.dtype, &g.n_rows, &g.n_seqs, &g.n_heads, &g.n_kv_heads, &g.head_dim,
                      &g.page, &g.table_ld, &g.shared_len, &g.max_rows, &g.max_len) != 11) return 1;
            const AttnPlan p = attn_plan(&g);
            printf("%d %d\n", 16 * p.qg * p.qt, p.shared > 0 && p.ns_s > 0);
        } else if (kind == 's') {
            int T, V;
            if (scanf("%d %d", &T, &V) != 2) return 1;
            const int n = select_ranges(V);
            printf("%d %d\n", select_rows_per(T, n), select_four_waves(select_wgs(T, n)));
        } else {
            int T, H, Hk;
            if (scanf("%d %d %d", &T, &H, &Hk) != 3) return 1;
            printf("%d 0\n", qk_heads_per(T, H, Hk));
        }
    }
}
"""
    asked, want = [], []
    for c in batch_large.ATTN:
        for dtype in c.dtypes:
            asked.append("a " + " ".join(map(str, c.plan_args(dtype))))
            want.append((f"{c.name} {dtype}", (c.tile, int(c.shared))))
    for *args, tile in batch_large.ODD:
        asked.append("a " + " ".join(map(str, batch_large.odd_plan_args(*args))))
        want.append((f"infinities {args[0]} {tile}", (tile, 1)))
    for rows, V, _, _, _, per, four in batch_large.SELECT:
        asked.append(f"s {sum(rows)} {V}")
        want.append((f"select {sum(rows)}", (per, int(four))))
    for T, H, Hk, _, _, heads in batch_large.QK:
        asked.append(f"q {T} {H} {Hk}")
        want.append((f"qk {T}", (heads, 0)))
    out = run_cpp(tmp_path, body, stdin="\n".join(asked)).split("\n")
    got = [(name, tuple(int(x) for x in line.split())) for (name, _), line in zip(want, out)]
    assert got == want
