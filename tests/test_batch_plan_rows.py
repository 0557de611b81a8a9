"""Positions of a plan's rows and the pages that they lie in, at the ends of their range (no GPU needed)."""
import subprocess
import textwrap

from paper_2609_36938_b200 import build


def test_positions_that_do_not_fit(tmp_path):
    """A cached length near 2^63 has no page in any table: neither the sum nor the page number may wrap into one."""
    src = tmp_path / "rows.cpp"
    src.write_text(textwrap.dedent("""
        #include "batch_plan_rows.h"
        using namespace janus;
        int main() {
            const int64_t top = INT64_MAX, cached[] = {top, top - 1, top - 5, int64_t(1) << 62, int64_t(1) << 40, INT64_MIN, -3, 0, 5, 1000};
            const int64_t row[] = {0, 1, 2, 7, 100, INT32_MAX};
            const int page[] = {1, 7, 24, 40, 64, 96, 128, 1 << 30};
            const int32_t pages[] = {0, 1, 17, INT32_MAX};
            for (int64_t c : cached)
                for (int64_t i : row) {
                    const __int128 sum = static_cast<__int128>(c > 0 ? c : 0) + i;
                    const int64_t pos = bp_position(c, i);
                    if (pos != (sum > top ? top : static_cast<int64_t>(sum))) return 1;
                    for (int p : page)
                        for (int32_t n : pages) {
                            int shift = -1;
                            for (int s = 0; s < 31; ++s)
                                if (p == 1 << s) shift = s;
                            const __int128 j = sum / p;
                            if (bp_page_of(pos, p, shift, n) != (j < n ? static_cast<int32_t>(j) : -1)) return 2;
                        }
                }
            return 0;
        }
    """))
    exe = tmp_path / "rows"
    subprocess.check_call(["g++", "-std=c++17", "-I", build.CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0


def test_the_kernel_goes_by_them():
    with open(build.CSRC + "/batch_plan.cu") as f:
        code = f.read()
    assert code.count("bp_position(") == 1 and code.count("bp_page_of(") == 1 and "ld_input(p.cached + b) +" not in code
