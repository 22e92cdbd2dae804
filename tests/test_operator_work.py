"""How the operators beside the step divide their work, checked on the CPU over sizes that no GPU test allocates: the program below is
compiled against the header that the kernels and their launchers use."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(tmp_path, body):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include "qadam_operator_work.h"\n#include <cstdio>\n#include <cstdlib>\n#include <initializer_list>\nusing namespace qadam;\n'
                   '#define CHECK(c, ...) do { if (!(c)) { std::puts(#c); std::printf(__VA_ARGS__); std::exit(1); } } while (0)\n'
                   "int main() {\n" + body + "\nreturn 0; }\n")
    inc = os.path.join(ROOT, "paper_2004_14180_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-unused", "-I", inc, "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_sums_of_a_sorted_list_fit_a_launch(tmp_path):
    """Whatever rows, columns and tokens a handle takes: fewer than 2^32 work-items, and every row is cleared."""
    _run(tmp_path, """
    for (long long rows = 1; rows <= 1ll << 28; rows = rows < (1ll << 28) && rows * 2 > 1ll << 28 ? 1ll << 28 : rows * 2 + (rows > 3) * 5)
        for (long long dim = 1; dim <= 1 << 20; dim = dim * 3 / 2 + 1)
            for (long long tokens = 1; tokens <= 1ll << 24; tokens *= 2) {
                if (sum_groups(tokens, (int)dim) >= kMostSums) continue;        // refused by the handle
                const long long clear = clear_groups(rows);
                CHECK((sum_groups(tokens, (int)dim) + clear) * 64 < kMostItems, "rows %lld dim %lld tokens %lld", rows, dim, tokens);
                // the kernel's turns
                const long long turn = clear * kClearRows, last = (rows - 1) / turn * turn;
                CHECK(clear > 0 && clear <= (rows + kClearRows - 1) / kClearRows && last < rows && last + turn >= rows, "rows %lld", rows);
            }
    CHECK((sum_groups((1 << 24), 512) + clear_groups(1 << 28)) * 64 < kMostItems, "the largest");
    CHECK(clear_groups(0) == 0 && clear_groups(1) == 1 && clear_groups(50257) == 25129, "a wavefront for every two rows");""")


def test_the_ends_of_a_run_are_found_in_few_looks(tmp_path):
    """Boundaries within the run from none to those of 2^24 tokens of one row: found, in one look up to 63 and in seven at most."""
    _run(tmp_path, """
    const int most = (1 << 24) / kRunPiece + 1;
    int worst = 0;
    for (int count = 0; count <= most; count += count < 300000 && count > 9000 ? 997 : 1) {
        RunSearch s;
        int looks = 0;
        for (bool more = true; more; ++looks) {
            int matched = 0;
            while (matched < 64 && s.place(matched) < count) ++matched;
            for (int lane = matched; lane < 64; ++lane) CHECK(s.place(lane) >= count && (long long)s.place(lane) * kRunPiece < 1ll << 30, "%d", count);
            more = s.next(matched);
        }
        CHECK(s.count == count && (count > 63 || looks == 1), "%d: %d in %d looks", count, s.count, looks);
        worst = looks > worst ? looks : worst;
    }
    CHECK(worst <= 7, "%d looks", worst);""")
