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


def test_scratch_of_the_gradient(tmp_path):
    """Every piece and every arrival has its place, whichever way the list's length takes, and none is reserved for a way that no list takes."""
    _run(tmp_path, """
    for (long long dim = 1; dim <= 1 << 20; dim = dim < 10000 ? dim + 1 : dim + dim / 7) {
        const int d = (int)dim, slices = column_slices(d), groups = groups_per_token(d);
        CHECK(slices * 64 * lane_columns(d) >= d && (slices - 1) * 64 * lane_columns(d) < d && d >= lane_columns(d), "dim %d", d);
        CHECK((groups << log_group_slices(d)) >= slices && ((groups - 1) << log_group_slices(d)) < slices && kDirectWaves >> log_group_slices(d), "dim %d", d);
        const long long direct = direct_tokens(d);
        CHECK(direct >= 1 && direct <= kDirectTokens && direct * groups <= kDirectGroups, "dim %d", d);
        CHECK(direct == kDirectTokens || (direct + 1) * groups > kDirectGroups, "dim %d", d);
        CHECK((direct * groups + direct_clear_groups(1 << 28)) * 64 * kDirectWaves < kMostItems, "dim %d", d);
        for (long long most : {1ll, 2ll, 39ll, 40ll, 41ll, 500ll, 512ll, 1023ll, 1024ll, 2047ll, 2048ll, 2049ll, 50000ll, 1ll << 24}) {
            const long long pieces = piece_places(most, d), arrivals = arrival_places(most, d);
            const long long shorter = most < direct ? most : direct, last = (most - 1) / kRunPiece;
            CHECK(pieces >= shorter && arrivals >= shorter, "dim %d, %lld tokens", d, most);
            CHECK(pieces >= 2 * last + 2 && arrivals >= last + 1, "dim %d, %lld tokens", d, most);
            CHECK(4 * pieces * dim <= (most * dim) / 5 + 8 * dim + (8 << 20), "dim %d, %lld tokens", d, most);
        }
    }
    CHECK(direct_tokens(768) == 2048 && direct_tokens(1024) == 2048 && direct_tokens(1025) == 1024 && direct_tokens(2048) == 1024 &&
          direct_tokens(4096) == 512, "the lengths that the comments name");""")


def test_launches_of_a_list_fit(tmp_path):
    """Whatever the tensors' sizes: fewer than 2^32 work-items of AdamW per launch, and its gradients' addresses fit."""
    _run(tmp_path, """
    CHECK(kMostLaunchTiles * kTileBlocks * 64 < kMostItems && (kMostLaunchTiles + 1) * kTileBlocks * 64 == kMostItems, "the most");
    for (long long tiles : {0ll, 1ll, 1000ll, 9362ll, 9363ll, 1ll << 18, (1ll << 22) - 1}) {
        long long tensors = 0, sum = 0;
        while (list_launch_takes(tensors, sum, tiles)) { ++tensors; sum += tiles; }
        CHECK(tensors >= 1 && tensors <= kListGrads && sum * kTileBlocks * 64 < kMostItems, "%lld tiles", tiles);
        CHECK(tensors == kListGrads || sum + tiles > kMostLaunchTiles, "%lld tiles: %lld tensors", tiles, tensors);
    }""")
