"""How layer norm and the product in 8-bit integers divide their work, checked on the CPU over sizes that no GPU test allocates: the program
below is compiled against the header that the kernels and their launchers use."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(tmp_path, body):
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text('#include "qadam_layer_work.h"\n#include <cstdio>\n#include <cstdlib>\n#include <vector>\nusing namespace qadam;\n'
                   '#define CHECK(c, ...) do { if (!(c)) { std::puts(#c); std::printf(__VA_ARGS__); std::exit(1); } } while (0)\n'
                   "int main() {\n" + body + "\nreturn 0; }\n")
    inc = os.path.join(ROOT, "paper_2004_14180_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-unused", "-I", inc, "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_every_tile_has_one_workgroup(tmp_path):
    _run(tmp_path, """
    for (int across : {1, 2, 3, 7, 8, 32, 33, 393})
        for (int down : {1, 2, 3, 4, 5, 8, 9, 63, 64, 65, 130}) {
            std::vector<int> seen(across * down);
            for (int b = 0; b < across * down; ++b) {
                int tm = -1, tn = -1;
                tile_place(b, across, down, &tm, &tn);
                CHECK(tm >= 0 && tm < down && tn >= 0 && tn < across, "%d x %d: block %d at %d, %d", across, down, b, tm, tn);
                CHECK(seen[tm * across + tn]++ == 0, "%d x %d: %d, %d twice", across, down, tm, tn);
            }
        }""")


def test_the_products_plan(tmp_path):
    """The integers that a workgroup makes fit its LDS and its threads, wavefronts that share the inputs divide a workgroup's."""
    _run(tmp_path, """
    for (long long tokens = 1; tokens <= 1 << 24; tokens = tokens * 5 / 4 + 1)
        for (long long outputs = 1; outputs <= 1 << 24; outputs = outputs * 3 / 2 + 1)
            for (int inputs = 1; inputs < 1 << 17; inputs = inputs * 3 / 2 + 1) {
                const Linear8Plan p(tokens, outputs, inputs, true), q(tokens, outputs, inputs, false);
                CHECK(!q.made && p.kind == q.kind, "kind");
                CHECK(!p.made || tokens * linear8_padded(inputs) <= kMadeInputs, "%lld %d", tokens, inputs);
                CHECK((tokens <= kRowsTokens) == (p.kind == Linear8Plan::kRows), "few tokens");
                CHECK(p.split >= 1 && p.split <= kRowWaves && kRowWaves % p.split == 0, "split %d", p.split);
                for (bool direct : {false, true}) {
                    const Linear8Plan s(tokens, outputs, inputs, true, direct);
                    const long long tiles = (tokens + 63) / 64 * ((outputs + 63) / 64);
                    CHECK(s.parts >= 1 && s.parts <= (inputs + 127) / 128, "parts %d", s.parts);
                    CHECK(s.parts == 1 || (tiles * s.parts <= kPartTiles && s.kind == Linear8Plan::kTiles64Deep), "parts %d", s.parts);
                    CHECK(s.parts == 1 || linear8_may_share(outputs, inputs, tokens), "scratch");
                }
            }
    CHECK(linear8_padded(1) == 128 && linear8_padded(128) == 128 && linear8_padded(129) == 256 && linear8_padded((1 << 17) - 1) == 1 << 17, "padded");""")


def test_scratch_of_the_norms_gradient(tmp_path):
    _run(tmp_path, """
    for (int dim = 1; dim <= 1 << 20; ++dim) {
        const int n = norm_partials(dim);
        CHECK(n >= 8 && n <= 512 && (long long)n * 8 * dim <= 64ll << 20, "dim %d: %d", dim, n);
    }""")
