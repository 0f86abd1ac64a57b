"""How the attention of the paged cache deals its work (csrc/paged_plan.h), compiled for the CPU and walked through: every tile
has one owner, and a sequence's tiles are the ones that its rows see."""
import pathlib
import shutil
import subprocess

import pytest

ROOT = pathlib.Path(__file__).resolve().parent.parent
CODE = r"""
#include <cstdio>
#include <cstdlib>
#include "../paper_2509_00579_amd/csrc/paged_plan.h"
using namespace kvc;
#define CHECK(x) do { if (!(x)) { printf("%s fails at line %d: %u %u\n", #x, __LINE__, A, Bv); exit(1); } } while (0)
static unsigned A, Bv;
int main() {
    for (unsigned total = 0; total < 700; total++)
        for (unsigned ways = 1; ways <= 70; ways++) {
            A = total; Bv = ways;
            const Deal d(total, ways);
            CHECK(d.begin(0) == 0 && d.begin(ways) == total);
            for (unsigned w = 0; w < ways; w++) {
                const unsigned n = d.begin(w + 1) - d.begin(w);
                CHECK(d.begin(w + 1) >= d.begin(w) && (n == total / ways || n == total / ways + 1));
                for (unsigned t = d.begin(w); t < d.begin(w + 1); t++) CHECK(d.owner(t) == w);
            }
        }
    const unsigned big = 0x7fffffffu;
    for (unsigned ways = 1; ways <= 256; ways++) {
        A = big; Bv = ways;
        const Deal d(big, ways);
        CHECK(d.begin(ways) == big);
        for (unsigned w = 0; w < ways; w++) CHECK(d.owner(d.begin(w)) == w && d.owner(d.begin(w + 1) - 1) == w);
    }
    for (int len = 1; len < 400; len++)
        for (int q = 1; q <= 40; q += 3)
            for (int window = 0; window < 400; window += window < 3 ? 1 : 31) {
                A = len; Bv = window;
                const TileRange r = tiles_of(len, q, window);
                CHECK(r.first >= 0 && r.count >= 1 && (r.first + r.count - 1) * kPBT < len && (r.first + r.count) * kPBT >= len);
                int low = len;  // the first key that any row sees
                for (int i = 0; i < q; i++) {
                    const int pos = len - q + i, from = window > 0 && pos - window + 1 > 0 ? pos - window + 1 : 0;
                    if (pos >= 0 && from < low) low = from;
                }
                CHECK(r.first * kPBT <= low && (window == 0 || len < q || low - r.first * kPBT < kPBT));
            }
    puts("ok");
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_tile_has_one_owner(tmp_path):
    src = tmp_path / "plan.cc"
    src.write_text(CODE.replace("../paper_2509_00579_amd", str(ROOT / "paper_2509_00579_amd")))
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout[-2000:]


DIVIDE = r"""
#include <cstdio>
#include <cstdlib>
#include "../paper_2509_00579_amd/csrc/paged_plan.h"
using namespace kvc;
static void check(unsigned d, unsigned n) {
    if (Divide(d).of(n) != n / d) { printf("%u / %u\n", n, d); exit(1); }
}
int main() {
    for (unsigned d = 1; d < (1u << 30); d += d < 5000 ? 1 : d / 97) {
        for (unsigned n = 0; n < 300; n++) check(d, n);
        for (unsigned k = 1; k && k <= 0x7fffffffu / d; k += 1 + k / 3)
            for (int off = -1; off <= 1; off++) check(d, k * d + off > 0x7fffffffu ? 0x7fffffffu : k * d + off);
        const unsigned last = 0x7fffffffu / d * d;
        check(d, last); check(d, last - 1); check(d, 0x7fffffffu); check(d, 0x7ffffffeu);
    }
    puts("ok");
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_division_by_multiplication(tmp_path):
    src = tmp_path / "divide.cc"
    src.write_text(DIVIDE.replace("../paper_2509_00579_amd", str(ROOT / "paper_2509_00579_amd")))
    exe = tmp_path / "divide"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout
