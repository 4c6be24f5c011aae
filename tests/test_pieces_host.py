"""The units of a row that the rotation hands to its lanes (csrc/pieces.h), compiled for the host: a unit's head is the quotient that its multiplier stands for, for every size that
is taken, heads of a single unit and the widest rows among them; the units of a head cover each of its pieces once."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include "pieces.h"
#include <stdio.h>
#include <vector>
using namespace poss;
int main() {
    long wrong = 0, taken = 0, single = 0, refused = 0;
    for (int E = 4; E <= 8; E += 4)
        for (int dh = E; dh <= 16384; dh += dh < 1024 ? E : 509 * E)
            for (int rot = 0; rot <= (dh < 256 ? dh : 256); rot += E)
                for (int inter = 0; inter < 2; ++inter)
                    for (int heads : {1, 2, 3, 7, 40, 1000, 65535, 300000, 2000000, 16777215}) {
                        Units n{};
                        if (!units_of(E, 300, heads, dh, rot, inter, n)) { refused += rot % (2 * E) == 0 && heads <= 65535 && dh <= 256; continue; }
                        ++taken;
                        single += n.units == 1;
                        // pieces of a head: those of the first half stand for two
                        const int turned = inter ? rot / E : rot / 2 / E;
                        if (n.units - turned < 0 || n.units + (inter ? 0 : turned) != dh / E) ++wrong;
                        const int64_t all = (int64_t)heads * n.units;
                        auto look = [&](int64_t j) {
                            if (j >= 0 && j < all && unit_head((int)j, n.of_units) != j / n.units && wrong++ < 5)
                                printf("E %d dh %d rot %d interleaved %d: unit %ld of %d is head %d\n", E, dh, rot, inter, (long)j, n.units, unit_head((int)j, n.of_units));
                        };
                        for (int64_t j = 0; j < all && j < 300; ++j) look(j);
                        // next to multiples, where a quotient would slip first, up to the last
                        for (int64_t h = heads, i = 0; i < 40; ++i, h -= 1 + h / 8) { look(h * n.units - 1); look(h * n.units); look(h * n.units + 1); }
                    }
    printf("taken %ld single %ld refused %ld wrong %ld\n", taken, single, refused, wrong);
    return wrong || !single || refused;
}
"""


def test_a_units_head_is_the_quotient(tmp_path):
    src, exe = tmp_path / "pieces.cc", tmp_path / "pieces"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2506_03566_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    print(r.stdout)
    assert r.returncode == 0
