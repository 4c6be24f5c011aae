"""Which kernel a microscaled product runs on (csrc/mx_plan.h), compiled for the host: the sizes that the GPU tests run reach every one of them, whole and
in K splits, and the choice stays within what a launch can hold over the documented range."""
import os
import subprocess

import pytest

from mx_sizes import SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

HARNESS = r"""
#include "mx_plan.h"
#include <stdio.h>
#include <string.h>
using namespace poss;
static long wrong = 0, seen = 0;
static void check(bool both, int parts, int M, int N, int K) {
    const MxPlan p = mx_plan_of(both, parts, M, N, K);
    const MxTile &t = both ? MX_BOTH_TILES[p.shape] : MX_TILES[p.shape];
    const int groups = mx_groups(K) * parts;
    const double tiles = (double)((M + t.tm - 1) / t.tm) * ((N + t.tn - 1) / t.tn);
    // a launch has fewer than 2^32 threads (768 of a workgroup at most; 512 of the largest tiles), a split at least one group, and planes are few
    const double threads = p.shape == MX_STREAM ? 1024. * ((N + 15) / 16) / (stream_waves((N + 15) / 16, mx_groups(K)) > 4 ? 1 : 4) : tiles * p.splits * (t.tm == 256 ? 512 : 768);
    bool ok = p.splits >= 1 && p.splits <= 16 && p.splits <= groups && threads < 4294967296.0 && (p.splits == 1 || tiles * p.splits <= 1024);
    if (p.shape == MX_STREAM) ok = ok && M <= 16 && p.splits == 1 && stream_waves((N + 15) / 16, mx_groups(K)) <= mx_groups(K);
    ++seen;
    if (!ok && wrong++ < 5) printf("M %d N %d K %d both %d parts %d: tile %d x %d, %d splits\n", M, N, K, both, parts, t.tm, t.tn, p.splits);
}
int main(int argc, char **argv) {
    if (argc > 1) {
        char kind[8];
        int M, N, K;
        while (scanf("%7s %d %d %d", kind, &M, &N, &K) == 4) {
            const bool both = !strcmp(kind, "mx");
            const MxPlan p = mx_plan_of(both, strcmp(kind, "f32") ? 1 : 3, M, N, K);
            const MxTile &t = both ? MX_BOTH_TILES[p.shape] : MX_TILES[p.shape];
            printf("%dx%d %d\n", t.tm, t.tn, p.splits);
        }
        return 0;
    }
    for (int form = 0; form < 3; ++form)
        for (long m = 1; m <= 1 << 24; m = m * 3 / 2 + 1)
            for (long n = 1; n <= 1 << 27 && m * n <= 1l << 38; n = n * 3 / 2 + 1)
                for (long k = 1; k <= 1 << 21; k = k * 2 + 1) check(form == 2, form == 1 ? 3 : 1, (int)m, (int)n, (int)k);
    for (int form = 0; form < 3; ++form) { check(form == 2, form == 1 ? 3 : 1, 1 << 24, 1 << 14, 64); check(form == 2, form == 1 ? 3 : 1, 1 << 11, 1 << 27, 1 << 21); }
    for (int n = 4; n <= 1 << 22; n = n * 5 / 4 + 4)
        for (int k = 8; k <= 1 << 21; k = k * 3 / 2 + 8) {
            const int s = mx_plane_splits(n, k), groups = mx_groups(k);
            bool ok = s >= 1 && s <= 16 && s <= groups;
            for (int i = 0; i < s; ++i) ok = ok && (long)(i + 1) * groups / s > (long)i * groups / s;      // (no split is empty)
            for (int m = 1; m <= 256; m += m < 20 ? 1 : 13) { const MxPlan p = best_plan(MX_TILES, m, n, groups, s); ok = ok && p.shape != MX_STREAM && p.splits == s; }
            ++seen;
            if (!ok && wrong++ < 5) printf("planes of N %d K %d: %d splits\n", n, k, s);
        }
    printf("wrong %ld of %ld\n", wrong, seen);
    return wrong != 0;
}
"""


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cc").write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2506_03566_amd", "csrc"), str(d / "plan.cc"), "-o", str(d / "plan")], check=True)
    return str(d / "plan")


def test_plans_fit_a_launch(planner):
    r = subprocess.run([planner], stdout=subprocess.PIPE, text=True)
    print(r.stdout)
    assert r.returncode == 0


def test_the_tested_sizes_reach_every_kernel(planner):
    lines = "".join("%s %d %d %d\n" % s[:4] for s in SIZES)
    got = subprocess.run([planner, "sizes"], input=lines, stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")
    assert [g for g in got if g] == ["%s %d" % s[4:] for s in SIZES]
    reached = {(kind, tile, splits > 1) for kind, _, _, _, tile, splits in SIZES}
    tiled = {"16": ["16x64", "32x128", "32x256", "64x128", "64x256", "256x256"], "mx": ["16x64", "32x128", "64x128", "64x256", "256x256"]}
    tiled["f32"] = tiled["16"]
    assert reached == {(kind, t, split) for kind, ts in tiled.items() for t in ts for split in (False, True)} | {(kind, "16x16", False) for kind in tiled}


def test_splits_of_a_contexts_matrices(tmp_path):
    """By the columns alone: half of 256 CUs a tile of 128 columns, two splits from a quarter on, none beyond three quarters."""
    (tmp_path / "splits.cc").write_text('#include "mx_plan.h"\n#include <stdio.h>\nint main() { int n, k; while (scanf("%d %d", &n, &k) == 2) printf("%d\\n", poss::mx_plane_splits(n, k)); }\n')
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2506_03566_amd", "csrc"), str(tmp_path / "splits.cc"), "-o", str(tmp_path / "splits")], check=True)
    cases = {(128, 1 << 21): 16, (1024, 8192): 16, (1024, 4096): 8, (4096, 4096): 4, (4096, 14336): 4, (5120, 5120): 3, (8192, 4096): 2, (8193, 4096): 2, (15360, 5120): 2, (24576, 4096): 2,
             (24577, 4096): 1, (28672, 4096): 1, (4096, 512): 1, (1024, 1536): 3, (1024, 5632): 11, (2048, 5120): 5}
    got = subprocess.run([str(tmp_path / "splits")], input="".join("%d %d\n" % c for c in cases), stdout=subprocess.PIPE, text=True, check=True).stdout.split()
    assert [int(g) for g in got] == list(cases.values())
