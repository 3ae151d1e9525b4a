"""Which kernels the loss takes for the cases of test_gpu_xent_paths.py (csrc/xent_sizes.h, compiled for the host): a rule that changes
may not leave a branch without a case."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "xent_sizes.h"
#include <algorithm>
#include <cstdio>
using namespace jitdb;
template <int WM> static bool is_long(const Sizes &s, int64_t b_tiles, int64_t nk) {
    const int pairs = pair_count(s.parts, s.g_parts), half = grad_ranges(kTilePlaces<WM> / 2, s.a_tiles);
    return (int)make_plan((uint32_t)b_tiles, (uint32_t)nk, pairs, kTilePlaces<WM>, s.a_tiles).ranges > half;
}
int main() {
    for (int element : {4, 2})
        for (int ct : {1, 2, 4})
            for (int nb : {1, 2, 4, 8})
                if (few_variant(element, ct, nb)) std::printf("variant %d %d %d\n", element, ct, nb);
    long long n, labelled;
    int H, C, dtype, grad;
    while (std::scanf("%lld %lld %d %d %d %d", &n, &labelled, &H, &C, &dtype, &grad) == 6) {
        Sizes s;
        if (!make_sizes(n, H, C, (jitdb_dtype)dtype, (jitdb_dtype)grad, s)) return 1;
        const FewSizes few = few_sizes(dtype == JITDB_F32 ? 4 : 2, H, C);
        const int64_t rows = std::min<int64_t>(labelled, s.grad_rows), rt = ceil_div(rows, kTileB), ct = ceil_div(C, kTileB);
        const bool lh = s.wm == 4 ? is_long<4>(s, rt, ceil_div(C, 32)) : s.wm == 5 ? is_long<5>(s, rt, ceil_div(C, 32)) : is_long<2>(s, rt, ceil_div(C, 32));
        const bool lv = s.wm == 4 ? is_long<4>(s, ct, ceil_div(rows, 32)) : s.wm == 5 ? is_long<5>(s, ct, ceil_div(rows, 32)) : is_long<2>(s, ct, ceil_div(rows, 32));
        std::printf("case few=(%d,%d) res=%d stat_chunks=%d stat_used=%d grad_chunks=%d grad_used=%d join=%d bands=%d grad_bands=%d wm=%d a_tiles=%d long_h=%d long_v=%d\n",
                    few.ct, few.nb, s.res, (int)ceil_div(n, s.stat_rows), (int)ceil_div(labelled, s.stat_rows), (int)ceil_div(n, s.grad_rows),
                    (int)ceil_div(labelled, s.grad_rows), join_waves(stat_sets(s)),
                    s.res ? 0 : (int)ceil_div(ceil_div(std::min<int64_t>(labelled, s.stat_rows), 256), kBand),
                    s.res ? 0 : (int)ceil_div(2 * rt, kBand), s.wm, s.a_tiles, lh, lv);
    }
}
"""

# rows, labelled rows, features, classes, dtype, type of the gradients, what the case is there for
CASES = [
    # wide states: several chunks of rows forward and backward, the last one ragged; long ranges of tiles of 160 features
    (90112, 90000, 520, 50021, "bf16", "bf16", "res == 0 and stat_used == 2 and grad_used >= 3 and wm == 5 and long_h and long_v and join == 16"),
    # ... and chunks that no labelled row reaches
    (90112, 30001, 520, 50021, "bf16", "f32", "res == 0 and stat_chunks == 2 and stat_used == 1 and 1 < grad_used < grad_chunks"),
    (88000, 87001, 200, 50021, "f32", "f32", "res == 0 and stat_used == 2 and grad_used >= 3"),
    (88000, 500, 200, 50021, "f32", "f32", "res == 0 and stat_chunks == 2 and stat_used == 1 and grad_used == 1 and grad_chunks > 1"),
    # wide states: more than one band of row tiles
    (2500, 2500, 600, 700, "bf16", "bf16", "res == 0 and bands > 1 and grad_bands > 1 and stat_chunks == 1"),
    (2500, 2400, 600, 700, "bf16", "f32", "res == 0 and bands > 1 and grad_bands > 1"),
    (2500, 2500, 200, 700, "f32", "f32", "res == 0 and bands > 1 and grad_bands > 1"),
    (4097, 4097, 1030, 300, "bf16", "f32", "res == 0 and bands > 2"),
    # states of ordinary width, long ranges: tiles of 256, 128 and 160 features
    (20000, 20000, 512, 40000, "bf16", "bf16", "res == 32 and wm == 4 and a_tiles > 1 and long_h and long_v"),
    (8000, 8000, 384, 40000, "bf16", "f32", "res == 24 and wm == 2 and a_tiles > 1 and long_h and long_v"),
    (5500, 5500, 300, 42000, "f32", "f32", "res == 0 and wm == 5 and a_tiles > 1 and long_h and long_v"),
    (9000, 9000, 150, 42000, "f32", "f32", "res == 10 and wm == 5 and a_tiles == 1 and not long_h"),
    # several chunks backward, operands resident, the last ones empty
    (60000, 31000, 256, 40000, "bf16", "f32", "res == 16 and 1 < grad_used < grad_chunks"),
    # few rows: many sets of statistics
    (64, 64, 150, 10007, "f32", "f32", "res == 10 and join == 16"),
    (70, 33, 512, 20011, "bf16", "f32", "res == 32 and join == 16"),
    (70, 70, 600, 5000, "bf16", "bf16", "res == 0 and join == 16"),
    (3000, 3000, 100, 4099, "f32", "f32", "res == 8 and join == 4"),
    # few classes: every variant, each at its widest and inside
    (700, 650, 256, 16, "f32", "f32", "few == (1, 1)"), (700, 700, 300, 5, "f32", "f32", "few == (1, 2)"), (700, 700, 512, 16, "f32", "f32", "few == (1, 2)"),
    (700, 600, 600, 3, "f32", "f32", "few == (1, 4)"), (300, 300, 1024, 16, "f32", "f32", "few == (1, 4)"),
    (700, 700, 1200, 7, "f32", "f32", "few == (1, 8)"), (200, 200, 2048, 16, "f32", "f32", "few == (1, 8)"),
    (700, 700, 256, 32, "f32", "f32", "few == (2, 1)"), (700, 700, 333, 17, "f32", "f32", "few == (2, 2)"), (700, 690, 512, 32, "f32", "f32", "few == (2, 2)"),
    (700, 700, 777, 31, "f32", "f32", "few == (2, 4)"), (300, 299, 1024, 32, "f32", "f32", "few == (2, 4)"),
    (700, 700, 256, 64, "f32", "f32", "few == (4, 1)"), (700, 610, 99, 33, "f32", "f32", "few == (4, 1)"),
    *[(n, k, H, C, "bf16", grad, want) for grad in ("f32", "bf16") for n, k, H, C, want in [
        (700, 700, 512, 16, "few == (1, 1)"), (700, 650, 600, 9, "few == (1, 2)"), (700, 700, 1024, 16, "few == (1, 2)"),
        (700, 700, 1300, 5, "few == (1, 4)"), (200, 200, 2048, 16, "few == (1, 4)"), (700, 700, 512, 32, "few == (2, 1)"),
        (700, 600, 555, 18, "few == (2, 2)"), (300, 300, 1024, 32, "few == (2, 2)"), (700, 700, 512, 64, "few == (4, 1)"),
        (700, 699, 77, 50, "few == (4, 1)")]],
    # more rows than the blocks of few classes take in one turn
    (140000, 130000, 600, 4, "f32", "f32", "few == (1, 4)"), (140000, 139000, 1030, 12, "bf16", "f32", "few == (1, 4)"),
    (140000, 70000, 500, 40, "bf16", "bf16", "few == (4, 1)"), (70001, 70001, 1100, 3, "f32", "f32", "few == (1, 8)"),
]


@pytest.fixture(scope="module")
def answers(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("paths")
    (at / "paths.cpp").write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_1904_07421_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                    "-o", str(at / "paths"), str(at / "paths.cpp")], check=True)
    types = {"f32": 0, "bf16": 1}
    asked = "\n".join(f"{n} {k} {H} {C} {types[d]} {types[g]}" for n, k, H, C, d, g, _ in CASES)
    out = subprocess.run([str(at / "paths")], input=asked, capture_output=True, text=True, check=True, timeout=20).stdout.splitlines()
    variants = {tuple(int(v) for v in line.split()[1:]) for line in out if line.startswith("variant")}
    cases = [{k: eval(v) for k, v in (f.split("=") for f in line.split()[1:])} for line in out if line.startswith("case")]
    return variants, cases


def test_each_case_takes_the_branch_it_is_there_for(answers):
    _, cases = answers
    assert len(cases) == len(CASES)
    for case, found in zip(CASES, cases):
        assert eval(case[-1], {}, found), (case, found)


def test_every_variant_of_few_classes_has_a_case(answers):
    variants, cases = answers
    seen = {(4 if case[4] == "f32" else 2, *found["few"]) for case, found in zip(CASES, cases) if found["few"][0]}
    assert seen == variants
