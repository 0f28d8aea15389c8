"""Which kernels the gated feed-forward block takes (csrc/ffn_plan.h compiled for the host), and that the GPU tests' shapes reach
every one that its rules choose over the range of real sizes: another constant there cannot leave a kernel untested."""
import math
import os
import random
import shutil
import subprocess

import pytest

from ffn_shapes import PLAN_SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LARGEST = 16384 * 2048 * 5632          # tokens d f of the largest timed block

# reads "t d f" per line; prints for each product its form, tile, workgroups a unit, tiles, whole ones, splits and K tiles
PROGRAM = r"""
#include <cstdio>
#include "ffn_plan.h"
using namespace mlc;
int main() {
  long t, d, f;
  while (std::scanf("%ld %ld %ld", &t, &d, &f) == 3) {
    auto put = [&](const char* form, const Plan& p, int n, const Size* s, long kt) {
      long tiles = 0;
      for (int i = 0; i < n; ++i) tiles += (s[i].M + p.bm - 1) / p.bm * ((s[i].N + p.bn - 1) / p.bn);
      std::printf("%s %d %d %d %ld %d %d %ld %zu ", form, p.bm, p.bn, p.per_unit, tiles, p.whole, p.splits, kt, partial_bytes(p));
    };
    const Size up{t, 2 * f}, down{t, d}, inner{t, f}, dw[3] = {{f, d}, {f, d}, {d, f}};
    if (few(t, f, d)) std::printf("UP 0 0 0 0 0 0 0 0 "); else put("UP", plan_up(t, d, f), 1, &up, k_tiles(d));
    if (few(t, d, f)) std::printf("NT 0 0 0 0 0 0 0 0 "); else put("NT", plan_down(t, d, f), 1, &down, k_tiles(f));
    put("DH", plan_inner(t, d, f), 1, &inner, k_tiles(d));
    put("NN", plan_dx(t, d, f), 1, &down, 2 * k_tiles(f));
    put("TN", plan_dw(t, d, f), 3, dw, k_tiles(t));
    std::printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    tmp = tmp_path_factory.mktemp("plan")
    (tmp / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "paper_2505_23725_amd", "csrc"),
                    str(tmp / "plan.cpp"), "-o", str(tmp / "plan")], check=True)

    def run(shapes):
        text = "".join("%d %d %d\n" % s for s in shapes)
        out = subprocess.run([str(tmp / "plan")], input=text, capture_output=True, text=True, check=True).stdout
        lines = [line.split() for line in out.splitlines()]
        return [[(w[i], *map(int, w[i + 1:i + 9])) for i in range(0, len(w), 9)] for w in lines]
    return run


def kind(plan, tokens):
    """What a plan runs that others do not: the form; the tile and how many workgroups share a unit (the kernel); whether its
    tiles are one round, run on over several, are all cut along K or only the last round's; and whether a tile has no more K tiles than
    are requested ahead, so that the requests run on into the next one or beyond the list."""
    form, bm, bn, per_unit, tiles, whole, splits, kt, _ = plan
    if not bm:
        return (form, "few", (tokens + 15) // 16)
    if splits > 1:
        how = "rounds, then cut" if whole else "cut"
    else:
        how = "rounds" if tiles > 256 * per_unit else "a round"
    return (form, bm, per_unit, how, kt // splits <= (4 if per_unit == 1 and bm < 256 else 2))


def draws(n, seed):
    rng = random.Random(seed)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    for _ in range(n):
        d, f = 8 * log(1, 1024), 8 * log(1, 2560)
        t = min(log(1, 32768), LARGEST // (d * f))
        if t:
            yield t, d, f


def test_the_gpu_tests_reach_every_choice(plans):
    reached = {kind(p, s[0]) for s, ps in zip(PLAN_SHAPES, plans(PLAN_SHAPES)) for p in ps}
    shapes, missing = list(draws(60000, 1)), {}
    for s, ps in zip(shapes, plans(shapes)):
        for p in ps:
            if kind(p, s[0]) not in reached:
                missing.setdefault(kind(p, s[0]), s)
    assert not missing, missing
    # every kernel of the tables is somebody's choice: five tiles for each form, two for few tokens of UP and NT
    assert len({k[:3] for k in reached}) == 5 * 5 + 2 * 2 and {k[3] for k in reached if k[1] != "few"} == {"a round", "rounds", "cut",
                                                                                                          "rounds, then cut"}


def test_plans_fit_their_launches_and_work_spaces(plans):
    shapes = list(draws(20000, 2)) + PLAN_SHAPES
    for s, ps in zip(shapes, plans(shapes)):
        for form, bm, bn, per_unit, tiles, whole, splits, kt, partial in ps:
            if not bm:
                continue
            assert (bm, bn, per_unit) in {(256, 256, 1), (128, 128, 1), (128, 128, 2), (64, 128, 1), (64, 128, 2)}
            if splits == 1:
                assert partial == 0 and whole == 0
                continue
            assert form not in ("UP", "DH"), (s, form)                         # their epilogues need whole sums
            rest = tiles - whole
            assert 0 <= whole < tiles and whole % (256 * per_unit) == 0 and rest * splits <= 256 * per_unit, s
            assert kt // splits >= 1 and rest * splits * bm * bn * 4 <= partial, s
