"""The launch rule of group norm, asked on the host: the shapes of the GPU tests
take the paths they are there for, and every grid has a block."""
import os
import subprocess
import tempfile

import pytest

from paper_2312_11841_amd import build
from refine_paths import PATHS

PROGRAM = r"""
#include <cstdio>
#include "mixrt_norm.hpp"
int main()
{
    int N, C, G, dt, how;
    long long P;
    const char *ways[3] = {"small", "fold", "large"};
    while (scanf("%d %lld %d %d %d %d", &N, &P, &C, &G, &dt, &how) == 6) {
        const mixrt::NormPlan p = mixrt::norm_plan(N, P, C, G, dt, how == 1, how == 2);
        int sums = 1;
        while (sums < p.V && (C / G) % (p.V / sums)) sums *= 2;
        printf("%s %d %d %d %d %d %d %d\n", ways[p.way], sums, p.S, p.share, p.slabs, p.R, p.lanes,
               p.V);
    }
}
"""


@pytest.fixture(scope="module")
def plans():
    """f(list of (N, P, C, G, dtype, how)) -> list of (way, sums, S, share,
    slabs, R, lanes, V); how: 0 forward, 1 keeping x, 2 backward."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "p.cpp"), os.path.join(d, "p")
        with open(src, "w") as f:
            f.write(PROGRAM)
        subprocess.run([build.HIPCC, "-x", "hip", "--cuda-host-only", "-O1", "-I", build.INCLUDE,
                        "-I", build.CSRC, src, "-o", exe], check=True, capture_output=True)

        def ask(calls):
            text = "\n".join(" ".join(str(v) for v in c) for c in calls)
            out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
            rows = [line.split() for line in out.stdout.splitlines()]
            assert len(rows) == len(calls)
            return [(r[0], *map(int, r[1:])) for r in rows]
        yield ask


def test_shapes_take_the_paths_they_are_there_for(plans):
    for shape, want in PATHS.items():
        for key, dtypes in (("f32", (0,)), ("16", (1, 3))):
            for dt in dtypes:
                got = plans([(*shape, dt, how) for how in range(3)])
                forward, keep, back, sums = want[key]
                assert tuple(g[0] for g in got) == (forward, keep, back), (shape, dt, got)
                if forward != "small":
                    assert got[0][1] == sums, (shape, dt, got)


def test_the_shapes_reach_every_path(plans):
    """Each way, each number of sums a thread, rows of one and of several
    slabs, one image and several, and more than dx's first block adds up."""
    for dt in (0, 1, 3):
        seen = set()
        for shape in PATHS:
            for how, p in enumerate(plans([(*shape, dt, how) for how in range(3)])):
                seen.add((how, p[0], "slabs" if p[4] > 1 else "one slab"))
                seen.add((how, p[0], "images" if shape[0] > 1 else "one image"))
                if how == 0 and p[0] != "small":
                    seen.add(("sums", p[1]))
        for how in (0, 1, 2):
            for kind in ("one slab", "slabs", "images", "one image"):
                assert (how, "large", kind) in seen, (dt, how, kind)
        for kind in ("one slab", "images"):
            assert (2, "fold", kind) in seen
        for kind in ("slabs", "images", "one image"):
            assert (0, "fold", kind) in seen and (1, "fold", kind) in seen
        assert {s[1] for s in seen if s[0] == "sums"} >= ({1, 2, 4} if dt == 0 else {1, 2, 4, 8})
    assert any(shape[0] > 64 for shape in PATHS)


def test_every_grid_has_a_block_and_rows_are_bounded(plans):
    calls = [(N, P, C, G, dt, how)
             for N in (1, 2, 65, 1024, 65535) for P in (0, 1, 7, 513, 20000, 1 << 20)
             for C, G in ((1, 1), (8, 2), (33, 11), (257, 1), (640, 640), (1024, 8), (4095, 1),
                          (4096, 32))
             for dt in (0, 1, 3) for how in range(3)]
    for c, (way, sums, S, share, slabs, R, lanes, V) in zip(calls, plans(calls)):
        assert S >= 1 and share >= 1 and slabs >= 1 and R >= 1, c
        assert lanes * R <= (1024 if way == "small" else 256), c
        if c[5] == 2:     # a thread of the backward's sums
            assert -(-c[1] // (S * R)) <= 128, c
