"""The attention kernels' limits, without a GPU: the order of what lanes pass to each
other, the rule that finds arrays which share memory, and the sizes of launches."""
import ctypes as C
import os
import random
import re
import subprocess
import tempfile

import pytest

from paper_2312_11841_amd import build, mixrt


def _compile(source, *flags):
    """What hipcc makes of a few lines of source, with the library's own flags."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "t.hip"), os.path.join(d, "t.out")
        with open(src, "w") as f:
            f.write(source)
        subprocess.run([build.HIPCC, *build.FLAGS, "-I", build.INCLUDE, "-I", build.CSRC, *flags,
                        "-x", "hip", src, "-o", out], check=True, capture_output=True)
        with open(out) as f:
            return f.read()


HALVES = r"""
#include "mixrt_attend_backward.hpp"
namespace mixrt {
namespace {
__global__ void halves(const f32x16 *g, const TilePos<32> *from, float *out)
{
    __shared__ TilePos<32> tile;
    __shared__ uint16_t place[kMaxBiasAxes * kReachRow];
    __shared__ float hist[4096];
    const int column[kMaxBiasAxes] = {1, 2, 3};
    if (threadIdx.x == 0) tile = *from;
    __syncthreads();
    add_table<32>(g[threadIdx.x], tile, 0, threadIdx.x >> 5 & 1, place, column, 1, 9,
                  hist + (threadIdx.x & 31), 960);
    __syncthreads();
    out[threadIdx.x] = hist[threadIdx.x];
}
}
void use(float *o) { halves<<<1, 64>>>((f32x16 *)o, (TilePos<32> *)o, o); }
}
"""


def test_a_wave_s_halves_add_to_shared_places_in_turn():
    """Both halves of a wave add to a column's places of the bias table's gradient.  To
    a compiler that looks at one lane the two turns are one, so something has to stand
    between them: a wave barrier, which the listing of the function names."""
    text = _compile(HALVES, "--cuda-device-only", "-S")
    body = re.search(r"^(\S*halves\S*):(.*?)s_endpgm", text, re.S | re.M).group(2)
    assert "wave barrier" in body


SHARED = r"""
#include <cstdio>
#include "mixrt_apart.hpp"
int main()
{
    mixrt::Extent e[2];
    long long at, run, n[3], st[3];
    for (int i = 0;; i ^= 1) {
        if (scanf("%lld %lld %lld %lld %lld %lld %lld %lld", &at, &run, n, n + 1, n + 2, st, st + 1,
                  st + 2) != 8)
            return 0;
        e[i] = mixrt::Extent{(uint64_t)at, run, {n[0], n[1], n[2]}, {st[0], st[1], st[2]}};
        if (i) printf("%d %d\n", mixrt::apart(e[0], e[1]), mixrt::apart(e[1], e[0]));
    }
}
"""


def _bytes(e):
    at, run, n0, n1, n2, s0, s1, s2 = e
    return {at + i * s0 + j * s1 + k * s2 + x for i in range(n0) for j in range(n1)
            for k in range(n2) for x in range(run)}


@pytest.fixture(scope="module")
def apart():
    """f([(extent, extent)]) -> [whether the rule calls them apart, either way round]."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "a.cpp"), os.path.join(d, "a")
        with open(src, "w") as f:
            f.write(SHARED)
        subprocess.run(["g++", "-std=c++17", "-I", build.CSRC, src, "-o", exe], check=True)

        def ask(pairs):
            text = "\n".join(" ".join(map(str, e)) for p in pairs for e in p)
            out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
            return [tuple(map(int, l.split())) for l in out.stdout.splitlines()]
        yield ask


def test_arrays_that_share_memory_are_found(apart):
    """Small layouts, each against all of its bytes: what the rule calls apart is."""
    rng = random.Random(3)
    pairs = []
    for _ in range(4000):
        pairs.append(tuple((rng.randint(1, 60), rng.randint(1, 6), rng.randint(1, 4),
                            rng.randint(1, 4), rng.randint(1, 3), rng.choice((0, 2, 6, 12, 24, 48)),
                            rng.choice((0, 3, 6, 8, 12, 24)), rng.choice((0, 2, 4, 6)))
                           for _ in range(2)))
    got = apart(pairs)
    assert len(got) == len(pairs)
    for p, g in zip(pairs, got):
        if any(g):
            assert not _bytes(p[0]) & _bytes(p[1]), p
    assert sum(all(g) for g in got) > 400


def test_slices_of_one_joint_array_are_apart(apart):
    """What programs have: arrays behind each other, heads of one token behind each
    other, halves of each head, tokens of two parts, and what is not there."""
    T, D = 7, 8
    joint = [[(1, 4 * D, T, 1, 1, 12 * D, 0, 0), (1 + 4 * D, 4 * D, T, 1, 1, 12 * D, 0, 0)],
             [(1, D, T, 4, 1, 12 * D, D, 0), (1 + 4 * D, D, T, 2, 1, 12 * D, D, 0)],
             [(1, D, 2, T, 4, 8 * D * T, 8 * D, 2 * D),
              (1 + D, D, 2, T, 4, 8 * D * T, 8 * D, 2 * D)],
             [(1, D, T, 4, 1, D, 2 * T * D, 0), (1 + T * D, D, T, 4, 1, D, 2 * T * D, 0)],
             [(1, 100, 1, 1, 1, 0, 0, 0), (101, 4, 1, 1, 1, 0, 0, 0)],
             [(0, 100, 1, 1, 1, 0, 0, 0), (1, 100, 1, 1, 1, 0, 0, 0)],
             [(1, 100, 0, 1, 1, 5, 0, 0), (1, 100, 1, 1, 1, 0, 0, 0)]]
    assert apart(joint) == [(1, 1)] * len(joint)


# --- grids ------------------------------------------------------------------------------

GRIDS = r"""
#include <cstdio>
#include "mixrt_attend.hpp"
int main()
{
    long long n;
    printf("%lld\n", (long long)mixrt::kMostBlocks256);
    while (scanf("%lld", &n) == 1) printf("%lld\n", (long long)mixrt::join_blocks(n));
}
"""


def test_no_launch_holds_2_to_the_32_threads_in_x():
    """The blocks of a call's kernels are bounded by its checks, those of the kernels that
    join splits by their own walk, whatever their rows."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    rows = [1, 7, 65535, 65536, 65537, 2 ** 24, 2 ** 30, 32 * 2 ** 30]
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "g.cpp"), os.path.join(d, "g")
        with open(src, "w") as f:
            f.write(GRIDS)
        subprocess.run([build.HIPCC, "-x", "hip", "--cuda-host-only", "-O1", "-I", build.INCLUDE,
                        "-I", build.CSRC, src, "-o", exe], check=True, capture_output=True)
        most, *got = map(int, subprocess.run([exe], input=" ".join(map(str, rows)), text=True,
                                             capture_output=True, check=True).stdout.split())
    assert most * 256 < 2 ** 32
    for n, g in zip(rows, got):
        assert 1 <= g <= n and g * 256 < 2 ** 32


def _workspace(backward=0, **kw):
    d = dict(batch=1, heads=16, kv_heads=16, head_dim=64, dtype=mixrt.MIXRT_F32, scale=0.125,
             queries=100, keys=300, lens=0)
    size = C.c_size_t(7)
    rc = mixrt.lib().mixrt_attention_workspace(C.byref(mixrt.Attention(**{**d, **kw})), None,
                                               backward, C.byref(size))
    return rc, size.value


@pytest.mark.parametrize("backward", [0, 1])
def test_calls_of_too_many_blocks_are_refused_and_others_not(backward):
    """A call of one query an entry and head has a block for each: 2^24 of them are more
    than a launch holds.  Calls of many rows and long keys are not too many blocks."""
    for kw in (dict(batch=2 ** 15, heads=512, kv_heads=512, queries=1, keys=8),
               dict(batch=65535, heads=257, kv_heads=257, queries=2, keys=8),
               dict(batch=2 ** 15, heads=1024, kv_heads=512, queries=1, keys=8)):
        assert _workspace(backward, **kw) == (-4, 0), kw
        assert b"too many blocks" in mixrt.lib().mixrt_thread_error()
    for kw in (dict(batch=128, queries=8193, keys=8193),
               dict(batch=16, queries=16385, keys=16385, head_dim=128),
               dict(batch=65535, heads=128, kv_heads=128, queries=1, keys=8),
               dict(batch=1024, queries=1, keys=9000),
               dict(queries=65536, keys=65536, head_dim=128)):
        assert _workspace(backward, **kw)[0] == 0, kw


@pytest.mark.parametrize("dtype,longest", [(mixrt.MIXRT_F32, 2048), (mixrt.MIXRT_BF16, 32768)])
@pytest.mark.parametrize("tokens", [8192, 40000, 65536, 262144])
def test_scratch_does_not_grow_with_the_square_of_the_tokens(tokens, dtype, longest):
    """Walks run in passes: at most four parts and what the passes before left, and one
    more for every 64 chains; the backward pass holds those of two arrays."""
    H, D = 16, 128
    array = 4 * H * D * tokens
    parts = 5 + tokens // longest // 64
    for backward in (0, 1):
        rc, size = _workspace(backward, head_dim=D, heads=H, kv_heads=H, queries=tokens,
                              keys=tokens, dtype=dtype)
        assert rc == 0
        sums = 16 * H * tokens * (parts + 1) + (1 << 20)
        assert size <= (2 if backward else 1) * parts * array + sums, size / array


def test_scales_that_leave_32_bits_in_units_of_log2_are_refused():
    assert _workspace(scale=2.0 ** 127)[0] == 0
    assert _workspace(scale=2.0 ** -149)[0] == 0
    for scale in (3e38, 2.4e38):
        assert _workspace(scale=scale) == (-1, 0)
