"""The attention kernels' limits, without a GPU: the order of what lanes pass to each
other."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2312_11841_amd import build


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
