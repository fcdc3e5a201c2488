"""How the large gradients' product dx = dz W is laid out, without a GPU: the sizes that the GPU tests have for a way stand for that way.

A program of a few lines asks the library's own planning functions; it is compiled for the host alone and linked to the built library."""
import os
import subprocess

import pytest

import paper_2112_00709_amd as fb
from paper_2112_00709_amd import build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "fb_affine.h"
using namespace fb;
int main(int n, char **a)                 // kind, type, M, N, K: log probabilities, gated layer (N of the outputs), affine layer
{
    const char kind = a[1][0];
    const int type = atoi(a[2]);
    const int64_t M = atoll(a[3]), N = atoll(a[4]), K = atoll(a[5]);
    const void *p = (const void *)4096;
    Product dx, last;
    int64_t pieces = 1;
    if (kind == 'l') {
        const ScoreGradPlan g = score_grad_plan(p, K, p, K, M, N, K, type);
        dx = g.dx;
        pieces = g.pieces;
    } else {
        dx = grad_plan(p, N, type, p, K, p, K, M, kind == 'g' ? 2 * N : N, K, type, kind == 'g' ? FB_ACT_SILU : FB_ACT_NONE).dx;
    }
    const int64_t rows = rows_in_rounds(dx, last);
    printf("%lld %d %d %lld %d\n", (long long)pieces, (int)dx.parts, dx.tile, (long long)rows, rows ? last.tile : 0);
}
"""

# (kind, M, N, K), type: pieces of the vocabulary, dx by way of shares in memory, its tiles, rows in whole rounds of them, the rest's tiles
TYPES = {"float32": 0, "bfloat16": 1, "float16": 2}
CUT = ["bfloat16", "float16"]
PLANS = ([(("l", 69120, 300, 1024), t, (1, 0, 256, 65536, 128)) for t in CUT] + [(("l", 40000, 7000, 1024), t, (2, 0, 256, 32768, 128)) for t in CUT] +
         [(("l", 70000, 4200, 256), t, (2, 0, 128, 0, 0)) for t in CUT] + [(("l", 70000, 4200, 256), "float32", (3, 0, 64, 0, 0))] +
         [(("a", 69120, 300, 1024), t, (1, 0, 256, 65536, 128)) for t in CUT] + [(("g", 69120, 150, 1024), t, (1, 0, 256, 65536, 128)) for t in CUT])


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(fb.LIB_PATH):
        build.build_library()
    d = tmp_path_factory.mktemp("plans")
    source, obj, exe = (str(d / f"plans{end}") for end in (".cpp", ".o", ""))
    with open(source, "w") as f:
        f.write(PROGRAM)
    subprocess.check_call([build.HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-fPIE", "-w", "-I", build.CSRC, "-c", source, "-o", obj])
    subprocess.check_call(["g++", obj, fb.LIB_PATH, "-Wl,-rpath," + os.path.dirname(fb.LIB_PATH), "-o", exe])
    return exe


@pytest.mark.parametrize("size,dtype,plan", PLANS)
def test_sizes_go_the_way_they_stand_for(program, size, dtype, plan):
    kind, *numbers = size
    out = subprocess.check_output([program, kind, str(TYPES[dtype]), *map(str, numbers)], text=True)
    assert tuple(map(int, out.split())) == plan
