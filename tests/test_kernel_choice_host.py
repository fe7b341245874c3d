"""The rules that choose the kernels of the dense layer and of the group norm (built with the host compiler; needs no GPU): the sizes of the GPU tests reach every one of them."""
import os
import shutil
import subprocess

import pytest

from conftest import ROOT
from kernel_sizes import DENSE_BACKWARD, DENSE_FORWARD, FEW, GROUP_NORM, TILES

DENSE = r"""
#include <cstdio>
#include "dense_way.h"
using namespace abt;
int main() {
    long M; int m, n, forward, kind;
    while (std::scanf("%ld %d %d %d %d", &M, &m, &n, &forward, &kind) == 5) {
        if (forward) {
            const DenseWay w = dense_way(M, m, n, kind != 0);
            std::printf("%d %d\n", w.tile, w.pieces);
        } else {
            const GradWay g = grad_way(M, m, n, kind);
            const bool together = dense_together(M, m, n, kind == 1 ? m : 2 * m, kind);
            std::printf("%d %d %d\n", together, together ? kDenseGrads[2].t : kDenseGrads[g.tile].t, !together && g.order.splits > 1);
        }
    }
    return 0;
}
"""

GROUP = r"""
#include <cstdio>
#include "group_norm_plan.h"
using namespace abt;
int main() {
    long N; int pixels, C, groups, bf16, backward;
    while (std::scanf("%ld %d %d %d %d %d", &N, &pixels, &C, &groups, &bf16, &backward) == 6) {
        const GroupPlan p = group_plan(N, pixels, C, groups, bf16 != 0, backward != 0);
        std::printf("%d %d\n", p.threads, p.vectors);
    }
    return 0;
}
"""


def answers(tmp_path, program, lines):
    (tmp_path / "ways.cpp").write_text(program)
    exe = str(tmp_path / "ways")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2405_01067_amd", "csrc"), str(tmp_path / "ways.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], input="\n".join(" ".join(str(int(v)) for v in line) for line in lines), stdout=subprocess.PIPE, text=True, check=True)
    return [tuple(int(v) for v in line.split()) for line in r.stdout.splitlines()]


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_dense(tmp_path):
    got = answers(tmp_path, DENSE, [(*s, 1, more) for s, more, _, _ in DENSE_FORWARD] + [(*s, 0, values) for s, values, _, _, _ in DENSE_BACKWARD])
    assert got == [(tile, pieces) for _, _, tile, pieces in DENSE_FORWARD] + [(int(one), tile, int(cut)) for _, _, one, tile, cut in DENSE_BACKWARD]
    # all there are
    assert {(tile, pieces > 1) for _, _, tile, pieces in DENSE_FORWARD} == {(t, False) for t in range(len(TILES))} | {(len(TILES) - 1, True), (FEW, False)}
    assert {(values, tile, cut) for _, values, one, tile, cut in DENSE_BACKWARD if not one} == {(v, t, c) for v in (1, 3) for t in (64, 128, 256) for c in (False, True)}
    assert {values for _, values, one, _, _ in DENSE_BACKWARD if one} == {1, 3}


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_group_norm(tmp_path):
    calls = [(*shape, bf16, backward) for shape in GROUP_NORM for bf16 in (0, 1) for backward in (0, 1)]
    got = set()
    for (_, _, C, groups, bf16, backward), (threads, vectors) in zip(calls, answers(tmp_path, GROUP, calls)):
        channels = C // groups                # the forward adds up the channels that lie in one group before it goes on: eight, four, or none
        units = 0 if backward or not threads else 1 if channels % 8 == 0 else 2 if channels % 4 == 0 else 8
        got.add((bf16, backward, threads, min(k for k in (0, 2, 4, 8, 16) if k >= vectors), units))
    # all there are: 0 threads are the kernels in pieces
    want = {(bf16, backward, 0, 0, 0) for bf16 in (0, 1) for backward in (0, 1)}
    for bf16 in (0, 1):
        want |= {(bf16, 0, *k, units) for k in ((256, 2), (256, 4), (512, 4), (512, 8), (1024, 8)) + ((1024, 16),) * bf16 for units in (1, 2, 8)}
        want |= {(bf16, 1, *k, 0) for k in ((256, 2), (256, 4), (256, 8), (512, 8)) + ((256, 16), (512, 16)) * bf16}
    assert got == want
