"""Which kernel a product of 4-bit floats runs, without a GPU: the plan is plain host code, compiled
here by itself.  The GPU tests name sizes for every kernel and border; this file checks that they
still lead there."""
import subprocess

import pytest

import test_gpu_operators as ops
from paper_2512_02541_amd import build as b

DRIVER = r"""
#include <stdio.h>
#include "agg_mx4_plan.h"
int main() {
  long long rows, N, K;
  int count, residual;
  while (scanf("%lld %lld %lld %d %d", &rows, &N, &K, &count, &residual) == 5) {
    const agg::Mx4Plan p = agg::plan_mx4(rows, N, K, count, residual);
    printf("%lld %d\n", (long long)p.split, (int)p.kernel);
  }
}
"""
NAMES = ["few", "tile64", "tile128", "many", "tile256", "panel"]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(DRIVER)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-unused-function", "-I", b.CSRC,
                           "-o", str(d / "plan"), str(d / "plan.cpp")])

    def ask(sizes):
        text = "".join("%d %d %d %d %d\n" % tuple(int(v) for v in s) for s in sizes)
        out = subprocess.run([str(d / "plan")], input=text, text=True, check=True, stdout=subprocess.PIPE).stdout
        return [(int(split), NAMES[int(k)]) for split, k in (line.split() for line in out.splitlines())]

    return ask


def test_sizes_reach_their_kernels(plan):
    for name, sizes in (("few", ops.FEW), ("tile64", ops.TILE64), ("tile128", ops.TILE128), ("many", ops.MANY),
                        ("tile256", ops.TILE256), ("panel", ops.PANEL)):
        assert plan(sizes) == [(0, name)] * len(sizes), name
    for (rows, _, _, _, _), (split, kernel) in zip(ops.SPLIT, plan(ops.SPLIT)):
        assert 0 < split < rows and split % 256 == 0 and kernel in ("tile64", "tile128", "many")
    assert len({k for _, k in plan(ops.SPLIT)}) > 1


def test_plans_are_sound(plan):
    """Every size has one: a split inside the rows, panels only where a panel fits."""
    sizes = [(rows, N, K, count, residual)
             for rows in (1, 5, 64, 1000, 4097, 30001, 137400, 2 ** 31) for N in (8, 1000, 4096)
             for K in (8, 1024, 1032, 4096, 1 << 22) for count in (1, 2, 3) for residual in (0, 1) if count * residual < 2]
    for (rows, N, K, count, residual), (split, kernel) in zip(sizes, plan(sizes)):
        assert 0 <= split < rows and split % 256 == 0
        assert split == 0 or (K > 1024 and kernel in ("tile64", "tile128", "many"))
        assert kernel != "panel" or (K <= 1024 and not residual)
        if kernel == "few":
            assert -(-rows // 16) * -(-N // 16) * count <= 512
