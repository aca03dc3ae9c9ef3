"""Which kernel a product of 4-bit floats runs, without a GPU: the plan is plain host code, compiled
here by itself.  The GPU tests name sizes for every kernel and border; this file checks that they
still lead there."""
import os
import re
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


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "agg_mx4.s"
    subprocess.check_call([b.HIPCC, *b.FLAGS, "-I", os.path.join(b.ROOT, "include"), "-I", b.CSRC, "-S",
                           "--cuda-device-only", os.path.join(b.CSRC, "agg_mx4.hip"), "-o", str(out)],
                          stderr=subprocess.DEVNULL)
    return out.read_text()


def test_product_kernels_leave_m0_to_their_copy_statements(assembly):
    """The copies global -> LDS set M0 inside assembly statements without declaring it: sound only
    while no instruction that the compiler emits touches M0."""
    inside, copies, offenders = False, 0, []
    for line in assembly.splitlines():
        code = line.split(";")[0] if not line.lstrip().startswith(";;#") else line
        if "#ASMSTART" in line:
            inside = True
        elif "#ASMEND" in line:
            inside = False
        elif inside:
            copies += "global_load_lds_dword" in code
        elif re.search(r"\bm0\b", code):
            offenders.append(line.strip())
    assert copies >= 32, "the copy statements were not found"
    assert not offenders, offenders[:5]


def test_panels_store_as_often_as_their_waits_count(assembly):
    """A pass's copies are awaited by the number of younger accesses, three passes' stores among them.
    Were the compiler to merge stores, or to put anything into scratch memory between them, that wait
    would end early: a whole pass's stores are exactly 16 in one run without a branch, for the
    wavefronts that store at a pass's end and those that store at the next one's beginning, and in the loop every
    wait that is not one of the three written ones belongs to the loading of a panel."""
    kernels = re.findall(r"^(\S*mx4_panel_kernelILi(\d)E\S*):[^\n]*\n(.*?)^\.Lfunc_end", assembly, flags=re.M | re.S)
    assert len(kernels) == 2, [k[0] for k in kernels]
    for name, steps, body in kernels:
        assert "scratch_" not in body, name
        loop = body[:body.rindex("v_mfma")]
        runs, run = [], 0
        for line in body.splitlines():
            if re.match(r"\s+\w*store", line):
                assert "global_store_dwordx2" in line, (name, line)
                run += 1
            elif re.match(r"\s+s_c?branch", line) or re.match(r"\.LBB", line):
                runs.append(run)
                run = 0
        assert runs.count(16) >= 2 and set(runs) <= {0, 1, 15, 16}, (name, runs)
        group = int(steps) // 2 + 2
        waits = [int(w) for w in re.findall(r"s_waitcnt vmcnt\((\d+)\)\n", loop)]
        assert 2 * group + 3 * 16 in waits and 2 * group in waits, (name, waits)
        copies = re.findall(r"global_load_lds_dword(?:x4)?", body)
        assert len(copies) % group == 0, (name, len(copies))
