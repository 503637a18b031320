"""Which form takes a product with step sizes per block of 128 (csrc/qmm_block_plan.h, compiled for the host): the sizes of tests/block_forms.py are taken by the
forms they are meant for."""
import os
import shutil
import subprocess

import pytest

import block_forms as F
from paper_2408_02897_amd import build

PROGRAM = """
#include <cstdio>
#include "qmm_block_plan.h"
int main()
{
    long long b, m, n, k;
    while (scanf("%lld %lld %lld %lld", &b, &m, &n, &k) == 4) {
        const qmm::Plan p = qmm::plan_of(m, n, k, b);
        printf("%d %d\\n", p.tile, p.splits);
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)

    def run(sizes):
        text = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, s)) for s in sizes), text=True, stdout=subprocess.PIPE, check=True).stdout
        return [tuple(map(int, line.split())) for line in text.splitlines()]
    return run


def workgroups(b, m, n, tile, splits):
    return -(-n // 16) * b if tile == 0 else -(-m // tile) * -(-n // tile) * b * splits


def test_sizes_are_taken_by_their_forms(plans):
    got = plans([f[:4] for f in F.FORMS])
    assert [(*f[:4], *p, workgroups(*f[:3], *p)) for f, p in zip(F.FORMS, got)] == F.FORMS
    assert all(f[6] > 256 for f in F.LARGE) and {f[5] for f in F.LARGE_SPLIT} == {2, 4, 8, 16} and {f[5] for f in F.MIDDLE_SPLIT} == {2, 4, 8, 16}


def test_the_workspace_is_the_parts(plans):
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2408_02897_amd import qmm
    for (b, m, n, k), (tile, splits) in zip((f[:4] for f in F.FORMS), plans([f[:4] for f in F.FORMS])):
        assert qmm.lib().qmm_gemm_blocks_workspace_size(b, m, n, k) == (4 * splits * b * m * n if splits > 1 else 0)


def test_no_form_asks_for_more_than_a_launch_takes(plans):
    """Less than 2^32 threads: 512 a workgroup with few tokens, 256 in tiles of 128 and 64; workgroups of 256 x 256 go round."""
    sizes = [(b, m, n, k) for b in (1, 3, 2 ** 16, 2 ** 23 - 1, 2 ** 23, 2 ** 24 + 1, 2 ** 28) for m in (1, 16, 17, 40, 64, 65, 129, 5000) for n in (1, 16, 17, 4000, 2 ** 28, 2 ** 31 - 1)
             for k in (16, 128, 4096, 2 ** 22)]
    for s, (tile, splits) in zip(sizes, plans(sizes)):
        assert tile == 256 or workgroups(*s[:3], tile, splits) * (512 if tile == 0 else 256) < 2 ** 32, (s, tile, splits)
    assert plans([(2 ** 24 - 1, 1, 1, 16), (2 ** 24, 1, 1, 16)]) == [(64, 1), (256, 1)]
