"""The choices of the products whose rows choose their weights (igemm_rows_plan.cpp, host
code) compiled with g++: the tiles of the GPU tests' sizes, and random ones."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2302_07594_amd as ig
from rows_tiles import ADAPTERS, GROUPED

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2302_07594_amd", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "rows_plan")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined",
                    "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I",
                    CSRC, os.path.join(CSRC, "igemm_rows_plan.cpp"),
                    os.path.join(ROOT, "tests", "rows_plan_driver.cpp"), "-o", exe],
                   check=True, capture_output=True)

    def run(lines):
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, x)) for x in lines),
                           capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr[-2000:]
        return [tuple(map(int, x.split())) for x in r.stdout.splitlines()]
    return run


def test_the_sizes_of_the_gpu_tests_run_the_tiles_they_name(plan):
    got = plan([(rows, n, k, groups, 0, 0, 256) for rows, n, k, groups in GROUPED])
    for (size, want), g in zip(GROUPED.items(), got):
        assert g[:4] == want, (size, g)
    got = plan([(m, n, k, 1, adapters, rank, 256) for m, n, k, adapters, rank in ADAPTERS])
    for (size, want), g in zip(ADAPTERS.items(), got):
        assert g[:6] == want, (size, g)
    every = {g[:3] for g in GROUPED.values()} | {(32, 128, False), (32, 128, True)}
    assert every == {(bm, bn, reg) for bm, bn in ((32, 128), (32, 256), (64, 128), (128, 128))
                     for reg in (False, True)} | {(256, 256, False)}


def test_random_sizes(plan):
    """Every tile is one that is built, k slices cover k, and the workspace is what the query
    says."""
    rng = np.random.default_rng(0)
    lines = []
    for _ in range(3000):
        rows, n = (int(2 ** rng.uniform(0, 17)) for _ in range(2))
        k = int(2 ** rng.uniform(0, 17) - 1)
        adapt = rng.random() < 0.5
        groups = 1 if adapt else int(2 ** rng.uniform(0, 16))
        rank = int(2 ** rng.uniform(0, 10)) if adapt else 0
        lines.append((rows, n, k, groups, int(adapt) * 7, rank, int(rng.choice([256, 64, 32]))))
    for line, (bm, bn, reg, slices, by_row, ranks, nbytes) in zip(lines, plan(lines)):
        rows, n, k, groups, adapters, rank, cu = line
        assert (bm, bn) in ((32, 128), (32, 256), (64, 128), (128, 128), (256, 256)), line
        assert not (reg and bm == 256), line
        assert 1 <= slices <= 16 and (slices == 1 or (bm <= 64 and bn == 128)), line
        assert slices == 1 or not adapters or by_row, line
        assert not by_row or rows * rank <= 4096, line
        assert ranks in ((16, 32) if adapters else (0,)), line
        if k <= 131071:
            want = ig.igemm_i8_adapters_query(
                ig.AdaptersDesc(rows, n, k, adapters, rank, 1, 1), cu) if adapters else \
                ig.igemm_i8_grouped_query(
                    ig.GroupedDesc(rows, n, k, groups, rows, rows, 0, 0, 1), cu)
            assert nbytes == want, line
