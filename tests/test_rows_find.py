"""The tile lookup of the products whose rows choose their weights, compiled for the
host (tests/rows_find_driver.cpp): with ascending offsets every tile is taken
once, and with any others no workgroup is led out of the arrays."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2302_07594_amd", "csrc")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("find") / "rows_find")
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined",
                    "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I",
                    CSRC, os.path.join(ROOT, "tests", "rows_find_driver.cpp"), "-o", exe],
                   check=True, capture_output=True)
    return exe


@pytest.mark.parametrize("what", ["legal", "hostile"])
def test_tiles(driver, what):
    r = subprocess.run([driver, what], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout[-2000:] + r.stderr[-2000:]
