"""Which tile the weights' gradient from kept rows takes, and that the GPU tests' cases take each (tests/host/kept_tiles.cpp)."""
import shutil
import subprocess

import pytest

from test_gpu_kept_tiles import CASES
from test_host_sanitized import HOST, SAN


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_cases_take_every_tile(tmp_path):
    exe = str(tmp_path / "kept_tiles")
    res = subprocess.run(["g++", "-std=c++17", *SAN, "-Wall", "-Werror", "-o", exe, "kept_tiles.cpp"], cwd=HOST, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    shapes = [(T * k, E, n, m) for _, T, E, k, n, m in CASES] + [(16384, 32, 2048, 8192), (9003, 16, 2765, 1031)]
    res = subprocess.run([exe], input="".join("%d %d %d %d\n" % s for s in shapes), capture_output=True, text=True)
    tiles = [int(line) for line in res.stdout.split()]
    assert tiles == [c[0] for c in CASES] + [0, 1]
    for tile in range(3):   # each with results in whole chunks of 8 columns, and not
        assert {c[5] % 8 == 0 for c in CASES if c[0] == tile} == {True, False}
