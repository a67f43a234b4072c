"""Which tiles, remainders and shared contractions sizes lead to in the head's loss (tests/host/head_paths.cpp), and that the GPU tests' cases
take all that are reached."""
import os
import random
import shutil
import subprocess

import pytest

from test_gpu_loss_paths import CASES
from test_host_sanitized import HOST, SAN

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
MEASURED = [(2048, 128, 512, 0), (1024, 2048, 50304, 0), (8192, 2048, 50304, 0), (4096, 2048, 50304, 1), (3001, 1031, 32003, 0)]


@pytest.fixture(scope="module")
def names(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("paths") / "head_paths")
    res = subprocess.run(["g++", "-std=c++17", *SAN, "-Wall", "-Werror", "-o", exe, "head_paths.cpp"], cwd=HOST, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def of(shapes):
        text = "".join("%d %d %d %d\n" % (*s[:3], int(s[3])) for s in shapes)
        res = subprocess.run([exe], input=text, capture_output=True, text=True)
        assert res.returncode == 0 and not res.stderr, res.stderr[-2000:]
        return [set(line.split()) for line in res.stdout.splitlines()]
    return of


def drawn(n, seed=5):
    r = random.Random(seed)

    def log(lo, hi):
        return int(round(lo * (hi / lo)**r.random()))
    shapes = []
    while len(shapes) < n:
        lo, hi = r.choice((((1, 1, 1), (10000, 4200, 70000)), ((500, 64, 200), (10000, 4200, 70000)), ((3900, 8, 30000), (10000, 1500, 90000))))
        T, d, V = (log(a, b) for a, b in zip(lo, hi))
        d, V = (max(8, v // 8 * 8) if r.random() < 0.6 else v for v in (d, V))
        if T * d * V <= 6e11 and T * V <= 6e8:
            shapes.append((T, d, V, r.randrange(2)))
    return shapes


def test_cases_take_every_path(names):
    tested = set().union(*names(CASES))
    # each kind of path is among them
    for kind in ("few", "loss/untied/rest", "loss/tied/rest", "G/half/untied/rest", "G/half/tied/rest", "G/two/untied/rest", "G/two/tied/rest",
                 *(f"d{p}/half/{m}{cut}/{t}" for p in "xw" for m in ("tied", "untied") for cut, tiles in
                   (("", ("0/one", "0/shared", "1/one", "1/shared", "3/one", "3/shared")), ("/rows", ("3",)), ("/columns", ("3",))) for t in tiles),
                 "dx/half/tied/more/columns", "dx/half/tied/more/rows", "dx/half/untied/more/columns", "dx/half/untied/more/rows",
                 *(f"dx/two/{m}/{t}/shared" for m in ("tied", "untied") for t in (0, 1, 3)),
                 *(f"dw/two/{m}/{t}/one" for m in ("tied", "untied") for t in (0, 1, 3))):
        assert any(n.startswith(kind) for n in tested), kind
    shapes = MEASURED + drawn(15000)
    for s, found in zip(shapes, names(shapes)):
        assert found <= tested, (s, found - tested)
