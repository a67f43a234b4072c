"""The rounds of the weights' gradient up to 2^31 - 1 places of one expert, on the host under UndefinedBehaviorSanitizer."""
import shutil

import pytest

from test_host_sanitized import SAN, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rounds_of_the_most_places(tmp_path):
    exe = str(tmp_path / "moe_rounds")
    _build_and_run(["g++", "-std=c++17", *SAN, "-Wall", "-Werror", "-o", exe, "moe_rounds_check.cpp"], exe, tmp_path, "rounds checked")
