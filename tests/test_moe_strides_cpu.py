"""The rule for 32-bit byte offsets at any stride, on the host under UndefinedBehaviorSanitizer."""
import shutil

import pytest

from test_host_sanitized import SAN, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rule_for_short_rows(tmp_path):
    exe = str(tmp_path / "moe_strides")
    _build_and_run(["g++", "-std=c++17", *SAN, "-Wall", "-Werror", "-o", exe, "moe_strides_check.cpp"], exe, tmp_path, "strides checked")
