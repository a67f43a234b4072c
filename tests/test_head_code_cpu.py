"""What the compiler made of the written-out matrix instruction in the kernels of the head's loss and of kept rows' gradient, in the AMD
assembly of this library's own sources (compiled here, no GPU needed); see test_kernel_code_cpu.py."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_19058_amd import build
from test_kernel_code_cpu import early_reads

pytestmark = pytest.mark.skipif(shutil.which(build.hipcc()) is None, reason="needs hipcc")
FILES = {"head_logits": 6, "head_products": 6, "kept_product": 2}   # and how many kernels keep their sums in accumulation registers


def listing(name, out):
    cmd = [build.hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Xclang",
           "-target-feature", "-Xclang", "-packed-fp32-ops", "--cuda-device-only", "-S", "-o", out,
           os.path.join(build.CSRC, name + ".hip")]
    return subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True)


def kernels(path):
    code, name = {}, None
    for line in open(path):
        line = line.split(";")[0].strip()
        label = re.match(r"^(_Z\w+):", line)
        if label:
            name = label.group(1)
            code[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name and line and (line.startswith(".LBB") or not line.startswith(".")):
            code[name].append(line.rstrip(":"))
    return code


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    at = tmp_path_factory.mktemp("asm")
    runs = {n: listing(n, str(at / (n + ".s"))) for n in FILES}
    for n, p in runs.items():
        err = p.communicate()[1]
        assert p.returncode == 0, (n, err[-2000:])
    return {n: str(at / (n + ".s")) for n in FILES}


@pytest.mark.parametrize("name", FILES)
def test_sums_are_read_after_the_wait(listings, name):
    seen = 0
    for kernel, body in kernels(listings[name]).items():
        if "s_nop 15" not in body:
            continue   # (its sums are the compiler's own)
        sums, early = early_reads(body)
        assert sums == 256, kernel
        assert not early, (kernel, len(early), early[:4])
        seen += 1
    assert seen == FILES[name]


@pytest.mark.parametrize("name", FILES)
def test_the_products_take_their_operands_type(listings, name):
    """Logits and kept rows bf16, the gradients of rows and weights float16, or bf16 (few tokens)."""
    ops = set(re.findall(r"v_mfma_f32_16x16x32_(\w+)", open(listings[name]).read()))
    assert ops == ({"f16", "bf16"} if name == "head_products" else {"bf16"})
