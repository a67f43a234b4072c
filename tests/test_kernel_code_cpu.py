"""What the compiler made of the kernels' written-out instructions, in the AMD assembly of this library's own sources
(compiled here, no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_19058_amd import build

pytestmark = pytest.mark.skipif(shutil.which(build.hipcc()) is None, reason="needs hipcc")


def registers(text, kind):
    out = set()
    for a, b in re.findall(rf"\b{kind}\[(\d+):(\d+)\]", text):
        out |= set(range(int(a), int(b) + 1))
    return out | {int(a) for a in re.findall(rf"\b{kind}(\d+)\b", text)}


def targets(x):
    return re.findall(r"\.LBB\w+", x) if x.startswith(("s_branch", "s_cbranch")) else []


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: [instruction or label]} of moe_product.hip, in the listing's order."""
    out = str(tmp_path_factory.mktemp("asm") / "product.s")
    cmd = [build.hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Xclang",
           "-target-feature", "-Xclang", "-packed-fp32-ops", "--cuda-device-only", "-S", "-o", out,
           os.path.join(build.CSRC, "moe_product.hip")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    code, name = {}, None
    for line in open(out):
        line = line.split(";")[0].strip()
        label = re.match(r"^(_Z\w+):", line)
        if label:
            name = label.group(1)
            code[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name and line and (line.startswith(".LBB") or not line.startswith(".")):
            code[name].append(line.rstrip(":"))
    assert code
    return code


def early_reads(body):
    """Instructions that read a matrix instruction's result (in accumulation registers) where one can have been issued
    since the last wait, followed along every branch."""
    sums = set()
    for x in body:
        if x.startswith("v_mfma"):
            sums |= registers(x.split(",")[0], "a")
    at = {x: i for i, x in enumerate(body) if x.startswith(".LBB")}
    seen, todo, early = set(), [(0, False)], set()
    while todo:
        i, pending = todo.pop()
        while i < len(body) and (i, pending) not in seen:
            seen.add((i, pending))
            x = body[i]
            op, _, args = x.partition(" ")
            if op.startswith("v_mfma"):
                pending = True
            elif x == "s_nop 15" and body[i - 1] == x:
                pending = False
            elif pending:
                read = args if "store" in op or op.startswith("ds_write") else args.partition(",")[2]
                if registers(read, "a") & sums:
                    early.add(i)
            todo += [(at[t], pending) for t in targets(x)]
            if op in ("s_branch", "s_endpgm"):
                break
            i += 1
    return len(sums), [body[i] for i in sorted(early)]


def test_sums_are_read_after_the_wait(kernels):
    """The compiler does not know the latency of the written-out matrix instruction: nothing but another one may
    read a sum before the wait."""
    seen = 0
    for name, body in kernels.items():
        if "s_nop 15" not in body:
            continue   # (its sums are the compiler's own)
        sums, early = early_reads(body)
        assert sums == 256, name   # a lane's 8 x 8 blocks of 4
        assert not early, (name, len(early), early[:4])
        seen += 1
    assert seen == 3


def test_early_reads_are_found():
    body = ["v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]", "s_cbranch_scc1 .LBB0_2", "s_nop 15", "s_nop 15",
            ".LBB0_2", "v_accvgpr_read_b32 v1, a2", "s_endpgm"]
    assert early_reads(body) == (4, ["v_accvgpr_read_b32 v1, a2"])
    del body[1]
    assert early_reads(body) == (4, [])


def written_out():
    """(file, statement) of every asm statement in the device sources."""
    for f in sorted(os.listdir(build.CSRC)):
        if f.endswith((".hip", ".h")):
            for s in re.findall(r"\basm volatile\((.*?)\);", open(os.path.join(build.CSRC, f)).read(), flags=re.S):
                yield f, s


def test_written_registers_are_named():
    """A fixed register that an asm statement writes (m0, which scalar code of the compiler's own may hold) is among its clobbers."""
    seen = 0
    for f, s in written_out():
        text = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', s.split(":")[0]))
        if re.search(r"\bs_mov_b32 m0\b", text):
            assert '"m0"' in s.split(":")[-1], (f, s)
            seen += 1
    assert seen
