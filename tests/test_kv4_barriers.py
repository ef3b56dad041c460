"""The barriers of the kernel whose wavefronts share keys of a 4-bit cache: each waits for the reads and writes of LDS in front of it in the same
statement, so that the compiler can place nothing in between (compiled here, no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2509_18824_amd import build as B


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "kv4_attn.s")
    subprocess.run([B.HIPCC, *B.FLAGS, *B.FILE_FLAGS["kv4_attn.hip"], "--cuda-device-only", "-S", os.path.join(B.CSRC, "kv4_attn.hip"), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    found = re.findall(r"^(_ZN\S*kv4_rows_kernel\S*):[^\n]*\n(.*?)^\.Lfunc_end", text, re.S | re.M)
    assert len(found) == 2
    return dict(found)


def test_waits_and_barriers_are_one_statement(kernels):
    for name, body in kernels.items():
        statements = [[line.strip() for line in s.splitlines() if line.strip()] for s in re.findall(r";+\s*#ASMSTART\n(.*?);+\s*#ASMEND", body, re.S)]
        barriers = [s for s in statements if "s_barrier" in s]
        assert len(barriers) >= 2 and all(s == ["s_waitcnt lgkmcnt(0)", "s_barrier"] for s in barriers), name
        # the others are __syncthreads(), which the compiler knows
        outside = re.sub(r";+\s*#ASMSTART\n.*?;+\s*#ASMEND", "", body, flags=re.S)
        assert len(re.findall(r"^\s*s_barrier", outside, re.M)) >= 1
