"""The kernels of the paged 4-bit KV cache keep their arrays in registers: an array that the compiler cannot take apart goes through scratch
memory, lane by lane, and shows as bytes written that no result has.  Read from the assembly of a build from source; no GPU needed.  (Single
registers that do not fit are another matter: the compiler marks those as spills.)"""

import os
import re
import subprocess

import pytest

from paper_2410_05265_amd import build

SOURCES = [os.path.basename(s) for s in build.sources() if os.path.basename(s).startswith("pq_kv4_")]

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")


@pytest.mark.parametrize("source", SOURCES)
def test_no_array_in_scratch_memory(source, tmp_path):
    asm = str(tmp_path / "kernels.s")
    subprocess.run([build.HIPCC, *build.FLAGS, "-w", "--offload-device-only", "-S", os.path.join(build.CSRC, source), "-o", asm], check=True, capture_output=True)
    with open(asm) as f:
        lines = [line.strip() for line in f if re.match(r"\s*scratch_(load|store)", line)]
    assert not [line for line in lines if "Folded" not in line]
