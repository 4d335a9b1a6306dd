"""The plan of the masked attention kernels for many rows and the way of their workgroups through it, on the CPU: whatever cu_q and the lengths hold,
no workgroup asks for an entry that was not listed, and every step is taken once (kv4_plan_walk.cpp)."""

import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_no_workgroup_leaves_the_list(tmp_path):
    exe = str(tmp_path / "kv4_plan_walk")
    subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-w", os.path.join(HERE, "kv4_plan_walk.cpp"), "-o", exe],
                   check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "kv4_plan_walk: ok" in r.stdout, r.stdout[-4000:] + r.stderr[-2000:]
