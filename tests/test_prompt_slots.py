"""The index arithmetic of sla_prefill's chunked kernels on the CPU, over random ragged
batches (tests/prompt_slots_driver.cpp): slots, passes, walk list, workspace, descriptors
and the addresses read in advance."""
import os
import shutil
import subprocess

import pytest

from paper_2607_16673_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which(build.HIPCC) is None, reason="needs hipcc")
def test_every_address_lies_in_its_buffer(tmp_path):
    objs = []
    for src in (os.path.join(build.CSRC, "prefill.hip"), os.path.join(ROOT, "tests", "prompt_slots_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([build.HIPCC] + build.COMMON + ["-x", "hip", "-c", src, "-o", objs[-1]], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    exe = str(tmp_path / "driver")
    # (the driver has the runtime's few functions itself: nothing here needs a GPU)
    r = subprocess.run([build.HIPCC, "-no-hip-rt"] + objs + ["-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "prompt slot checks passed" in out, out[-6000:]
