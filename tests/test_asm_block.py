"""The generated code of the operators around the layer: no barrier passed with LDS writes under way, no lane mask of a loop that decides for
the wave behind it, nothing spilled, no packed fp32 arithmetic.  CPU only."""
import os
import re
import subprocess

import pytest

from paper_2605_23764_amd.asm_check import barrier_violations, stale_lane_masks
from paper_2605_23764_amd.build import BLOCK_SOURCES, HIPCC_FLAGS

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")


@pytest.mark.parametrize("source", BLOCK_SOURCES, ids=[os.path.basename(s) for s in BLOCK_SOURCES])
def test_generated_code(source, tmp_path):
    flags = [f for f in HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = str(tmp_path / "device.s")
    res = subprocess.run([HIPCC, *flags, "--cuda-device-only", "-S", source, "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    asm = open(out).read()
    n, bad = barrier_violations(asm)
    assert n >= 8 and not bad, bad[:5]
    n, bad = stale_lane_masks(asm)
    assert n >= 1 and not bad, bad[:5]
    kernels = re.findall(r"\.amdhsa_kernel (\S+)", asm)
    spilled = [k for k, s in zip(kernels, re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", asm)) if s != "0"]
    assert len(kernels) >= 10 and not spilled, spilled
    assert not re.findall(r"\bv_pk_(?:add|mul|fma)_f32\b", asm)
