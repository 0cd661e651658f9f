"""What the compiler gives the operators' kernels (its own resource report): none touches scratch memory but the gradient's product in large
tiles with one operand across its rows, whose 256 registers leave 12 over; and the wavefronts a SIMD that the large kernels are written for."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2502_11058_amd import build

SOURCES = ["ddp_attention.hip", "ddp_cross_entropy.hip", "ddp_norm.hip", "ddp_rotary.hip"]


def _report(hipcc, src, tmp_path):
    r = subprocess.run([hipcc] + build.FLAGS + ["--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-x", "hip", "-c", os.path.join(build.CSRC, src),
                                                "-o", str(tmp_path / (src + ".o"))], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    seen, kernel = {}, ""
    for ln in r.stderr.splitlines():
        if m := re.search(r"remark: .*Function Name: (\S+)", ln):
            kernel = m[1]
        elif m := re.search(r"remark: .* (SGPRs Spill|VGPRs Spill|ScratchSize|Occupancy)[^:]*: (\d+)", ln):
            seen.setdefault(kernel, {})[m[1]] = int(m[2])
    return seen


@pytest.mark.timeout(600)
def test_operators(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        seen = {k: v for part in ex.map(lambda s: _report(hipcc, s, tmp_path), SOURCES) for k, v in part.items()}
    assert len(seen) > 100 and all(len(v) == 4 for v in seen.values())
    spills = {k: v for k, v in seen.items() if v["VGPRs Spill"] or v["ScratchSize"]}
    # grad_kernel<Shape<T, 2, 4, 4, 2>, true, false>, of bf16 and of planes
    assert all(re.search(r"grad_kernelI.*Li2ELi4ELi4ELi2EEELb1ELb0E", k) and v["VGPRs Spill"] <= 12 and v["ScratchSize"] <= 52 for k, v in spills.items()), spills
    # scalar registers kept in vector ones: the large logits kernel's, outside its loop
    assert {k: v["SGPRs Spill"] for k, v in seen.items() if v["SGPRs Spill"] > (210 if re.search(r"13logits_kernelI.*Li2ELi4ELi4ELi2E", k) else 60)} == {}
    two = [v["Occupancy"] for k, v in seen.items() if re.search(r"attention_(forward|dq|dkdv)_kernelI(DF16b|.*TripleELi64)", k) and not re.search(r"dkdv_kernelI.*Triple", k)]
    assert len(two) == 8 and min(two) >= 2
