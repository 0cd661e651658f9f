"""What the operators' kernels read and write, on the CPU: their sources compiled by the host's clang over stand-ins for the device's
instructions (tests/sanitize/host_device) and run a thread at a time under AddressSanitizer and UndefinedBehaviorSanitizer, through the
entry points, on tensors and workspaces of exactly their size (tests/sanitize/operators.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_11058_amd", "csrc")
SOURCES = {"norm": "ddp_norm.hip", "rotary": "ddp_rotary.hip", "attention": "ddp_attention.hip", "entropy": "ddp_cross_entropy.hip"}
# (addresses within a tensor without rows, which may be null, are formed and not read: not looked at)
SAN = ["-fsanitize=address,undefined", "-fno-sanitize=pointer-overflow", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-gline-tables-only",
       "-O1"]

# Threads run one after the other, so the wavefront's search over 64 sequences at a time is one sequence after the other.
SEARCH = """    int before = 0;
    for (int b = 0; b <= a.batch; ++b) {
        int64_t q0, q1, k0, k1;
        bounds<KEYS>(a, b, q0, q1, k0, k1);
        const int mine = (int)(((KEYS ? k1 - k0 : q1 - q0) + kRows - 1) / kRows);
        if (before + mine > block) {
            s.b = b, s.block = block - before, s.q0 = q0, s.k0 = k0, s.q_len = (int)(q1 - q0), s.k_len = (int)(k1 - k0);
            return true;
        }
        before += mine;
    }
"""


def _on_the_host(which):
    text = open(os.path.join(CSRC, SOURCES[which])).read()
    text = text.replace('asm volatile("s_waitcnt vmcnt(0)" ::: "memory");', "").replace('asm volatile("" ::: "memory");', "")
    assert "asm" not in text.replace("same", "")
    if which == "attention":
        a = text.index("    const int lane = threadIdx.x & 63;\n    int before = 0;")
        b = text.index("    return false;\n}", a)
        text = text[:a] + SEARCH + text[b:]
    return text


@pytest.mark.timeout(900)
@pytest.mark.parametrize("which", sorted(SOURCES))
def test_inside_their_tensors(tmp_path, which):
    clang = "/opt/rocm/bin/amdclang++"
    if not shutil.which(clang):
        pytest.skip("no clang")
    (tmp_path / "kernels.cpp").write_text(_on_the_host(which))
    inc = ["-I" + os.path.join(ROOT, "tests", "sanitize", "host_device"), "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]
    exe = str(tmp_path / which)
    objs = []
    for src, extra in ((str(tmp_path / "kernels.cpp"), ["-Wno-everything"]), (os.path.join(ROOT, "tests", "sanitize", "operators.cpp"), ["-D" + which.upper()])):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        r = subprocess.run([clang, "-x", "c++", "-std=c++17"] + inc + SAN + extra + ["-c", src, "-o", objs[-1]], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([clang] + SAN + objs + ["-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=800)
    assert r.returncode == 0, r.stdout + r.stderr[-4000:]
    assert "ok, " in r.stdout
