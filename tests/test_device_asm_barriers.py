"""Hand-written barriers of the 4-bit sources in the generated gfx950 code (CPU only): the wait
in front of one covers the wave's LDS accesses.  Direct loads and stores of the waves that
have passed overwrite what those accesses read, and where the compiler would put a wait of
its own depends on what it moves past the barrier.  (In front of __syncthreads the compiler
waits for what is still under way.)"""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_07008_amd", "csrc")


def _instructions(src, out):
    from paper_2609_07008_amd.build import HIPCC_FLAGS
    cc = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
    if cc is None:
        pytest.skip("hipcc not found")
    subprocess.run([cc, *HIPCC_FLAGS, "-I", CSRC, "--cuda-device-only", "-S", os.path.join(CSRC, src), "-o", str(out)], check=True,
                   capture_output=True)
    got, in_asm = [], False
    for line in open(out):
        if ";;#ASM" in line:
            in_asm = "START" in line
        x = line.split(";")[0].strip()
        if x and not x.startswith("."):
            got.append((x, in_asm))
    return got


# at least two a kernel: 16 kernels of W_b, three of the attention
@pytest.mark.parametrize("src,least", [("mx4.hip", 32), ("cache_attend.hip", 6)])
def test_lds_accesses_end_before_a_hand_written_barrier(src, least, tmp_path):
    code = _instructions(src, tmp_path / "code.s")
    at = [i for i, (x, _) in enumerate(code) if re.match(r"s_barrier\b", x) and code[i - 1][1]]
    assert len(at) >= least
    bad = [code[max(0, i - 4): i + 1] for i in at if not re.match(r"s_waitcnt .*lgkmcnt\(0\)", code[i - 1][0])]
    assert not bad, (len(bad), bad[:4])
