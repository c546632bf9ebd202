"""Hand-written barriers of the 8-bit products in the generated gfx950 code (CPU only): as in the 4-bit sources, the wait in
front of one covers the wave's LDS accesses, which direct loads of the waves that have passed overwrite."""
import re

import pytest

from test_device_asm_barriers import _instructions


@pytest.mark.parametrize("src,least", [("i8.hip", 32), ("experts.hip", 12)])
def test_lds_accesses_end_before_a_hand_written_barrier(src, least, tmp_path):
    code = _instructions(src, tmp_path / "code.s")
    at = [i for i, (x, _) in enumerate(code) if re.match(r"s_barrier\b", x) and code[i - 1][1]]
    assert len(at) >= least
    bad = [code[max(0, i - 4): i + 1] for i in at if not re.match(r"s_waitcnt .*lgkmcnt\(0\)", code[i - 1][0])]
    assert not bad, (len(bad), bad[:4])
