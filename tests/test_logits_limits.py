"""How many words a row may have, as the header says.  No GPU: the rows are never looked at."""
import ctypes
import os
import re

from paper_1811_00206_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MOST = (1 << 31) - 65


def test_the_longest_row():
    lib = b.load_library()
    p, odd, null = (ctypes.c_void_p(a) for a in (1 << 20, (1 << 20) + 1, 0))      # never dereferenced: validation fails first
    for dtype in (0, 1, 2):
        assert b.bs_beam_step_workspace_bytes(dtype, 1, 4, MOST, 4) > 0 == b.bs_beam_step_workspace_bytes(dtype, 1, 4, MOST + 1, 4)
        assert lib.bs_logprobs_workspace_bytes(dtype, 1, MOST, 4) > 0 == lib.bs_logprobs_workspace_bytes(dtype, 1, MOST + 1, 4)
        for V, want in ((MOST, 4), (MOST + 1, 3)):      # 4: refused later, for the alignment of an output
            assert lib.bs_beam_step(p, dtype, 1, 4, V, V, p, null, -1, 4, odd, p, p, p, null, 0, null) == want
            assert lib.bs_logprobs(p, dtype, 1, V, V, p, 0, odd, p, p, null, null, null, 0, null) == want
            assert lib.bs_logprobs_backward(p, dtype, 1, V, V, odd if want == 4 else p, p, null, p, null, p, V, null) == want


def test_the_header_says_so():
    with open(os.path.join(ROOT, "include", "bs.h")) as f:
        limits = re.findall(r"\(V < (2\^31[^;]*);", f.read())
    assert limits == ["2^31 - 64"] * 2
