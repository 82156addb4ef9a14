"""Outputs that share memory with what a call reads, or with one another, are refused before anything is launched.  No GPU: the addresses
are never looked at."""
import ctypes
import os
import subprocess
import sys
import textwrap

from paper_1811_00206_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_pitch_of_a_single_row_does_not_count():
    """Whatever a leading dimension times the type's size is in 64 bits, 0 among it: in a process of its own, which must not end."""
    code = """
        import ctypes
        from paper_1811_00206_amd import binding as b
        lib, p, null = b.load_library(), ctypes.c_void_p(4096), ctypes.c_void_p(0)
        far, beside = ctypes.c_void_p(1 << 30), ctypes.c_void_p(1 << 31)
        for ld in (64, 65, 1 << 40, 1 << 60, 1 << 61, 1 << 62, (1 << 62) + 64, (1 << 63) - 1):
            for other in (64, ld):
                assert lib.bs_mx4_gemm(p, p, 64, 64, far, 0, 1, other, null, far, ld, null, 0, null) == 3, ld
                assert lib.bs_mx4_gemm(p, p, 64, 64, far, 0, 1, ld, null, far, other, null, 0, null) == 3, ld
                # a gradient one element behind the logits, and (refused later, for its alignment) one beside them
                for first, want in ((far.value + 4, 3), (beside.value, 4)):
                    assert lib.bs_logprobs_backward(far, 0, 1, 64, ld, p, ctypes.c_void_p(4098), p, p, p, ctypes.c_void_p(first), other, null) == want, ld
        # rows that no memory holds are not told apart
        for ld in (1 << 61, 1 << 62, (1 << 62) + 64, (1 << 63) - 1):
            assert lib.bs_mx4_gemm(p, p, 64, 64, far, 0, 2, 64, null, beside, ld, null, 0, null) == 3, ld
            assert lib.bs_mx4_gemm(p, p, 64, 64, far, 0, 2, ld, null, beside, 64, null, 0, null) == 3, ld
    """
    out = subprocess.run([sys.executable, "-c", textwrap.dedent(code)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, (out.returncode, out.stdout + out.stderr)
