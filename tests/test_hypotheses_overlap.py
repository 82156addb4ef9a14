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


def test_products_refuse_a_result_over_what_they_read():
    """Workgroups store their part of y while others still read the matrix, x or the bias."""
    lib, null, far = b.load_library(), ctypes.c_void_p(0), 1 << 40
    M, K, N = 40, 300, 9      # rows of the matrix are 192 bytes of codes and 12 of scales
    at = {"codes": 1 << 20, "scales": 2 << 20, "x": 3 << 20, "x_scales": 4 << 20, "bias": 5 << 20}
    sizes = {"codes": M * 192, "scales": M * 12, "x_scales": N * 12, "bias": M * 4}
    for dtype, size in ((0, 4), (1, 2), (2, 2)):
        for ldy in (M, M + 7):
            span = ((N - 1) * ldy + M) * size
            for packed in (False, True):
                x_bytes = N * 192 if packed else ((N - 1) * (K + 3) + K) * size

                def status(y):
                    p = {k: ctypes.c_void_p(v) for k, v in at.items()}
                    if packed:
                        return lib.bs_mx4_gemm_packed(p["codes"], p["scales"], M, K, p["x"], p["x_scales"], N, p["bias"], ctypes.c_void_p(y), dtype, ldy, null,
                                                      0, null)
                    return lib.bs_mx4_gemm(p["codes"], p["scales"], M, K, p["x"], dtype, N, K + 3, p["bias"], ctypes.c_void_p(y), ldy, ctypes.c_void_p(far), 1 << 20,
                                           null)

                for what, first in at.items():
                    if what == "x_scales" and not packed:
                        continue
                    last = first + (x_bytes if what == "x" else sizes[what]) - size
                    for y in (first, last, first - span + size):
                        assert status(y) == 3, (what, dtype, ldy, packed, y - first)


def test_packing_refuses_codes_and_scales_over_the_matrix_or_each_other():
    lib, null = b.load_library(), ctypes.c_void_p(0)
    M, K = 7, 300
    for dtype, size in ((0, 4), (1, 2), (2, 2)):
        for ld in (K, K + 5):
            W, far, span = 1 << 20, 1 << 30, ((M - 1) * ld + K) * size

            def pack(codes, scales):
                return lib.bs_mx4_pack(ctypes.c_void_p(W), dtype, M, K, ld, ctypes.c_void_p(codes), ctypes.c_void_p(scales), null)

            end = (W + span - 1) // 16 * 16      # in the last row, whose end no boundary of 16 bytes has to be
            for codes in (W, W + 16, W - M * 192 + 16, end):
                assert pack(codes, far) == 3, (dtype, ld, codes - W)
            for scales in (W, W - M * 12 + 4, (W + span - 1) // 4 * 4):
                assert pack(far, scales) == 3, (dtype, ld, scales - W)
            for scales in (far, far + M * 192 - 4, far - M * 12 + 4):
                assert pack(far, scales) == 3, (dtype, ld, scales - far)


def test_unpacking_refuses_a_matrix_over_its_codes_and_scales():
    lib, null = b.load_library(), ctypes.c_void_p(0)
    M, K, codes, scales = 7, 300, 1 << 20, 1 << 30
    for dtype, size in ((0, 4), (1, 2), (2, 2)):
        for at, there in ((codes, M * 192), (scales, M * 12)):
            for W in (at, at + there - size, at - M * K * size + size):
                assert lib.bs_mx4_unpack(ctypes.c_void_p(codes), ctypes.c_void_p(scales), M, K, ctypes.c_void_p(W), dtype, null) == 3, (dtype, W - at)


def test_a_step_refuses_outputs_over_inputs_or_one_another():
    """A sequence's workgroup stores while others still read.  Scores and finished flags alone may take their inputs' place, whole."""
    lib, null = b.load_library(), ctypes.c_void_p(0)
    B, W, V = 3, 5, 300
    for n in (W, 4, 9):
        for dtype, size in ((0, 4), (1, 2), (2, 2)):
            for ld in (V, V + 11):
                inputs = {"logits": (1 << 20, ((B * W - 1) * ld + V) * size), "scores": (2 << 20, B * W * 4), "finished": (3 << 20, B * W)}
                outputs = {"scores": 4 * B * n, "tokens": 4 * B * n, "parents": 4 * B * n, "finished": B * n}

                def status(**places):
                    out = {k: ctypes.c_void_p(places.get(k, (5 + i) << 20)) for i, k in enumerate(outputs)}
                    p = {k: ctypes.c_void_p(v[0]) for k, v in inputs.items()}
                    return lib.bs_beam_step(p["logits"], dtype, B, W, V, ld, p["scores"], p["finished"], 2, n, out["scores"], out["tokens"], out["parents"], out["finished"],
                                            ctypes.c_void_p(1 << 30), 1 << 30, null)

                for k, mine in outputs.items():
                    unit = 1 if k == "finished" else 4
                    for what, (first, there) in inputs.items():
                        places = {first, (first + there - 1) // unit * unit, -(-(first - mine + 1) // unit) * unit}
                        if what == k and n == W:
                            places.remove(first)      # in place
                        for at in places:
                            assert status(**{k: at}) == 3, (k, what, n, dtype, ld, at - first)
                    for other, there in outputs.items():
                        if other != k:
                            for at in (20 << 20, (20 << 20) + (there - 1) // unit * unit, (20 << 20) - mine + 4):
                                assert status(**{other: 20 << 20, k: at}) == 3, (k, other, n, at)
