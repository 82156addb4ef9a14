"""MX 4-bit matrices, beam search's step and the states that follow it where no GPU is needed: sizes, refusals before anything is
launched, the native marshalling behind a stand-in for the library, and what the compiler made of the kernels."""
import ctypes
import os
import random
import re
import subprocess
import sys
import textwrap
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from paper_1811_00206_amd import binding as b
from paper_1811_00206_amd import build as bs_build
from test_language_host import FAKE
from test_native_calls import PREAMBLE, STAND_IN

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = ["bs_mx4_pack.hip", "bs_mx4_gemm.hip", "bs_beam.hip"]


def test_sizes():
    assert b.bs_mx4_codes_bytes(6000, 3000) == 6000 * 24 * 64 and b.bs_mx4_scales_bytes(6000, 3000) == 6000 * 24 * 4
    assert b.bs_mx4_codes_bytes(1, 1) == 64 and b.bs_mx4_scales_bytes(1, 128) == 4 and b.bs_mx4_scales_bytes(1, 129) == 8
    assert b.bs_mx4_codes_bytes(1 << 24, 1 << 24) == 1 << 47
    for M, K in ((0, 8), (8, 0), (-1, 8), ((1 << 24) + 1, 8), (8, (1 << 24) + 1)):
        assert b.bs_mx4_codes_bytes(M, K) == b.bs_mx4_scales_bytes(M, K) == 0


def test_workspaces():
    gemm, packed, beam = b.bs_mx4_gemm_workspace_bytes, b.bs_mx4_gemm_packed_workspace_bytes, b.bs_beam_step_workspace_bytes
    for dtype in (b.BS_F32, b.BS_F16, b.BS_BF16):
        assert gemm(dtype, 10000, 1500, 1) == packed(dtype, 10000, 1500, 1) == 0        # rounded inside the product's kernel
        for M, K, N in ((10000, 1500, 7), (4096, 25088, 77), (16384, 8192, 4096), (1, 1, 1 << 20), (377, 1 << 20, 64)):
            x = (N * 68 * -(-K // 128) + 15) // 16 * 16
            assert gemm(dtype, M, K, N) == packed(dtype, M, K, N) + x
            assert packed(dtype, M, K, N) % (4 * M * N) == 0 and packed(dtype, M, K, N) <= 16 * 4 * M * N      # sums of shares of K
        assert beam(dtype, 1, 4, 10000, 4) > 0 and beam(dtype, 1 << 24, 64, 7, 64) > 1 << 38
        # all lists of a sequence go into one workgroup's LDS
        for W in (1, 7, 64):
            for n in (1, 13, 64):
                each = 16 * W + 8 * n * W
                assert beam(dtype, 1, W, 1 << 30, n) <= each * min(16, max(1, 4096 // (W * n)))
    for args in ((3, 8, 8, 8), (0, 0, 8, 8), (0, 8, 0, 8), (0, 8, 8, 0), (0, 8, 8, (1 << 24) + 1), (0, (1 << 24) + 1, 8, 8), (0, 1 << 20, 8, (1 << 16) + 1)):
        assert gemm(*args) == packed(*args) == 0
    for args in ((5, 1, 4, 100, 4), (0, 0, 4, 100, 4), (0, 1, 0, 100, 4), (0, 1, 65, 100, 4), (0, 1, 4, 0, 4), (0, 1, 4, 100, 0), (0, 1, 4, 100, 65),
                 (0, 1, 4, 1 << 31, 4), (0, (1 << 24) + 1, 4, 100, 4)):
        assert beam(*args) == 0


def test_plans_of_products():
    """What the kernels assume of their launch, over random shapes and the largest ones."""
    g = random.Random(3)
    shapes = [(round(2 ** g.uniform(0, 24)), round(2 ** g.uniform(0, 24)), round(2 ** g.uniform(0, 12))) for _ in range(4000)]
    shapes += [(round(2 ** g.uniform(0, 18)), round(2 ** g.uniform(0, 14)), round(2 ** g.uniform(0, 18))) for _ in range(2000)]
    for M, K, N in shapes + [(1 << 24, 1 << 24, 1), (1 << 24, 128, 4096), (4096, 128, 1 << 24), (1 << 18, 1 << 24, 1 << 18)]:
        p = b.bs_mx4_gemm_plan(M, K, N)
        chunks = -(-K // 128)
        if p["tile_rows"]:
            stages = -(-chunks // 2)
            assert p["split"] * p["stages"] >= stages > (p["split"] - 1) * p["stages"], (M, K, N)
            assert p["lds_bytes"] == (p["tile_rows"] + p["tile_columns"]) * (128 * p["buffers"] + 64) <= 160 * 1024
            assert p["workgroups"] == -(-M // p["tile_columns"]) * -(-N // p["tile_rows"]) * p["split"] and p["workgroups"] * 256 < 1 << 32, (M, K, N, p)
        else:
            assert p["workgroups"] * 16 * p["r"] * p["groups"] >= M and 16 * p["nt"] >= N and p["lds_bytes"] <= 48 * 1024, (M, K, N, p)
            threads = 64 * p["ways"] * p["groups"]
            assert threads <= (1024 if p["r"] * p["nt"] == 1 else 512) and p["workgroups"] * threads < 1 << 32
    for args in ((0, 8, 8), (8, 0, 8), (8, 8, 0)):
        with pytest.raises(b.BsError) as e:
            b.bs_mx4_gemm_plan(*args)
        assert e.value.status == 2
    for args in (((1 << 24) + 1, 8, 8), (8, (1 << 24) + 1, 8), (8, 8, (1 << 24) + 1), (1 << 20, 8, (1 << 16) + 1)):
        with pytest.raises(b.BsError) as e:
            b.bs_mx4_gemm_plan(*args)
        assert e.value.status == 3


def test_bad_arguments_are_refused_before_launch():
    lib = b.load_library()
    p, odd, null = (ctypes.c_void_p(a) for a in (4096, 4097, 0))      # never dereferenced: validation fails first
    two = ctypes.c_void_p(4098)                                       # aligned for 16 bits, not for 32
    four, far = ctypes.c_void_p(4100), ctypes.c_void_p(1 << 30)

    def refused(f, good, changes):
        for status, change in changes:
            args = list(good)
            for at, v in change.items():
                args[at] = v
            assert f(*args) == status, (f.__name__, status, change)

    big = (1 << 24) + 1
    refused(lib.bs_mx4_pack, (p, 0, 4, 64, 64, p, p, null),
            ((1, {0: null}), (1, {5: null}), (1, {6: null}), (2, {2: 0}), (2, {3: 0}), (2, {4: 63}), (3, {1: 3}), (3, {2: big}), (3, {3: big, 4: big}),
             (4, {0: two}), (4, {0: odd, 1: 1}), (4, {5: four}), (4, {6: two})))
    refused(lib.bs_mx4_unpack, (p, p, 4, 64, p, 0, null),
            ((1, {0: null}), (1, {1: null}), (1, {4: null}), (2, {2: -1}), (2, {3: 0}), (3, {5: 7}), (3, {2: big}), (4, {0: four}), (4, {1: two}),
             (4, {4: two}), (4, {4: odd, 5: 2})))
    refused(lib.bs_mx4_gemm, (p, p, 40, 64, p, 0, 1, 64, null, far, 40, null, 0, null),
            ((3, {9: p}), (3, {9: ctypes.c_void_p(4096 + 63 * 4)}), (3, {9: ctypes.c_void_p(4096 - 39 * 4)}), *((1, {at: null}) for at in (0, 1, 4, 9)), (2, {2: 0}), (2, {3: 0}), (2, {6: 0}), (2, {7: 63}), (2, {10: 39}), (3, {5: 3}), (3, {6: big}),
             (3, {2: 1 << 20, 6: (1 << 16) + 1, 10: 1 << 20}), (4, {0: four}), (4, {1: two}), (4, {4: two}), (4, {8: two}), (4, {9: two}), (4, {9: odd, 5: 1}),
             (6, {6: 60}), (6, {6: 60, 11: p, 12: 60 * 68 - 1}), (6, {6: 60, 11: four, 12: 1 << 30})))
    refused(lib.bs_mx4_gemm_packed, (p, p, 40, 64, p, p, 9, null, p, 0, 40, null, 0, null),
            (*((1, {at: null}) for at in (0, 1, 4, 5, 8)), (2, {6: 0}), (2, {10: 39}), (2, {3: 0}), (3, {9: 3}), (3, {6: big}), (3, {2: big, 10: big}),
             (4, {4: four}), (4, {5: two}), (4, {7: odd}), (4, {8: two}), (6, {2: 4096, 10: 4096, 3: 25088, 6: 77}),
             (6, {2: 4096, 10: 4096, 3: 25088, 6: 77, 11: p, 12: 1024})))
    refused(lib.bs_beam_step, (p, 0, 2, 3, 100, 100, p, p, 5, 4, p, p, p, p, p, 1 << 30, null),
            (*((1, {at: null}) for at in (0, 6, 10, 11, 12, 13)), (2, {2: 0}), (2, {3: 0}), (2, {4: 0}), (2, {9: 0}), (2, {5: 99}), (2, {8: 100}),
             (3, {1: 3}), (3, {2: big}), (3, {3: 65}), (3, {9: 65}), (3, {4: 1 << 31, 5: 1 << 31}), (4, {0: two}), (4, {0: odd, 1: 2}), (4, {6: two}),
             (4, {10: two}), (4, {11: odd}), (4, {12: two}), (6, {14: null}), (6, {15: 64}), (6, {14: four})))


def test_reorder_refusals():
    lib = b.load_library()

    def call(states, outs, size, pitch, out_pitch, B=2, W=3, parents=1 << 20, count=None):
        n = max(len(states), 1)
        return lib.bs_beam_reorder(len(states) if count is None else count, (ctypes.c_void_p * n)(*states), (ctypes.c_void_p * n)(*outs), (ctypes.c_int64 * n)(*size),
                                   (ctypes.c_int64 * n)(*pitch), (ctypes.c_int64 * n)(*out_pitch), B, W, ctypes.c_void_p(parents), ctypes.c_void_p(0))

    a, c = 1 << 30, 1 << 31
    ok = ([a], [c], [8], [8], [8])
    for status, args, more in (
            (1, ([0], [c], [8], [8], [8]), {}), (1, ([a], [0], [8], [8], [8]), {}), (1, ok, {"parents": 0}),
            (2, ok, {"B": 0}), (2, ok, {"W": 0}), (2, ok, {"count": 0}), (2, ([a], [c], [0], [8], [8]), {}), (2, ([a], [c], [8], [7], [8]), {}),
            (2, ([a], [c], [8], [8], [7]), {}), (3, ok, {"W": 65}), (3, ok, {"B": (1 << 24) + 1}), (3, ok, {"count": 33}),
            (3, ([a], [c], [(1 << 30) + 1], [1 << 31], [1 << 31]), {}), (3, ([a], [c], [8], [1 << 32], [8]), {}), (3, ([a], [c], [8], [8], [1 << 32]), {}),
            (4, ok, {"parents": (1 << 20) + 2}),
            # overlaps: an output with its own input at another place or pitch, with another's, with another output, with the parents
            (3, ([a], [a + 8], [8], [8], [8]), {}), (3, ([a], [a - 47], [8], [8], [8]), {}), (3, ([a], [a], [8], [8], [16]), {}), (3, ([a], [a + 4], [8], [16], [16]), {}),
            (3, ([a, c], [c, a], [8, 8], [8, 8], [8, 8]), {}), (3, ([a, a + 48], [c, c + 40], [8, 8], [8, 8], [8, 8]), {}),
            (3, ([a, a], [a, a], [8, 8], [8, 8], [8, 8]), {}), (3, ([a], [c], [8], [8], [8]), {"parents": c + 44}), (3, ([a], [a], [8], [8], [8]), {"parents": a - 4})):
        assert call(*args, **more) == status, (status, args, more)


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    """That of the older calls, and these."""
    older = STAND_IN.replace("    static const auto real", FAKE + "    static const auto real").replace("int out_of_memory = 0,", "int host_memory = 0, out_of_memory = 0,")
    assert older.count("host_memory") == 2
    more = r"""
extern "C" {
int bs_mx4_pack(const void* first, int, int64_t, int64_t, int64_t, uint8_t*, uint8_t*, void*) CALL
int bs_mx4_unpack(const uint8_t* first, const uint8_t*, int64_t, int64_t, void*, int, void*) CALL
int bs_mx4_gemm(const uint8_t* first, const uint8_t*, int64_t, int64_t, const void*, int, int64_t, int64_t, const float*, void*, int64_t, void*,
                size_t, void*) CALL
int bs_mx4_gemm_packed(const uint8_t* first, const uint8_t*, int64_t, int64_t, const uint8_t*, const uint8_t*, int64_t, const float*, void*, int,
                       int64_t, void*, size_t, void*) CALL
int bs_beam_step(const void* first, int, int64_t, int, int64_t, int64_t, const float*, const uint8_t*, int64_t, int, float*, int32_t*, int32_t*,
                 uint8_t*, void*, size_t, void*) CALL
int64_t seen[6];
int bs_beam_reorder(int count, const void* const* states, void* const* outs, const int64_t* bytes, const int64_t* pitch, const int64_t* out_pitch,
                    int64_t, int, const int32_t*, void*) {
    const void* first = states[0];
    seen[0] = count; seen[1] = bytes[count - 1]; seen[2] = pitch[count - 1]; seen[3] = out_pitch[count - 1]; seen[4] = states[0] == outs[0];
    CALL
}
}
"""
    tmp = tmp_path_factory.mktemp("stand_in")
    src, lib = str(tmp / "stand_in.cpp"), str(tmp / "stand_in.so")
    with open(src, "w") as f:
        f.write(older + more)
    subprocess.check_call([*bs_build.native_compiler(), "-I" + os.path.join(ROOT, "include"), "-shared", "-o", lib, src,
                           "-L" + os.path.join(os.path.dirname(torch.__file__), "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu"])
    return lib


QUERIES = PREAMBLE.replace('("bs_status_str",', '("bs_status_str", "bs_mx4_gemm_workspace_bytes", "bs_mx4_gemm_packed_workspace_bytes", "bs_beam_step_workspace_bytes",')
CALLS = """
    u8, types = torch.uint8, (torch.float32, torch.float16, torch.bfloat16)
    def apart(*size, stride, dtype=torch.float32):
        '''rows of a wider tensor, or a view of a larger one'''
        host = torch.zeros(4096, dtype=dtype)
        kept.append(host)
        storage = torch._C._construct_storage_from_data_pointer(host.data_ptr(), torch.device("cuda", 0), host.numel() * host.element_size())
        return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(dict(size=size, stride=stride, dtype=dtype, storage_offset=3), storage)
    def calls(dtype=torch.float32, rows=13):
        '''name -> call; all but the last two allocate what they return'''
        codes, scales, x_codes, x_scales = gpu(40, 64, dtype=u8), gpu(40, 4, dtype=u8), gpu(13, 64, dtype=u8), gpu(13, 4, dtype=u8)
        x, x1, bias, logits, scores = gpu(rows, 100, dtype=dtype), gpu(100, dtype=dtype), gpu(40), gpu(6, 500, dtype=dtype), gpu(2, 3)
        W, y, states, parents = gpu(2, 5, 130, dtype=dtype), gpu(40, dtype=dtype), [gpu(6, 7, dtype=dtype), gpu(2, 3, 5, dtype=torch.int32)], gpu(2, 3, dtype=torch.int32)
        done = gpu(2, 3, dtype=torch.bool)
        return {"bs_mx4_pack": lambda **k: bs.bs_mx4_pack(W),
                "bs_mx4_unpack": lambda **k: bs.bs_mx4_unpack(codes, scales, 100, dtype=dtype),
                "bs_mx4_gemm": lambda **k: bs.bs_mx4_gemm(codes, scales, x, bias=bias, **k),
                "bs_mx4_gemm_packed": lambda **k: bs.bs_mx4_gemm_packed(codes, scales, x_codes, x_scales, 100, dtype=dtype, **k),
                "bs_beam_step": lambda **k: bs.bs_beam_step(logits, scores, done, end=7, n=5, **k),
                "bs_mx4_gemm ": lambda **k: bs.bs_mx4_gemm(codes, scales, x1, out=y),
                "bs_beam_reorder": lambda **k: bs.bs_beam_reorder(states, parents)}
"""


def _run(stand_in, body):
    code = textwrap.dedent(QUERIES + CALLS) + textwrap.dedent(body)
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env={**os.environ, "BS_STAND_IN": stand_in}, capture_output=True, text=True,
                         timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr


def test_a_status_is_raised_after_one_attempt(stand_in):
    _run(stand_in, """
        ctypes.c_int.in_dll(stand_in, "host_memory").value = 1
        for dtype in types:
            for name, f in calls(dtype).items():
                for status in range(1, 9):
                    ctypes.c_int.in_dll(stand_in, "status").value = status
                    attempts.value = 0
                    try:
                        f()
                    except bs.BsError as e:
                        assert e.status == status and str(e).startswith(name.strip() + ":"), (name, e)
                    else:
                        raise AssertionError(name + ": no error")
                    assert attempts.value == 1, (name, status, attempts.value)
    """)


def test_results(stand_in):
    """Shapes and types of what the native code allocates, and what is refused before the library is called."""
    _run(stand_in, """
        ctypes.c_int.in_dll(stand_in, "host_memory").value = 1
        ctypes.c_int.in_dll(stand_in, "status").value = 0
        for dtype in types:
            c = calls(dtype)
            codes, scales = c["bs_mx4_pack"]()
            assert tuple(codes.shape) == (2, 5, 128) and tuple(scales.shape) == (2, 5, 8) and codes.dtype == scales.dtype == u8
            W = c["bs_mx4_unpack"]()
            assert tuple(W.shape) == (40, 100) and W.dtype == dtype
            for name in ("bs_mx4_gemm", "bs_mx4_gemm_packed"):
                y = c[name]()
                assert tuple(y.shape) == (13, 40) and y.dtype == dtype
            out = c["bs_beam_step"]()
            assert all(tuple(t.shape) == (2, 5) for t in out) and [t.dtype for t in out] == [torch.float32, torch.int32, torch.int32, torch.bool]
            assert tuple(c["bs_mx4_gemm "]().shape) == (40,)
        codes, scales, x, bias = gpu(40, 64, dtype=u8), gpu(40, 4, dtype=u8), gpu(2, 100), gpu(40)
        logits, scores, parents, state = gpu(6, 500), gpu(2, 3), gpu(2, 3, dtype=torch.int32), gpu(6, 7)
        seen = (ctypes.c_int64 * 6).in_dll(stand_in, "seen")
        wide, other = apart(6, 5, stride=(20, 1), dtype=torch.float16), apart(6, 5, stride=(9, 1), dtype=torch.float16)
        assert bs.bs_beam_reorder([state, wide], parents)[0] is state and list(seen[:5]) == [2, 10, 40, 40, 1]
        assert bs.bs_beam_reorder(wide, parents, out=other) is other and list(seen[:5]) == [1, 10, 40, 18, 0]
        attempts.value = 0
        bad = (lambda: bs.bs_mx4_gemm(codes, scales, x, out=gpu(2, 41)), lambda: bs.bs_mx4_gemm(codes, scales, x, out=gpu(3, 40)),
               lambda: bs.bs_mx4_gemm(codes, scales, gpu(2, 129)), lambda: bs.bs_mx4_gemm(codes, gpu(40, 5, dtype=u8), x),
               lambda: bs.bs_mx4_gemm(codes, scales, x, bias=gpu(41)), lambda: bs.bs_mx4_gemm(gpu(2, 20, 64, dtype=u8), gpu(2, 20, 4, dtype=u8), x),
               lambda: bs.bs_mx4_gemm_packed(codes, scales, gpu(2, 128, dtype=u8), gpu(2, 8, dtype=u8), 100),
               lambda: bs.bs_mx4_unpack(codes, scales, 100, out=gpu(40, 99)), lambda: bs.bs_mx4_unpack(codes, scales, 129),
               lambda: bs.bs_beam_step(logits, gpu(2, 4)), lambda: bs.bs_beam_step(logits, gpu(6)), lambda: bs.bs_beam_step(logits, scores, gpu(3, 2, dtype=u8)),
               lambda: bs.bs_beam_step(logits, scores, gpu(2, 3, dtype=torch.int32)),
               lambda: bs.bs_beam_reorder([gpu(5, 7)], parents), lambda: bs.bs_beam_reorder([state], parents, out=[gpu(6, 8)]),
               lambda: bs.bs_beam_reorder([state], parents, out=[gpu(6, 7, dtype=torch.int32)]), lambda: bs.bs_beam_reorder([state], gpu(6, dtype=torch.int32)),
               lambda: bs.bs_beam_reorder([state], parents, out=[gpu(6, 7), gpu(6, 7)]), lambda: bs.bs_beam_reorder([apart(6, 4, 3, stride=(24, 6, 1))], parents),
               lambda: bs.bs_beam_reorder([apart(6, 4, stride=(3, 1))], parents), lambda: bs.bs_beam_reorder([apart(6, 4, stride=(8, 2))], parents),
               lambda: bs.bs_beam_step(apart(6, 500, stride=(499, 1)), scores), lambda: bs.bs_mx4_gemm(codes, scales, apart(2, 100, stride=(1, 2))))
        types_wrong = (lambda: bs.bs_mx4_gemm(codes, scales, gpu(2, 100, dtype=torch.float64)), lambda: bs.bs_mx4_gemm(torch.zeros(40, 64, dtype=u8), scales, x),
                       lambda: bs.bs_mx4_gemm(codes, gpu(40, 4, dtype=torch.float16), x), lambda: bs.bs_mx4_gemm(codes, scales, x, bias=gpu(40, dtype=torch.float16)),
                       lambda: bs.bs_mx4_pack(gpu(4, 4, dtype=torch.int32)), lambda: bs.bs_mx4_unpack(codes, scales, 100, dtype=torch.int32),
                       lambda: bs.bs_beam_step(logits, gpu(2, 3, dtype=torch.float16)), lambda: bs.bs_beam_reorder([state], gpu(2, 3, dtype=torch.int64)))
        for kind, fs in ((ValueError, bad), (TypeError, types_wrong)):
            for i, f in enumerate(fs):
                try:
                    f()
                except kind:
                    pass
                else:
                    raise AssertionError((kind, i))
        for f in (lambda: bs.bs_beam_step(logits, scores, n=0), lambda: bs.bs_beam_step(logits, scores, n=-1)):
            try:
                f()
            except bs.BsError as e:
                assert e.status == 2
            else:
                raise AssertionError("no error")
        assert attempts.value == 0
    """)


def test_tensors_of_another_device_are_refused(stand_in):
    _run(stand_in, """
        ctypes.c_int.in_dll(stand_in, "host_memory").value = 1
        ctypes.c_int.in_dll(stand_in, "status").value = 0
        here = gpu
        def there(*size, dtype=torch.float32):
            host = torch.zeros(size, dtype=dtype)
            kept.append(host)
            storage = torch._C._construct_storage_from_data_pointer(host.data_ptr(), torch.device("cuda", 1), host.numel() * host.element_size())
            return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(dict(size=tuple(size), stride=host.stride(), dtype=dtype, storage_offset=0), storage)
        def mixed(at):
            '''gpu(), but the at-th tensor is on the second device'''
            count = [0]
            def make(*size, dtype=torch.float32):
                count[0] += 1
                return (there if count[0] - 1 == at else here)(*size, dtype=dtype)
            return make
        # in the order in which calls() makes them
        order = ["codes", "scales", "x_codes", "x_scales", "x", "x1", "bias", "logits", "scores", "W", "y", "state", "state", "parents", "done"]
        takes = {"bs_mx4_pack": ("W",), "bs_mx4_unpack": ("codes", "scales"), "bs_mx4_gemm": ("codes", "scales", "x", "bias"),
                 "bs_mx4_gemm_packed": ("codes", "scales", "x_codes", "x_scales"), "bs_beam_step": ("logits", "scores", "done"),
                 "bs_mx4_gemm ": ("codes", "scales", "x1", "y"), "bs_beam_reorder": ("state", "parents")}
        for at, what in enumerate(order):
            gpu = mixed(at)
            c = calls()
            for name, f in c.items():
                attempts.value = 0
                try:
                    f()
                except ValueError as e:
                    assert what in takes[name] and "current device" in str(e), (name, what, e)
                else:
                    assert what not in takes[name], (name, what)
                assert attempts.value == (what not in takes[name]), (name, what)
    """)


def test_exceptions_keep_their_types_and_allocations_give_the_lock_up(stand_in):
    _run(stand_in, """
        from torch.utils._python_dispatch import TorchDispatchMode

        class Refuses(TorchDispatchMode):
            def __torch_dispatch__(self, func, types, args=(), kwargs=None):
                raise KeyError("refused")

        fails, held = ctypes.c_int.in_dll(stand_in, "out_of_memory"), ctypes.c_int.in_dll(stand_in, "lock_held")
        for name, f in list(calls().items())[:-2]:
            for want, text in ((KeyError, "refused"), (torch.OutOfMemoryError, "no memory left")):
                fails.value, held.value = want is not KeyError, -1
                try:
                    if want is KeyError:
                        with Refuses():
                            f()
                    else:
                        f()
                except Exception as e:
                    assert type(e) is want and text in str(e), (name, type(e), e)
                else:
                    raise AssertionError(name + ": no error")
                assert held.value == (-1 if want is KeyError else 0), (name, held.value)
            fails.value = 0
        assert attempts.value == 0
    """)


def test_a_workspace_in_host_memory_is_refused(stand_in):
    _run(stand_in, """
        ctypes.c_int.in_dll(stand_in, "host_memory").value = 1
        ctypes.c_int.in_dll(stand_in, "status").value = 0
        c = calls(rows=60)      # more than every workgroup rounds for itself
        for name in ("bs_mx4_gemm", "bs_beam_step"):
            for host in (torch.empty(1 << 20, dtype=u8), bytearray(1 << 20)):
                attempts.value = 0
                try:
                    c[name](workspace=host)
                except TypeError as e:
                    assert "workspace" in str(e), e
                else:
                    raise AssertionError(name + ": no error")
                assert attempts.value == 0
            c[name](workspace=gpu(1 << 20, dtype=u8))
            assert attempts.value == 1
    """)


def _assembly(src):
    flags = [f for f in bs_build.FLAGS if f != "-fPIC"]
    return subprocess.run([bs_build.HIPCC, *flags, "-S", "--cuda-device-only", "-o", "-", os.path.join(bs_build.CSRC, src)],
                          stderr=subprocess.DEVNULL, stdout=subprocess.PIPE, check=True, text=True).stdout


@pytest.fixture(scope="module")
def texts():
    with ThreadPoolExecutor(3) as ex:
        return dict(zip(SOURCES, ex.map(_assembly, SOURCES)))


def test_no_kernel_spills_registers_or_packs_fp32(texts):
    for src, text in texts.items():
        spills = re.findall(r"\.vgpr_spill_count:\s+(\d+)", text)
        assert spills and not any(map(int, spills)), src
        assert not any(map(int, re.findall(r"\.private_segment_fixed_size:\s+(\d+)", text))), src
        assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text), src


def test_tiles_wait_for_their_stages(texts):
    """Loads to LDS are written in assembly and waited for by counting: in front of the barrier in the loop a wavefront may have no more on
    their way than it has sent for since the stage that comes next, whole stages, and the compiler has put no wait of its own among the
    loads and none of what it does goes through M0."""
    found = 0
    for name, body in re.findall(r"^(_ZN2bs16mx4_tiles_kernel\w+):(.*?)\.Lfunc_end", texts["bs_mx4_gemm.hip"], re.S | re.M):
        tn, tm, _, _, buffers = map(int, re.findall(r"Li(\d+)E", name)[:5])
        each = (tn + tm) // 32      # loads of codes of a wavefront and stage
        lines = [s.strip() for s in body.splitlines()]
        ins = [s for s in lines if s and not s.startswith((";", "."))]
        barriers = [i for i, s in enumerate(ins) if s == "s_barrier"]
        waits = [int(re.search(r"vmcnt\((\d+)\)", ins[i - 1]).group(1)) for i in barriers if ins[i - 1].startswith("s_waitcnt vmcnt")]
        assert waits[:2] == [(buffers - 2) * each] * 2, (name, waits)
        # between the barrier in the loop and itself: the loop, whichever way the compiler turned it
        first = next(i for i, s in enumerate(ins) if s.startswith("global_load_lds_dwordx4"))
        sends = [i for i, s in enumerate(ins) if s.startswith("global_load_lds")]
        assert sends[0] == first and all(ins[i - 1] == "s_nop 0" and ins[i - 2].startswith("s_mov_b32 m0") for i in sends), name
        assert all(ins[i + 1] == "s_mov_b64 exec, -1" for i in sends), name
        assert sum("m0" in s for s in ins) == len(sends), name
        inside = [s for s in ins[barriers[0]:sends[-1]] if s.startswith("s_waitcnt") and "vmcnt" in s]
        assert len(inside) == 1, (name, inside)
        found += 1
    assert found == 4 * 6      # three types and the sums of shares of K


def test_the_package_offers_them():
    import paper_1811_00206_amd as package
    for name in ("bs_mx4_codes_bytes", "bs_mx4_scales_bytes", "bs_mx4_pack", "bs_mx4_unpack", "bs_mx4_gemm_workspace_bytes", "bs_mx4_gemm",
                 "bs_mx4_gemm_packed_workspace_bytes", "bs_mx4_gemm_packed", "bs_mx4_gemm_plan", "bs_beam_step_workspace_bytes", "bs_beam_step", "bs_beam_reorder"):
        assert name in package.__all__ and callable(getattr(package, name))
