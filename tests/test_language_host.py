"""The calls on 4-bit matrices, expert layers and logits where no GPU is needed: sizes, refusals before anything is launched, the
native marshalling where the library or torch fails, and what the compiler made of the kernels."""
import ctypes
import os
import re
import subprocess
import sys
import textwrap
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from paper_1811_00206_amd import binding as b
from paper_1811_00206_amd import build as bs_build
from test_native_calls import PREAMBLE, STAND_IN

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = ["bs_q4_pack.hip", "bs_q4_gemv.hip", "bs_q4_moe.hip", "bs_logprobs.hip"]


def test_sizes():
    assert b.bs_q4_codes_bytes(6000, 3000) == 6000 * 1504 and b.bs_q4_scales_bytes(6000, 3000, 64) == 6000 * 47 * 2
    assert b.bs_q4_codes_bytes(1, 1) == 16 and b.bs_q4_scales_bytes(1, 1, 128) == 2
    assert b.bs_q4_codes_bytes(1 << 24, 1 << 24) == 1 << 47
    for M, K, group in ((0, 8, 32), (8, 0, 32), (-1, 8, 32), (8, 8, 0), (8, 8, 33), (8, 8, 256), ((1 << 24) + 1, 8, 32), (8, (1 << 24) + 1, 32)):
        assert b.bs_q4_scales_bytes(M, K, group) == 0
    assert b.bs_q4_codes_bytes(0, 8) == 0 and b.bs_q4_codes_bytes(8, (1 << 24) + 1) == 0


def test_workspaces():
    gemv, moe, lp = b.bs_q4_gemv_workspace_bytes, b.bs_q4_moe_workspace_bytes, b.bs_logprobs_workspace_bytes
    for dtype in (b.BS_F32, b.BS_F16, b.BS_BF16):
        assert gemv(dtype, 10000, 1500, 32, 1) == 0                   # one vector needs none
        assert gemv(dtype, 4096, 25088, 64, 65535) > 0
        assert moe(dtype, 1, 1500, 1500, 8, 2, 32) > 0
        # 64 tokens pass together: more need no more
        sizes = [moe(dtype, T, 512, 300, 16, 4, 64) for T in range(1, 200)]
        assert max(sizes) == max(sizes[:64]) and min(sizes) > 0 and sizes[63] == sizes[127]
        assert moe(dtype, b.MOE_TOKENS_MAX, 512, 300, 16, 4, 64) == sizes[63]
        assert lp(dtype, 4096, 1000, 64) == 0 and lp(dtype, 1, 131072, 20) > 0
    for args in ((9, 8, 8, 32, 8), (0, 0, 8, 32, 8), (0, 8, 0, 32, 8), (0, 8, 8, 16, 8), (0, 8, 8, 32, 0), (0, 8, 8, 32, 65536)):
        assert gemv(*args) == 0
    good = (0, 4, 64, 32, 8, 2, 32)
    assert moe(*good) > 0
    for at, values in ((0, (3, -1)), (1, (0, b.MOE_TOKENS_MAX + 1)), (2, (0, (1 << 24) + 1)), (3, (0, (1 << 23) + 1)), (4, (0, 1, 1025)), (5, (0, 9, 33)),
                       (6, (0, 48))):
        for v in values:
            assert moe(*good[:at], v, *good[at + 1:]) == 0, (at, v)
    for args in ((3, 1, 131072, 1), (0, 0, 131072, 1), (0, 1, 0, 0), (0, 1, 131072, 65), (0, 1, 131072, -1), (0, 1, 1 << 31, 1)):
        assert lp(*args) == 0


def test_bad_arguments_are_refused_before_launch():
    lib = b.load_library()
    p, odd, null = (ctypes.c_void_p(a) for a in (4096, 4097, 0))      # never dereferenced: validation fails first
    two = ctypes.c_void_p(4098)                                       # aligned for 16 bits, not for 32

    def refused(f, good, changes):
        for status, change in changes:
            args = list(good)
            for at, v in change.items():
                args[at] = v
            assert f(*args) == status, (f.__name__, status, change)

    refused(lib.bs_q4_pack, (p, 0, 4, 64, 32, p, p, null),
            ((1, {0: null}), (1, {5: null}), (1, {6: null}), (2, {2: 0}), (2, {3: 0}), (3, {1: 3}), (3, {4: 31}), (3, {2: (1 << 24) + 1}),
             (4, {0: two}), (4, {0: odd, 1: 1}), (4, {5: two}), (4, {6: odd})))
    refused(lib.bs_q4_unpack, (p, p, 4, 64, 32, p, 0, null),
            ((1, {0: null}), (1, {5: null}), (2, {2: -1}), (3, {6: 7}), (3, {4: 96}), (4, {0: two}), (4, {5: two}), (4, {5: odd, 6: 2})))
    refused(lib.bs_q4_gemv, (p, p, 40, 64, 32, p, 0, 1, 64, p, 40, null, 0, null),
            ((1, {0: null}), (1, {5: null}), (1, {9: null}), (2, {7: 0}), (2, {8: 63}), (2, {10: 39}), (3, {6: 3}), (3, {7: 65536}), (3, {4: 8}),
             (4, {0: two}), (4, {5: two}), (4, {9: odd, 6: 1}), (6, {7: 9}), (6, {7: 9, 11: p, 12: 16}), (6, {7: 9, 11: two, 12: 1 << 30})))
    good = (p, 0, 2, 64, 64, p, 8, p, p, p, p, 32, 32, 2, 1, p, 64, p, p, p, 1 << 30, null)
    refused(lib.bs_q4_moe, good,
            (*((1, {at: null}) for at in (0, 5, 7, 8, 9, 10, 15, 17, 18)), (2, {2: 0}), (2, {3: 63}), (2, {16: 63}), (2, {6: 0}), (2, {13: 0}),
             (2, {13: 9}), (2, {11: 0}), (3, {1: 3}), (3, {2: 65537}), (3, {6: 1025}), (3, {6: 40, 13: 33}), (3, {12: 16}), (3, {11: (1 << 23) + 1}),
             (4, {0: two}), (4, {7: two}), (4, {8: odd}), (4, {9: two}), (4, {17: two}), (6, {19: null}), (6, {20: 64}), (6, {19: two})))
    refused(lib.bs_logprobs, (p, 0, 3, 100, 100, p, 5, p, p, p, p, p, null, 0, null),
            (*((1, {at: null}) for at in (0, 5, 7, 8, 9, 10, 11)), (2, {2: 0}), (2, {3: 0}), (2, {4: 99}), (2, {6: -1}), (2, {3: 4, 6: 5}),
             (3, {1: 5}), (3, {6: 65}), (3, {3: 1 << 31, 4: 1 << 31}), (4, {0: two}), (4, {5: ctypes.c_void_p(4100)}), (4, {7: two}),
             (6, {3: 131072, 4: 131072}), (6, {3: 131072, 4: 131072, 12: p, 13: 16})))
    refused(lib.bs_logprobs_backward, (p, 0, 3, 100, 100, p, p, p, p, p, ctypes.c_void_p(8192), 100, null),
            ((1, {0: null}), (1, {6: null}), (1, {7: null}), (1, {9: null}), (1, {8: null}), (1, {10: null}), (2, {4: 99}), (2, {11: 99}),
             (3, {1: 4}), (3, {10: p, 11: 101}), (4, {10: two}), (4, {6: two})))


def test_older_calls_know_no_bfloat16():
    lib = b.load_library()
    p, null = ctypes.c_void_p(4096), ctypes.c_void_p(0)
    two = b.BS_BF16
    assert b.bs_vals_bytes(4, 8, 4, 2, two) == 0
    assert lib.bs_prune_pack(p, two, 4, 8, 4, 2, p, p, null) == 3
    assert lib.bs_spmv(p, p, two, 4, 8, 4, 2, p, p, null) == 3
    assert lib.bs_spmm(p, p, two, 4, 8, 4, 2, p, 4, 4, p, 4, null, 0, null) == 3
    assert lib.bs_reprune(p, p, two, 4, 8, 4, 2, 1, p, p, null) == 3
    assert lib.bs_dense_gemv(p, two, 4, 8, p, p, null) == 3


FAKE = r"""
    // told so, host memory that claims to be on the GPU
    if (host_memory && device && device->is_cuda()) {
        size_t bytes = c10::elementSize(*dtype);
        c10::SmallVector<int64_t, 4> sizes;
        for (const auto& n : size) {
            sizes.push_back(n.expect_int());
            bytes *= (size_t)sizes.back();
        }
        c10::Storage storage(c10::Storage::use_byte_size_t(), bytes, c10::DataPtr(calloc(bytes + 1, 1), Device(kCUDA, 0)), nullptr, false);
        Tensor t = at::detail::make_tensor<c10::TensorImpl>(::std::move(storage), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                            c10::scalarTypeToTypeMeta(*dtype));
        t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
        return t;
    }
"""


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    """That of the older calls, and these."""
    older = STAND_IN.replace("    static const auto real", FAKE + "    static const auto real").replace("int out_of_memory = 0,", "int host_memory = 0, out_of_memory = 0,")
    assert older.count("host_memory") == 2
    more = r"""
extern "C" {
int bs_q4_pack(const void* first, int, int64_t, int64_t, int, uint8_t*, uint16_t*, void*) CALL
int bs_q4_unpack(const uint8_t* first, const uint16_t*, int64_t, int64_t, int, void*, int, void*) CALL
int bs_q4_gemv(const uint8_t* first, const uint16_t*, int64_t, int64_t, int, const void*, int, int64_t, int64_t, void*, int64_t, void*,
               size_t, void*) CALL
int bs_q4_moe(const void* first, int, int64_t, int64_t, int64_t, const void*, int, const uint8_t*, const uint16_t*, const uint8_t*,
              const uint16_t*, int64_t, int, int, int, void*, int64_t, int32_t*, float*, void*, size_t, void*) CALL
int bs_logprobs(const void* first, int, int64_t, int64_t, int64_t, const int64_t*, int, float*, float*, float*, float*, int32_t*, void*,
                size_t, void*) CALL
int bs_logprobs_backward(const void* first, int, int64_t, int64_t, int64_t, const int64_t*, const float*, const float*, const float*,
                         const float*, void*, int64_t, void*) CALL
}
"""
    tmp = tmp_path_factory.mktemp("stand_in")
    src, lib = str(tmp / "stand_in.cpp"), str(tmp / "stand_in.so")
    with open(src, "w") as f:
        f.write(older + more)
    subprocess.check_call([*bs_build.native_compiler(), "-I" + os.path.join(ROOT, "include"), "-shared", "-o", lib, src,
                           "-L" + os.path.join(os.path.dirname(torch.__file__), "lib"), "-lc10", "-lc10_hip", "-ltorch_cpu"])
    return lib


QUERIES = PREAMBLE.replace('("bs_status_str",', '("bs_status_str", "bs_q4_gemv_workspace_bytes", "bs_q4_moe_workspace_bytes", "bs_logprobs_workspace_bytes",')
CALLS = """
    types = (torch.float32, torch.float16, torch.bfloat16)
    def calls(dtype=torch.float32, V=131072):
        '''name -> call; all but the last two allocate what they return'''
        E, D, F, T, group = 3, 64, 32, 2, 32
        codes, scales = gpu(40, 32, dtype=torch.uint8), gpu(40, 2, dtype=torch.float16)
        w1, s1 = gpu(E, 2 * F, 32, dtype=torch.uint8), gpu(E, 2 * F, 2, dtype=torch.float16)
        w2, s2 = gpu(E, D, 16, dtype=torch.uint8), gpu(E, D, 1, dtype=torch.float16)
        x, x1, router, logits, targets, one = gpu(13, D, dtype=dtype), gpu(D, dtype=dtype), gpu(E, D, dtype=dtype), gpu(1, V, dtype=dtype), gpu(1, dtype=torch.int64), gpu(1)
        W, y, grad = gpu(2, 5, 70, dtype=dtype), gpu(40, dtype=dtype), gpu(1, V, dtype=dtype)
        return {"bs_q4_pack": lambda **k: bs.bs_q4_pack(W, group),
                "bs_q4_unpack": lambda **k: bs.bs_q4_unpack(codes, scales, D, group, dtype=dtype),
                "bs_q4_gemv": lambda **k: bs.bs_q4_gemv(codes, scales, group, x, **k),
                "bs_q4_moe": lambda **k: bs.bs_q4_moe(x, router, w1, s1, w2, s2, group, 2, **k),
                "bs_logprobs": lambda **k: bs.bs_logprobs(logits, targets, top_n=3, **k),
                "bs_logprobs_backward": lambda **k: bs.bs_logprobs_backward(logits, targets, one, one, one, one),
                "bs_q4_gemv ": lambda **k: bs.bs_q4_gemv(codes, scales, group, x1, out=y),
                "bs_logprobs_backward ": lambda **k: bs.bs_logprobs_backward(logits, targets, one, None, one, None, out=grad)}
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
    """Shapes and types of what the native code allocates, and its refusals of outputs that do not fit."""
    _run(stand_in, """
        ctypes.c_int.in_dll(stand_in, "host_memory").value = 1
        ctypes.c_int.in_dll(stand_in, "status").value = 0
        for dtype in types:
            c = calls(dtype)
            codes, scales = c["bs_q4_pack"]()
            assert tuple(codes.shape) == (2, 5, 48) and tuple(scales.shape) == (2, 5, 3), (codes.shape, scales.shape)
            assert codes.dtype == torch.uint8 and scales.dtype == torch.float16
            W = c["bs_q4_unpack"]()
            assert tuple(W.shape) == (40, 64) and W.dtype == dtype
            y = c["bs_q4_gemv"]()
            assert tuple(y.shape) == (13, 40) and y.dtype == dtype
            y, ids, weights = c["bs_q4_moe"]()
            assert tuple(y.shape) == (13, 64) and y.dtype == dtype and tuple(ids.shape) == tuple(weights.shape) == (13, 2)
            assert ids.dtype == torch.int32 and weights.dtype == torch.float32
            *three, values, ids = c["bs_logprobs"]()
            assert all(tuple(t.shape) == (1,) and t.dtype == torch.float32 for t in three)
            assert tuple(values.shape) == tuple(ids.shape) == (1, 3) and values.dtype == torch.float32 and ids.dtype == torch.int32
            grad = c["bs_logprobs_backward"]()
            assert tuple(grad.shape) == (1, 131072) and grad.dtype == dtype
            assert tuple(c["bs_q4_gemv "]().shape) == (40,)
        attempts.value = 0
        x, codes, scales = gpu(2, 64), gpu(40, 32, dtype=torch.uint8), gpu(40, 2, dtype=torch.float16)
        logits, targets, one = gpu(2, 50), gpu(2, dtype=torch.int64), gpu(2)
        for f in (lambda: bs.bs_q4_gemv(codes, scales, 32, x, out=gpu(2, 41)), lambda: bs.bs_q4_gemv(codes, scales, 32, x, out=gpu(3, 40)),
                  lambda: bs.bs_q4_unpack(codes, scales, 64, 32, out=gpu(40, 63)),
                  lambda: bs.bs_logprobs_backward(logits, targets, one, one, one, one, out=gpu(2, 51)),
                  lambda: bs.bs_logprobs_backward(logits, targets, one, one, one, None)):
            try:
                f()
            except ValueError:
                pass
            else:
                raise AssertionError("no error")
        assert attempts.value == 0
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
        c = calls()
        for name in ("bs_q4_gemv", "bs_q4_moe", "bs_logprobs"):
            for host in (torch.empty(1 << 20, dtype=torch.uint8), bytearray(1 << 20)):
                attempts.value = 0
                try:
                    c[name](workspace=host)
                except TypeError as e:
                    assert "workspace" in str(e), e
                else:
                    raise AssertionError(name + ": no error")
                assert attempts.value == 0
            c[name](workspace=gpu(1 << 20, dtype=torch.uint8))
            assert attempts.value == 1
    """)


def _assembly(src):
    flags = [f for f in bs_build.FLAGS if f != "-fPIC"]
    return subprocess.run([bs_build.HIPCC, *flags, "-S", "--cuda-device-only", "-o", "-", os.path.join(bs_build.CSRC, src)],
                          stderr=subprocess.DEVNULL, stdout=subprocess.PIPE, check=True, text=True).stdout


def test_no_kernel_spills_registers_or_packs_fp32():
    with ThreadPoolExecutor(4) as ex:
        texts = list(ex.map(_assembly, SOURCES))
    for src, text in zip(SOURCES, texts):
        spills = re.findall(r"\.vgpr_spill_count:\s+(\d+)", text)
        assert spills and not any(map(int, spills)), src
        assert not any(map(int, re.findall(r"\.private_segment_fixed_size:\s+(\d+)", text))), src
        assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text), src
