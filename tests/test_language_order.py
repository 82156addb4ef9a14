"""Workgroups that share a sum: each stores its own, waits for the stores, and only then counts itself.  Stores and count are relaxed
atomics that nothing else orders, so the assembly the compiler emits for these sources is read.  No GPU needed."""
import os
import re
import subprocess

import pytest

from paper_1811_00206_amd import build as bs_build


def _kernels(src):
    """name -> instructions, and "pin" where nothing that touches memory may pass"""
    flags = [f for f in bs_build.FLAGS if f != "-fPIC"]
    text = subprocess.run([bs_build.HIPCC, *flags, "-S", "--cuda-device-only", "-o", "-", os.path.join(bs_build.CSRC, src)],
                          stderr=subprocess.DEVNULL, stdout=subprocess.PIPE, check=True, text=True).stdout
    name, kernels = None, {}
    for line in text.splitlines():
        m = re.match(r"^(_ZN2bs\w+_kernel\w+):", line)
        s = line.strip()
        if m:
            name = m.group(1)
            kernels[name] = []
        elif s.startswith(".Lfunc_end"):
            name = None
        elif name and s.startswith("; bs_pin"):
            kernels[name].append("pin")
        elif name and s and not s.startswith((";", ".")):
            kernels[name].append(s)
    return kernels


# every type (3) with every group (3): tiles of x with 1, 2 or 4 rows for one tile of vectors and for two, one row for four
@pytest.mark.parametrize("src,count", [("bs_q4_gemv.hip", 3 * 3 * 7), ("bs_q4_moe.hip", 3 * 3 * 2)])
def test_a_workgroup_counts_itself_behind_its_stores(src, count):
    found = 0
    for name, ins in _kernels(src).items():
        adds = [i for i, s in enumerate(ins) if s.startswith("global_atomic_add")]
        if not adds:
            continue
        found += 1
        assert len(adds) == 1, name
        pins = [i for i, s in enumerate(ins[:adds[0]]) if s == "pin"]
        assert len(pins) >= 2, name + ": nothing keeps the stores in front of the wait"
        first, second = pins[-2:]
        assert any(s.startswith("s_waitcnt") and "vmcnt(0)" in s for s in ins[first:second]), name
        assert any(s == "s_barrier" for s in ins[second:adds[0]]), name
        assert not any(s.startswith(("global_store", "flat_store", "buffer_store")) for s in ins[first:adds[0]]), name
        assert any(s.startswith("global_store") and "sc1" in s for s in ins[:first]), name
    assert found == count
