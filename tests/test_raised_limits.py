"""The table of raised LDS limits (csrc/acc_plan.h): a kernel that is launched with more than it was allowed so far is raised again."""
import ctypes
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_SOURCE = r'''
#include "paper_2605_01255_amd/csrc/acc_plan.h"
static acc::RaisedLimits table;
extern "C" {
int has(intptr_t kernel, int device, uint32_t bytes) { return table.has((const void*)kernel, device, bytes); }
void add(intptr_t kernel, int device, uint32_t bytes) { table.add((const void*)kernel, device, bytes); }
int capacity() { return acc::RaisedLimits::kKernels; }
}
'''


def _table():
    with tempfile.TemporaryDirectory() as tmp:
        src, out = os.path.join(tmp, "raised.cpp"), os.path.join(tmp, "raised.so")
        with open(src, "w") as f:
            f.write(_SOURCE)
        subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + ROOT, src, "-o", out], check=True)
        so = ctypes.CDLL(out)
    so.has.argtypes = so.add.argtypes = [ctypes.c_ssize_t, ctypes.c_int, ctypes.c_uint32]
    return so


def test_limits_are_known_by_kernel_device_and_size():
    t = _table()
    assert not t.has(8, 0, 66000)
    t.add(8, 0, 70784)
    assert t.has(8, 0, 70784) and t.has(8, 0, 66000) and not t.has(8, 0, 82816)
    t.add(8, 0, 98304)
    assert t.has(8, 0, 98304)
    t.add(8, 0, 82816)                                           # a smaller one is not kept
    assert t.has(8, 0, 98304) and not t.has(8, 0, 98305)
    assert not t.has(8, 1, 66000) and not t.has(16, 0, 66000)    # another device, another kernel
    t.add(8, 63, 66000)
    assert t.has(8, 63, 66000) and not t.has(8, 63, 70784) and not t.has(8, 64, 1) and not t.has(8, -1, 1)
    t.add(8, 64, 66000)
    for kernel in range(100, 100 + t.capacity()):                # more kernels than places: those without one are set every time
        t.add(kernel, 0, 66000)
    assert t.has(100, 0, 66000) and not t.has(99 + t.capacity(), 0, 66000) and t.has(8, 0, 98304)
