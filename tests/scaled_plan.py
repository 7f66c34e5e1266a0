"""ctypes access to the host build of the plans of the 8-bit products with block scales (tests/scaled_plan_host.hip)."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def load(folder):
    so = str(folder / "scaled_plan_host.so")
    subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wno-inline-asm", "-o", so,
                    os.path.join(ROOT, "tests", "scaled_plan_host.hip")], check=True, capture_output=True)
    lib = ctypes.CDLL(so)
    lib.host_plan_scaled.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.POINTER(ctypes.c_int)]
    lib.host_plan_grad.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    return lib


def product(lib, M, N, K, workspace, narrow=False):
    """"few" (rows in one kernel), "256x256" or "128x256" (tile and program in one kernel), or (tile, ranges) of a divided contraction.  narrow: a program
    without row reductions and 8-bit outputs on a B stored [N x K]."""
    out = (ctypes.c_int * 4)()
    lib.host_plan_scaled(M, N, K, int(workspace), int(narrow), out)
    bm, bn, ranges, few = out
    tile = "%dx%d" % (bm, bn)
    return "few" if few else tile if ranges == 0 else (tile, ranges)


def gradient(lib, M, N, K, workspace):
    """(tile, ranges)"""
    out = (ctypes.c_int * 2)()
    lib.host_plan_grad(M, N, K, int(workspace), out)
    return tuple(out)
