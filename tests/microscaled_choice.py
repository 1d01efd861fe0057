"""The rule by which a call of scores_microscaled takes a kernel, compiled from the library's own header for the host."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = ("online", "few", "held", "small", "large")
SOURCE = '''#include "xc_microscaled_choice.h"
static_assert(xc::kMicroOnline == 0 && xc::kMicroFew == 1 && xc::kMicroHeld == 2 && xc::kMicroSmall == 3 && xc::kMicroLarge == 4, "");
extern "C" int choose(int64_t B, int64_t L, int units) { return xc::choose_micro(B, L, units); }
'''


def build(folder):
    """A function (B, L, d) -> name of the kernel."""
    src, so = os.path.join(folder, "micro_choice.cpp"), os.path.join(folder, "micro_choice.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "paper_2409_20156_amd", "csrc"), src, "-o", so],
                   check=True)
    fn = ctypes.CDLL(so).choose
    fn.argtypes, fn.restype = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int], ctypes.c_int
    return lambda B, L, d: KERNELS[fn(B, L, (d + 127) // 128)]
