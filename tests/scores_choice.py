"""The rule by which a call of scores_quantized takes a kernel, compiled from the library's own header for the host."""
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = ("online", "thin", "narrow", "few", "low", "small", "some", "held", "mid", "many")
SOURCE = '''#include "xc_scores_choice.h"
static_assert(xc::kScoresOnline == 0 && xc::kScoresThin == 1 && xc::kScoresNarrow == 2 && xc::kScoresFew == 3 && xc::kScoresLow == 4 &&
              xc::kScoresSmall == 5 && xc::kScoresSome == 6 && xc::kScoresHeld == 7 && xc::kScoresMid == 8 && xc::kScoresMany == 9, "");
extern "C" int choose(int64_t B, int64_t L, int ppitch, int out_bytes) { return xc::choose_scores(B, L, ppitch, out_bytes); }
'''


def build(folder):
    """A function (B, L, d, bytes of a score) -> name of the kernel."""
    src, so = os.path.join(folder, "choice.cpp"), os.path.join(folder, "choice.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I" + os.path.join(ROOT, "paper_2409_20156_amd", "csrc"), src, "-o", so],
                   check=True)
    fn = ctypes.CDLL(so).choose
    fn.argtypes, fn.restype = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int], ctypes.c_int
    return lambda B, L, d, out: KERNELS[fn(B, L, (d + 127) // 128 * 128, out)]
