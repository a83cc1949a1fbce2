"""The short form of GELU (normal_below in csrc/arena_gemm.h) by itself: its source, compiled
for the host with a reciprocal and an exponential rounded once, against 64 bits."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest
from scipy.special import erfc, erfcx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = open(os.path.join(ROOT, "paper_2403_16125_amd", "csrc", "arena_gemm.h")).read()
T = np.linspace(0.0, 13.0, 260001).astype(np.float32)


def body():
    return re.search(r"^__device__ __forceinline__ void normal_below\(.*?^\}", SOURCE, flags=re.S | re.M)[0]


@pytest.fixture(scope="module")
def normal_below(tmp_path_factory):
    at = tmp_path_factory.mktemp("gelu")
    (at / "gelu.cpp").write_text(
        "#include <cmath>\n#define __device__\n#define __forceinline__ static inline\n"
        "#define __builtin_amdgcn_rcpf(x) ((float)(1.0 / (double)(x)))\n"
        "#define __builtin_amdgcn_exp2f(x) ((float)std::exp2((double)(x)))\n" + body() +
        '\nextern "C" void run(const float* t, float* q, float* e, int n)\n'
        "{ for (int i = 0; i < n; ++i) normal_below(t[i], q + i, e + i); }\n")
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-shared", "-fPIC", str(at / "gelu.cpp"), "-o",
                    str(at / "gelu.so")], check=True)
    lib = ctypes.CDLL(str(at / "gelu.so"))
    q, e = np.empty_like(T), np.empty_like(T)
    p = [v.ctypes.data_as(ctypes.c_void_p) for v in (T, q, e)]
    lib.run(*p, len(T))
    return q.astype(np.float64), e.astype(np.float64)


def test_polynomial():
    """9e-8 of half the scaled complementary error function, as said beside it."""
    lead = re.search(r"float r = ([-\d.e]+)f;", body())[1]
    rest = re.findall(r"r = __builtin_fmaf\(r, s, ([-\d.e]+)f\)", body())
    assert len(rest) == 8
    t = T.astype(np.float64)
    s, r = 1.0 / (1.0 + float(np.float32(0.3)) * t), 0.0
    for c in (lead, *rest):
        r = r * s + float(np.float32(c))
    assert np.abs(r / (0.5 * erfcx(t / math.sqrt(2.0))) - 1.0).max() <= 9e-8


def test_value(normal_below):
    """Roundings of 2^-24 of the value each.  The exponential: its own and the addition that takes
    up what rounding left of its argument (of the second order less than 1 %).  The rest: the fit
    (9e-8, 1.51); the polynomial's eight additions, whose results are together 4.1 times the last one where s
    is 1 and fewer where it is less; the reciprocal and its argument, of which R, about as steep as s,
    takes up at most both; the product."""
    q, e = normal_below
    t = T.astype(np.float64)
    assert np.abs(e / np.exp(-t * t / 2.0) - 1.0).max() <= 2.02 * 2.0 ** -24
    assert np.abs(q / (0.5 * erfc(t / math.sqrt(2.0))) - 1.0).max() <= (2.02 + 1.51 + 4.1 + 2.0 + 1.0) * 2.0 ** -24
