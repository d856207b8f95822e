"""A step of the rounding to 4 bits, compiled for the host without contraction:
its result must not depend on what the compiler fuses by itself."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from paper_2006_12645_amd import build as B  # noqa: E402

from test_kernel_resources_cpu import _have_hipcc  # noqa: E402

pytestmark = pytest.mark.skipif(not _have_hipcc(), reason="hipcc not available")


@pytest.fixture(scope="module")
def offset(tmp_path_factory):
    at = tmp_path_factory.mktemp("rounding")
    src, lib = at / "offset.hip", at / "liboffset.so"
    src.write_text('#include "decode/gba_q4_cache.hpp"\nextern "C" float offset(float low, float scale) { return gba::q4_offset(low, scale); }\n')
    r = subprocess.run([B._hipcc(), "--offload-host-only", "-O3", "-std=c++17", "-ffp-contract=off", "-fPIC", "-shared", "-I", B.INCLUDE, "-I", B.CSRC,
                        str(src), "-o", str(lib)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    f = ctypes.CDLL(os.fspath(lib)).offset
    f.argtypes, f.restype = [ctypes.c_float] * 2, ctypes.c_float
    return f


@pytest.mark.parametrize("low,high", [(-1.0, 1.0), (-3.0, 2.5), (0.1, 0.7), (-1e-30, 4e-30), (-3e38, 3e38), (-float(torch.finfo(torch.bfloat16).max),
                                      float(torch.finfo(torch.bfloat16).max))])
def test_offsets_are_rounded_once(offset, low, high):
    low, high = (torch.tensor(v).bfloat16().double() for v in (low, high))
    scale = ((high / 2 - low / 2).float() * torch.tensor(2 / 15, dtype=torch.float64).float()).bfloat16().double()
    want = (low + 8 * scale).float()  # (exact in 64 bits: two numbers of 8 bits that are less than 2^44 apart)
    assert want.isfinite() and offset(float(low), float(scale)) == float(want)
