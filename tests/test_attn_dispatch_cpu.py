"""What calls of the 8-bit cache operators launch, without a GPU: their host code is
linked with launchers that write down what they are asked (tests/c/
attn_dispatch_record.cpp) and called with made-up addresses, which nothing reads."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2403_01876_amd import attn, dv
from tests.test_attn_cpu import FAKE, KEPT, POS, SCALE, TABLE, WEIGHT

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("dispatch") / "libattndispatch.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wall", "-Werror",
                    "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                    os.path.join(ROOT, "paper_2403_01876_amd", "csrc", "dv_attn.cpp"),
                    os.path.join(ROOT, "tests", "c", "attn_dispatch_record.cpp"),
                    "-L", os.path.join(ROCM, "lib"), "-lamdhip64",
                    "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-o", out], check=True, timeout=300)
    lib = ctypes.CDLL(out)
    for name in attn.EXPORTS:
        getattr(lib, name).argtypes = getattr(attn.lib, name).argtypes
    lib.dispatch_record_take.restype = ctypes.c_char_p
    return lib


def taken(lib):
    return [(ln.split()[0], {k: int(v) for k, v in (f.split("=") for f in ln.split()[1:])})
            for ln in lib.dispatch_record_take().decode().splitlines()]


def paged(H, B, cap, bs=16, D=16):
    """A cache whose sequences may share or lack most of their blocks."""
    c = dv.Cache(dv.DV_PAGED, 1, H, D, B, [FAKE], elem_bytes=1, block_size=bs, num_blocks=64,
                 max_blocks=-(-cap // bs), block_tables=[TABLE])
    far = 1 << 48  # (the companions of so many heads are large)
    return attn.QuantCache(c, [SCALE], scale_block=bs, weights=[WEIGHT + far],
                           positions=[POS + 2 * far])


@pytest.mark.parametrize("H,B,length", [(1 << 15, 192, 5000), (1 << 15, 192, 4096), (1 << 16, 70, 9000),
                                        (1 << 20, 5, 4097), (40, 450, 6000)])
def test_evict_launches_stay_within_a_grid(lib, H, B, length):
    """Lanes of a launch are counted in 32 bits; every sequence is selected and moved."""
    c = paged(H, B, length)
    n, keep = np.full(B, length, np.int32), np.ones(B, np.int32)
    kept = KEPT + (1 << 52)
    assert lib.dv_evict(c.ref, 0, c.ref, 0, 0, 1, n.ctypes.data, keep.ctypes.data, 0, kept, 1,
                        None) == 0
    ran = taken(lib)
    for name in ("select", "move"):
        at = [f for k, f in ran if k == name]
        assert [f["b0"] for f in at] == list(np.cumsum([0] + [f["nseq"] for f in at[:-1]]))
        assert sum(f["nseq"] for f in at) == B
    for k, f in ran:
        if k == "select":
            assert f["nseq"] * f["heads"] * (1024 if f["most"] > 4096 else 256) < 1 << 32
        else:
            assert f["items"] * 256 < 1 << 32
