"""What slh_attend_paged_e4m3 would launch (attend8_api.cpp against cache_stub.cpp), without a GPU."""
import ctypes
import os
import subprocess

from paper_2607_19368_amd import build as BUILD
from paper_2607_19368_amd import slh as B

_P = 4096                                         # an aligned address that nothing reads


def build(folder):
    out = os.path.join(str(folder), "libcachestub.so")
    cmd = [BUILD.HIPCC, "--offload-host-only", "-x", "hip", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-w",
           "-I", os.path.join(BUILD.ROOT, "include"), "-I", BUILD.CSRC, os.path.join(BUILD.CSRC, "attend8_api.cpp"),
           os.path.join(BUILD.ROOT, "tests", "cache_stub.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return Planner(out)


class Planner:
    """paged() gives a call's launches, as tuples (kernel, rows of a block, blocks, splits of the own keys, row tiles of the
    prefix, its splits, chain); of a join (its name, partial results of a row, rows)."""

    def __init__(self, path):
        self.lib = ctypes.CDLL(path)
        self.lib.stub_log.restype = ctypes.c_char_p
        real = B.load()
        for name in ("slh_attend_paged_e4m3", "slh_attend_paged_e4m3_workspace"):
            f = getattr(self.lib, name)
            f.restype, f.argtypes = getattr(real, name).restype, getattr(real, name).argtypes

    def paged(self, n, n_q, Hq, Hkv, d, page, pages, prefix, block=16, dtype=B.SLH_BF16):
        """pages: the width of the page table."""
        need = self.lib.slh_attend_paged_e4m3_workspace(n, n_q, Hq, Hkv, d, pages * page, prefix)
        assert need >= 0, need
        rc = self.lib.slh_attend_paged_e4m3(_P, Hq * d, d, _P, _P, _P, _P, dtype, 8, page, block, n, n_q, Hq, Hkv, d, _P, pages, pages,
                                            _P, _P, prefix, 0.1, _P, Hq * d, d, None, _P, need, None)
        out = [tuple(x if i == 0 else int(x) for i, x in enumerate(t.split())) for t in self.lib.stub_log().decode().splitlines()]
        self.lib.stub_clear()
        assert rc == B.SLH_OK, rc
        return [t[:3] if t[0] == "join" else t for t in out]
