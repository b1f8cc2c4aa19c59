"""What the attention entry points would launch (attend_api.cpp against attend_stub.cpp), without a GPU."""
import ctypes
import os
import subprocess

from paper_2607_19368_amd import build as BUILD
from paper_2607_19368_amd import slh as B

_P = 4096                                         # an aligned address that nothing reads


def build(folder):
    out = os.path.join(str(folder), "libattendstub.so")
    cmd = [BUILD.HIPCC, "--offload-host-only", "-x", "hip", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-w",
           "-I", os.path.join(BUILD.ROOT, "include"), "-I", BUILD.CSRC, os.path.join(BUILD.CSRC, "attend_api.cpp"),
           os.path.join(BUILD.ROOT, "tests", "attend_stub.cpp"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return Planner(out)


class Planner:
    """packed() and paged() give a call's launches, as tuples (kernel, paged, rows of a block, blocks, splits of the
    own keys, row tiles of the prefix, its splits, chain); of a join (its name, 0, partial results of a row, rows)."""

    def __init__(self, path):
        self.lib = ctypes.CDLL(path)
        self.lib.stub_log.restype = ctypes.c_char_p
        real = B.load()
        for name in ("slh_attend", "slh_attend_workspace", "slh_attend_paged", "slh_attend_paged_workspace"):
            f = getattr(self.lib, name)
            f.restype, f.argtypes = getattr(real, name).restype, getattr(real, name).argtypes

    def _log(self, rc):
        out = [tuple(x if i == 0 else int(x) for i, x in enumerate(t.split())) for t in self.lib.stub_log().decode().splitlines()]
        self.lib.stub_clear()
        assert rc == B.SLH_OK, rc
        return [t[:4] if t[0] == "join" else t for t in out]

    def packed(self, Tq, Tk, n, Hq, Hkv, d, causal=True, dtype=B.SLH_BF16):
        need = self.lib.slh_attend_workspace(Tq, Tk, n, Hq, Hkv, d, causal)
        assert need >= 0, need
        return self._log(self.lib.slh_attend(_P, Hq * d, d, _P, Hkv * d, d, _P, Hkv * d, d, dtype, Tq, Tk, n, Hq, Hkv, d, _P, _P,
                                             0.1, causal, _P, Hq * d, d, None, _P, need, None))

    def paged(self, n, n_q, Hq, Hkv, d, page, pages, prefix, dtype=B.SLH_BF16):
        """pages: the width of the page table."""
        need = self.lib.slh_attend_paged_workspace(n, n_q, Hq, Hkv, d, pages * page, prefix)
        assert need >= 0, need
        return self._log(self.lib.slh_attend_paged(_P, Hq * d, d, _P, _P, dtype, 8, page, n, n_q, Hq, Hkv, d, _P, pages, pages, _P,
                                                   _P, prefix, 0.1, _P, Hq * d, d, None, _P, need, None))
