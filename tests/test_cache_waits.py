"""The wait states between a matrix product and the first use of its result, in the built kernels of 8-bit attention and of
attention weights (as in test_matrix_waits.py).  No GPU."""
import os
import re
import shutil
import subprocess

from paper_2607_19368_amd import build as BUILD
from paper_2607_19368_amd import slh as B
from test_matrix_waits import OBJDUMP, early_uses, needed, probe  # noqa: F401


def test_no_result_is_used_early(needed, tmp_path):  # noqa: F811
    lib = shutil.copy(B.LIB_PATH, tmp_path)
    r = subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels = {}
    for name in sorted(os.listdir(tmp_path)):
        if not name.endswith(BUILD.ARCH):
            continue
        r = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", "--no-leading-addr", name],
                           cwd=tmp_path, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        for f, kind, body in re.findall(r"^<(_Z\w*\d(k_rows8|k_tiles8|k_both8|k_weights|k_weights_tiles)I\w*)>:\n(.*?)(?=^<_Z|\Z)", r.stdout, re.S | re.M):
            n, early = early_uses(body.split("\n"), needed)
            assert not early, (f, early[:3])
            kernels[kind] = kernels.get(kind, 0) + (n > 0)
    # types, head sizes, and rows of a block or kinds of cache
    assert kernels == {"k_rows8": 16, "k_tiles8": 8, "k_both8": 16, "k_weights": 16, "k_weights_tiles": 16}
