"""The wait states between a matrix product and the first use of its result, in the attention kernels as they are
built: the hardware does not wait by itself, the compiler counts the states and fills them, and where it is known to
miscount (two ways of different lengths behind a product) the kernels spend them.  No GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_19368_amd import build as BUILD
from paper_2607_19368_amd import slh as B

OBJDUMP = os.path.join(os.path.dirname(os.path.realpath(BUILD.HIPCC)), "..", "llvm", "bin", "llvm-objdump")
SHAPES = {"32x32x16": "k32", "16x16x32": "k16", "16x16x16": "k16h"}

PROBE = """
#include "attend.h"
using namespace slh;
template <class TY> __global__ void k32(const at_u32x4* x, float* y) {
  at_f32x16 c = {};
  c = TY::mfma(x[threadIdx.x], x[threadIdx.x], c);
  y[threadIdx.x] = c[0] * 3.f;
}
template <class TY> __global__ void k16(const at_u32x4* x, float* y) {
  at_f32x4 c = {};
  c = TY::mfma16(x[threadIdx.x], x[threadIdx.x], c);
  y[threadIdx.x] = c[0] * 3.f;
}
template <class TY> __global__ void k16h(const at_u32x2* x, float* y) {
  at_f32x4 c = {};
  c = TY::mfma16k16(x[threadIdx.x], x[threadIdx.x], c);
  y[threadIdx.x] = c[0] * 3.f;
}
__global__ void spent32(float* y) {
  at_f32x16 c[1] = {};
  at_products_done(c);
  y[threadIdx.x] = c[0][0];
}
__global__ void spent16(float* y) {
  at_f32x4 c[1] = {};
  at_products_done(c);
  y[threadIdx.x] = c[0][0];
}
#define ALL(TY) template __global__ void k32<TY>(const at_u32x4*, float*); \\
  template __global__ void k16<TY>(const at_u32x4*, float*); template __global__ void k16h<TY>(const at_u32x2*, float*);
ALL(AtBf16)
ALL(AtF16)
"""


def nops(lines):
    return sum(int(x, 0) + 1 for x in re.findall(r"^\s*s_nop\s+(\w+)", "\n".join(lines), re.M))


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    """Functions of the probe: {name: lines of assembly}."""
    folder = tmp_path_factory.mktemp("waits")
    src, out = folder / "probe.hip", folder / "probe.s"
    src.write_text(PROBE)
    r = subprocess.run([BUILD.HIPCC, *BUILD.FLAGS, "--offload-device-only", "-x", "hip", "-S", str(src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return {m[1]: m[2].split("\n") for m in re.finditer(r"^(_Z\w+):[^\n]*\n(.*?)\.Lfunc_end", out.read_text(), re.S | re.M)}


@pytest.fixture(scope="module")
def needed(probe):
    """States that the compiler fills between a product and an instruction that reads its result."""
    need = {}
    for shape, name in SHAPES.items():
        for f in [f for f in probe if re.search(rf"\d{name}I", f)]:
            at = next(i for i, x in enumerate(probe[f]) if "v_mfma" in x)
            assert shape in probe[f][at]
            end = next(i for i, x in enumerate(probe[f]) if i > at and "v_mul_f32" in x)
            assert all("s_nop" in x or not x.split(";")[0].strip() for x in probe[f][at + 1:end])
            need[shape] = max(need.get(shape, 0), nops(probe[f][at + 1:end]))
    assert set(need) == set(SHAPES) and min(need.values()) > 0
    return need


def test_spent_states_are_those_that_the_products_need(probe, needed):
    for name, shapes in (("spent32", ["32x32x16"]), ("spent16", ["16x16x32", "16x16x16"])):
        body = "\n".join(next(v for f, v in probe.items() if name in f))
        spent = nops("\n".join(re.findall(r"#ASMSTART(.*?)#ASMEND", body, re.S)).split("\n"))
        assert spent >= max(needed[s] for s in shapes), name


# ---------------------------------------------------------------- the built kernels, along every path
def registers(text):
    out = set()
    for m in re.finditer(r"\bv\[(\d+):(\d+)\]", text):
        out |= set(range(int(m[1]), int(m[2]) + 1))
    return out | {int(x) for x in re.findall(r"\bv(\d+)\b", text)}


def early_uses(lines, needed):
    """(products, uses of a product's result before its states have passed) of a function."""
    code, label = [], {}
    for x in lines:
        x = x.split("//")[0].strip()
        m = re.match(r"<(L\d+)>:", x)
        if m:
            label[m[1]] = len(code)
        elif x:
            op, _, rest = x.partition(" ")
            code.append((op, re.split(r",(?![^\[]*\])", rest)))

    def ways(i):
        op, args = code[i]
        if op == "s_endpgm":
            return []
        to = [label[args[0].strip()]] if "branch" in op else []
        return to if op == "s_branch" else to + [i + 1]

    products, early = 0, []
    for i, (op, args) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        products += 1
        need = next(v for k, v in needed.items() if k in op)
        result = registers(args[0])
        best, left = {}, [(j, 0) for j in ways(i)]
        while left:
            j, passed = left.pop()
            if j >= len(code) or passed >= need or best.get(j, need) <= passed:
                continue
            best[j] = passed
            o, a = code[j]
            if o.startswith("v_mfma"):
                # its third source may be the result: products that add up follow each other
                if (registers(a[1]) | registers(a[2])) & result:
                    early.append((i, j, passed, need, o))
                if registers(a[0]) >= result:
                    continue
            elif o.startswith(("v_", "ds_", "global_", "buffer_", "scratch_", "flat_")) and registers(",".join(a)) & result:
                early.append((i, j, passed, need, o))
                continue
            left += [(n, passed + (int(a[0], 0) + 1 if o == "s_nop" else 1)) for n in ways(j)]
    return products, early


def test_no_result_is_used_early(needed, tmp_path):
    lib = shutil.copy(B.LIB_PATH, tmp_path)
    r = subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels = products = 0
    for name in sorted(os.listdir(tmp_path)):
        if not name.endswith(BUILD.ARCH):
            continue
        r = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", "--no-leading-addr", name],
                           cwd=tmp_path, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        for f, body in re.findall(r"^<(_Z\w*k_attend\w*)>:\n(.*?)(?=^<_Z|\Z)", r.stdout, re.S | re.M):
            n, early = early_uses(body.split("\n"), needed)
            assert not early, (f, early[:3])
            kernels += n > 0
            products += n
    assert kernels == 72 and products > 0


def test_paths_are_followed():
    """The walk itself, on listings made up here: a branch, a loop, a wait that is long enough and one that is not."""
    need = {"32x32x16": 12}
    product = "v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]"

    def early(*lines):
        return len(early_uses([product, *lines, "s_endpgm"], need)[1])

    assert early("s_nop 11", "v_add_f32_e32 v30, v3, v4") == 0
    assert early("s_nop 10", "v_add_f32_e32 v30, v3, v4") == 1
    assert early("s_nop 10", "v_add_f32_e32 v30, v31, v32", "v_add_f32_e32 v30, v3, v4") == 0
    assert early("s_cbranch_scc0 L0", "s_nop 11", "<L0>:", "v_add_f32_e32 v30, v3, v4") == 1
    assert early("s_cbranch_scc0 L0", "s_nop 11", "<L0>:", "s_nop 10", "v_add_f32_e32 v30, v3, v4") == 0
    assert early("s_branch L1", "<L0>:", "s_nop 9", "v_mov_b32_e32 v1, 0", "s_endpgm", "<L1>:", "s_cbranch_vccz L0") == 0
    assert early("s_branch L1", "<L0>:", "s_nop 8", "v_mov_b32_e32 v1, 0", "s_endpgm", "<L1>:", "s_cbranch_vccz L0") == 1
    assert early("s_nop 2", product, "s_nop 11", "ds_write_b32 v40, v15") == 0
    assert early("s_nop 2", "v_mfma_f32_32x32x16_bf16 v[30:45], v[12:15], v[24:27], v[30:45]") == 1
    assert early("global_store_dword v40, v15, s[0:1]") == 1
