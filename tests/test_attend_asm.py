"""The attention's kernels as the compiler makes them (CPU only, gfx950 code
from hipcc): the copies to LDS set M0 in inline assembly and nothing else uses
it; the main loop's operands are read ahead of their matrix instructions; no
kernel keeps registers in memory."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2408_05235_amd import build
from test_kernel_resources import _resources

IMPLICIT_M0 = re.compile(r"^\s*(s_sendmsg\w*|s_movrel\w*|v_movrel\w*|s_set_gpr_idx\w*|ds_gws\w*|v_interp\w*)\b")
INSTR = re.compile(r"^\s+[a-z_][a-z0-9_]*(\s|$)")

needs_hipcc = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                 reason="no hipcc")


def _device_asm(tmp_path, name):
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = str(tmp_path / "out.s")
    cmd = [build.hipcc(), *flags, "--cuda-device-only", "-S", "-I", build.INCLUDE, "-I", build.CSRC, "-x", "hip",
           os.path.join(build.CSRC, name), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    return open(out).read().splitlines()


@needs_hipcc
def test_tiles_in_assembly(tmp_path):
    lines = _device_asm(tmp_path, "attend_tiles.hip")
    instrs = [ln.split(";")[0].rstrip() for ln in lines if INSTR.match(ln) and not ln.lstrip().startswith(".")]
    writes = 0
    for i, ins in enumerate(instrs):
        assert not IMPLICIT_M0.match(ins), f"{ins.strip()} reads M0"
        if re.search(r"\bm0\b", ins):
            assert re.fullmatch(r"\s*s_mov_b32 m0, s\d+", ins), f"unexpected use of M0: {ins.strip()}"
            assert instrs[i + 1].split()[0] in ("global_load_lds_dwordx4", "global_load_lds_dword"), instrs[i + 1]
            writes += 1
    assert writes > 0
    # a read that its matrix instruction waits for at once would be
    # `ds_read; s_waitcnt lgkmcnt(0); v_mfma_f32_32x32`: only the last ones may be
    at_once = sum(a.split()[0].startswith("ds_read") and "lgkmcnt(0)" in b and c.split()[0].startswith("v_mfma_f32_32x32")
                  for a, b, c in zip(instrs, instrs[1:], instrs[2:]))
    matrix = sum(ins.split()[0].startswith("v_mfma_f32_32x32") for ins in instrs)
    assert matrix > 300 and at_once <= matrix // 32, (at_once, matrix)


@needs_hipcc
@pytest.mark.parametrize("name", ["attend.hip", "attend_tiles.hip", "pages.hip"])
def test_no_registers_in_memory(tmp_path, name):
    kernels = _resources(tmp_path, name)
    assert len(kernels) >= 8
    for k, r in kernels.items():
        assert r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (k, r)
