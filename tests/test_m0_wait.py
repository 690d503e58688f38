"""The wait state between a write of M0 and the copy to LDS that reads it, in
the machine code (CPU only, gfx950 code from hipcc).

A scalar write of M0 needs one wait state before a load to LDS that reads it.
The compiler puts an instruction between its own such pairs, but nothing into
inline assembly, where the kernels write theirs.
"""
import os
import shutil
import subprocess

import pytest

from paper_2408_05235_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.mark.skipif((shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"))
                    or not os.path.exists(OBJDUMP), reason="no hipcc or no llvm-objdump")
@pytest.mark.parametrize("name", ["attend_tiles.hip", "forest.hip", "column.hip"])
def test_a_wait_state_between_m0_and_the_copy(tmp_path, name):
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    obj = str(tmp_path / "out.o")
    cmd = [build.hipcc(), *flags, "--cuda-device-only", "--no-gpu-bundle-output", "-c", "-I", build.INCLUDE, "-I",
           build.CSRC, "-x", "hip", os.path.join(build.CSRC, name), "-o", obj]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    lines = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", obj], check=True, capture_output=True,
                           text=True).stdout.splitlines()
    instrs = [ln.split("//")[0].split() for ln in lines if ln.startswith("\t")]
    copies = 0
    for i, ins in enumerate(instrs):
        if ins and ins[0].startswith("global_load_lds"):
            assert "m0," not in instrs[i - 1], f"{name}: {' '.join(instrs[i - 1])} directly before {' '.join(ins)}"
            copies += 1
    assert copies > 0
