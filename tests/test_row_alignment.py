"""The norm's and the sampling's kernels as the compiler makes them (CPU only): rows begin
at any element, so no access of several elements is taken for aligned to more than one of them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2408_05235_amd import build

needs_hipcc = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                 reason="no hipcc")
ACCESS = re.compile(r"\b(load|store) <(\d+) x (\w+)>.*ptr addrspace\(1\).*, align (\d+)")


@needs_hipcc
@pytest.mark.parametrize("name", ["norm.hip", "sample.hip"])
def test_accesses(tmp_path, name):
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = str(tmp_path / "out.ll")
    cmd = [build.hipcc(), *flags, "--cuda-device-only", "-S", "-emit-llvm", "-I", build.INCLUDE, "-I", build.CSRC, "-x",
           "hip", os.path.join(build.CSRC, name), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    kernel, seen = None, 0
    for line in open(out):
        if line.startswith("define"):
            kernel = re.search(r"kernelILi(\d)", line)      # (its type: TL_BF16 1, TL_F16 2, TL_F32 3)
        access = ACCESS.search(line)
        if not access or not kernel:
            continue
        # 16 bytes are elements of that type, 8 bytes are elements in 8 bits
        size = int(access[2]) * {"i32": 4, "float": 4, "i16": 2, "half": 2, "bfloat": 2}[access[3]]
        element = {16: 4 if kernel[1] == "3" else 2, 8: 1}[size]
        seen += 1
        assert int(access[4]) <= element, line
    assert seen > 50
