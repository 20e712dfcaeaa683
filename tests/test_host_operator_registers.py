"""The operators' kernels keep their registers: what the compiler cannot hold goes to scratch memory, a round trip each way, without a word. Each
kernel's scratch per lane by the compiler's own resource remarks, with the flags that the library is built with."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2304_14698_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="no HIP compiler")
@pytest.mark.parametrize("file,at_least", [("op_embedding.hip", 20), ("op_token_logp.hip", 15), ("op_muon.hip", 12)])
def test_no_kernel_spills(tmp_path, file, at_least):
    run = subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                          "-mllvm", "-amdgpu-mfma-vgpr-form", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-x", "hip", "--cuda-device-only", "-S",
                          "-Rpass-analysis=kernel-resource-usage", "-o", str(tmp_path / "out.s"), os.path.join(CSRC, file)],
                         capture_output=True, text=True)
    assert run.returncode == 0, run.stderr[-2000:]
    scratch = dict(zip(re.findall(r"Function Name: (\S+)", run.stderr), map(int, re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", run.stderr))))
    assert len(scratch) >= at_least
    assert not {k: v for k, v in scratch.items() if v}
