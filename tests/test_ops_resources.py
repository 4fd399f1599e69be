"""What the compiler gives the kernels of the operators for gfx950: none keeps anything of a lane in scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2507_11941_amd import build


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_no_scratch(tmp_path):
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    for source in build.OPERATOR_SOURCES:
        done = subprocess.run(["/opt/rocm/bin/hipcc", *flags, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", "-o",
                               str(tmp_path / "ops.o"), source], capture_output=True, text=True)
        assert done.returncode == 0, done.stderr[-2000:]
        found = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", done.stderr, flags=re.S)
        assert len(found) > 20
        assert not [name for name, scratch in found if int(scratch)]
