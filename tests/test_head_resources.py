"""What the compiler gives the kernels of a model's output end for gfx950: none keeps anything of a lane in scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2507_11941_amd import build


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_no_scratch(tmp_path):
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    jobs = [subprocess.Popen(["/opt/rocm/bin/hipcc", *flags, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", "-o",
                              str(tmp_path / (os.path.basename(source) + ".o")), source], stderr=subprocess.PIPE, text=True)
            for source in build.HEAD_SOURCES]
    for job in jobs:
        said = job.communicate()[1]
        assert job.returncode == 0, said[-2000:]
        found = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", said, flags=re.S)
        assert len(found) > 10
        assert not [name for name, scratch in found if int(scratch)]
