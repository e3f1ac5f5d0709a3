"""What the compiler needs for the kernels of pages, adapters and filtered draws: nothing of a lane's goes to scratch memory, and the adapters of the
largest ranks, whose waves stage 18 KB each, fit a unit."""
import os
import re
import subprocess

import pytest

from paper_2510_25739_amd import build


@pytest.mark.parametrize("source,least", [("adapters.hip", 37), ("filtered.hip", 12), ("pages.hip", 5)])
def test_nothing_is_kept_in_scratch_memory(tmp_path, source, least):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    cmd = [build.HIPCC, *build.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(build.CSRC, source), "-o", str(tmp_path / "k.o")]
    report = subprocess.run(cmd, capture_output=True, text=True, check=True).stderr
    use = {name: [int(re.search(k + r": (\d+)", text).group(1)) for k in (r"VGPRs Spill", r"ScratchSize \[bytes/lane\]", r"LDS Size \[bytes/block\]")]
           for name, text in re.findall(r"Function Name: (\S+)(.*?LDS Size \[bytes/block\]: \d+)", report, flags=re.S)}
    assert len(use) >= least
    assert {k: v for k, v in use.items() if v[0] or v[1] or v[2] > 160 * 1024} == {}
