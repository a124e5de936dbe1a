"""The kernels of rotated positions and of windows keep everything in registers: what the compiler reports of each instance."""
import re
import subprocess

import pytest

from paper_2401_09670_amd import build


@pytest.mark.parametrize("source,least", [("attn_window.hip", 2), ("kv_rotary.hip", 18)])
def test_no_instance_uses_scratch(source, least, tmp_path):
    out = subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S",
                          f"{build.CSRC}/{source}", "-o", str(tmp_path / "out.s")], check=True, capture_output=True, text=True)
    used = re.findall(r"Function Name: (\S+)[\s\S]*?ScratchSize \[bytes/lane\]: (\d+)[\s\S]*?VGPRs Spill: (\d+)", out.stderr)
    assert len({name for name, _, _ in used}) >= least
    assert not [u for u in used if u[1:] != ("0", "0")]
