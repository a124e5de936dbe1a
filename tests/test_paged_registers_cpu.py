"""The kernels over pages of 8 bits and in tiles keep everything in registers: what the compiler reports of each instance.  They
are held to as many registers as let 3 or 4 waves share a SIMD, and what does not fit would go through memory in the loop."""
import re
import subprocess

import pytest

from paper_2401_09670_amd import build


@pytest.mark.parametrize("source,least", [("attn_paged.hip", 26), ("kv_quant.hip", 12)])
def test_no_instance_uses_scratch(source, least, tmp_path):
    out = subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S",
                          f"{build.CSRC}/{source}", "-o", str(tmp_path / "out.s")], check=True, capture_output=True, text=True)
    found = re.findall(r"Function Name: (\S+)|ScratchSize \[bytes/lane\]: (\d+)|VGPRs Spill: (\d+)", out.stderr)
    kernels, name = {}, None
    for function, scratch, spilled in found:
        if function:
            name = function
        else:
            kernels.setdefault(name, []).append(int(scratch or spilled))
    assert len(kernels) >= least and all(len(v) == 2 for v in kernels.values())
    assert not {k: v for k, v in kernels.items() if any(v)}
