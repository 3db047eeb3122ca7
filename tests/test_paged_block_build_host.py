"""No kernel of the caches with scales by block keeps registers in memory: the compiler has been
seen to lose one of a 128-bit operand that it had put partly there."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2603_08739_amd import build as B


@pytest.mark.parametrize("source, kernels", [("k_attn_block.hip", 36), ("k_block.hip", 28)])
def test_no_vector_register_is_spilled(source, kernels):
    with tempfile.TemporaryDirectory() as d:
        cmd = [B.HIPCC, *B.FLAGS, "--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
               os.path.join(B.CSRC, source), "-o", os.path.join(d, "k.o")]
        r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    spills = [int(x) for x in re.findall(r"VGPRs Spill: (\d+)", r.stderr)]
    scratch = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    assert len(names) == len(spills) == len(scratch) == kernels
    assert [n for n, s, m in zip(names, spills, scratch) if s or m] == []
