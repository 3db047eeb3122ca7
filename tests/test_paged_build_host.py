"""No attention kernel keeps registers in memory.  The compiler has been seen to lose one
register of a 128-bit operand that it had put partly into accumulation registers and
partly into memory; the kernels are sized so that it never has to."""
import os
import re
import subprocess
import tempfile

from paper_2603_08739_amd import build as B


def test_attention_kernels_spill_no_vector_registers():
    with tempfile.TemporaryDirectory() as d:
        cmd = [B.HIPCC, *B.FLAGS, "--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
               os.path.join(B.CSRC, "k_attn.hip"), "-o", os.path.join(d, "k.o")]
        r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    spills = [int(x) for x in re.findall(r"VGPRs Spill: (\d+)", r.stderr)]
    assert len(names) == len(spills) and sum("k_attn" in n for n in names) >= 26
    assert [n for n, s in zip(names, spills) if s] == []
