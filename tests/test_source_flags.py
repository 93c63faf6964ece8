"""Sources that are compiled with flags of their own, as they are built: they wait for
their matrix products, and keep everything in registers."""
import os
import re
import subprocess

import pytest

from paper_2607_04181_amd import build as B
from test_mfma_waits import early_reads, hipcc


@hipcc
@pytest.mark.parametrize("source", sorted(B.SOURCE_FLAGS))
def test_a_source_with_flags_of_its_own(source, tmp_path):
    out = tmp_path / (source + ".s")
    subprocess.run([B.HIPCC, *B.flags_of(source), "--cuda-device-only", "-S",
                    os.path.join(B.CSRC, source), "-o", str(out)], check=True,
                   stderr=subprocess.DEVNULL)
    text = out.read_text()
    n, bad = early_reads(text)
    assert n > 0 and not bad, bad[:5]
    spilled = re.findall(r"\.vgpr_spill_count:\s*(\d+)", text)
    assert spilled and set(spilled) == {"0"}
