"""CPU check of what the compiler gives the kernels of the 8-bit integer layers: nothing
of theirs lies in scratch memory.  Their tiles hold up to 256 rows' sums in registers; a
spill among them costs a trip to memory a stage, and no output shows it."""
import os
import re
import subprocess

import pytest

from paper_2606_15789_amd import build


@pytest.mark.parametrize("source", ["wc_i8.hip", "wc_experts.hip", "wc_route.hip"])
def test_nothing_in_scratch(source, tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    asm = tmp_path / "kernels.s"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-lpthread")]
    subprocess.run([build.HIPCC, *flags, "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, source), "-o", str(asm)],
                   check=True, capture_output=True, text=True, timeout=600)
    kernels = re.findall(r"^    \.name: +(\S*wc_\w*)\n(.*?)\.wavefront_size:", asm.read_text(),
                         re.M | re.S)
    assert kernels
    for name, meta in kernels:
        fields = dict(re.findall(r"\.(\w+): +(\d+)", meta))
        got = {k: int(fields[k]) for k in ("private_segment_fixed_size", "vgpr_spill_count")}
        assert not any(got.values()), (name, got)
