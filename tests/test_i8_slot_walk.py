"""CPU: the waves of the slot-by-slot down product of wc_experts_i8 take every block of
every slot that has an expert once, wherever a token's empty slots lie."""
import os
import subprocess

import pytest

from paper_2606_15789_amd import build


def test_every_block_once(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    here = os.path.dirname(os.path.abspath(__file__))
    program = tmp_path / "walk"
    flags = [f for f in build.FLAGS if f not in ("-shared", "-lpthread")]
    subprocess.run([build.HIPCC, *flags, "-I", build.CSRC, os.path.join(here, "i8_slot_walk_driver.hip"),
                    "-o", str(program)],
                   check=True, capture_output=True, text=True, timeout=600)
    out = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.endswith(" 0 wrong\n"), out.stdout
