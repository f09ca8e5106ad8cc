"""CPU: which kernels the microscaled layers' calls run, by their sizes alone: the rules of
the library's sources, compiled for the host."""
import os
import subprocess

import pytest

from paper_2606_15789_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def _answers(tmp_path, driver, calls):
    """The driver's answer to each call."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    build.ensure_built()
    program = str(tmp_path / driver)
    flags = [f for f in build.FLAGS if f not in ("-shared", "-lpthread", "-O3", "-Wall")]
    where = os.path.dirname(build.LIB)
    for cmd in ([build.HIPCC, *flags, "-w", "--offload-host-only", "-I", build.CSRC, "-c",
                 os.path.join(HERE, driver + ".hip"), "-o", program + ".o"],
                # the kernels themselves are left out
                [build.HIPCC, program + ".o", "-o", program, "-L", where, "-lwc",
                 "-Wl,--unresolved-symbols=ignore-all", f"-Wl,-rpath,{where}"]):
        res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
        assert res.returncode == 0, res.stderr
    text = "\n".join(" ".join(str(v) for v in c) for c in calls) + "\n"
    out = subprocess.run([program], input=text, capture_output=True, text=True, timeout=60)
    assert out.returncode == 0
    answers = out.stdout.split("\n")[:-1]
    assert len(answers) == len(calls)
    return answers


# (tokens, k, experts, hidden, ffn): places to a block, 0 for the two kernels of few tokens
PLACES = [((1, 2, 8, 8192, 64), 0), ((16, 32, 40, 4096, 64), 0), ((1, 2, 8, 8193, 64), 16),
          ((2, 2, 8, 8193, 64), 16), ((16, 2, 8, 65536, 64), 16), ((7, 33, 40, 96, 64), 16),
          ((17, 2, 8, 8193, 64), 64), ((17, 2, 8, 96, 64), 64), ((200, 2, 8, 96, 64), 128),
          ((1000, 2, 8, 96, 64), 256),
          # codes of x past 2^31 bytes
          ((65536, 1, 2, 65536, 33), 16), ((65535, 1, 2, 65536, 33), 256)]


def test_places_of_experts(tmp_path):
    """The kernels go by the sizes' orders: one token's are not others than two tokens'."""
    got = _answers(tmp_path, "mx_places_driver", [c for c, _ in PLACES])
    assert [int(v) for v in got] == [p for _, p in PLACES]
