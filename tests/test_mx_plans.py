"""CPU: which kernels the microscaled layers' calls run, by their sizes alone: the rules of
the library's sources, compiled for the host."""
import os
import subprocess

import pytest

from mx_plans import PLANS
from paper_2606_15789_amd import build, wc

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


def test_every_kernel_of_a_product(tmp_path):
    calls = [(m, k, n, wc.mx_row_bytes(k), wc.mx_blocks(k)) for (m, k, n), _ in PLANS]
    assert _answers(tmp_path, "mx_plan_driver", calls) == [plan for _, plan in PLANS]
    seen = {tuple(plan.split()[:2]) for _, plan in PLANS}
    assert seen >= {(tile, parts) for tile in ("tile64", "tile128", "tile128deep", "tile256") for parts in "1248"}


def test_rows_far_apart(tmp_path):
    """Rows that tiles' offsets do not reach go without tiles, or without streams."""
    far, further = (1 << 22) + 16, (1 << 27) + 16
    got = _answers(tmp_path, "mx_plan_driver", [
        (300, 4096, 4096, 2048, 128), (300, 4096, 4096, far, 128), (300, 4096, 4096, 2048, far),
        (5, 4096, 4096, far, far), (5, 4096, 4096, further, 128), (5, 4096, 4096, 2048, further),
        ((1 << 24) - 1, 64, 64, 32, 2), (1 << 24, 64, 64, 32, 2)])
    kinds = [g[:4] for g in got]
    assert kinds == ["tile", "slim", "slim", "stre", "slim", "slim", "tile", "slim"]
