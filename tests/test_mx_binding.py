"""CPU: the binding of the microscaled layers: its first call from two threads at once, and refusals."""
import sys

import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")


def test_first_calls_of_two_threads(monkeypatch):
    """A call that begins while another one fills the tables of element types, after any line of it,
    takes valid tensors for what they are (refused here for lying in host memory alone)."""
    q = torch.zeros((4, 32), dtype=torch.uint8)
    scale = torch.zeros((4, 2), dtype=torch.uint8)
    lines = 0

    def call():
        with pytest.raises(ValueError, match="on a device"):
            wc.dequantize_mx_torch(q, scale, 64)

    def first_call(at):
        nonlocal lines
        lines = 0

        def trace(frame, event, arg):
            nonlocal lines
            if frame.f_code is not wc._mx_types.__code__:
                return None
            if event == "line":
                lines += 1
                if lines == at:
                    call()  # what another thread does here
            return trace
        for name in [n for n in vars(wc) if n.startswith("_bytes_of_")]:
            monkeypatch.setattr(wc, name, ())
        before = sys.gettrace()
        sys.settrace(trace)
        try:
            wc._mx_types()
        finally:
            sys.settrace(before)
        call()
    first_call(0)
    assert lines >= 4
    for at in range(1, lines + 1):
        first_call(at)
