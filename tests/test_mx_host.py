"""CPU: what the microscaled layers' entry points refuse before anything is launched, and the
workspace they ask for.  Pointers are made up and never followed."""
import ctypes as C
import math

import pytest

from paper_2606_15789_amd import wc

EINVAL = -1
A = 1 << 20  # an aligned address that is never read


def _job(**more):
    f = dict(w=A, scale=A + 1, bias=None, y=A, ldw=32, lds=2, ldy=8, n=8, bias_dtype=0, y_dtype=1)
    f.update(more)
    return wc._MxJob(**f)


def _jobs(*jobs):
    return (wc._MxJob * max(1, len(jobs)))(*jobs)


def test_sizes():
    assert [wc.mx_blocks(k) for k in (1, 32, 33, 64, 65536)] == [1, 1, 2, 2, 2048]
    assert [wc.mx_row_bytes(k) for k in (1, 32, 33, 64, 65536)] == [16, 16, 32, 32, 32768]
    assert C.sizeof(wc._MxJob) == wc._MX_JOB.size == 72
    assert C.sizeof(wc._MxExperts) == 32


def test_quantize_refusals():
    ok = [A, 1, 4, 64, 64, A, 32, A + 1, 2, None]
    bad = ((0, None), (0, A + 1), (1, 3), (1, 0), (3, 0), (3, 65537), (4, 63), (4, 1 << 31),
           (5, None), (5, A + 8), (6, 16), (6, 40), (6, 1 << 31), (7, None), (8, 1), (8, 1 << 31), (2, 1 << 31))
    for at, v in bad:
        args = list(ok)
        args[at] = v
        assert wc.lib().wc_quantize_mx(*args) == EINVAL, (at, v)
    assert wc.lib().wc_quantize_mx(None, 1, 0, 64, 64, None, 0, None, 0, None) == 0  # no rows


def test_dequantize_refusals():
    ok = [A, 32, A + 1, 2, 4, 64, A, 1, 64, None]
    for at, v in ((0, None), (0, A + 8), (1, 16), (1, 40), (2, None), (3, 1), (4, 1 << 31), (5, 0),
                  (5, 65537), (6, None), (6, A + 1), (7, 3), (8, 63), (8, 1 << 31)):
        args = list(ok)
        args[at] = v
        assert wc.lib().wc_dequantize_mx(*args) == EINVAL, (at, v)
    assert wc.lib().wc_dequantize_mx(None, 0, None, 0, 0, 64, None, 1, 64, None) == 0


@pytest.mark.parametrize("bad", [
    dict(w=None), dict(w=A + 8), dict(scale=None), dict(y=None), dict(n=0), dict(n=1 << 27), dict(ldw=16),
    dict(ldw=40), dict(ldw=1 << 31), dict(lds=1), dict(lds=1 << 31), dict(ldy=7), dict(ldy=1 << 31),
    dict(y_dtype=5), dict(y_dtype=0), dict(bias=A, bias_dtype=0), dict(y=A + 1),
    dict(bias=A + 2, bias_dtype=8), dict(y=A + 2, y_dtype=8)])
def test_job_refusals(bad):
    L = wc.lib()
    need = C.c_uint64(7)
    jobs = _jobs(_job(), _job(**bad))
    assert L.wc_linear_mx_workspace_bytes(4, 64, 2, jobs, C.byref(need)) == EINVAL
    assert need.value == 0
    assert L.wc_matmul_mx_workspace_bytes(4, 64, 2, jobs, C.byref(need)) == EINVAL
    assert L.wc_matmul_mx(A, 32, A, 2, 4, 64, 2, jobs, A, 1 << 30, None) == EINVAL
    assert L.wc_linear_mx(A, 1, 4, 64, 64, 2, jobs, A, 1 << 30, None) == EINVAL


def test_linear_refusals():
    L = wc.lib()
    need = C.c_uint64(0)
    jobs = _jobs(_job())
    # a few rows are quantised by the product's own kernel, more in the workspace
    assert L.wc_linear_mx_workspace_bytes(16, 64, 1, jobs, C.byref(need)) == 0
    assert need.value == 0
    assert L.wc_linear_mx_workspace_bytes(100, 64, 1, jobs, C.byref(need)) == 0
    assert need.value >= 100 * (wc.mx_row_bytes(64) + 2) and need.value % 256 == 0
    n = need.value
    for args in ((4, 64, 0, jobs), (4, 64, 33, jobs), (4, 0, 1, jobs), (4, 65537, 1, jobs),
                 (1 << 31, 64, 1, jobs), (4, 64, 1, None)):
        assert L.wc_linear_mx_workspace_bytes(*args, C.byref(need)) == EINVAL
    assert L.wc_linear_mx_workspace_bytes(4, 64, 1, jobs, None) == EINVAL
    for x, dt, ldx, ws, size in ((None, 1, 64, A, n), (A + 1, 1, 64, A, n), (A, 4, 64, A, n),
                                 (A, 1, 63, A, n), (A, 1, 64, None, n), (A, 1, 64, A + 16, n),
                                 (A, 1, 64, A, n - 1)):
        assert L.wc_linear_mx(x, dt, 100, 64, ldx, 1, jobs, ws, size, None) == EINVAL
    for q, ldq, s, lds in ((None, 32, A, 2), (A + 8, 32, A, 2), (A, 16, A, 2), (A, 40, A, 2), (A, 32, None, 2),
                           (A, 32, A, 1)):
        assert L.wc_matmul_mx(q, ldq, s, lds, 4, 64, 1, jobs, A, 1 << 30, None) == EINVAL
    # together 2^27 rows
    many = _jobs(*[_job(n=1 << 26, ldy=1 << 26)] * 2)
    assert L.wc_linear_mx_workspace_bytes(4, 64, 2, many, C.byref(need)) == EINVAL
    none = _jobs(_job(y=None))
    assert L.wc_matmul_mx(None, 0, None, 0, 0, 64, 1, none, None, 0, None) == 0
    assert L.wc_linear_mx(None, 1, 0, 64, 64, 1, none, None, 0, None) == 0


def _bank(n, k, **more):
    f = dict(w=A, scale=A + 1, stride=n * wc.mx_row_bytes(k), scale_stride=n * wc.mx_blocks(k))
    f.update(more)
    return C.byref(wc._MxExperts(**f))


def test_experts_refusals():
    L = wc.lib()
    need = C.c_uint64(0)
    T, k, E, H, F = 40, 2, 8, 96, 160
    assert L.wc_experts_mx_workspace_bytes(T, k, E, H, F, C.byref(need)) == 0
    size = need.value
    assert size >= T * k * (wc.mx_row_bytes(F) + H * 4) and size % 256 == 0
    for sizes in ((T, 0, E, H, F), (T, 9, E, H, F), (T, k, 0, H, F), (T, k, 513, H, F), (T, k, E, 0, F),
                  (T, k, E, 65537, F), (T, k, E, H, 0), (T, k, E, H, 65537), (1 << 23, 2, E, H, F)):
        assert L.wc_experts_mx_workspace_bytes(*sizes, C.byref(need)) == EINVAL
    assert L.wc_experts_mx_workspace_bytes(T, k, E, H, F, None) == EINVAL

    def call(T=T, **more):
        f = dict(x=A, dt=1, ldx=H, ids=A, weights=A, offsets=A, order=A, gate=_bank(F, H), up=_bank(F, H),
                 down=_bank(H, F), y=A, ldy=H, ws=A, size=size)
        f.update(more)
        return L.wc_experts_mx(f["x"], f["dt"], T, f["ldx"], k, E, H, F, f["ids"], f["weights"], f["offsets"],
                               f["order"], f["gate"], f["up"], f["down"], f["y"], f["ldy"], f["ws"], f["size"],
                               None)
    for bad in (dict(x=None), dict(x=A + 1), dict(dt=3), dict(ldx=H - 1), dict(ldx=1 << 31), dict(ids=None),
                dict(ids=A + 2), dict(weights=None), dict(weights=A + 1), dict(offsets=None),
                dict(offsets=A + 2), dict(order=None), dict(order=A + 1), dict(gate=None), dict(up=None),
                dict(down=None), dict(gate=_bank(F, H, w=None)), dict(gate=_bank(F, H, w=A + 8)),
                dict(up=_bank(F, H, scale=None)), dict(down=_bank(H, F, stride=H * 80 - 16)),
                dict(down=_bank(H, F, stride=H * 80 + 8)), dict(gate=_bank(F, H, scale_stride=F * 3 - 1)),
                dict(y=None), dict(y=A + 1), dict(ldy=H - 1), dict(ws=None), dict(ws=A + 64), dict(size=size - 1)):
        assert call(**bad) == EINVAL, bad
    assert call(T=0, x=None, ids=None, weights=None, offsets=None, order=None, y=None, ws=None, size=0) == 0


def test_moe_refusals():
    L = wc.lib()
    need = C.c_uint64(0)
    H, F = 96, 160

    def params(**more):
        f = dict(experts=16, k=2, score=0, renormalize=1, groups=1, top_groups=1, group_top=1, scale=1.0)
        f.update(more)
        return C.byref(wc._RouteParams(*f.values()))
    for bad in (dict(experts=0), dict(experts=513), dict(k=0), dict(k=17), dict(score=2), dict(groups=3),
                dict(top_groups=2), dict(group_top=3), dict(scale=math.nan)):
        assert L.wc_moe_mx_workspace_bytes(4, params(**bad), H, F, C.byref(need)) == EINVAL, bad
    for T, hidden, ffn in ((4, 0, F), (4, 65537, F), (4, H, 0), (4, H, 65537), (1 << 23, H, F)):
        assert L.wc_moe_mx_workspace_bytes(T, params(), hidden, ffn, C.byref(need)) == EINVAL
    assert L.wc_moe_mx_workspace_bytes(4, params(), H, F, None) == EINVAL
    assert L.wc_moe_mx_workspace_bytes(4, None, H, F, C.byref(need)) == EINVAL
    for T in (4, 40):
        assert L.wc_moe_mx_workspace_bytes(T, params(), H, F, C.byref(need)) == 0
        size = need.value
        assert size > 0 and size % 256 == 0

        def call(T=T, **more):
            f = dict(x=A, dt=1, ldx=H, logits=A, lt=8, ld=16, p=params(), bias=None, gate=_bank(F, H),
                     up=_bank(F, H), down=_bank(H, F), y=A, ldy=H, ws=A, size=size)
            f.update(more)
            return L.wc_moe_mx(f["x"], f["dt"], T, f["ldx"], f["logits"], f["lt"], f["ld"], f["p"], f["bias"],
                               H, F, f["gate"], f["up"], f["down"], f["y"], f["ldy"], f["ws"], f["size"], None)
        for bad in (dict(x=None), dict(dt=0), dict(ldx=H - 1), dict(logits=None), dict(logits=A + 2), dict(lt=4),
                    dict(ld=15), dict(ld=1 << 31), dict(p=None), dict(bias=A + 1), dict(gate=None),
                    dict(down=_bank(H, F, w=A + 4)), dict(y=None), dict(ldy=H - 1), dict(ws=None),
                    dict(ws=A + 16), dict(size=size - 1)):
            assert call(**bad) == EINVAL, (T, bad)
    assert call(T=0, x=None, logits=None, y=None, ws=None, size=0) == 0


def test_python_refusals():
    """What the binding refuses: tensors of host memory stand for ones on the wrong device."""
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 64))
    with pytest.raises(ValueError, match="on a device"):
        wc.quantize_mx_torch(x)
    with pytest.raises(ValueError, match="on a device"):
        wc.linear_mx_torch(x, [], [])
    with pytest.raises(ValueError, match="packed 4-bit codes"):
        wc.dequantize_mx_torch(x, x, 64)
    with pytest.raises(ValueError, match="e8m0"):
        wc.dequantize_mx_torch(x.to(torch.uint8), x, 64)
    with pytest.raises(ValueError, match="on a device"):
        wc.experts_mx_torch(x, None, x, x, x, x, x, x)
    with pytest.raises(ValueError, match="on a device"):
        wc.moe_mx_torch(x, x, 2, x, x, x, x, x, x)
