"""CPU: what the 8-bit layers' entry points refuse before anything is launched, and
the workspace they ask for.  Pointers are made up and never followed."""
import ctypes as C
import math

import pytest

from paper_2606_15789_amd import wc

EINVAL = -1
A = 1 << 20  # an aligned address that is never read


def _job(**more):
    f = dict(w=A, scale=A, bias=None, y=A, ldw=64, ldy=8, n=8, scale_dtype=2, bias_dtype=0, y_dtype=1)
    f.update(more)
    return wc._I8Job(**f)


def _jobs(*jobs):
    return (wc._I8Job * max(1, len(jobs)))(*jobs)


def test_quantize_refusals():
    ok = [A, 1, 4, 64, 64, A, A, None]
    for at, v in ((0, None), (0, A + 1), (1, 3), (1, 0), (3, 0), (3, 65537), (4, 63), (4, 1 << 31),
                  (5, None), (5, A + 8), (6, None), (6, A + 2), (2, 1 << 31)):
        args = list(ok)
        args[at] = v
        assert wc.lib().wc_quantize_i8(*args) == EINVAL, (at, v)
    assert wc.lib().wc_quantize_i8(None, 1, 0, 64, 64, None, None, None) == 0  # no rows


@pytest.mark.parametrize("bad", [
    dict(w=None), dict(scale=None), dict(y=None), dict(n=0), dict(n=1 << 31), dict(ldw=63),
    dict(ldw=1 << 31), dict(ldy=7), dict(ldy=1 << 31), dict(scale_dtype=3), dict(scale_dtype=0),
    dict(y_dtype=5), dict(bias=A, bias_dtype=0), dict(scale=A + 1), dict(y=A + 1),
    dict(bias=A + 2, bias_dtype=8), dict(y=A + 2, y_dtype=8)])
def test_job_refusals(bad):
    L = wc.lib()
    need = C.c_uint64(7)
    jobs = _jobs(_job(), _job(**bad))
    assert L.wc_linear_i8_workspace_bytes(4, 64, 2, jobs, C.byref(need)) == EINVAL
    assert need.value == 0
    assert L.wc_matmul_i8_workspace_bytes(4, 64, 2, jobs, C.byref(need)) == EINVAL
    assert L.wc_matmul_i8(A, A, 4, 64, 2, jobs, A, 1 << 30, None) == EINVAL
    assert L.wc_linear_i8(A, 1, 4, 64, 64, 2, jobs, A, 1 << 30, None) == EINVAL


def test_linear_refusals():
    L = wc.lib()
    need = C.c_uint64(0)
    jobs = _jobs(_job())
    # a few rows are quantised by the product's own kernel, more in the workspace
    assert L.wc_linear_i8_workspace_bytes(4, 64, 1, jobs, C.byref(need)) == 0
    assert need.value == 0
    assert L.wc_linear_i8_workspace_bytes(100, 64, 1, jobs, C.byref(need)) == 0
    assert need.value >= 100 * wc.i8_row_bytes(64) + 400 and need.value % 256 == 0
    n = need.value
    for args in ((4, 64, 0, jobs), (4, 64, 33, jobs), (4, 0, 1, jobs), (4, 65537, 1, jobs),
                 (1 << 31, 64, 1, jobs), (4, 64, 1, None)):
        assert L.wc_linear_i8_workspace_bytes(*args, C.byref(need)) == EINVAL
    assert L.wc_linear_i8_workspace_bytes(4, 64, 1, jobs, None) == EINVAL
    for x, dt, ldx, ws, size in ((None, 1, 64, A, n), (A + 1, 1, 64, A, n), (A, 4, 64, A, n),
                                 (A, 1, 63, A, n), (A, 1, 64, None, n), (A, 1, 64, A + 16, n),
                                 (A, 1, 64, A, n - 1)):
        assert L.wc_linear_i8(x, dt, 100, 64, ldx, 1, jobs, ws, size, None) == EINVAL
    for q, s in ((None, A), (A, None), (A + 4, A), (A, A + 1)):
        assert L.wc_matmul_i8(q, s, 4, 64, 1, jobs, A, 1 << 30, None) == EINVAL
    none = _jobs(_job(y=None))
    assert L.wc_matmul_i8(None, None, 0, 64, 1, none, None, 0, None) == 0
    assert L.wc_linear_i8(None, 1, 0, 64, 64, 1, none, None, 0, None) == 0


def test_route_refusals():
    L = wc.lib()
    need = C.c_uint64(0)

    def params(**more):
        f = dict(experts=16, k=2, score=0, renormalize=1, groups=1, top_groups=1, group_top=1, scale=1.0)
        f.update(more)
        return C.byref(wc._RouteParams(**f))
    assert L.wc_route_workspace_bytes(10, params(), C.byref(need)) == 0
    for bad in (dict(experts=0), dict(experts=513), dict(k=0), dict(k=17), dict(experts=64, k=33),
                dict(score=2), dict(score=-1), dict(groups=0), dict(groups=3), dict(top_groups=0),
                dict(top_groups=2), dict(group_top=0), dict(group_top=3),
                dict(groups=16, top_groups=1, group_top=2), dict(scale=float("nan")),
                dict(scale=float("inf"))):
        assert L.wc_route_workspace_bytes(10, params(**bad), C.byref(need)) == EINVAL, bad
    assert L.wc_route_workspace_bytes(1 << 30, params(), C.byref(need)) == EINVAL
    assert L.wc_route_workspace_bytes(10, None, C.byref(need)) == EINVAL
    # 65536 tokens: more than one workgroup sorts, so there is a workspace
    ok = [A, 1, 65536, 16, params(), None, A, A, A, A, A, 1 << 30, None]
    for at, v in ((0, None), (0, A + 1), (1, 6), (3, 15), (3, 1 << 31), (5, A + 2), (6, None),
                  (7, None), (8, None), (9, None), (6, A + 1), (7, A + 1), (8, A + 2), (9, A + 3),
                  (10, None), (10, A + 8), (11, 16)):
        args = list(ok)
        args[at] = v
        assert L.wc_route(*args) == EINVAL, (at, v)


def test_experts_refusals():
    L = wc.lib()
    need = C.c_uint64(0)
    assert L.wc_experts_i8_workspace_bytes(4, 2, 8, 64, 32, C.byref(need)) == 0
    size = need.value
    assert size % 256 == 0
    for args in ((4, 0, 8, 64, 32), (4, 9, 8, 64, 32), (4, 2, 0, 64, 32), (4, 2, 513, 64, 32),
                 (4, 2, 8, 0, 32), (4, 2, 8, 65537, 32), (4, 2, 8, 64, 0), (4, 2, 8, 64, 65537),
                 (1 << 24, 2, 8, 64, 32)):
        assert L.wc_experts_i8_workspace_bytes(*args, C.byref(need)) == EINVAL, args

    def bank(**more):
        f = dict(w=A, scale=A, stride=64 * 32, scale_dtype=2, reserved=0)
        f.update(more)
        return C.byref(wc._I8Experts(**f))
    ok = [A, 1, 4, 64, 2, 8, 64, 32, A, A, A, A, bank(), bank(), bank(), A, 64, A, size, None]
    for at, v in ((0, None), (0, A + 1), (1, 3), (3, 63), (3, 1 << 31), (8, None), (9, None),
                  (10, None), (11, A + 2), (12, None), (13, bank(w=None)), (14, bank(stride=2047)),
                  (12, bank(scale=None)), (13, bank(scale_dtype=4)), (14, bank(scale=A + 1)),
                  (12, bank(stride=1 << 40)), (15, None), (15, A + 1), (16, 63), (17, None),
                  (17, A + 128), (18, size - 1)):
        args = list(ok)
        args[at] = v
        assert L.wc_experts_i8(*args) == EINVAL, (at, v)
    args = list(ok)
    args[2] = 0
    args[0] = args[15] = args[17] = None
    assert L.wc_experts_i8(*args) == 0  # no tokens


class _OnDevice:
    """What a tensor on a device looks like to the checks of wc.py; nothing follows its
    address."""

    def __init__(self, shape, dtype, index=0):
        torch = pytest.importorskip("torch")
        self.shape, self.dtype, self.index = tuple(shape), dtype, index
        self.is_cuda, self.device = True, torch.device("cuda", index)
        self._size = torch.empty((), dtype=dtype).element_size()

    def get_device(self):
        return self.index

    def stride(self):
        return tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self._size

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return A

    def new_empty(self, shape, dtype=None):
        return _OnDevice(shape if isinstance(shape, tuple) else (shape,), dtype or self.dtype, self.index)


class _Stream:
    cuda_stream = 0
    device_index = 0


class _NoLibrary:
    """Sizes and status of a library that must not launch anything."""

    def __getattr__(self, name):
        assert name.endswith("_workspace_bytes"), f"{name} was called"

        def workspace_bytes(*args):
            args[-1]._obj.value = 4096
            return 0
        return workspace_bytes


def _calls(torch, at, put, index=0, m=40, k=64, n=16, F=32):
    """Each torch entry point with everything on device `index`, but argument `at`."""
    i8, i32, f32, bf = torch.int8, torch.int32, torch.float32, torch.bfloat16

    def t(name, shape, dtype):
        return put(shape, dtype) if name == at else _OnDevice(shape, dtype, index)

    def ws():
        return t("workspace", (1 << 16,), torch.uint8)
    st = _Stream()
    E = 8
    x, w = (lambda: t("x", (m, k), bf)), (lambda: t("w", (n, k), i8))
    s, b = (lambda: t("w_scale", (n,), f32)), (lambda: t("bias", (n,), f32))
    y, q, qs = (lambda: t("y", (m, n), bf)), (lambda: t("q", (m, 128), i8)), (lambda: t("q_scale", (m,), f32))

    def routing():
        return wc.Routing(t("ids", (m, 2), i32), t("weights", (m, 2), f32), t("offsets", (E + 1,), i32),
                          t("order", (2 * m,), i32))
    bank = (lambda: [t("gate", (E, F, k), i8), t("gate_scale", (E, F), f32), t("up", (E, F, k), i8),
                     t("up_scale", (E, F), f32), t("down", (E, k, F), i8), t("down_scale", (E, k), f32)])
    return {
        "quantize": lambda: wc.quantize_i8_torch(x(), q=q(), scale=qs(), stream=st),
        "matmul": lambda: wc.matmul_i8_torch(q(), qs(), k, [w()], [s()], [b()], ys=[y()], workspace=ws(),
                                             stream=st),
        "linear": lambda: wc.linear_i8_torch(x(), [w()], [s()], [b()], ys=[y()], workspace=ws(), stream=st),
        "route": lambda: wc.route_torch(t("logits", (m, E), f32), 2, "sigmoid", t("route_bias", (E,), f32),
                                        out=routing(), workspace=ws(), stream=st),
        "experts": lambda: wc.experts_i8_torch(x(), routing(), *bank(), y=t("out", (m, k), bf),
                                               workspace=ws(), stream=st),
    }


_ARGUMENTS = {"quantize": ["x", "q", "q_scale"],
              "matmul": ["q", "q_scale", "w", "w_scale", "bias", "y", "workspace"],
              "linear": ["x", "w", "w_scale", "bias", "y", "workspace"],
              "route": ["logits", "route_bias", "ids", "weights", "offsets", "order", "workspace"],
              "experts": ["x", "ids", "weights", "offsets", "order", "gate", "gate_scale", "up", "up_scale",
                          "down", "down_scale", "out", "workspace"]}


@pytest.mark.parametrize("call,argument", [(c, a) for c, names in _ARGUMENTS.items() for a in names])
@pytest.mark.parametrize("where", ["host", "device 1"])
def test_every_tensor_on_one_device(monkeypatch, call, argument, where):
    """A tensor in host memory, or on another device than the others, is refused before
    the library has its address."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(wc, "lib", lambda: _NoLibrary())

    def put(shape, dtype):
        return torch.zeros(shape, dtype=dtype) if where == "host" else _OnDevice(shape, dtype, 1)
    with pytest.raises(ValueError):
        _calls(torch, argument, put)[call]()


@pytest.mark.parametrize("call", list(_ARGUMENTS))
def test_tensors_on_one_device_pass_the_checks(monkeypatch, call):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(wc, "lib", lambda: _NoLibrary())
    with pytest.raises(AssertionError, match="was called"):
        _calls(torch, None, None)[call]()


def test_a_stream_of_another_device(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(wc, "lib", lambda: _NoLibrary())
    monkeypatch.setattr(_Stream, "device_index", 1)
    for call in _calls(torch, None, None).values():
        with pytest.raises(ValueError):
            call()


def test_launches_with_the_tensors_device_current(monkeypatch):
    """The current stream of a device that is not the current one: the library is called
    while that device is."""
    torch = pytest.importorskip("torch")
    current, seen = [0], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            current.append(self.index)

        def __exit__(self, *_):
            current.pop()

    class Library(_NoLibrary):
        def __getattr__(self, name):
            if name.endswith("_workspace_bytes"):
                return _NoLibrary.__getattr__(self, name)
            return lambda *args: seen.append((name, current[-1])) or 0
    monkeypatch.setattr(wc, "lib", lambda: Library())
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[-1], raising=False)
    monkeypatch.setattr(_Stream, "__new__", lambda cls: None)  # the current stream

    def on(index):
        seen.clear()
        for call in _calls(torch, None, None, index).values():
            call()
        return [device for _, device in seen]
    assert on(0) == [0] * len(_ARGUMENTS) and on(1) == [1] * len(_ARGUMENTS)


@pytest.mark.parametrize("m", [1, 16, 40, 700])
def test_workspace_does_not_depend_on_the_jobs_order(m):
    """A matrix past the tiles' offsets takes the kernel that needs no shifted copies of x,
    and no workspace, whichever matrix is named first."""
    L = wc.lib()
    odd, far = _job(ldw=65, w=A + 1), _job(ldw=(1 << 20) + 4)
    sizes = []
    for jobs in ((odd, far), (far, odd), (odd, odd, far), (far, far)):
        need = C.c_uint64(7)
        assert L.wc_matmul_i8_workspace_bytes(m, 64, len(jobs), _jobs(*jobs), C.byref(need)) == 0
        assert need.value == 0, jobs
        assert L.wc_linear_i8_workspace_bytes(m, 64, len(jobs), _jobs(*jobs), C.byref(need)) == 0
        sizes.append(need.value)
    assert len(set(sizes)) == 1, sizes


BIG = 1 << 32


@pytest.mark.parametrize("call,sizes", [
    ("quantize", dict(m=BIG + 3)), ("matmul", dict(m=BIG + 3)), ("linear", dict(m=BIG + 1)),
    ("linear", dict(m=BIG + 40, k=8)), ("linear", dict(k=BIG + 64)), ("linear", dict(n=BIG + 16)),
    ("route", dict(m=BIG + 3)), ("experts", dict(m=BIG + 3)), ("experts", dict(k=BIG + 64)),
    ("experts", dict(F=BIG + 32))])
def test_sizes_past_32_bits(monkeypatch, call, sizes):
    """Sizes that 32 bits do not hold are refused, not taken for what is left of them."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(wc, "lib", lambda: _NoLibrary())
    with pytest.raises(wc.WcError):
        _calls(torch, None, None, **sizes)[call]()


@pytest.mark.parametrize("bad", [dict(k=BIG + 2), dict(k=-BIG + 2), dict(k=-1), dict(groups=BIG + 1),
                                 dict(groups=-BIG + 1), dict(groups=2, top_groups=BIG + 1),
                                 dict(group_top=BIG + 1)])
def test_route_parameters_past_32_bits(monkeypatch, bad):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(wc, "lib", lambda: _NoLibrary())
    how = dict(k=2)
    how.update(bad)
    for tokens in (0, 4):
        with pytest.raises(wc.WcError):
            wc.route_torch(_OnDevice((tokens, 16), torch.float32), stream=_Stream(), **how)
