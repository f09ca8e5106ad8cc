"""GPU: int8 linear layers (wc_quantize_i8, wc_matmul_i8, wc_linear_i8) against the
definition in 64 bits.

Quantisation is checked bit for bit against the fp32 formula and against the definition
in 64 bits.  A product's int32 sum is exact; float(sum) * x scale * W scale + bias is
four fp32 roundings, of relative error 2^-24 each, and y one rounding to its type:
    |y - ref| <= 4 2^-24 (|product| + |bias|) + u |ref| (+ half of the smallest number)
with u = 2^-8 (bf16, 8 bits of significand), 2^-11 (fp16), 2^-24 (fp32), and 1 % on top for the products of
these errors.
"""
import numpy as np
import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _codes(g, n, k):
    return torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int8)


def _quantised(x):
    """The formula, in fp32 on the CPU: codes (as float) and scales."""
    x = x.float()
    top = x.abs().amax(dim=1)
    none = top < 1e-30
    # (a number divided by a tensor is the tensor's reciprocal times the number: rounded twice)
    inv = torch.where(none, torch.zeros(()), torch.full_like(top, 127.0) / top)
    return torch.round(x * inv[:, None]).clamp(-127, 127), \
        torch.where(none, torch.zeros(()), top / torch.full_like(top, 127.0))


def _check(y, q, scale, w, ws, bias):
    """y against the products of the codes in 64 bits."""
    p = (q.double() @ w.double().T) * scale.double()[:, None] * ws.double()[None]
    b = torch.zeros(()) if bias is None else bias.double()
    ref = p + b
    tol = 1.01 * (4 * 2.0 ** -24 * (p.abs() + b.abs()) + UNIT[y.dtype] * ref.abs()) + LEAST[y.dtype]
    off = (y.cpu().double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,k", [(1, 1), (3, 16), (1, 127), (2, 128), (5, 129), (64, 1000),
                                 (7, 2048), (3, 4097), (2, 8192), (1, 16385), (2, 40000), (1, 65536)])
def test_quantize(dev, dtype, m, k):
    x = torch.randn((m, k), generator=_gen(m * k)).to(DT[dtype])
    x[:, ::97] *= 30
    q, s = wc.quantize_i8_torch(x.to(dev))
    rq, rs = _quantised(x)
    assert torch.equal(s.cpu(), rs)
    assert torch.equal(q.cpu()[:, :k].float(), rq)
    assert not bool(q[:, k:].any())  # the padding
    # the definition: every value within half a step (and the roundings of x * (127 / top))
    off = (q.cpu()[:, :k].double() * rs.double()[:, None] - x.double()).abs()
    assert bool((off <= rs.double()[:, None] * (0.5 + 127 * 2.0 ** -22)).all())


def test_quantize_special_rows(dev):
    x = torch.randn((9, 300), generator=_gen(1))
    x[0] = 0
    x[1] *= 1e-35                        # counts as zeros
    x[2, 7] = float("nan")
    x[3, 299] = float("inf")
    x[4, 0] = -float("inf")
    x[5] *= 1e-20
    x[6] = torch.finfo(torch.float32).max
    x[7] = 0
    x[7, 150] = -3.0
    q, s = (t.cpu() for t in wc.quantize_i8_torch(x.to(dev)))
    for r in (0, 1):
        assert s[r] == 0 and not bool(q[r].any())
    assert torch.isnan(s[2]) and not torch.isfinite(s[3]) and not torch.isfinite(s[4])
    rq, rs = _quantised(x)
    for r in (5, 6, 7, 8):
        assert s[r] == rs[r] and torch.equal(q[r, :300].float(), rq[r])
    assert q[7, 150] == -127 and int(q[7].abs().sum()) == 127
    # in a product these rows are NaN and no other is
    w = _codes(_gen(2), 20, 300)
    y = wc.linear_i8_torch(x.to(dev), [w.to(dev)], [torch.ones(20, device=dev) * 1e-3])[0].cpu()
    assert torch.isnan(y).all(dim=1).tolist() == [False, False, True, True, True] + [False] * 4
    assert not bool(y[0].any()) and not bool(y[1].any()) and bool(torch.isfinite(y[7:]).all())


SIZES = [(1, 1, 1), (1, 16, 16), (1, 127, 15), (2, 128, 17), (15, 129, 31), (16, 255, 16),
         (17, 256, 33), (31, 1000, 100), (33, 64, 1), (63, 384, 255), (64, 4096, 48),
         (65, 515, 257), (100, 1, 300), (129, 130, 128), (200, 2048, 520), (256, 1024, 256),
         (257, 1153, 700), (700, 640, 1030), (1, 65536, 40), (40, 65535, 20), (1, 4096, 4099),
         (3, 30000, 17), (1, 132, 50), (9, 1004, 70), (40, 260, 90), (300, 1460, 300), (600, 2052, 516),
         (1, 4097, 3), (16, 126, 2), (16, 257, 1), (30, 1023, 301), (128, 1290, 66), (520, 2049, 1027)]


@pytest.mark.parametrize("m,k,n", SIZES)
def test_linear_sizes(dev, m, k, n):
    g = _gen(m + 7 * k + 13 * n)
    x = torch.randn((m, k), generator=g).bfloat16()
    w = _codes(g, n, k)
    ws = (torch.rand(n, generator=g) * 0.01).half()
    bias = torch.randn(n, generator=g)
    q, s = _quantised(x)
    for out in (torch.float32, torch.bfloat16):
        y, = wc.linear_i8_torch(x.to(dev), [w.to(dev)], [ws.to(dev)], [bias.to(dev)], dtype=out)
        assert y.dtype == out
        _check(y, q, s, w, ws, bias)
    y, = wc.matmul_i8_torch(*wc.quantize_i8_torch(x.to(dev)), k, [w.to(dev)], [ws.to(dev)])
    assert y.dtype == torch.bfloat16
    _check(y, q, s, w, ws, None)
    assert torch.equal(y, wc.linear_i8_torch(x.to(dev), [w.to(dev)], [ws.to(dev)])[0])


@pytest.mark.parametrize("m", [1, 20, 300])
@pytest.mark.parametrize("xt", list(DT))
@pytest.mark.parametrize("st", list(DT))
@pytest.mark.parametrize("yt", list(DT))
def test_linear_types(dev, m, xt, st, yt):
    g = _gen(m)
    x = (torch.randn((m, 272), generator=g) * 3).to(DT[xt])
    w = _codes(g, 90, 272)
    ws = (torch.rand(90, generator=g) * 1e-3).to(DT[st])
    bias = torch.randn(90, generator=g).to(DT[xt])
    y, = wc.linear_i8_torch(x.to(dev), [w.to(dev)], [ws.to(dev)], [bias.to(dev)], dtype=DT[yt])
    _check(y, *_quantised(x), w, ws, bias)


@pytest.mark.parametrize("m", [1, 13, 64, 150, 600])
def test_jobs_share_x(dev, m):
    """Several matrices of different heights, types, strides and biases in one call."""
    g = _gen(m)
    k = 384
    x = torch.randn((m, k), generator=g).half()
    ns = [300, 1, 16, 17, 129, 64, 500]
    ws = [_codes(g, n, k) for n in ns]
    scales = [(torch.rand(n, generator=g) * 0.01).to(list(DT.values())[i % 3]) for i, n in enumerate(ns)]
    biases = [None if i % 2 else torch.randn(n, generator=g) for i, n in enumerate(ns)]
    ys = [torch.zeros((m, n), device=dev, dtype=list(DT.values())[i % 3]) for i, n in enumerate(ns)]
    got = wc.linear_i8_torch(x.to(dev), [w.to(dev) for w in ws], [s.to(dev) for s in scales],
                             [None if b is None else b.to(dev) for b in biases], ys=ys)
    q, s = _quantised(x)
    for y, mine, w, ss, b in zip(got, ys, ws, scales, biases):
        assert y is mine
        _check(y, q, s, w, ss, b)


@pytest.mark.parametrize("m", [1, 16, 40, 130, 520])
@pytest.mark.parametrize("k", [96, 301])
def test_strides_and_alignment(dev, m, k):
    """Rows apart by odd strides, starting at odd addresses, and nothing written
    between them."""
    g = _gen(m * k)
    n = 77
    wide = torch.randint(-128, 128, (n, k + 13), generator=g, dtype=torch.int8).to(dev)
    w = wide[:, 3:3 + k]
    xw = torch.randn((m, k + 9), generator=g).bfloat16().to(dev)
    x = xw[:, 1:1 + k]
    ws = torch.rand(n + 1, generator=g).half().to(dev)[1:]
    yw = torch.full((m + 2, n + 5), 7.0, dtype=torch.float32, device=dev)
    y = yw[1:m + 1, 2:2 + n]
    wc.linear_i8_torch(x, [w], [ws], ys=[y])
    _check(y, *_quantised(x.cpu()), w.cpu(), ws.cpu(), None)
    yw[1:m + 1, 2:2 + n] = 7.0
    assert bool((yw == 7.0).all())


@pytest.mark.parametrize("m", [1, 50, 400])
def test_extreme_sums(dev, m):
    """Every product of the same sign and of the largest magnitude, k = 65536."""
    k, n = 65536, 33
    x = torch.ones((m, k)) * -5.0
    w = torch.full((n, k), -128, dtype=torch.int8)
    y, = wc.linear_i8_torch(x.to(dev), [w.to(dev)], [torch.ones(n, device=dev)])
    _check(y, *_quantised(x), w, torch.ones(n), None)


def test_codes_as_decoded_bytes(dev):
    """uint8 buffers as the decoder fills them: a blob's int8 matrix and its scales."""
    g = _gen(5)
    n, k = 200, 515
    w = _codes(g, n, k)
    ws = (torch.rand(n, generator=g) * 0.01).half()
    blob = wc.encode([("u8", w.numpy()), ("fp16", ws.view(torch.int16).numpy())], chunk_bytes=16384)
    codes, scales = wc.decode_torch(blob, wc.to_device(blob, dev))
    x = torch.randn((9, k), generator=g).bfloat16()
    y, = wc.linear_i8_torch(x.to(dev), [codes.view(n, k)], [scales.view(torch.float16)])
    _check(y, *_quantised(x), w, ws, None)


def test_past_32_bit_offsets(dev):
    """A matrix and a batch of more than 4 GiB: the last rows."""
    k, n = 65536, 66000
    w = torch.randint(-128, 128, (n, k), dtype=torch.int8, device=dev)
    ws = torch.rand(n, device=dev) * 1e-4
    x = torch.randn((2, k), generator=_gen(3))
    q, s = _quantised(x)
    y, = wc.linear_i8_torch(x.to(dev), [w], [ws])
    for rows in (slice(0, 40), slice(32760, 32780), slice(n - 40, n)):
        _check(y[:, rows], q, s, w[rows].cpu(), ws[rows].cpu(), None)
    m = 70000
    x = torch.randn((m, k), dtype=torch.float16, device=dev)
    y, = wc.linear_i8_torch(x, [w[:24]], [ws[:24]], dtype=torch.float32)
    for rows in (slice(0, 8), slice(m - 40, m)):
        _check(y[rows], *_quantised(x[rows].cpu()), w[:24].cpu(), ws[:24].cpu(), None)


def test_no_rows(dev):
    w = torch.zeros((8, 64), dtype=torch.int8, device=dev)
    y, = wc.linear_i8_torch(torch.zeros((0, 64), device=dev), [w], [torch.ones(8, device=dev)])
    assert tuple(y.shape) == (0, 8)
    q, s = wc.quantize_i8_torch(torch.zeros((0, 64), device=dev))
    assert q.shape[0] == 0 and s.numel() == 0


@pytest.mark.parametrize("m,k,n", [(1, 4096, 600), (200, 2048, 256), (96, 8192, 64)])
def test_same_result_every_time(dev, m, k, n):
    g = _gen(9)
    x = torch.randn((m, k), generator=g).to(dev)
    w = _codes(g, n, k).to(dev)
    ws = torch.rand(n, generator=g).to(dev)
    first = wc.linear_i8_torch(x, [w], [ws])[0]
    for _ in range(5):
        assert torch.equal(first, wc.linear_i8_torch(x, [w], [ws])[0])


@pytest.mark.parametrize("m", [1, 48, 300])
def test_another_stream_and_a_graph(dev, m):
    g = _gen(m)
    k, n = 1024, 320
    w = _codes(g, n, k).to(dev)
    ws = (torch.rand(n, generator=g) * 0.01).to(dev)
    xs = [torch.randn((m, k), generator=g).bfloat16() for _ in range(4)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x = xs[0].to(dev)
    y, = wc.linear_i8_torch(x, [w], [ws], stream=side)
    side.synchronize()
    _check(y, *_quantised(xs[0]), w.cpu(), ws.cpu(), None)
    x, ys = xs[0].to(dev), [torch.zeros((m, n), dtype=torch.bfloat16, device=dev)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wc.linear_i8_torch(x, [w], [ws], ys=ys)
    for v in xs:
        x.copy_(v)
        ys[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager, = wc.linear_i8_torch(x, [w], [ws])
        assert torch.equal(eager, ys[0])
        _check(ys[0], *_quantised(v), w.cpu(), ws.cpu(), None)


def test_refusals(dev):
    x = torch.zeros((4, 64), device=dev)
    w = torch.zeros((8, 64), dtype=torch.int8, device=dev)
    s = torch.ones(8, device=dev)
    bad = [lambda: wc.linear_i8_torch(x.double(), [w], [s]),
           lambda: wc.linear_i8_torch(x[0], [w], [s]),
           lambda: wc.linear_i8_torch(x.T, [w], [s]),
           lambda: wc.linear_i8_torch(x[:, :60], [w], [s]),
           lambda: wc.linear_i8_torch(x, [w.float()], [s]),
           lambda: wc.linear_i8_torch(x, [w], [s[:7]]),
           lambda: wc.linear_i8_torch(x, [w], [s.double()]),
           lambda: wc.linear_i8_torch(x, [w], [s], [s[:4]]),
           lambda: wc.linear_i8_torch(x, [w], [s, s]),
           lambda: wc.linear_i8_torch(x, [w], [s], ys=[torch.zeros((4, 7), device=dev)]),
           lambda: wc.linear_i8_torch(torch.zeros((40, 64), device=dev), [w], [s],
                                      workspace=torch.zeros(8, dtype=torch.uint8, device=dev)),
           lambda: wc.linear_i8_torch(x.cpu(), [w], [s]),
           lambda: wc.quantize_i8_torch(x, q=torch.zeros((4, 64), dtype=torch.int8, device=dev)),
           lambda: wc.matmul_i8_torch(w, s, 64, [w], [s])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: wc.linear_i8_torch(x, [], []),
                 lambda: wc.linear_i8_torch(x, [w] * 33, [s] * 33),
                 lambda: wc.linear_i8_torch(x.expand(4, 64)[:1].expand(4, 64), [w], [s]),
                 lambda: wc.linear_i8_torch(torch.zeros((1, 65537), device=dev),
                                            [torch.zeros((1, 65537), dtype=torch.int8, device=dev)],
                                            [s[:1]])):
        with pytest.raises(wc.WcError):
            call()
    assert np.isfinite(wc.linear_i8_torch(x, [w], [s])[0].float().cpu().numpy()).all()


def test_more_rows_than_a_launch_has_threads_for(dev):
    """2^24 rows and a few: a grid of one workgroup of 256 threads to each is too large.

    The codes are the formula's, on the device with the same fp32 operations; W's rows
    start at every byte of a dword, so copies of x are made, beside the codes and from them.
    """
    m, k, n = (1 << 24) + 5, 3, 6
    g = torch.Generator(device=dev).manual_seed(24)
    x = torch.randn((m, k), generator=g, device=dev).half()
    q, scale = wc.quantize_i8_torch(x)
    top = x.float().abs().amax(dim=1)
    want = torch.round(x.float() * (torch.full_like(top, 127.0) / top)[:, None])
    assert torch.equal(q[:, :k].float(), want) and not bool(q[-70:, k:].any())
    assert torch.equal(scale, top / torch.full_like(top, 127.0))
    w, ws = _codes(_gen(1), n, k).to(dev), torch.rand(n, generator=_gen(2)).to(dev)
    p = (want.double() @ w.double().T) * scale.double()[:, None] * ws.double()
    for y in (wc.linear_i8_torch(x, [w], [ws], dtype=torch.float32)[0],
              wc.matmul_i8_torch(q, scale, k, [w], [ws], dtype=torch.float32)[0]):
        off = (y.double() - p).abs()
        assert bool((off <= 1.01 * 5 * 2.0 ** -24 * p.abs() + LEAST[y.dtype]).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m", [20, 130, 520])
@pytest.mark.parametrize("n,off", [(140, 1), (140, 2), (268, 3), (77, 1), (301, 2), (5, 3)])
def test_results_at_any_element(dev, dtype, m, n, off):
    """y's rows start at any element of a larger matrix, nothing beside them is written."""
    g = _gen(m + n)
    k = 256
    x = torch.randn((m, k), generator=g).half()
    w, ws, b = _codes(g, n, k), torch.rand(n, generator=g) * 0.01, torch.randn(n, generator=g)
    wide = torch.full((m + 2, n + 7), 7.0, dtype=DT[dtype], device=dev)
    y = wide[1:m + 1, off:off + n]
    wc.linear_i8_torch(x.to(dev), [w.to(dev)], [ws.to(dev)], [b.to(dev)], ys=[y])
    _check(y, *_quantised(x), w, ws, b)
    y.fill_(7.0)
    assert bool((wide == 7.0).all())


# Matrices past the tiles' 32-bit offsets: rows more than 2^20 bytes apart, 2^20 rows or
# more, results 2^20 elements or more apart.

@pytest.mark.parametrize("m", [1, 16, 17, 64, 200])
@pytest.mark.parametrize("k,off", [(1, 0), (31, 3), (128, 0), (700, 1), (65536, 2)])
def test_rows_far_apart(dev, m, k, off):
    g = _gen(m + k)
    n, far = 53, (1 << 20) + 5
    wide = torch.randint(-128, 128, (n, far), dtype=torch.int8, device=dev)
    far_w, near_w = wide[:, off:off + k], _codes(g, 21, k).to(dev)
    ws = [torch.rand(n, generator=g) * 0.01, (torch.rand(21, generator=g) * 0.01).half()]
    bias = torch.randn(n, generator=g).bfloat16()
    x = torch.randn((m, k), generator=g).half()
    q, s = _quantised(x)
    yw = torch.full((m + 2, n + 3), 7.0, device=dev)
    near_y = torch.zeros((m, 21), dtype=torch.bfloat16, device=dev)
    wc.linear_i8_torch(x.to(dev), [far_w, near_w], [v.to(dev) for v in ws], [bias.to(dev), None],
                       ys=[yw[1:-1, 1:1 + n], near_y])
    _check(yw[1:-1, 1:1 + n], q, s, far_w.cpu(), ws[0], bias)
    _check(near_y, q, s, near_w.cpu(), ws[1], None)
    y, again = wc.matmul_i8_torch(*wc.quantize_i8_torch(x.to(dev)), k, [near_w, far_w],
                                  [ws[1].to(dev), ws[0].to(dev)], [None, bias.to(dev)], dtype=torch.float32)
    assert torch.equal(again, yw[1:-1, 1:1 + n])
    _check(y, q, s, near_w.cpu(), ws[1], None)
    yw[1:-1, 1:1 + n] = 7.0
    assert bool((yw == 7.0).all())


def test_many_columns(dev):
    """2^20 + 3 rows of W; and results that far apart."""
    g = _gen(20)
    n, m, k = (1 << 20) + 3, 20, 24
    w, ws = _codes(g, n, k), torch.rand(n, generator=g) * 0.01
    x = torch.randn((m, k), generator=g)
    y, = wc.linear_i8_torch(x.to(dev), [w.to(dev)], [ws.to(dev)])
    _check(y, *_quantised(x), w, ws, None)
    m = 70
    x = torch.randn((m, k), generator=g)
    wide = torch.full((m, n), 7.0, device=dev)
    wc.linear_i8_torch(x.to(dev), [w[:50].to(dev)], [ws[:50].to(dev)], ys=[wide[:, 9:59]])
    _check(wide[:, 9:59], *_quantised(x), w[:50], ws[:50], None)
    wide[:, 9:59] = 7.0
    assert bool((wide == 7.0).all())


def test_rows_far_apart_and_many_of_x(dev):
    """More rows of x than a grid's second axis has blocks for, the last ones a few."""
    m, k, n = 65535 * 64 + 9, 3, 2
    g = torch.Generator(device=dev).manual_seed(6)
    x = torch.randn((m, k), generator=g, device=dev).half()
    w = torch.randint(-128, 128, (n, (1 << 20) + 1), dtype=torch.int8, device=dev)[:, :k]
    ws = torch.rand(n, generator=_gen(2)).to(dev)
    y, = wc.linear_i8_torch(x, [w], [ws], dtype=torch.float32)
    q, scale = wc.quantize_i8_torch(x)
    p = (q[:, :k].double() @ w.double().T) * scale.double()[:, None] * ws.double()
    assert bool(((y.double() - p).abs() <= 1.01 * 5 * 2.0 ** -24 * p.abs() + LEAST[y.dtype]).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m", [511, 512, 513])
@pytest.mark.parametrize("k", [2041, 2048, 2049, 4095, 4096, 4097, 8191, 8192, 8193, 16384, 16385, 32769])
def test_quantize_at_its_bounds(dev, dtype, m, k):
    """Both sides of every bound of the kernel's choice, codes and scales bit for bit."""
    x = torch.randn((m, k), generator=torch.Generator(device=dev).manual_seed(k), device=dev).to(DT[dtype])
    x[:, ::97] *= 30
    q, s = wc.quantize_i8_torch(x)
    top = x.float().abs().amax(dim=1)
    assert torch.equal(s, top / torch.full_like(top, 127.0))
    want = torch.round(x.float() * (torch.full_like(top, 127.0) / top)[:, None])
    assert torch.equal(q[:, :k].float(), want) and not bool(q[:, k:].any())
