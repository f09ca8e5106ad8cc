"""GPU: MXFP4 linear layers (wc_quantize_mx, wc_dequantize_mx, wc_matmul_mx, wc_linear_mx)
against the definition in 64 bits.

Quantisation is exact: the codes, scales and values have to be the definition's.  A
product sums blocks of 32, each exact in fp32, in fp32: blocks and parts of k, in some
order, each addition off by at most 2^-23 of the magnitudes added so far (2^-24 where it
rounds to nearest, which the matrix unit need not):
    |y - ref| <= (blocks + 32) 2^-23 sum |x w| + 2^-24 |ref| + u |ref| (+ half the smallest number)
with u = 2^-8 (bf16), 2^-11 (fp16), 2^-24 (fp32), 2^-24 the bias's addition, and 1 % on top for the
products of these errors.
"""
import numpy as np
import pytest

from paper_2606_15789_amd import synth, wc

torch = pytest.importorskip("torch")
import mx_reference as mx  # noqa: E402
from mx_reference import DT, LEAST, UNIT  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _x(g, m, k, dtype):
    x = torch.randn((m, k), generator=g)
    x[:, ::97] *= 20
    return x.to(DT[dtype])


def _check(y, xv, w, s, bias=None):
    """y against the product of x's values (64 bits) and the matrix w, s."""
    k = xv.shape[1]
    wv = mx.values(w, s, k)
    ref = xv @ wv.T
    mag = xv.abs() @ wv.abs().T
    if bias is not None:
        ref = ref + bias.double()
    tol = 1.01 * ((mx.blocks(k) + 32) * 2.0 ** -23 * mag + (2.0 ** -24 + UNIT[y.dtype]) * ref.abs()) \
        + LEAST[y.dtype]
    off = (y.cpu().double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


def _xv(x):
    c, b = mx.quantize(x)
    return mx.values(mx.pack(c), b, x.shape[1])


# --- quantisation -------------------------------------------------------------

SIZES = [(1, 1), (3, 31), (1, 32), (5, 33), (64, 1000), (7, 2048), (300, 64), (3, 4097), (2, 8192),
         (1, 16385), (2, 40000), (1, 65536), (1000, 8), (129, 2055)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,k", SIZES)
def test_quantize(dev, dtype, m, k):
    x = _x(_gen(m * k), m, k, dtype)
    q, s = wc.quantize_mx_torch(x.to(dev))
    codes, byte = mx.quantize(x)
    assert torch.equal(s.cpu(), byte)
    assert torch.equal(q.cpu(), mx.pack(codes))  # the padding's zeros too


@pytest.mark.parametrize("dtype", list(DT))
def test_quantize_every_exponent(dev, dtype):
    """Blocks of every exponent of the type, with ties, neighbours of ties, zeros of both signs and
    denormal numbers."""
    info = torch.finfo(DT[dtype])
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.0, 0.5, 1.5, 3.0])
    rows = []
    for e in range(int(np.log2(info.smallest_normal)) - 12, int(np.log2(info.max)) + 1):
        for top in (4.0, 6.0, 7.9):
            r = torch.cat([ties, torch.nextafter(ties, torch.zeros(14)), torch.tensor([top, -0.25, -2.5, -5.0])])
            rows.append(r.clamp(-top, top).double() * 2.0 ** (e - 2))
    x = torch.stack(rows)
    x = x.clamp(-info.max, info.max).to(DT[dtype])
    q, s = wc.quantize_mx_torch(x.to(dev))
    codes, byte = mx.quantize(x)
    assert torch.equal(s.cpu(), byte)
    assert torch.equal(q.cpu(), mx.pack(codes))
    # the framework's own quantiser of checkpoints, where it does not drop the sign of zeros
    pk, sc = synth.quant_mxfp4(x.float().numpy())
    big = x.abs().amax(dim=1) > 1e-25
    assert torch.equal(torch.from_numpy(sc)[big], byte[big])
    assert torch.equal(mx.values(torch.from_numpy(pk), torch.from_numpy(sc), 32)[big],
                       mx.values(mx.pack(codes), byte, 32)[big])


@pytest.mark.parametrize("dtype", list(DT))
def test_quantize_not_finite(dev, dtype):
    x = _x(_gen(1), 4, 100, dtype)
    x[0, 3] = float("nan")
    x[1, 40] = float("inf")
    x[2, 99] = -float("inf")
    x[3, 32:64] = 0
    q, s = wc.quantize_mx_torch(x.to(dev))
    codes, byte = mx.quantize(x)
    assert byte[0, 0] == byte[1, 1] == byte[2, 3] == 255 and byte[3, 1] == 0
    assert torch.equal(s.cpu(), byte) and torch.equal(q.cpu(), mx.pack(codes))
    y = wc.dequantize_mx_torch(q, s, 100, dtype=DT[dtype]).cpu()
    nan = torch.zeros((4, 100), dtype=torch.bool)
    nan[0, :32] = nan[1, 32:64] = nan[2, 96:] = True
    assert torch.equal(torch.isnan(y), nan)


@pytest.mark.parametrize("dtype", list(DT))
def test_quantize_strides(dev, dtype):
    """Rows at any element, in rows of a larger result whose other bytes stay."""
    m, k = 37, 141
    g = _gen(5)
    wide = _x(g, m, 200, dtype).to(dev)
    x = wide[:, 7:7 + k]
    q = torch.full((m, 112), 0xA5, dtype=torch.uint8, device=dev)
    s = torch.full((m, 11), 0xA5, dtype=torch.uint8, device=dev)
    wc.quantize_mx_torch(x, q[:, 16:96], s[:, 3:8])
    codes, byte = mx.quantize(x.cpu())
    assert torch.equal(q[:, 16:96].cpu(), mx.pack(codes)) and torch.equal(s[:, 3:8].cpu(), byte)
    for rest in (q[:, :16], q[:, 96:], s[:, :3], s[:, 8:]):
        assert bool((rest == 0xA5).all())
    y = torch.zeros((m, 200), dtype=DT[dtype], device=dev)
    wc.dequantize_mx_torch(q[:, 16:96], s[:, 3:8], k, y=y[:, 9:9 + k])
    assert torch.equal(y[:, 9:9 + k].cpu().double(), mx.values(mx.pack(codes), byte, k).to(DT[dtype]).double())
    assert not bool(y[:, :9].any()) and not bool(y[:, 9 + k:].any())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,k", SIZES)
def test_dequantize(dev, dtype, m, k):
    w, s = mx.matrix(_gen(m + k), m, k, spread=256, base=0)
    y = wc.dequantize_mx_torch(w.to(dev), s.to(dev), k, dtype=DT[dtype]).cpu()
    v = mx.values(w, s, k)
    ref = v.float().to(DT[dtype])  # exact in fp32, then one rounding
    assert torch.equal(torch.isnan(y), torch.isnan(ref))
    assert torch.equal(torch.nan_to_num(y.double(), 7.0), torch.nan_to_num(ref.double(), 7.0))


def test_every_code_and_scale(dev):
    codes = torch.arange(16, dtype=torch.uint8).repeat(2).expand(256, 1, 32)
    s = torch.arange(256, dtype=torch.int32).to(torch.uint8)[:, None]
    y = wc.dequantize_mx_torch(mx.pack(codes).contiguous().to(dev), s.to(dev), 32, dtype=torch.float32).cpu()
    ref = mx.values(mx.pack(codes), s, 32)
    ref = torch.where(ref.abs() > torch.finfo(torch.float32).max, ref.sign() * float("inf"), ref)
    assert bool(torch.isnan(y[255]).all()) and torch.equal(y[:255].double(), ref[:255])


# --- products -----------------------------------------------------------------

@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 33, 64, 65, 130, 257])
@pytest.mark.parametrize("k,n", [(1, 1), (31, 17), (32, 16), (33, 100), (512, 32), (513, 33),
                                 (1000, 260), (4096, 96), (5461, 131), (256, 515), (224, 64)])
def test_linear_sizes(dev, m, k, n):
    g = _gen(m * 7 + k * 3 + n)
    dtype = list(DT)[(m + k) % 3]
    x = _x(g, m, k, dtype)
    w, s = mx.matrix(g, n, k)
    y, = wc.linear_mx_torch(x.to(dev), [w.to(dev)], [s.to(dev)])
    assert y.dtype == DT[dtype]
    _check(y, _xv(x), w, s)


@pytest.mark.parametrize("m", [3, 40, 200, 600])
@pytest.mark.parametrize("x_dtype", list(DT))
@pytest.mark.parametrize("y_dtype", list(DT))
def test_linear_types_bias_jobs(dev, m, x_dtype, y_dtype):
    """Several matrices of one x, with biases of every type and without."""
    g = _gen(m)
    k = 352
    x = _x(g, m, k, x_dtype)
    mats = [mx.matrix(g, n, k) for n in (48, 1, 129, 300)]
    biases = [torch.randn(48, generator=g).bfloat16(), None, torch.randn(129, generator=g),
              torch.randn(300, generator=g).half()]
    ys = wc.linear_mx_torch(x.to(dev), [w.to(dev) for w, _ in mats], [s.to(dev) for _, s in mats],
                            [None if b is None else b.to(dev) for b in biases], dtype=DT[y_dtype])
    for y, (w, s), b in zip(ys, mats, biases):
        assert y.dtype == DT[y_dtype]
        _check(y, _xv(x), w, s, b)


@pytest.mark.parametrize("m", [5, 16, 50, 300, 700])
def test_matmul_of_quantised(dev, m):
    """quantize then matmul is linear, bit for bit where both run the same product."""
    g = _gen(m)
    k, n = 800, 200
    x = _x(g, m, k, "bf16").to(dev)
    w, s = mx.matrix(g, n, k)
    q, qs = wc.quantize_mx_torch(x)
    y, = wc.matmul_mx_torch(q, qs, k, [w.to(dev)], [s.to(dev)], dtype=torch.float32)
    _check(y, _xv(x.cpu()), w, s)
    z, = wc.linear_mx_torch(x, [w.to(dev)], [s.to(dev)], dtype=torch.float32)
    assert torch.equal(y, z)


@pytest.mark.parametrize("m", [4, 60, 400])
@pytest.mark.parametrize("k", [608, 601])
def test_strides(dev, m, k):
    """Every operand inside a larger one: rows further apart, results at odd elements, the
    elements between them as they were."""
    g = _gen(m)
    n = 77
    big = _x(g, m + 2, k + 31, "fp16").to(dev)
    x = big[1:m + 1, 5:5 + k]
    w, s = mx.matrix(g, n, k)
    W = torch.randint(0, 256, (n + 1, 480), generator=g, dtype=torch.uint8).to(dev)
    S = torch.full((n, 40), 255, dtype=torch.uint8, device=dev)
    W[1:, 32:32 + w.shape[1]] = w.to(dev)
    S[:, 11:11 + s.shape[1]] = s.to(dev)
    Y = torch.full((m + 2, n + 9), 3.0, device=dev)
    bias = torch.randn(n + 1, generator=g).to(dev)[1:]
    wc.linear_mx_torch(x, [W[1:, 32:32 + w.shape[1]]], [S[:, 11:11 + s.shape[1]]], [bias],
                       ys=[Y[1:m + 1, 3:3 + n]])
    _check(Y[1:m + 1, 3:3 + n], _xv(x.cpu()), w, s, bias.cpu())
    Y[1:m + 1, 3:3 + n] = 3.0
    assert bool((Y == 3.0).all())
    # x of quantised rows inside larger ones, NaN scales between them
    q, qs = wc.quantize_mx_torch(x)
    Q = torch.full((m, q.shape[1] + 48), 0x77, dtype=torch.uint8, device=dev)
    QS = torch.full((m, qs.shape[1] + 5), 255, dtype=torch.uint8, device=dev)
    Q[:, 16:16 + q.shape[1]], QS[:, 2:2 + qs.shape[1]] = q, qs
    y, = wc.matmul_mx_torch(Q[:, 16:16 + q.shape[1]], QS[:, 2:2 + qs.shape[1]], k, [w.to(dev)], [s.to(dev)],
                            dtype=torch.float32)
    _check(y, _xv(x.cpu()), w, s)


@pytest.mark.parametrize("m", [1, 16, 48, 300])
def test_not_finite(dev, m):
    """A NaN scale of a row of W, or a NaN or infinity in a row of x, makes its results NaN and no
    others."""
    g = _gen(m)
    k, n = 1056, 90
    x = _x(g, m, k, "bf16")
    w, s = mx.matrix(g, n, k)
    s[4, 32] = s[17, 0] = s[89, 20] = 255
    x[m // 2, 1055] = float("inf")
    y, = wc.linear_mx_torch(x.to(dev), [w.to(dev)], [s.to(dev)])
    nan = torch.zeros((m, n), dtype=torch.bool)
    nan[:, [4, 17, 89]] = True
    nan[m // 2] = True
    assert torch.equal(torch.isnan(y.cpu()), nan)


@pytest.mark.parametrize("m", [3, 40, 300])
def test_scales_far_apart(dev, m):
    """Scales of every size: sums that are rounded, results beyond the range of fp32."""
    g = _gen(m)
    k, n = 416, 64
    x = _x(g, m, k, "fp32")
    x *= torch.exp2(torch.randint(-60, 60, (m, k // 32), generator=g).float()).repeat_interleave(32, 1)
    w, s = mx.matrix(g, n, k, spread=60, base=90)
    y, = wc.linear_mx_torch(x.to(dev), [w.to(dev)], [s.to(dev)])
    _check(y, _xv(x), w, s)
    s[:] = 250
    y, = wc.linear_mx_torch(x.abs().to(dev), [(w & 0x77).to(dev)], [s.to(dev)])
    assert bool((torch.isinf(y) | (y == 0) | (y > 0)).all()) and not bool(torch.isnan(y).any())


@pytest.mark.parametrize("m", [0, 1, 100])
def test_nothing_behind_the_rows(dev, m):
    n, k = 40, 96
    w, s = mx.matrix(_gen(1), n, k)
    Y = torch.full((m + 3, n), 9.0, device=dev)
    x = _x(_gen(2), m, k, "fp32").to(dev)
    wc.linear_mx_torch(x, [w.to(dev)], [s.to(dev)], ys=[Y[:m]])
    assert bool((Y[m:] == 9.0).all())


@pytest.mark.parametrize("m", [1, 9, 16])
@pytest.mark.parametrize("k", [8192, 8193, 12288, 12289, 16400])
@pytest.mark.parametrize("n", [48, 5000, 17000])
def test_few_rows_of_many(dev, m, k, n):
    """Up to 16 rows: x held on chip and not, tiles of 16, 32 and 64 rows of W, several to a
    workgroup."""
    g = torch.Generator(device=dev).manual_seed(m + k + n)
    w = torch.randint(0, 256, (n, mx.blocks(k) * 16), generator=g, device=dev, dtype=torch.uint8)
    s = torch.randint(120, 123, (n, mx.blocks(k)), generator=g, device=dev, dtype=torch.uint8)
    x = _x(_gen(m), m, k, list(DT)[m % 3])
    bias = torch.randn(n, generator=g, device=dev)
    y, = wc.linear_mx_torch(x.to(dev), [w], [s], [bias], dtype=torch.float32)
    some = torch.unique(torch.cat([torch.arange(0, n, 257), torch.arange(n - 40, n)]))
    on = some.to(dev)
    _check(y[:, on], _xv(x), w[on].cpu(), s[on].cpu(), bias[on].cpu())


def test_many_jobs(dev):
    """As many matrices as a call takes, of every tile's sizes."""
    g = _gen(4)
    k = 288
    mats = [mx.matrix(g, 1 + 13 * i, k) for i in range(32)]
    for m in (2, 30, 140):
        x = _x(g, m, k, "bf16")
        ys = wc.linear_mx_torch(x.to(dev), [w.to(dev) for w, _ in mats], [s.to(dev) for _, s in mats])
        for y, (w, s) in zip(ys, mats):
            _check(y, _xv(x), w, s)


@pytest.mark.parametrize("m,k,n", [(300, 2048, 700), (520, 4096, 1030), (1100, 1024, 2300), (90, 20000, 300)])
def test_tiles_and_parts(dev, m, k, n):
    """Tiles of every size, parts of k, in every type of result."""
    g = _gen(m)
    x = _x(g, m, k, "bf16")
    w, s = mx.matrix(g, n, k)
    bias = torch.randn(n, generator=g)
    for dtype in DT.values():
        y, = wc.linear_mx_torch(x.to(dev), [w.to(dev)], [s.to(dev)], [bias.to(dev)], dtype=dtype)
        _check(y, _xv(x), w, s, bias)


def test_scales_past_a_gigabyte(dev):
    """So many rows that a group's scales of all of them lie further apart than a tile's offsets
    reach: they are kept in rows."""
    m, k, n = (1 << 20) + 77, 32768, 40
    if torch.cuda.mem_get_info(dev)[0] < 120 << 30:
        pytest.skip("needs 120 GiB")
    g = torch.Generator(device=dev).manual_seed(1)
    some = torch.randn((64, k), generator=g, device=dev).bfloat16()
    x = torch.empty((m, k), dtype=torch.bfloat16, device=dev)
    for i in range(0, m, 64):
        x[i:i + 64] = some[:min(64, m - i)]
    x[-1] = some[5] * 3
    w, s = (t.to(dev) for t in mx.matrix(_gen(1), n, k))
    y, = wc.linear_mx_torch(x, [w], [s], dtype=torch.float32)
    rows = torch.tensor([0, 63, 64, 65535 * 16, (1 << 20) - 1, 1 << 20, m - 2, m - 1])
    on = rows.to(dev)
    _check(y[on], _xv(x[on].cpu()), w.cpu(), s.cpu())
    assert torch.equal(y[:64], y[64:128]) and torch.equal(y[:64], y[(1 << 20) - 64:1 << 20])


def test_two_streams_at_once(dev):
    """Calls on two streams at the same time, each with its own workspace."""
    g = _gen(8)
    k, n = 1024, 640
    w, s = (t.to(dev) for t in mx.matrix(g, n, k))
    xs = [_x(g, m, k, "bf16").to(dev) for m in (3, 400)]
    want = [wc.linear_mx_torch(x, [w], [s])[0].clone() for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(wc.linear_mx_torch(xs[i], [w], [s])[0])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_padding_of_weights(dev):
    """Codes past k of W's rows may be any (mx.matrix makes them random); those of x are zeros."""
    g = _gen(3)
    k, n = 45, 30
    w, s = mx.matrix(g, n, k)
    clean = mx.unpack(w).clone()
    clean[:, k:] = 0
    other = mx.pack(clean.view(n, 2, 32))
    for m in (2, 90, 300):
        x = _x(g, m, k, "bf16").to(dev)
        a, = wc.linear_mx_torch(x, [w.to(dev)], [s.to(dev)])
        b, = wc.linear_mx_torch(x, [other.to(dev)], [s.to(dev)])
        assert torch.equal(a, b)


@pytest.mark.parametrize("m", [7, 20, 300])
def test_streams_and_graphs(dev, m):
    """On another stream, and captured and replayed with eager calls between the replays."""
    g = _gen(m)
    k, n = 768, 320
    w, s = (t.to(dev) for t in mx.matrix(g, n, k))
    xs = [_x(g, m, k, "bf16").to(dev) for _ in range(3)]
    want = [wc.linear_mx_torch(x, [w], [s])[0].clone() for x in xs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = wc.linear_mx_torch(xs[1], [w], [s], stream=side)[0]
    side.synchronize()
    assert torch.equal(got, want[1])
    x, y = xs[0].clone(), torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wc.linear_mx_torch(x, [w], [s], ys=[y])
        q, qs = wc.quantize_mx_torch(y)
        back = wc.dequantize_mx_torch(q, qs, n)
    for i in (0, 1, 2, 0, 1):
        x.copy_(xs[i])
        graph.replay()
        assert torch.equal(wc.linear_mx_torch(xs[2], [w], [s])[0], want[2])
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])
        q2, s2 = wc.quantize_mx_torch(want[i])
        assert torch.equal(back, wc.dequantize_mx_torch(q2, s2, n))


@pytest.mark.parametrize("m", [3, 100, 400])
def test_same_on_every_run(dev, m):
    g = _gen(m)
    k, n = 8192, 512
    w, s = (t.to(dev) for t in mx.matrix(g, n, k, spread=40, base=100))
    x = _x(g, m, k, "fp32").to(dev)
    first, = wc.linear_mx_torch(x, [w], [s])
    for _ in range(5):
        assert torch.equal(wc.linear_mx_torch(x, [w], [s])[0], first)


@pytest.mark.parametrize("m", [2, 40, 300])
def test_past_32_bits(dev, m):
    """A matrix of more than 4 GiB, and rows of x and y behind 2^32 bytes."""
    k, n = 65536, 140000
    g = torch.Generator(device=dev).manual_seed(1)
    w = torch.randint(0, 256, (n, k // 2), generator=g, device=dev, dtype=torch.uint8)
    s = torch.randint(120, 123, (n, k // 32), generator=g, device=dev, dtype=torch.uint8)
    x = torch.randn((m, k), generator=g, device=dev).bfloat16()
    y, = wc.linear_mx_torch(x, [w], [s], dtype=torch.float32)
    some = torch.tensor([0, 1, 33, 65535, 131071, 131072, 139990, 139999])
    _check(y[:, some.to(dev)], _xv(x.cpu()), w[some.to(dev)].cpu(), s[some.to(dev)].cpu())


def test_many_rows(dev):
    """More rows of x than 2^31 of its elements."""
    m, k, n = 70000, 32768, 16
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.empty((m, k), dtype=torch.bfloat16, device=dev)
    for i in range(0, m, 10000):
        x[i:i + 10000] = torch.randn((10000, k), generator=g, device=dev)
    w, s = (t.to(dev) for t in mx.matrix(_gen(1), n, k))
    y, = wc.linear_mx_torch(x, [w], [s], dtype=torch.float32)
    some = torch.tensor([0, 1, 65534, 65535, 65536, 69999])
    _check(y[some.to(dev)], _xv(x[some.to(dev)].cpu()), w.cpu(), s.cpu())
    q, qs = wc.quantize_mx_torch(x)
    back = wc.dequantize_mx_torch(q, qs, k)
    assert torch.equal(back[some.to(dev)].cpu().double(), _xv(x[some.to(dev)].cpu()))


def test_checkpoint_to_layer(dev):
    """A checkpoint's MXFP4 matrix from its blob through the decoder to a layer."""
    g = _gen(9)
    w = torch.randn((96, 512), generator=g) * 0.02
    codes, scales = synth.quant_mxfp4(w.numpy())
    blob = wc.encode([("fp4_e2m1", codes, (96, 512)), ("u8", scales)])
    outs = wc.decode_torch(blob, wc.to_device(blob, dev))
    x = torch.randn((5, 512), generator=g).bfloat16()
    y, = wc.linear_mx_torch(x.to(dev), [outs[0].view(96, 256)], [outs[1].view(96, 16)])
    _check(y, _xv(x), torch.from_numpy(codes), torch.from_numpy(scales))
