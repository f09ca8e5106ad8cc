"""GPU: products of MXFP4 matrices on every kernel that wc_linear_mx has and with every number of
parts of k (test_mx_plans checks on the CPU that these sizes take them); rows far apart; results
beyond fp32; torch's own 4-bit and scale types.  Tolerances are those of test_gpu_mx."""
import pytest

from mx_plans import PLANS
from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
import mx_reference as mx  # noqa: E402
import test_gpu_mx as base  # noqa: E402
import test_gpu_mx_experts as ex  # noqa: E402
from mx_reference import DT, LEAST  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _some(g, n):
    """Indexes below n: around the tiles' borders, the last ones, and some by chance."""
    at = [i + d for i in (0, 16, 32, 64, 128, 192, 256, 512, 1024) for d in (-1, 0, 1)] + list(range(n - 5, n))
    at += torch.randint(0, n, (30,), generator=g).tolist()
    return torch.tensor(sorted({i for i in at if 0 <= i < n}))


@pytest.mark.parametrize("size,plan", PLANS, ids=[f"{p.replace(' ', '-')}-{s[0]}x{s[1]}x{s[2]}" for s, p in PLANS])
def test_every_kernel(dev, size, plan):
    """With a bias and results of every type, stored inside a larger matrix whose other elements stay."""
    m, k, n = size
    g = base._gen(m + k)
    on = torch.Generator(device=dev).manual_seed(n)
    w = torch.randint(0, 256, (n, mx.blocks(k) * 16), generator=on, device=dev, dtype=torch.uint8)
    s = torch.randint(119, 122, (n, mx.blocks(k)), generator=on, device=dev, dtype=torch.uint8)
    x = base._x(g, m, k, list(DT)[n % 3])
    bias = torch.randn(n, generator=g).to(list(DT.values())[m % 3])
    rows, cols = _some(g, m), _some(g, n)
    xv = base._xv(x[rows])
    for dtype in DT.values():
        Y = torch.full((m + 1, n + 11), 3.0, dtype=dtype, device=dev)
        wc.linear_mx_torch(x.to(dev), [w], [s], [bias.to(dev)], ys=[Y[:m, 5:5 + n]])
        y = Y[:m, 5:5 + n]
        base._check(y[rows.to(dev)][:, cols.to(dev)], xv, w[cols.to(dev)].cpu(), s[cols.to(dev)].cpu(), bias[cols])
        Y[:m, 5:5 + n] = 3.0
        assert bool((Y == 3.0).all())


@pytest.mark.parametrize("m", [3, 40, 300])
@pytest.mark.parametrize("apart", [(1 << 22) + 16, (1 << 27) + 16])
def test_rows_far_apart(dev, m, apart):
    """Rows of W, and of x already quantised, and their scales, further apart than tiles' and streams'
    offsets reach."""
    k, n = 1000, 33
    if m * apart > 40 << 30:
        m = 70
    g = base._gen(m)
    x = base._x(g, m, k, "bf16").to(dev)
    w, s = mx.matrix(g, n, k)
    space = torch.empty(max(m, n) * apart + 4096, dtype=torch.uint8, device=dev)
    W = space.as_strided((n, w.shape[1]), (apart, 1))
    S = space.as_strided((n, s.shape[1]), (apart, 1), 1024)
    W.copy_(w)
    S.copy_(s)
    for ww, ss in ((W, s.to(dev)), (w.to(dev), S), (W, S)):
        y, = wc.linear_mx_torch(x, [ww], [ss], dtype=torch.float32)
        base._check(y, base._xv(x.cpu()), w, s)
    q, qs = wc.quantize_mx_torch(x)
    Q = space.as_strided((m, q.shape[1]), (apart, 1))
    QS = space.as_strided((m, qs.shape[1]), (apart, 1), 1024)
    Q.copy_(q)
    QS.copy_(qs)
    for qq, ss in ((Q, qs), (q, QS), (Q, QS)):
        y, = wc.matmul_mx_torch(qq, ss, k, [w.to(dev)], [s.to(dev)], dtype=torch.float32)
        base._check(y, base._xv(x.cpu()), w, s)


@pytest.mark.parametrize("m", [3, 40, 300, 1100])
def test_results_beyond_fp32(dev, m):
    """Sums of one sign: where the exact one is clearly beyond fp32 the result is an infinity of that
    sign, where it is clearly within, within the usual tolerance; zeros stay zeros under any scale."""
    g = base._gen(m)
    k, n = 416, 64
    x = base._x(g, m, k, "fp32").abs() + 0.1
    x *= torch.exp2(torch.randint(-60, 60, (m, 1), generator=g).float())
    x[m // 2] = 0
    w, s = mx.matrix(g, n, k)
    w = w & 0x77 | 0x11  # above zero
    w[n // 2:] |= 0x88   # and below
    s[:] = torch.randint(180, 252, (n, 1), generator=g, dtype=torch.uint8)
    w[5] = 0
    s[5] = 254
    xv = base._xv(x)
    wv = mx.values(w, s, k)
    ref = xv @ wv.T
    y, = wc.linear_mx_torch(x.to(dev), [w.to(dev)], [s.to(dev)])
    y = y.cpu().double()
    tol = 1.01 * ((mx.blocks(k) + 32) * 2.0 ** -23 + 2.0 ** -24)  # of |ref|: no terms cancel
    most = torch.finfo(torch.float32).max
    beyond, within = ref.abs() > most * (1 + tol), ref.abs() < most * (1 - tol)
    assert bool(beyond.any()) and int((within & (ref != 0)).sum()) > 100
    assert torch.equal(y[beyond], ref[beyond].sign() * float("inf"))
    off = (y - ref).abs()
    assert bool((off <= tol * ref.abs() + LEAST[torch.float32])[within].all())
    assert not bool(y[m // 2].any()) and not bool(y[:, 5].any())


def test_torch_types(dev):
    """Codes and scales as torch's own 4-bit and e8m0 types, where it has them."""
    if not hasattr(torch, "float4_e2m1fn_x2") or not hasattr(torch, "float8_e8m0fnu"):
        pytest.skip("torch has no such types")

    def own(codes, scales):
        return codes.view(torch.float4_e2m1fn_x2), scales.view(torch.float8_e8m0fnu)
    g = base._gen(2)
    k, n = 288, 96
    w, s = (t.to(dev) for t in mx.matrix(g, n, k))
    tw, ts = own(w, s)
    for m in (3, 40, 300):
        x = base._x(g, m, k, "bf16").to(dev)
        assert torch.equal(wc.linear_mx_torch(x, [tw], [ts])[0], wc.linear_mx_torch(x, [w], [s])[0])
        q, qs = wc.quantize_mx_torch(x)
        tq, tqs = own(torch.empty_like(q), torch.empty_like(qs))
        wc.quantize_mx_torch(x, tq, tqs)
        assert torch.equal(tq.view(torch.uint8), q) and torch.equal(tqs.view(torch.uint8), qs)
        assert torch.equal(wc.dequantize_mx_torch(tq, tqs, k), wc.dequantize_mx_torch(q, qs, k))
        a, = wc.matmul_mx_torch(tq, tqs, k, [tw], [ts])
        assert a.dtype == torch.bfloat16 and torch.equal(a, wc.matmul_mx_torch(q, qs, k, [w], [s])[0])
    E, kk, hidden, ffn = 4, 2, 96, 64
    layer = [t.to(dev) for pair in ex._layer(3, E, hidden, ffn) for t in pair]
    named = [t for i in (0, 2, 4) for t in own(layer[i], layer[i + 1])]
    for tokens in (3, 50):
        x = torch.randn((tokens, hidden), generator=g).bfloat16().to(dev)
        lo = torch.randn((tokens, E), generator=g).to(dev)
        r = wc.route_torch(lo, kk)
        assert torch.equal(wc.experts_mx_torch(x, r, *named), wc.experts_mx_torch(x, r, *layer))
        assert torch.equal(wc.moe_mx_torch(x, lo, kk, *named), wc.moe_mx_torch(x, lo, kk, *layer))
