"""GPU: more rows than one launch of the microscaled layers' kernels takes (2^23 rows of a
quantisation, 65535 blocks of 64 rows of a product without tiles), with the tolerances of the other
tests of these layers."""
import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
import mx_reference as mx  # noqa: E402
import test_gpu_mx as base  # noqa: E402
import test_gpu_mx_experts as ex  # noqa: E402

pytestmark = pytest.mark.gpu
ROWS = (1 << 23) + 1037


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _rows(dev, m, k):
    """m rows of which neighbours, and those 2^23 apart, differ."""
    g = torch.Generator(device=dev).manual_seed(k)
    return torch.randn((m, k), generator=g, device=dev).bfloat16()


def _some(m):
    return torch.tensor([0, 1, 255, 256, 65535 * 64 - 1, 65535 * 64, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, m - 2, m - 1])


@pytest.mark.parametrize("k", [3, 40])
def test_quantize_and_back(dev, k):
    x = _rows(dev, ROWS, k)
    q, s = wc.quantize_mx_torch(x)
    some = _some(ROWS)
    codes, byte = mx.quantize(x[some.to(dev)].cpu())
    assert torch.equal(q[some.to(dev)].cpu(), mx.pack(codes)) and torch.equal(s[some.to(dev)].cpu(), byte)
    back = wc.dequantize_mx_torch(q, s, k, dtype=torch.float32)
    assert torch.equal(back[some.to(dev)].cpu().double(), mx.values(mx.pack(codes), byte, k))


@pytest.mark.parametrize("m", [ROWS, (1 << 24) + 5])
def test_linear(dev, m):
    """On tiles, and from 2^24 rows on without."""
    k, n = 70, 6
    x = _rows(dev, m, k)
    w, s = mx.matrix(base._gen(1), n, k)
    bias = torch.randn(n, generator=base._gen(2))
    y, = wc.linear_mx_torch(x, [w.to(dev)], [s.to(dev)], [bias.to(dev)], dtype=torch.float32)
    some = _some(m)
    base._check(y[some.to(dev)], base._xv(x[some.to(dev)].cpu()), w, s, bias)


def test_experts(dev):
    E, hidden, ffn = 3, 34, 33
    x = _rows(dev, ROWS, hidden)
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(-1, E, (ROWS, 1), generator=g)
    weights = torch.rand((ROWS, 1), generator=g) + 0.1
    r = ex._routing(ids, weights, E)
    layer = ex._layer(3, E, hidden, ffn)
    y = wc.experts_mx_torch(x, wc.Routing(*(t.to(dev) for t in r)), *ex._on(dev, layer))
    some = torch.cat([_some(ROWS), torch.randint(0, ROWS, (200,), generator=g)])
    ex._check(y[some.to(dev)], x[some.to(dev)].cpu(), ex._routing(ids[some], weights[some], E), layer)
