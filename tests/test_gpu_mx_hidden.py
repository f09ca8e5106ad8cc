"""GPU: the codes of a mixture layer's hidden values next to the borders between codes.

h = silu(g) u is brought to MXFP4, so the least error of h decides the code of a value next to a
border.  Here g and u are sums that fp32 holds exactly, and h lies on either side of a border (a
half step between two codes, or the power of two at which a block's scale changes), 2^-40 to 2^-31
of its size away: less than fp32 tells apart, more than the 2^-49 that 64 bits are off by.  With
down a unit matrix and weights of 1, the results are the hidden values themselves, exact in fp32,
and have to be the definition's, all of them.
"""
import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
import mx_reference as mx  # noqa: E402

pytestmark = pytest.mark.gpu
DIGITS = 12  # a number of 24 bits as digits of two, a block's product each


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _silu(g):
    return g / (1 + torch.exp(-g))


def _fp32(v):
    return v.float().double()


def _near_borders(gen, n):
    """n pairs (g, u) whose h lies next to a border at 2^-2 .. 5 times a block's scale of 1."""
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    tries = 1 << 19
    g = _fp32((torch.rand(tries, generator=gen).double() * 12 + 0.2) * (1 - 2 * (torch.rand(tries, generator=gen) < 0.4).double()))
    b = border[torch.randint(0, 7, (tries,), generator=gen)] * (1 - 2 * (torch.rand(tries, generator=gen) < 0.5).double())
    u = _fp32(b / _silu(g))
    off = (_silu(g) * u / b - 1).abs()
    at = ((off < 2.0 ** -31) & (off > 2.0 ** -40)).nonzero()[:, 0][:n]
    assert len(at) == n
    return g[at], u[at]


def _near_power(gen, power, n):
    """n pairs whose h lies within 2^-31 below or above 2^power."""
    tries = 1 << 19
    g = _fp32(torch.rand(tries, generator=gen).double() * 6 + 0.5)
    u = _fp32(2.0 ** power / _silu(g))
    off = (_silu(g) * u * 2.0 ** -power - 1).abs()
    at = ((off < 2.0 ** -31) & (off > 2.0 ** -40)).nonzero()[:, 0][:n]
    assert len(at) == n
    return g[at], u[at]


def _rows(v, hidden):
    """MXFP4 rows whose product with ones at the first element of the first DIGITS blocks is v, exactly."""
    n = len(v)
    mant, e = torch.frexp(v.abs())
    whole = (mant * 2.0 ** 24).long()
    codes = torch.zeros((n, mx.blocks(hidden), 32), dtype=torch.uint8)
    scale = torch.full((n, mx.blocks(hidden)), 127, dtype=torch.uint8)
    code = torch.tensor([0, 2, 4, 5], dtype=torch.uint8)  # of 0, 1, 2, 3
    for i in range(DIGITS):
        codes[:, i, 0] = code[whole >> 2 * i & 3] + 8 * (v < 0).to(torch.uint8)
        scale[:, i] = (127 + e - 24 + 2 * i).to(torch.uint8)
    w = mx.pack(codes)
    assert torch.equal(mx.values(w, scale, hidden).sum(dim=1), v)
    return w, scale


def _layer(gen, hidden, ffn):
    """(g, u, the three matrices of one expert)."""
    g, u = _near_borders(gen, ffn)
    g, u = g.clone(), u.clone()
    for block in range(ffn // 32):
        at = block * 32
        if block % 3 == 0:    # a value that says the scale, and borders between codes
            g[at + 5], u[at + 5] = 8.0, 6.0 / 8.0
        elif block % 3 == 1:  # the largest lies next to a power of two
            a, b = _near_power(gen, 3, 1)
            g[at + 11], u[at + 11] = a[0], b[0]
    down = torch.zeros((hidden, mx.blocks(ffn), 32), dtype=torch.uint8)
    for c in range(ffn):
        down[c, c // 32, c % 32] = 2  # 1.0
    return g, u, [_rows(g, hidden), _rows(u, hidden),
                  (mx.pack(down), torch.full((hidden, mx.blocks(ffn)), 127, dtype=torch.uint8))]


def _run(dev, tokens, hidden, layer):
    x = torch.zeros((tokens, hidden))
    x[:, :DIGITS * 32:32] = 1.0
    n = torch.arange(tokens, dtype=torch.int32)
    r = wc.Routing(torch.zeros((tokens, 1), dtype=torch.int32), torch.ones((tokens, 1)),
                   torch.tensor([0, tokens], dtype=torch.int32), n)
    return wc.experts_mx_torch(x.to(dev), wc.Routing(*(t.to(dev) for t in r)),
                               *(t[None].to(dev) for pair in layer for t in pair)).cpu()


def _check(y, g, u):
    h = (_silu(g) * u)[None]
    c, b = mx.quantize(h)
    want = torch.zeros(y.shape[1], dtype=torch.float64)
    want[:len(g)] = mx.values(mx.pack(c), b, len(g))[0]
    wrong = (y.double() != want).sum(dim=0)
    assert not bool(wrong.any()), (int((wrong > 0).sum()), len(g))


# few tokens in two kernels; blocks of 64, 128 and 256 places; a row past what two kernels take
@pytest.mark.parametrize("tokens,hidden", [(1, 384), (16, 384), (3, 2304), (20, 384), (100, 384), (200, 384),
                                           (1, 8224), (2, 8224)])
@pytest.mark.parametrize("ffn", [384, 343])
def test_codes_next_to_borders(dev, tokens, hidden, ffn):
    g, u, layer = _layer(torch.Generator().manual_seed(ffn), hidden, ffn)
    _check(_run(dev, tokens, hidden, layer), g, u)
