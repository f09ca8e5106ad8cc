"""GPU: mixture layers with MXFP4 experts in blocks of 16 places, straight from memory: up to 16
tokens that the two kernels of few tokens do not take (wider than 8192, or more than 32 slots a
token), and more codes of x than 32-bit offsets reach.  Tolerances are those of the other tests
of these layers (test_gpu_mx_experts)."""
import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
import test_gpu_mx_experts as ex  # noqa: E402
from mx_reference import DT  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("tokens,E,k,hidden,ffn", [
    (1, 3, 2, 8193, 96), (2, 3, 2, 8193, 96), (16, 5, 3, 8225, 33), (16, 1, 1, 8704, 64), (3, 40, 33, 8224, 31),
    (7, 40, 33, 96, 64), (16, 34, 34, 45, 545), (1, 2, 1, 65536, 1), (5, 2, 1, 9000, 1030)])
def test_sizes(dev, dtype, tokens, E, k, hidden, ffn):
    g = torch.Generator().manual_seed(tokens + hidden)
    x = torch.randn((tokens, hidden), generator=g).to(DT[dtype])
    r = ex._routing(ex._ids(g, tokens, E, k), torch.rand((tokens, k), generator=g) + 0.1, E)
    layer = ex._layer(hidden, E, hidden, ffn)
    ex._check(ex._run(dev, x, r, layer), x, r, layer)


@pytest.mark.parametrize("tokens", [4, 16])
def test_empty_slots_and_tokens(dev, tokens):
    """Slots without an expert, a token without any, an expert of two of a token's slots, so that it has
    more places than there are tokens."""
    E, k, hidden, ffn = 5, 3, 8257, 77
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    ids = ex._ids(g, tokens, E - 1, k)
    ids[:, 0] = 2
    ids[:, 2] = 2
    ids[1] = -1
    ids[tokens - 1] = torch.tensor([3, -1, 0])
    r = ex._routing(ids, torch.rand((tokens, k), generator=g), E)
    layer = ex._layer(1, E, hidden, ffn)
    y = ex._run(dev, x, r, layer)
    ex._check(y, x, r, layer)
    assert not bool(y[1].any())
    none = ex._routing(torch.full((tokens, k), -1), torch.ones((tokens, k)), E)
    assert not bool(ex._run(dev, x, none, layer).any())


def test_not_finite(dev):
    """A NaN or an infinity of a token, its weight or an expert's scales reaches that token's results, or
    those of the expert's tokens, and no others."""
    E, k, hidden, ffn, tokens = 4, 2, 8230, 65, 9
    g = torch.Generator().manual_seed(1)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    ids = ex._ids(g, tokens, E - 1, k)
    ids[3] = torch.tensor([3, 0])
    ids[4, 1] = -1
    weights = torch.rand((tokens, k), generator=g)
    x[0, 8229] = float("nan")
    x[1, 8192] = float("inf")
    weights[2, 0] = weights[4, 1] = float("nan")
    layer = ex._layer(1, E, hidden, ffn)
    layer[0][1][3, 64, 257] = 255
    y = ex._run(dev, x, ex._routing(ids, weights, E), layer).cpu()
    bad = torch.arange(tokens) < 5
    assert torch.equal(torch.isnan(y).all(dim=1), bad) and torch.equal(torch.isnan(y).any(dim=1), bad)


@pytest.mark.parametrize("tokens", [1, 13])
def test_strides_and_any_workspace(dev, tokens):
    """Rows of x and y inside larger tensors, experts apart; a workspace of NaN and one of zeros."""
    E, k, hidden, ffn = 3, 2, 8199, 75
    g = torch.Generator().manual_seed(tokens)
    big = torch.randn((tokens, hidden + 21), generator=g).half()
    x = big[:, 3:3 + hidden]
    r = ex._routing(ex._ids(g, tokens, E, k), torch.rand((tokens, k), generator=g), E)
    layer = ex._layer(2, E, hidden, ffn)
    apart = []
    for w, s in layer:
        W = torch.full((E, w.shape[1] + 1, w.shape[2]), 0x77, dtype=torch.uint8, device=dev)
        S = torch.full((E, s.shape[1] + 1, s.shape[2]), 255, dtype=torch.uint8, device=dev)
        W[:, :-1], S[:, :-1] = w.to(dev), s.to(dev)
        apart += [W[:, :-1], S[:, :-1]]
    on = wc.Routing(*(t.to(dev) for t in r))
    for fill in (0, 255):
        space = torch.full((1 << 24,), fill, dtype=torch.uint8, device=dev)
        Y = torch.full((tokens + 1, hidden + 9), 3.0, dtype=torch.float16, device=dev)
        wc.experts_mx_torch(big.to(dev)[:, 3:3 + hidden], on, *apart, y=Y[:tokens, 5:5 + hidden], workspace=space)
        ex._check(Y[:tokens, 5:5 + hidden], x, r, layer)
        Y[:tokens, 5:5 + hidden] = 3.0
        assert bool((Y == 3.0).all())


def test_garbage_routing_stays_inside(dev):
    E, k, hidden, ffn, tokens = 6, 2, 8224, 96, 11
    layer = ex._on(dev, ex._layer(7, E, hidden, ffn))
    g = torch.Generator().manual_seed(1)
    x = torch.randn((tokens, hidden), generator=g).bfloat16().to(dev)
    wild = lambda *shape: torch.randint(-2 ** 31, 2 ** 31 - 1, shape, generator=g,  # noqa: E731
                                        dtype=torch.int64).int().to(dev)
    Y = torch.full((tokens + 2, hidden), 5.0, dtype=torch.bfloat16, device=dev)
    need = wc.C.c_uint64(0)
    assert wc.lib().wc_experts_mx_workspace_bytes(tokens, k, E, hidden, ffn, wc.C.byref(need)) == 0
    space = torch.full((need.value + 4096,), 77, dtype=torch.uint8, device=dev)
    r = wc.Routing(wild(tokens, k), torch.rand((tokens, k), generator=g).to(dev), wild(E + 1), wild(tokens * k))
    wc.experts_mx_torch(x, r, *layer, y=Y[1:tokens + 1], workspace=space[:need.value])
    torch.cuda.synchronize()
    assert bool((space[need.value:] == 77).all())
    assert bool((Y[0] == 5.0).all()) and bool((Y[-1] == 5.0).all())


def test_codes_of_x_past_32_bits(dev):
    tokens, E, k, hidden, ffn = (1 << 16) + 21, 2, 1, 65536, 33
    if torch.cuda.mem_get_info(dev)[0] < 60 << 30:
        pytest.skip("needs 60 GiB")
    g = torch.Generator().manual_seed(1)
    base = torch.randn((64, hidden), generator=g).bfloat16()
    x = torch.empty((tokens, hidden), dtype=torch.bfloat16, device=dev)
    for i in range(0, tokens, 64):
        x[i:i + 64] = base[:min(64, tokens - i)].to(dev) if i in (0, tokens // 64 * 64) else x[:64]
    x[-1] = base[5].to(dev) * 3
    ids = (torch.rand((tokens, 1), generator=g) < 0.5).long()
    weights = torch.rand((tokens, 1), generator=g) + 0.1
    r = ex._routing(ids, weights, E)
    layer = ex._layer(3, E, hidden, ffn)
    y = wc.experts_mx_torch(x, wc.Routing(*(t.to(dev) for t in r)), *ex._on(dev, layer))
    some = torch.tensor([0, 1, 63, 32767, 65535, 65536, tokens - 2, tokens - 1])
    ex._check(y[some.to(dev)], x[some.to(dev)].cpu(), ex._routing(ids[some], weights[some], E), layer)
