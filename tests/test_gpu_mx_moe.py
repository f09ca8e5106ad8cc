"""GPU: wc_moe_mx where its first kernel has eight waves (more than 2048 columns of x): the choice
of experts by every number of logits to a lane, up to the width that a workgroup holds, and past
it, where the routing is a call of its own.  Results against the definition in 64 bits with the
experts that wc_route chooses, with the tolerance of test_gpu_mx_experts; the weights may differ
in their last bits between the numbers of lanes that a choice takes."""
import math

import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
import test_gpu_mx_experts as ex  # noqa: E402
from mx_reference import DT, UNIT  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _compare(dev, x, logits, k, layer, bias, more):
    banks = ex._on(dev, layer)
    on = None if bias is None else bias.to(dev)
    y = wc.moe_mx_torch(x.to(dev), logits.to(dev), k, *banks, bias=on, **more)
    r = wc.Routing(*(t.cpu() for t in wc.route_torch(logits.to(dev), k, bias=on, **more)))
    ref, tol = ex.reference(x, r, layer)
    slack = ex.reference(x, wc.Routing(r.ids, r.weights * 2.0 ** -20, r.offsets, r.order), layer)[0].abs()
    least = 2.0 ** -25 if y.dtype == torch.float16 else 1e-37
    off = (y.cpu().double() - ref).abs()
    tol = 1.01 * (tol + slack + UNIT[y.dtype] * ref.abs()) + least
    assert bool((off <= tol).all()), float((off / tol).max())
    return y


CHOICES = [
    (64, 6, dict(renormalize=False)), (61, 4, dict(score="sigmoid")), (128, 3, {}),
    (128, 8, dict(score="sigmoid", groups=8, top_groups=4, group_top=2, scale=2.5)),
    (256, 8, dict(groups=4, top_groups=2)), (512, 3, {}),
    (512, 32, dict(score="sigmoid", groups=16, top_groups=5, group_top=2))]


@pytest.mark.parametrize("tokens", [1, 7, 16])
@pytest.mark.parametrize("E,k,more", CHOICES)
def test_eight_waves(dev, tokens, E, k, more):
    hidden, ffn = 2049, 33
    g = torch.Generator().manual_seed(tokens + E)
    x = torch.randn((tokens, hidden), generator=g).to(list(DT.values())[tokens % 3])
    logits = torch.randn((tokens, E), generator=g)
    logits[:, 3] = -math.inf
    if tokens > 4:
        logits[4] = -math.inf  # no expert left
        logits[5, 6:] = -math.inf  # fewer than k
    bias = torch.randn(E, generator=g) * 0.1 if more.get("score") == "sigmoid" else None
    y = _compare(dev, x, logits, k, ex._layer(E, E, hidden, ffn), bias, more)
    if tokens > 4:
        assert not bool(y[4].any())


# the widest that the two kernels take, and the first that they do not
@pytest.mark.parametrize("tokens", [1, 16])
@pytest.mark.parametrize("hidden", [2048, 8192, 8193])
@pytest.mark.parametrize("E", [64, 512])
def test_widths(dev, tokens, hidden, E):
    g = torch.Generator().manual_seed(hidden)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    layer = ex._layer(E, E, hidden, 34)
    _compare(dev, x, torch.randn((tokens, E), generator=g), 2, layer, None, {})


def test_eight_waves_nan_logit_and_graph(dev):
    """A NaN logit makes its token's results NaN and no others; captured and replayed with other calls
    between the replays."""
    E, k, hidden, ffn, tokens = 256, 4, 2304, 64, 11
    banks = ex._on(dev, ex._layer(4, E, hidden, ffn))
    g = torch.Generator().manual_seed(3)
    xs = [torch.randn((tokens, hidden), generator=g).bfloat16().to(dev) for _ in range(2)]
    ls = [torch.randn((tokens, E), generator=g) for _ in range(2)]
    ls[1][6, 200] = float("nan")
    ls = [t.to(dev) for t in ls]
    want = [wc.moe_mx_torch(x, lo, k, *banks) for x, lo in zip(xs, ls)]
    bad = torch.arange(tokens) == 6
    assert not bool(torch.isnan(want[0]).any())
    assert torch.equal(torch.isnan(want[1]).all(dim=1).cpu(), bad) and torch.equal(torch.isnan(want[1]).any(dim=1).cpu(), bad)
    x, lo, y = xs[0].clone(), ls[0].clone(), torch.empty_like(xs[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wc.moe_mx_torch(x, lo, k, *banks, y=y)
    for i in (0, 1, 0, 1):
        x.copy_(xs[i])
        lo.copy_(ls[i])
        graph.replay()
        assert torch.equal(wc.moe_mx_torch(xs[0], ls[0], k, *banks), want[0])
        torch.cuda.synchronize()
        assert torch.equal(y.nan_to_num(7.0), want[i].nan_to_num(7.0))


def test_scale_beyond_fp32_is_refused(dev):
    """A factor of the weights that is no fp32 number is refused like any other argument."""
    E, hidden, ffn = 4, 96, 64
    layer = [t.to(dev) for pair in ex._layer(3, E, hidden, ffn) for t in pair]
    x, lo = torch.zeros((3, hidden), device=dev), torch.zeros((3, E), device=dev)
    for scale in (1e39, float("inf"), float("nan")):
        with pytest.raises(wc.WcError):
            wc.route_torch(lo, 2, scale=scale)
        with pytest.raises(wc.WcError):
            wc.moe_mx_torch(x, lo, 2, *layer, scale=scale)
