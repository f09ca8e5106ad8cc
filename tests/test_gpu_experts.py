"""GPU: wc_experts_i8 against the definition in 64 bits.

The reference quantises x by the fp32 formula (bit for bit, as tests of wc_quantize_i8
establish) and everything after it in 64 bits.  Two things separate a result from it:

* roundings: h is a product of two fp32 products and a silu (|gate x| < 5 here), of error under
  2^-19; a down product, its scales, the weights and the sum over the slots add under
  (k + 8) 2^-24 each of the terms' magnitudes; y is rounded once to its type;
* codes of h next to a half: |h / step| <= 127, so an error of 2^-19 moves a quotient
  by less than 127 2^-18 = 5e-4 (with the step's own error), and a code within that of
  a half may be the next one.  Each such code adds one step times its weight's magnitude
  to the tolerance of a result.
"""
import math

import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
NEAR = 5e-4


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _bank(g, E, n, k, dtype):
    return (torch.randint(-128, 128, (E, n, k), generator=g, dtype=torch.int8),
            (torch.rand((E, n), generator=g) * 0.002 / math.sqrt(k) + 1e-5).to(DT[dtype]))


def _layer(seed, E, hidden, ffn, scales="fp16"):
    g = torch.Generator().manual_seed(seed)
    return [_bank(g, E, ffn, hidden, scales), _bank(g, E, ffn, hidden, scales),
            _bank(g, E, hidden, ffn, scales)]


def _routing(ids, weights, E):
    flat = ids.flatten().long()
    flat = torch.where(flat < 0, E, flat)
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    return wc.Routing(ids.int(), weights.float(), offsets.int(),
                      torch.sort(flat, stable=True)[1].int())


def _ids(g, tokens, E, k):
    return torch.argsort(torch.rand((tokens, E), generator=g), dim=1)[:, :k]


def _quantised(x):
    x = x.float()
    top = x.abs().amax(dim=1)
    none = top < 1e-30
    # (a number divided by a tensor is the tensor's reciprocal times the number: rounded twice)
    inv = torch.where(none, torch.zeros(()), torch.full_like(top, 127.0) / top)
    return torch.round(x * inv[:, None]).clamp(-127, 127).double(), \
        torch.where(none, torch.zeros(()), top / torch.full_like(top, 127.0)).double()


def reference(x, r, layer):
    """y in 64 bits and how far a result may be from it."""
    (gate, gs), (up, us), (down, ds) = layer
    T, hidden = x.shape
    k, E = r.ids.shape[1], gate.shape[0]
    y = torch.zeros((T, hidden), dtype=torch.float64)
    tol = torch.zeros_like(y)
    q, s = _quantised(x)
    for e in range(E):
        t, j = (r.ids == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        a = (q[t] @ gate[e].double().T) * s[t][:, None] * gs[e].double()
        b = (q[t] @ up[e].double().T) * s[t][:, None] * us[e].double()
        h = a / (1 + torch.exp(-a)) * b
        step = h.abs().amax(dim=1, keepdim=True) / 127
        quot = torch.where(step < 1e-30 / 127, torch.zeros(()).double(), h / step)
        codes = torch.round(quot)
        unsure = ((quot - quot.floor() - 0.5).abs() < NEAR).double()
        w = r.weights.double()[t, j][:, None]
        m = down[e].double()
        o = (codes @ m.T) * step * ds[e].double()
        mag = (codes.abs() @ m.abs().T) * step * ds[e].double()
        flips = (unsure @ m.abs().T) * step * ds[e].double()
        y.index_add_(0, t, o * w)
        # the step's own error scales a whole row of results
        tol.index_add_(0, t, (flips + o.abs() * 2.0 ** -18 + mag * (k + 8) * 2.0 ** -24) * w.abs())
    return y, tol


def _check(y, x, r, layer):
    ref, tol = reference(x, r, layer)
    tol = 1.01 * (tol + UNIT[y.dtype] * ref.abs()) + (2.0 ** -25 if y.dtype == torch.float16 else 1e-37)
    off = (y.cpu().double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


def _run(dev, x, r, layer, **more):
    banks = [t.to(dev) for pair in layer for t in pair]
    return wc.experts_i8_torch(x.to(dev), wc.Routing(*(t.to(dev) for t in r)), *banks, **more)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("tokens,E,k,hidden,ffn", [
    (1, 1, 1, 1, 1), (1, 4, 2, 64, 48), (3, 8, 8, 130, 257), (16, 2, 1, 128, 128),
    (17, 2, 2, 100, 300), (65, 5, 3, 272, 96), (33, 64, 6, 256, 160), (128, 3, 2, 515, 129),
    (300, 8, 2, 384, 512), (520, 4, 2, 256, 640), (40, 100, 1, 31, 17), (2, 16, 4, 2048, 1408),
    (1200, 2, 1, 160, 144), (800, 2, 2, 272, 304), (900, 2, 1, 131, 77),
    (2, 8, 2, 84, 60), (20, 4, 2, 140, 92), (300, 4, 2, 204, 132),
    (300, 4, 2, 203, 130), (4, 4, 2, 129, 66), (1300, 3, 1, 97, 258),
    (3000, 2, 1, 515, 640), (4100, 3, 2, 515, 386), (3000, 5, 2, 260, 1100), (6000, 3, 1, 256, 512)])
def test_sizes(dev, dtype, tokens, E, k, hidden, ffn):
    g = torch.Generator().manual_seed(tokens + E)
    x = torch.randn((tokens, hidden), generator=g).to(DT[dtype])
    layer = _layer(E, E, hidden, ffn)
    r = _routing(_ids(g, tokens, E, k), torch.rand((tokens, k), generator=g), E)
    y = _run(dev, x, r, layer)
    assert y.dtype == x.dtype
    _check(y, x, r, layer)


@pytest.mark.parametrize("scales", list(DT))
@pytest.mark.parametrize("tokens", [5, 150])
def test_scale_types(dev, scales, tokens):
    g = torch.Generator().manual_seed(3)
    x = torch.randn((tokens, 200), generator=g).bfloat16()
    layer = _layer(1, 6, 200, 144, scales)
    r = _routing(_ids(g, tokens, 6, 2), torch.rand((tokens, 2), generator=g), 6)
    _check(_run(dev, x, r, layer), x, r, layer)


@pytest.mark.parametrize("tokens", [2, 40, 400])
def test_skewed_and_empty(dev, tokens):
    """All rows on one expert, experts without rows, slots and tokens without experts."""
    g = torch.Generator().manual_seed(tokens)
    E, k, hidden, ffn = 9, 2, 144, 208
    layer = _layer(2, E, hidden, ffn)
    x = torch.randn((tokens, hidden), generator=g)
    ids = torch.full((tokens, k), -1)
    ids[:, 0] = 4
    ids[::3, 1] = 8
    ids[1::5] = -1
    weights = torch.where(ids < 0, torch.zeros(()), torch.rand((tokens, k), generator=g))
    r = _routing(ids, weights, E)
    y = _run(dev, x, r, layer)
    _check(y, x, r, layer)
    assert not bool(y[1::5].any())
    # nothing routed at all
    r = _routing(torch.full((tokens, k), -1), torch.zeros((tokens, k)), E)
    assert not bool(_run(dev, x, r, layer).any())
    # a NaN weight of an empty slot makes its token NaN, as the router meant it
    r.weights[0] = math.nan
    y = _run(dev, x, r, layer)
    assert bool(torch.isnan(y[0]).all()) and not bool(y[1:].any())


def test_uneven_and_many(dev):
    """Many rows to an expert on average, and one expert with 3, one with none."""
    g = torch.Generator().manual_seed(11)
    tokens, E, hidden, ffn = 4100, 5, 515, 386
    layer = _layer(4, E, hidden, ffn)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    ids = torch.tensor([[0, 3]]).repeat(tokens, 1)
    ids[2000:, 1] = 4
    ids[77:80, 0] = 1
    ids[500::7, 1] = -1
    weights = torch.where(ids < 0, torch.zeros(()), torch.rand((tokens, 2), generator=g))
    r = _routing(ids, weights, E)
    _check(_run(dev, x, r, layer), x, r, layer)


@pytest.mark.parametrize("tokens", [4, 200])
def test_bad_rows_stay_their_own(dev, tokens):
    """A token with a NaN or an infinity is NaN, the others are as without it."""
    g = torch.Generator().manual_seed(1)
    layer = _layer(5, 3, 96, 80)
    x = torch.randn((tokens, 96), generator=g)
    r = _routing(_ids(g, tokens, 3, 2), torch.rand((tokens, 2), generator=g), 3)
    clean = _run(dev, x, r, layer)
    x[1, 5] = math.nan
    x[3, 90] = math.inf
    y = _run(dev, x, r, layer)
    assert bool(torch.isnan(y[[1, 3]]).all())
    keep = [t for t in range(tokens) if t not in (1, 3)]
    assert torch.equal(y[keep], clean[keep])


def test_strides_views_and_interleaved_banks(dev):
    """x and y as slices; gate and up as the halves of one tensor per expert."""
    g = torch.Generator().manual_seed(8)
    E, hidden, ffn, T = 4, 129, 70, 45
    layer = _layer(7, E, hidden, ffn)
    both = torch.cat([layer[0][0], layer[1][0]], dim=1).to(dev)  # E x 2 ffn x hidden
    wide = torch.randn((T, hidden + 7), generator=g).half().to(dev)
    x = wide[:, 5:5 + hidden]
    r = _routing(_ids(g, T, E, 2), torch.rand((T, 2), generator=g), E)
    out = torch.full((T + 2, hidden + 3), 7.0, dtype=torch.half, device=dev)
    y = out[1:-1, 1:1 + hidden]
    wc.experts_i8_torch(x, wc.Routing(*(t.to(dev) for t in r)), both[:, :ffn], layer[0][1].to(dev),
                        both[:, ffn:], layer[1][1].to(dev), layer[2][0].to(dev),
                        layer[2][1].to(dev), y=y)
    _check(y, x.cpu(), r, layer)
    out[1:-1, 1:1 + hidden] = 7.0
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("tokens", [1, 24, 260])
def test_a_stream_a_graph_and_repeats(dev, tokens):
    g = torch.Generator().manual_seed(tokens)
    E, k, hidden, ffn = 8, 2, 256, 320
    layer = _layer(3, E, hidden, ffn)
    banks = [t.to(dev) for pair in layer for t in pair]
    xs = [torch.randn((tokens, hidden), generator=g).bfloat16().to(dev) for _ in range(4)]
    logits = [torch.randn((tokens, E), generator=g).to(dev) for _ in range(4)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = wc.route_torch(logits[0], k, stream=side)
    y = wc.experts_i8_torch(xs[0], r, *banks, stream=side)
    side.synchronize()
    eager = [wc.experts_i8_torch(x, wc.route_torch(v, k), *banks) for x, v in zip(xs, logits)]
    assert torch.equal(y, eager[0])
    _check(y, xs[0].cpu(), wc.Routing(*(t.cpu() for t in r)), layer)
    x, v, out = xs[0].clone(), logits[0].clone(), torch.zeros_like(xs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wc.experts_i8_torch(x, wc.route_torch(v, k), *banks, y=out)
    for i in (0, 1, 2, 3, 1):
        x.copy_(xs[i])
        v.copy_(logits[i])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i])


def test_broken_routing_stays_in_bounds(dev):
    """Offsets and an order that no router wrote: the result is meaningless, but a
    buffer around every argument is untouched and the call ends."""
    g = torch.Generator().manual_seed(2)
    E, T, k = 5, 30, 2
    layer = _layer(4, E, 64, 96)
    x = torch.randn((T, 64), generator=g)
    r = _routing(_ids(g, T, E, k), torch.rand((T, k), generator=g), E)
    out = torch.full((T + 2, 64), 7.0, device=dev)
    for offsets in ([0, 10, 5, 70, 2 ** 31 - 1, -3], [60] * 6, [-5, 60, 60, 60, 60, 60]):
        bad = wc.Routing(r.ids, r.weights, torch.tensor(offsets, dtype=torch.int32),
                         torch.randint(-2 ** 31, 2 ** 31 - 1, (T * k,), generator=g).int())
        _run(dev, x, bad, layer, y=out[1:-1])
        torch.cuda.synchronize()
        assert bool((out[0] == 7.0).all()) and bool((out[-1] == 7.0).all())


def test_refusals(dev):
    layer = [t.to(dev) for pair in _layer(1, 4, 64, 32) for t in pair]
    x = torch.zeros((3, 64), device=dev)
    r = wc.route_torch(torch.zeros((3, 4), device=dev), 2)

    def call(x=x, r=r, at=None, to=None, **more):
        args = list(layer)
        if at is not None:
            args[at] = to
        return wc.experts_i8_torch(x, r, *args, **more)
    assert not bool(call().any())
    for bad in (dict(x=x.double()), dict(x=x[:2]), dict(x=x[:, :60]), dict(x=x.T),
                dict(r=r._replace(ids=r.ids.long())), dict(r=r._replace(offsets=r.offsets[:4])),
                dict(r=r._replace(order=r.order[:5])), dict(r=r._replace(weights=r.weights.half())),
                dict(at=0, to=layer[0].float()), dict(at=2, to=layer[2][:3]),
                dict(at=4, to=layer[4][:, :, :30]), dict(at=1, to=layer[1][:, :30]),
                dict(at=3, to=layer[3].double()), dict(y=torch.zeros((3, 64), device=dev).half()),
                dict(y=torch.zeros((2, 64), device=dev)),
                dict(workspace=torch.zeros(100, dtype=torch.uint8, device=dev))):
        with pytest.raises(ValueError):
            call(**bad)
    none = wc.experts_i8_torch(torch.zeros((0, 64), device=dev),
                               wc.route_torch(torch.zeros((0, 4), device=dev), 2), *layer)
    assert tuple(none.shape) == (0, 64)


@pytest.mark.parametrize("tokens", [1, 2, 4, 5, 10, 40, 300])
@pytest.mark.parametrize("ffn", [8, 256, 768, 1024, 1408])
def test_empty_slots_anywhere(dev, tokens, ffn):
    """Empty slots before, between and after used ones, with weights of their own that count
    for nothing: few tokens slot by slot, few rows to an expert, many."""
    g = torch.Generator().manual_seed(tokens * ffn)
    E, k, hidden = 40, 8, 256
    layer = _layer(6, E, hidden, ffn)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    for empty in (torch.tensor([1, 0, 0, 0, 0, 0, 0, 0]), torch.tensor([0, 0, 0, 1, 0, 0, 0, 0]),
                  torch.tensor([1, 1, 1, 1, 1, 1, 1, 0]), torch.rand((tokens, k), generator=g) < 0.5):
        ids = torch.where(empty.bool().expand(tokens, k), -1, _ids(g, tokens, E, k))
        r = _routing(ids, torch.rand((tokens, k), generator=g), E)
        _check(_run(dev, x, r, layer), x, r, layer)


@pytest.mark.parametrize("tokens,off", [(1, 0), (4, 0), (20, 0), (20, 1)])
@pytest.mark.parametrize("low", [-80, -24])
def test_silu_over_its_range(dev, tokens, off, low):
    """h to fp32's precision, where the exponential is largest and where it is least: slot by
    slot, few rows to an expert, many, and matrices that start at different bytes.

    Expert e has one value of h, which reaches y's column e alone: gate x = 127/128 times a
    code and up x = 8128, both exact.  h is an exponential (2 ulp, 2^-22), a sum, a quotient
    and a product; then its code is 127, and h / 127, the down product, and the slot's weight
    are a rounding each.  2^-22 + 6 2^-24 = 10 2^-24, and 1 % for products of these.
    """
    g = torch.Generator().manual_seed(tokens + low)
    E, k, hidden, ffn = 64, 32, 64, 8
    code = torch.cat([torch.tensor([low, 87, -1, 0, 1]), torch.randint(low, 88, (E - 5,), generator=g)])
    gate, up = torch.zeros((2, E, ffn, hidden), dtype=torch.int8)
    down = torch.zeros((E, hidden, ffn), dtype=torch.int8)
    gate[:, 3, 5] = code.to(torch.int8)
    up[:, 3, 5] = 1
    down[torch.arange(E), torch.arange(E), 3] = 100
    one = torch.ones((E, ffn))
    layer = [(gate, one), (up, one * 8192), (down, torch.ones((E, hidden)))]
    banks = [t.to(dev) for pair in layer for t in pair]
    # gate at another byte of a dword than up, as a view of a larger buffer
    flat = torch.zeros(gate.numel() + 16, dtype=torch.int8, device=dev)
    flat[off:off + gate.numel()] = banks[0].flatten()
    banks[0] = flat[off:off + gate.numel()].view(gate.shape)
    x = torch.zeros((tokens, hidden))
    x[:, 5] = 127 / 128  # its code 127, its scale 2^-7
    r = _routing(_ids(g, tokens, E, k), torch.rand((tokens, k), generator=g) + 0.5, E)
    y = wc.experts_i8_torch(x.to(dev), wc.Routing(*(t.to(dev) for t in r)), *banks).cpu().double()
    a = code.double() * 127 / 128
    h = a / (1 + torch.exp(-a)) * (127 / 128 * 8192)
    assert bool(((h.abs() > 1e-29) | (h == 0)).all())  # none of them counts as a row of zeros
    ref = torch.zeros((tokens, E), dtype=torch.float64)
    ref.scatter_(1, r.ids.long(), r.weights.double() * (100 * h)[r.ids.long()])
    assert bool(((y - ref).abs() <= 1.01 * 10 * 2.0 ** -24 * ref.abs()).all()), \
        float(((y - ref).abs() / ref.abs().clamp_min(1e-300)).max())
