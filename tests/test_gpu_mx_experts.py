"""GPU: mixture layers with MXFP4 experts (wc_experts_mx, wc_moe_mx) against the definition in 64
bits.

x is quantised exactly.  What separates a result from the reference:
* roundings: gate x and up x are fp32 sums of blocks (as in the tests of wc_linear_mx; the
  layers here keep them exact or nearly), silu and the product of h are off by less than
  2^-19 (|gate x| < 30); a down product, the weights and the sum over the slots add under
  (blocks + k + 40) 2^-23 of the terms' magnitudes; y is rounded once to its type;
* codes of h: one within 2^-18 of a border between codes, or in a block whose largest
  magnitude is within 2^-18 of a power of two, may be another.  The tolerance takes the
  furthest of the codes that h (1 - 2^-18) and h (1 + 2^-18) have under either scale.
"""
import math

import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
import mx_reference as mx  # noqa: E402
from mx_reference import DT, UNIT  # noqa: E402

pytestmark = pytest.mark.gpu
D = 2.0 ** -18


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _bank(g, E, n, k):
    base = 125 - round(math.log2(k) / 2)
    pairs = [mx.matrix(g, n, k, base=base) for _ in range(E)]
    return torch.stack([w for w, _ in pairs]), torch.stack([s for _, s in pairs])


def _layer(seed, E, hidden, ffn):
    g = torch.Generator().manual_seed(seed)
    return [_bank(g, E, ffn, hidden), _bank(g, E, ffn, hidden), _bank(g, E, hidden, ffn)]


def _routing(ids, weights, E):
    flat = ids.flatten().long()
    flat = torch.where(flat < 0, E, flat)
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    return wc.Routing(ids.int(), weights.float(), offsets.int(),
                      torch.sort(flat, stable=True)[1].int())


def _ids(g, tokens, E, k):
    return torch.argsort(torch.rand((tokens, E), generator=g), dim=1)[:, :k]


def _h_codes(h):
    """(values of h in MXFP4, how far other codes of it may be)."""
    p = mx.padded(h)
    sure = mx.exponents(p)

    def at(v, byte):
        scale = mx.power(byte)[..., None]
        return mx.GRID[mx.nearest(v.abs() / scale).long()] * v.sign() * scale
    v = at(p, sure)
    far = torch.zeros_like(v)
    for byte in (mx.exponents(p * (1 - D)), mx.exponents(p * (1 + D))):
        for d in (1 - D, 1 + D):
            far = torch.maximum(far, (at(p * d, byte) - v).abs())
    return v.flatten(1)[:, :h.shape[1]], far.flatten(1)[:, :h.shape[1]]


def reference(x, r, layer):
    (gate, gs), (up, us), (down, ds) = layer
    T, hidden = x.shape
    k, E, ffn = r.ids.shape[1], gate.shape[0], gate.shape[1]
    y = torch.zeros((T, hidden), dtype=torch.float64)
    tol = torch.zeros_like(y)
    c, b = mx.quantize(x)
    xv = mx.values(mx.pack(c), b, hidden)
    for e in range(E):
        t, j = (r.ids == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        a = xv[t] @ mx.values(gate[e], gs[e], hidden).T
        h = a * torch.sigmoid(a) * (xv[t] @ mx.values(up[e], us[e], hidden).T)
        v, far = _h_codes(h)
        w = r.weights.double()[t, j][:, None]
        m = mx.values(down[e], ds[e], ffn)
        o = v @ m.T
        y.index_add_(0, t, o * w)
        tol.index_add_(0, t, (far @ m.abs().T + (v.abs() @ m.abs().T) * (mx.blocks(ffn) + k + 40) * 2.0 ** -23)
                       * w.abs())
    return y, tol


def _check(y, x, r, layer):
    ref, tol = reference(x, r, layer)
    tol = 1.01 * (tol + UNIT[y.dtype] * ref.abs()) + (2.0 ** -25 if y.dtype == torch.float16 else 1e-37)
    off = (y.cpu().double() - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


def _on(dev, layer):
    return [t.to(dev) for pair in layer for t in pair]


def _run(dev, x, r, layer, **more):
    return wc.experts_mx_torch(x.to(dev), wc.Routing(*(t.to(dev) for t in r)), *_on(dev, layer), **more)


SIZES = [(1, 1, 1, 1, 1), (1, 4, 2, 64, 48), (3, 8, 8, 130, 257), (16, 2, 1, 128, 128),
         (16, 64, 6, 544, 96), (17, 2, 2, 100, 300), (65, 5, 3, 272, 96), (33, 64, 6, 256, 160),
         (128, 3, 2, 515, 129), (300, 8, 2, 384, 512), (520, 4, 2, 256, 640), (40, 100, 1, 31, 17),
         (2, 16, 4, 2048, 1408), (1200, 2, 1, 160, 144), (900, 2, 1, 131, 77), (10, 40, 33, 96, 64),
         (1300, 3, 1, 97, 258), (3000, 2, 1, 515, 640), (2500, 5, 2, 1056, 352), (4, 4, 2, 8192, 64),
         (3, 3, 2, 8193, 96), (16, 300, 8, 2049, 33), (5, 2, 1, 4097, 700), (100, 4, 2, 1024, 2048)]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("tokens,E,k,hidden,ffn", SIZES)
def test_sizes(dev, dtype, tokens, E, k, hidden, ffn):
    g = torch.Generator().manual_seed(tokens + E)
    x = torch.randn((tokens, hidden), generator=g).to(DT[dtype])
    r = _routing(_ids(g, tokens, E, k), torch.rand((tokens, k), generator=g) + 0.1, E)
    layer = _layer(hidden, E, hidden, ffn)
    y = _run(dev, x, r, layer)
    assert y.dtype == DT[dtype]
    _check(y, x, r, layer)


@pytest.mark.parametrize("tokens", [4, 16, 90, 700])
def test_empty_slots_and_tokens(dev, tokens):
    """Slots without an expert, tokens without any, experts without tokens, a token with the same
    expert twice."""
    E, k, hidden, ffn = 9, 3, 192, 160
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    ids = _ids(g, tokens, E - 2, k)
    ids[:, 2][torch.rand(tokens, generator=g) < 0.5] = -1
    ids[1] = -1
    ids[tokens - 1] = torch.tensor([5, -1, 5])
    weights = torch.rand((tokens, k), generator=g)
    r = _routing(ids, weights, E)
    layer = _layer(1, E, hidden, ffn)
    y = _run(dev, x, r, layer)
    _check(y, x, r, layer)
    assert not bool(y[1].any())
    # nothing to do at all
    none = _routing(torch.full((tokens, k), -1), weights, E)
    assert not bool(_run(dev, x, none, layer).any())


@pytest.mark.parametrize("tokens", [5, 60, 500])
def test_not_finite(dev, tokens):
    """A NaN in a token's x or weights, or in an expert's scales, reaches that token's results, or
    those of the expert's tokens, and no others."""
    E, k, hidden, ffn = 4, 2, 160, 128
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    ids = _ids(g, tokens, E - 1, k)
    ids[3] = torch.tensor([3, 0])
    ids[4, 1] = -1
    weights = torch.rand((tokens, k), generator=g)
    x[0, 7] = float("nan")
    x[1, 159] = float("inf")
    weights[2, 0] = float("nan")
    weights[4, 1] = float("nan")
    layer = _layer(1, E, hidden, ffn)
    layer[0][1][3, 5, 1] = 255  # a row of expert 3's gate
    y = _run(dev, x, _routing(ids, weights, E), layer)
    bad = torch.zeros(tokens, dtype=torch.bool)
    bad[:5] = True
    assert torch.equal(torch.isnan(y.cpu()).all(dim=1), bad)
    assert torch.equal(torch.isnan(y.cpu()).any(dim=1), bad)


@pytest.mark.parametrize("tokens", [3, 40, 400])
def test_strides(dev, tokens):
    """Rows of x and y and experts of the banks inside larger tensors."""
    E, k, hidden, ffn = 5, 2, 173, 141
    g = torch.Generator().manual_seed(tokens)
    big = torch.randn((tokens, hidden + 21), generator=g).half()
    x = big[:, 3:3 + hidden]
    r = _routing(_ids(g, tokens, E, k), torch.rand((tokens, k), generator=g), E)
    layer = _layer(2, E, hidden, ffn)
    apart = []
    for w, s in layer:
        W = torch.full((E, w.shape[1] + 1, w.shape[2]), 0x77, dtype=torch.uint8, device=dev)
        S = torch.full((E, s.shape[1] + 1, s.shape[2]), 255, dtype=torch.uint8, device=dev)
        W[:, :-1], S[:, :-1] = w.to(dev), s.to(dev)
        apart += [W[:, :-1], S[:, :-1]]
    Y = torch.full((tokens + 1, hidden + 9), 3.0, dtype=torch.float16, device=dev)
    wc.experts_mx_torch(big.to(dev)[:, 3:3 + hidden], wc.Routing(*(t.to(dev) for t in r)), *apart,
                        y=Y[:tokens, 5:5 + hidden])
    _check(Y[:tokens, 5:5 + hidden], x, r, layer)
    Y[:tokens, 5:5 + hidden] = 3.0
    assert bool((Y == 3.0).all())


@pytest.mark.parametrize("tokens", [1, 7, 16, 17, 100])
@pytest.mark.parametrize("E,k,more", [
    (8, 2, {}), (64, 6, dict(renormalize=False)), (61, 4, dict(score="sigmoid")),
    (128, 8, dict(score="sigmoid", groups=8, top_groups=4, group_top=2, scale=2.5)),
    (256, 8, dict(groups=4, top_groups=2)), (512, 3, {})])
def test_moe_is_route_and_experts(dev, tokens, E, k, more):
    hidden, ffn = 224, 96
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    logits = torch.randn((tokens, E), generator=g)
    logits[:, 3] = -math.inf
    if tokens > 4:
        logits[4] = -math.inf  # no expert left
    bias = torch.randn(E, generator=g) * 0.1 if more.get("score") == "sigmoid" else None
    layer = _layer(tokens, E, hidden, ffn)
    on = None if bias is None else bias.to(dev)
    y = wc.moe_mx_torch(x.to(dev), logits.to(dev), k, *_on(dev, layer), bias=on, **more)
    r = wc.route_torch(logits.to(dev), k, bias=on, **more)
    z = wc.experts_mx_torch(x.to(dev), r, *_on(dev, layer))
    cpu = wc.Routing(*(t.cpu() for t in r))
    _check(z, x, cpu, layer)
    # the choice's weights may differ in their last bits between the number of lanes it takes
    w = r.weights.cpu()
    ref, tol = reference(x, cpu, layer)
    off = (y.cpu().double() - ref).abs()
    slack = reference(x, wc.Routing(cpu.ids, w * 2.0 ** -20, cpu.offsets, cpu.order), layer)[0].abs()
    assert bool((off <= 1.01 * (tol + slack + UNIT[y.dtype] * ref.abs()) + 1e-30).all())
    if tokens > 4:
        assert not bool(y[4].any())


@pytest.mark.parametrize("dtype", list(DT))
def test_moe_types(dev, dtype):
    """Activations and logits of every type, logits inside wider rows."""
    E, k, hidden, ffn = 16, 3, 288, 160
    layer = _layer(4, E, hidden, ffn)
    g = torch.Generator().manual_seed(3)
    for tokens in (2, 50):
        x = torch.randn((tokens, hidden), generator=g).to(DT[dtype])
        for lt in DT.values():
            wide = torch.randn((tokens, E + 5), generator=g).to(lt).to(dev)
            logits = wide[:, 2:2 + E]
            y = wc.moe_mx_torch(x.to(dev), logits, k, *_on(dev, layer))
            r = wc.route_torch(logits, k)
            assert y.dtype == DT[dtype]
            _check(y, x, wc.Routing(*(t.cpu() for t in r)), layer)


def test_moe_nan_logit(dev):
    E, k, hidden, ffn = 16, 2, 96, 64
    layer = _on(dev, _layer(4, E, hidden, ffn))
    for tokens in (3, 40):
        g = torch.Generator().manual_seed(3)
        x = torch.randn((tokens, hidden), generator=g).to(dev)
        logits = torch.randn((tokens, E), generator=g)
        logits[1, 5] = float("nan")
        y = wc.moe_mx_torch(x, logits.to(dev), k, *layer)
        assert bool(torch.isnan(y[1]).all()) and not bool(torch.isnan(y[0]).any()) \
            and not bool(torch.isnan(y[2:]).any())


@pytest.mark.parametrize("tokens", [1, 16, 60, 600])
def test_streams_graphs_and_runs(dev, tokens):
    """On another stream; two captured calls that share a workspace, replayed with eager calls between;
    the same bits on every run."""
    E, k, hidden, ffn = 8, 2, 320, 192
    layer = _on(dev, _layer(7, E, hidden, ffn))
    g = torch.Generator().manual_seed(tokens)
    xs = [torch.randn((tokens, hidden), generator=g).bfloat16().to(dev) for _ in range(3)]
    ls = [torch.randn((tokens, E), generator=g).to(dev) for _ in range(3)]
    want = [wc.moe_mx_torch(x, lo, k, *layer).clone() for x, lo in zip(xs, ls)]
    for x, lo, w in zip(xs, ls, want):
        assert torch.equal(wc.moe_mx_torch(x, lo, k, *layer), w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = wc.moe_mx_torch(xs[1], ls[1], k, *layer, stream=side)
    side.synchronize()
    assert torch.equal(got, want[1])
    x, lo = xs[0].clone(), ls[0].clone()
    ya, yb = torch.empty_like(want[0]), torch.empty_like(want[0])
    space = torch.empty(1 << 26, dtype=torch.uint8, device=dev)
    a, b = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(a):
        wc.moe_mx_torch(x, lo, k, *layer, y=ya, workspace=space)
    with torch.cuda.graph(b):
        wc.moe_mx_torch(x, lo, k, *layer, y=yb, workspace=space)
    for i in (0, 1, 2, 1, 0):
        x.copy_(xs[i])
        lo.copy_(ls[i])
        a.replay()
        b.replay()
        assert torch.equal(wc.moe_mx_torch(xs[2], ls[2], k, *layer), want[2])
        torch.cuda.synchronize()
        assert torch.equal(ya, want[i]) and torch.equal(yb, want[i])
        space.fill_(255)


def test_same_order_in_any_workspace(dev):
    """A workspace full of NaN and one of zeros: nothing in it is read before it is written."""
    E, k = 5, 2
    for tokens, hidden, ffn in ((7, 100, 70), (90, 100, 70), (500, 1000, 200)):
        layer = _on(dev, _layer(7, E, hidden, ffn))
        g = torch.Generator().manual_seed(tokens)
        x = torch.randn((tokens, hidden), generator=g).to(dev)
        r = _routing(_ids(g, tokens, E, k), torch.rand((tokens, k), generator=g), E)
        r = wc.Routing(*(t.to(dev) for t in r))
        ys = []
        for fill in (0, 255):
            space = torch.full((1 << 26,), fill, dtype=torch.uint8, device=dev)
            ys.append(wc.experts_mx_torch(x, r, *layer, workspace=space))
        assert torch.equal(*ys) and not bool(torch.isnan(ys[0]).any())


def test_garbage_routing_stays_inside(dev):
    """Entries out of range are taken as the nearest in range: the results are wrong, the memory
    around the arguments is as it was."""
    E, k, hidden, ffn = 6, 2, 128, 96
    layer = _on(dev, _layer(7, E, hidden, ffn))
    g = torch.Generator().manual_seed(1)
    for tokens in (5, 70, 500):
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


@pytest.mark.parametrize("tokens", [2, 50, 400])
def test_layer_together(dev, tokens):
    """A block's run: q, k and v, then the mixture layer on the sum, through the public calls."""
    E, k, hidden, ffn = 8, 2, 256, 224
    g = torch.Generator().manual_seed(tokens)
    mats = [mx.matrix(g, n, hidden) for n in (256, 64, 64)]
    layer = _layer(3, E, hidden, ffn)
    router = torch.randn((E, hidden), generator=g).bfloat16()
    x = torch.randn((tokens, hidden), generator=g).bfloat16()
    q, _, v = wc.linear_mx_torch(x.to(dev), [w.to(dev) for w, _ in mats], [s.to(dev) for _, s in mats])
    mid = (x.to(dev) + q / 64).contiguous()
    logits = mid.float() @ router.to(dev).float().T
    y = wc.moe_mx_torch(mid, logits, k, *_on(dev, layer))
    r = wc.route_torch(logits, k)
    assert v.shape == (tokens, 64)
    _check(y, mid.cpu(), wc.Routing(*(t.cpu() for t in r)), layer)


def test_bank_past_32_bits(dev):
    """Experts behind 2^32 bytes of a bank."""
    E, k, hidden, ffn, tokens = 300, 1, 8192, 4096, 3
    g = torch.Generator(device=dev).manual_seed(1)

    def bank(n, kk):
        w = torch.randint(0, 256, (E, n, kk // 2), generator=g, device=dev, dtype=torch.uint8)
        return w, torch.randint(118, 121, (E, n, kk // 32), generator=g, device=dev, dtype=torch.uint8)
    layer = [bank(ffn, hidden), bank(ffn, hidden), bank(hidden, ffn)]
    cpu = torch.Generator().manual_seed(1)
    for T in (tokens, 20):
        x = torch.randn((T, hidden), generator=cpu).bfloat16()
        ids = torch.full((T, 1), E - 1)
        r = _routing(ids, torch.ones((T, 1)), E)
        y = wc.experts_mx_torch(x.to(dev), wc.Routing(*(t.to(dev) for t in r)), *(t for p in layer for t in p))
        few = slice(0, 2)
        # the first tokens, and of y the first and last columns: the reference in 64 bits is slow
        c, b = mx.quantize(x[few])
        xv = mx.values(mx.pack(c), b, hidden).to(dev)
        on = [tuple(t[E - 1:].cpu() for t in p) for p in layer]
        a = xv @ mx.values(on[0][0][0], on[0][1][0], hidden).T.to(dev)
        u = xv @ mx.values(on[1][0][0], on[1][1][0], hidden).T.to(dev)
        v, far = _h_codes((a * torch.sigmoid(a) * u).cpu())
        rows = [0, 1, 8190, 8191]
        m = mx.values(on[2][0][0][rows], on[2][1][0][rows], ffn)
        ref = v @ m.T
        tol = far @ m.abs().T + (v.abs() @ m.abs().T) * (mx.blocks(ffn) + 41) * 2.0 ** -23 + 2.0 ** -8 * ref.abs()
        off = (y[few][:, rows].cpu().double() - ref).abs()
        assert bool((off <= 1.01 * tol).all()), float((off / tol).max())
