"""GPU: wc_route against a plain router in 64 bits, token by token.

The choice has to be the plain router's exactly: logits are spaced numbers no two of
which are equal in a row unless a test is about ties, so keys differ by far more than
fp32's rounding.  Where sums (with a bias, or of a group's two best) can fall close, rows
with two keys nearer than MARGIN are left out: a key's error is at most
(E + 16) 2^-24 s + 2^-23 |key|, under 1e-6 with the scores there.  Weights: exp in fp32 is within 2 ulp, the softmax's sum of E terms
within E 2^-24, the division, the renormalisation of k terms and the scale a rounding
each: (E + k + 16) 2^-24 relative.
"""
import math

import pytest

from paper_2606_15789_amd import wc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

MARGIN = 4e-6


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def plain(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_top=1,
          renormalize=True, scale=1.0):
    """ids and weights, with Python floats (64 bits) and the definition."""
    ids, weights, margins = [], [], []
    for row in logits.tolist():
        margin = math.inf
        E = len(row)
        b = [0.0] * E if bias is None else bias.tolist()
        on = [e for e in range(E) if row[e] != -math.inf and b[e] != -math.inf]
        bad = any(math.isnan(row[e]) for e in on)
        good = [e for e in on if not math.isnan(row[e])]
        s = [0.0] * E
        if score == "softmax":
            top = max((row[e] for e in good), default=0.0)
            total = sum(math.exp(row[e] - top) for e in good)
            for e in good:
                s[e] = math.exp(row[e] - top) / total
        else:
            for e in good:
                s[e] = 1 / (1 + math.exp(-row[e])) if row[e] > -700 else 0.0
        key = [-math.inf] * E
        for e in good:
            # the scores' own order, where they are too small to differ
            key[e] = row[e] if score == "softmax" and bias is None and group_top == 1 else s[e] + b[e]
        if groups > 1:
            per = E // groups
            rank = []
            for g in range(groups):
                best = sorted(key[g * per:(g + 1) * per], reverse=True)[:group_top]
                rank.append((-sum(best), g))
            rank.sort()
            kept = {g for _, g in rank[:top_groups]}
            if top_groups < groups and rank[top_groups][0] < math.inf:
                margin = rank[top_groups][0] - rank[top_groups - 1][0]
            key = [key[e] if e // per in kept else -math.inf for e in range(E)]
        chosen = sorted((-key[e], e) for e in range(E) if key[e] != -math.inf)[:k + 1]
        margin = min([margin] + [b[0] - a[0] for a, b in zip(chosen, chosen[1:])])
        margins.append(margin)
        chosen = [e for _, e in chosen][:k]
        w = [s[e] for e in chosen]
        if renormalize and sum(w):
            w = [v / sum(w) for v in w]
        w = [math.nan if bad else v * scale for v in w]
        ids.append(chosen + [-1] * (k - len(chosen)))
        weights.append(w + [math.nan if bad else 0.0] * (k - len(chosen)))
    return (torch.tensor(ids, dtype=torch.int32).view(-1, k),
            torch.tensor(weights, dtype=torch.float64).view(-1, k), torch.tensor(margins))


def _logits(tokens, experts, seed, dtype="fp32", step=1 / 16):
    g = torch.Generator().manual_seed(seed)
    order = torch.argsort(torch.rand((tokens, experts), generator=g), dim=1)
    return ((order - experts // 2) * step).to(DT[dtype])


def _check(r, logits, k, margin=0.0, **how):
    E = logits.shape[1]
    ids, weights, margins = plain(logits.double(), k, **how)
    clear = margins >= margin
    assert float(clear.float().mean()) > 0.8
    ids, weights, got = ids[clear], weights[clear], r.ids.cpu()[clear]
    assert torch.equal(got, ids), [t for t in range(len(ids)) if not torch.equal(got[t], ids[t])][:3]
    w = r.weights.cpu().double()[clear]
    assert torch.equal(torch.isnan(w), torch.isnan(weights))
    tol = (E + k + 16) * 2.0 ** -24 * weights.abs() + 1e-37
    assert bool(((w - weights).abs() <= tol)[~torch.isnan(weights)].all())
    check_order(r, E)


def check_order(r, E):
    flat = r.ids.cpu().flatten().long()
    flat = torch.where(flat < 0, E, flat)
    assert torch.equal(r.order.cpu().long(), torch.sort(flat, stable=True)[1])
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    assert r.offsets.cpu().tolist() == [0] + torch.cumsum(counts, 0).tolist()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("tokens,experts,k", [
    (1, 1, 1), (1, 8, 2), (2, 2, 2), (5, 7, 3), (64, 16, 4), (17, 63, 6), (30, 64, 8), (9, 65, 8),
    (33, 100, 32), (12, 128, 1), (7, 160, 6), (40, 192, 8), (25, 256, 8), (6, 257, 10), (8, 511, 9),
    (11, 512, 32), (700, 8, 2), (300, 61, 7)])
def test_sizes(dev, dtype, score, tokens, experts, k):
    # 16-bit types and sigmoid's flat ends: the values stay within +-16
    x = _logits(tokens, experts, tokens + experts, dtype, 1 / 16 if experts <= 128 else 1 / 32)
    if dtype == "bf16" and experts > 128:
        x = x * 0 + _logits(tokens, experts, tokens, "fp32", 1.0).to(torch.bfloat16) / 32
        if experts > 256:
            pytest.skip("more values than bf16 tells apart")
    for renorm, scale in ((True, 1.0), (False, 2.5)):
        r = wc.route_torch(x.to(dev), k, score, renormalize=renorm, scale=scale)
        _check(r, x, k, score=score, renormalize=renorm, scale=scale)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("experts,groups,top_groups,k", [
    (8, 4, 2, 3), (64, 8, 3, 8), (256, 8, 4, 8), (160, 8, 3, 6), (60, 5, 1, 12), (512, 16, 4, 32),
    (24, 12, 12, 5), (16, 1, 1, 4)])
@pytest.mark.parametrize("biased", [False, True])
def test_groups_and_bias(dev, score, group_top, experts, groups, top_groups, k, biased):
    tokens = 37
    x = _logits(tokens, experts, experts + k, step=1 / 64)
    # keys further apart than rounding, the bias decides between near scores
    bias = _logits(1, experts, 3, step=1 / 1024)[0] if biased else None
    how = dict(score=score, bias=bias, groups=groups, top_groups=top_groups, group_top=group_top)
    r = wc.route_torch(x.to(dev), k, score, None if bias is None else bias.to(dev), groups=groups,
                       top_groups=top_groups, group_top=group_top)
    _check(r, x, k, MARGIN, **how)


def test_ties_go_to_the_lowest_index(dev):
    x = torch.zeros((6, 70))
    x[1, 50:] = 1
    x[2, 69] = 2
    x[3, 3] = -1
    x[4] = -1e4
    x[5, ::2] = -0.0
    for score in ("softmax", "sigmoid"):
        r = wc.route_torch(x.to(dev), 4, score)
        want = [[0, 1, 2, 3], [50, 51, 52, 53], [69, 0, 1, 2], [0, 1, 2, 4], [0, 1, 2, 3], [0, 1, 2, 3]]
        assert r.ids.cpu().tolist() == want, score
    # equal groups: the lower one
    r = wc.route_torch(torch.zeros((3, 16), device=dev), 3, "sigmoid", groups=4, top_groups=1,
                       group_top=2)
    assert r.ids.cpu().tolist() == [[0, 1, 2]] * 3


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masks(dev, score):
    ninf, low = -math.inf, torch.finfo(torch.float32).min
    x = _logits(9, 40, 4)
    x[0] = ninf                       # nothing to choose
    x[1, 2:] = ninf                   # fewer than k
    x[2, ::3] = ninf
    x[3] = low                        # the type's lowest value is a number
    x[4, 5:] = low
    r = wc.route_torch(x.to(dev), 5, score)
    _check(r, x, 5, score=score)
    assert r.ids[0].tolist() == [-1] * 5 and not bool(r.weights[0].any())
    assert r.ids[1].tolist()[2:] == [-1] * 3
    # a bias of -inf masks whatever the logit holds, and its logit is not in the softmax's sum
    bias = torch.zeros(40)
    bias[[0, 7, 39]] = ninf
    x = _logits(9, 40, 5, step=1 / 8)
    x[0, 7] = math.nan
    x[1, 39] = math.inf
    r = wc.route_torch(x.to(dev), 5, score, bias.to(dev))
    _check(r, x, 5, score=score, bias=bias)
    assert bool(torch.isfinite(r.weights).all())
    # every expert masked in every group
    r = wc.route_torch(torch.full((3, 32), ninf, device=dev), 4, score, groups=4, top_groups=2)
    assert bool((r.ids == -1).all()) and not bool(r.weights.any())
    check_order(r, 32)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_nan_and_infinity(dev, score):
    x = _logits(4, 24, 8)
    x[1, 20] = math.nan
    x[2] = math.nan
    r = wc.route_torch(x.to(dev), 6, score)
    _check(r, x, 6, score=score)
    assert 20 not in r.ids[1].tolist()
    x = _logits(2, 24, 9)
    x[0, 11] = math.inf
    r = wc.route_torch(x.to(dev), 2, score)
    assert r.ids[0, 0] == 11
    assert bool(torch.isfinite(r.weights[1]).all())
    if score == "sigmoid":
        assert bool(torch.isfinite(r.weights[0]).all())


@pytest.mark.parametrize("tokens,experts,k", [(1000, 64, 8), (2048, 1, 1), (2049, 3, 1),
                                              (4099, 61, 7), (30000, 512, 16), (16384, 8, 2),
                                              (17000, 61, 6), (5000, 200, 3), (900, 40, 9),
                                              (140000, 16, 16), (300000, 60, 5), (40000, 300, 2)])
def test_order_of_many_slots(dev, tokens, experts, k):
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, experts), generator=g) + torch.randn(experts, generator=g)
    x[::7, experts // 2:] = -math.inf
    x[-tokens // 9:] = -math.inf
    r = wc.route_torch(x.to(dev), k)
    check_order(r, experts)
    top = torch.sort(x, dim=1, descending=True, stable=True)
    want = torch.where(top[0][:, :k] == -math.inf, -1, top[1][:, :k])
    assert torch.equal(r.ids.cpu().long(), want)
    again = wc.route_torch(x.to(dev), k)
    assert all(torch.equal(a.nan_to_num() if a.is_floating_point() else a,
                           b.nan_to_num() if b.is_floating_point() else b) for a, b in zip(r, again))


def test_no_tokens(dev):
    r = wc.route_torch(torch.zeros((0, 12), device=dev), 3)
    assert r.offsets.cpu().tolist() == [0] * 13 and r.ids.shape == (0, 3)


def test_strides_streams_and_a_graph(dev):
    wide = _logits(50, 40, 1).to(dev)
    x = wide[:, 3:36]
    _check(wc.route_torch(x, 4), x.cpu(), 4)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = _logits(80, 33, 2).to(dev)
    r = wc.route_torch(y, 4, stream=side)
    side.synchronize()
    _check(r, y.cpu(), 4)
    for tokens in (3, 900):
        data = [_logits(tokens, 33, s).to(dev) for s in range(4)]
        x = data[0].clone()
        out = wc.route_torch(x, 4, "sigmoid")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            wc.route_torch(x, 4, "sigmoid", out=out)
        for v in data:
            x.copy_(v)
            for t in out:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, wc.route_torch(v, 4, "sigmoid")):
                assert torch.equal(a, b)


def test_refusals(dev):
    x = torch.zeros((4, 16), device=dev)
    for call in (lambda: wc.route_torch(x, 2, "tanh"), lambda: wc.route_torch(x.double(), 2),
                 lambda: wc.route_torch(x.T, 2), lambda: wc.route_torch(x[0], 2),
                 lambda: wc.route_torch(x, 2, bias=torch.zeros(15, device=dev)),
                 lambda: wc.route_torch(x, 2, bias=torch.zeros(16, device=dev).half()),
                 lambda: wc.route_torch(x.cpu(), 2),
                 lambda: wc.route_torch(x, 2, out=wc.route_torch(x, 3))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: wc.route_torch(x, 0), lambda: wc.route_torch(x, 17),
                 lambda: wc.route_torch(x, 2, groups=3), lambda: wc.route_torch(x, 2, groups=0),
                 lambda: wc.route_torch(x, 2, groups=4, top_groups=5),
                 lambda: wc.route_torch(x, 2, groups=4, top_groups=0),
                 lambda: wc.route_torch(x, 2, groups=16, top_groups=2, group_top=2),
                 lambda: wc.route_torch(x, 2, group_top=3),
                 lambda: wc.route_torch(x, 2, scale=math.inf),
                 lambda: wc.route_torch(torch.zeros((2, 513), device=dev), 2),
                 lambda: wc.route_torch(torch.zeros((2, 64), device=dev), 33)):
        with pytest.raises(wc.WcError):
            call()


def test_more_tokens_than_a_launch_has_threads_for(dev):
    """2^26 tokens and a few, of a whole wave each."""
    tokens, experts = (1 << 26) + 3, 33
    x = torch.randint(-128, 128, (tokens, experts), dtype=torch.int8, device=dev).bfloat16()
    r = wc.route_torch(x, 1, "sigmoid", bias=torch.arange(experts, device=dev) * -0.125)
    at, ids = r.order.long(), r.ids[:, 0].long()
    key = ids[at] * 2 ** 32 + at
    assert bool((key[1:] > key[:-1]).all())
    assert torch.equal(r.offsets[1:].long(), torch.bincount(ids, minlength=experts).cumsum(0))
    for part in (slice(0, 1 << 20), slice((1 << 24) - 5, (1 << 24) + 5), slice(tokens - (1 << 20), tokens)):
        keys = torch.sigmoid(x[part].double()) - torch.arange(experts, device=dev) * 0.125
        top, best = keys.sort(dim=1, descending=True)
        clear = top[:, 0] - top[:, 1] > 1e-6
        assert float(clear.float().mean()) > 0.5
        assert torch.equal(ids[part][clear], best[:, 0][clear])


def _limits(x):
    """Rows with an infinite logit as their limit: it has all of the softmax, equal ones
    share it, and the others' scores are 0."""
    out = torch.where(torch.isposinf(x), 0.0, torch.full_like(x, -2000.0))
    out = torch.where(x.isnan() | torch.isneginf(x), x, out)
    return torch.where(torch.isposinf(x).any(dim=1, keepdim=True), out, x)


@pytest.mark.parametrize("experts", [16, 32, 64, 256, 512])
@pytest.mark.parametrize("biased,groups,group_top", [(False, 4, 2), (True, 1, 1), (True, 4, 1), (True, 4, 2)])
@pytest.mark.parametrize("renormalize", [False, True])
def test_infinity_and_nan_among_scores(dev, experts, groups, group_top, renormalize, biased):
    """Softmax keys that are scores: a token with an infinite or a NaN logit has NaN weights,
    and still the experts that its other logits give."""
    k = 6
    x = _logits(7, experts, experts, step=1 / 64)
    x[0, 11] = math.inf
    x[1, [3, 9]] = math.inf
    x[2, 5] = math.nan
    x[3] = math.nan
    x[4, [1, 6]] = math.inf
    x[4, [0, 12]] = -math.inf
    x[4, 13] = math.nan
    x[5] = math.inf
    bias = _logits(1, experts, 3, step=1 / 1024)[0] if biased else None
    how = dict(groups=groups, top_groups=max(1, groups // 2), group_top=group_top, renormalize=renormalize)
    r = wc.route_torch(x.to(dev), k, "softmax", None if bias is None else bias.to(dev), **how)
    ids, weights, margins = plain(_limits(x).double(), k, bias=bias, **how)
    # scores of 0, 1 and 1 / 2^n and the bias are exact, and so are their sums and ties
    clear = torch.isposinf(x).any(dim=1) | (margins >= MARGIN)
    assert torch.equal(r.ids.cpu()[clear], ids[clear])
    assert torch.isnan(r.weights).all(dim=1).tolist() == [True] * 6 + [False]
    assert bool(clear[6])
    w = r.weights[6].cpu().double()
    assert bool(((w - weights[6]).abs() <= (experts + k + 16) * 2.0 ** -24 * weights[6]).all())
    check_order(r, experts)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("tokens,experts,k", [(6, 257, 10), (8, 511, 9), (11, 512, 32), (600, 512, 8)])
def test_many_experts_in_bf16(dev, score, tokens, experts, k):
    """512 numbers of bf16 that differ: 128 of either sign to each of two powers of two, up
    to 4, where sigmoids of neighbours are 2^-13 apart."""
    v = (1 + torch.arange(128) / 128.0)[None] * torch.tensor([[1.0], [2.0]])
    v = torch.cat([v.flatten(), -v.flatten()])
    g = torch.Generator().manual_seed(tokens)
    x = v[torch.argsort(torch.rand((tokens, 512), generator=g), dim=1)][:, :experts].bfloat16()
    assert torch.equal(x.float().sort(dim=1)[0].diff(dim=1) > 0, torch.ones((tokens, experts - 1), dtype=torch.bool))
    r = wc.route_torch(x.to(dev), k, score)
    _check(r, x, k, score=score)


@pytest.mark.parametrize("experts,k,blocks", [(512, 32, 31), (512, 32, 32), (255, 16, 63), (255, 16, 64),
                                              (61, 8, 264), (61, 8, 265), (3, 2, 4095), (3, 2, 4096),
                                              (16, 16, 963), (16, 16, 964), (1, 1, 8192), (300, 20, 700)])
@pytest.mark.parametrize("last", [1, 2048])
def test_order_where_counts_are_summed(dev, experts, k, blocks, last):
    """Blocks of 2048 slots on both sides of 16384 counts, the last one full or begun."""
    tokens = ((blocks - 1) * 2048 + last + k - 1) // k
    g = torch.Generator(device=dev).manual_seed(blocks)
    x = torch.randn((tokens, experts), generator=g, device=dev) \
        + torch.randn(experts, generator=g, device=dev)
    x[::7, experts // 2:] = -math.inf
    r = wc.route_torch(x, k)
    flat = torch.where(r.ids < 0, experts, r.ids).flatten().long()
    assert torch.equal(r.order.long(), torch.sort(flat, stable=True)[1])
    counts = torch.bincount(flat, minlength=experts + 1)[:experts]
    assert torch.equal(r.offsets[1:].long(), counts.cumsum(0)) and int(r.offsets[0]) == 0
    top, ids = torch.sort(x, dim=1, descending=True, stable=True)
    assert torch.equal(r.ids.long(), torch.where(top == -math.inf, -1, ids)[:, :k])


def test_time_grows_with_the_tokens(dev):
    """Eight times the tokens, eight times the time: within half as much again for what the
    caches no longer hold.  (A sort whose every block reads all blocks' counts takes 46 times.)"""
    def us(tokens):
        x = torch.randn((tokens, 256), device=dev, dtype=torch.bfloat16)
        out = wc.route_torch(x, 8)
        times = []
        for _ in range(5):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            wc.route_torch(x, 8, out=out)
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        return min(times)
    assert us(1 << 22) < 12 * us(1 << 19)
