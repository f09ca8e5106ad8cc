"""Measured calls of the microscaled 4-bit operators: what a program that serves an
MXFP4 checkpoint (e2m1 codes, two to a byte, and an e8m0 scale for each 32 of a row,
as the decoder gives them back) runs.

A case's `op` is the operator:

* quantize: rows to MXFP4 and back: the values that the codes and scales stand for;
* linear: activations quantised to MXFP4, times MXFP4 matrices that share them (q, k
  and v, or one matrix), with an optional bias, in the activations' type or another;
* experts: the gated feed-forward of a mixture layer with MXFP4 experts, for tokens
  that a router has given experts: the weighted sum of down(silu(gate x) * up x), x and
  the hidden values quantised to MXFP4;
* moe: the same layer from the router's logits, for a few tokens.
"""

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]  # of the codes 0..7; 8..15 are their negatives


def _quantize(name, m, k, x="bf16"):
    return {"name": name, "op": "quantize", "m": m, "k": k, "x": x}


def _linear(name, m, k, n, kv=0, x="bf16", out="", bias=False):
    """kv: two more matrices of that many rows share x (0: none)."""
    return {"name": name, "op": "linear", "m": m, "k": k, "n": n, "kv": kv, "x": x,
            "out": out or x, "bias": bias}


def _experts(name, tokens, experts, k, hidden, ffn, x="bf16", pad=0):
    """pad: trailing tokens with nothing to route."""
    return {"name": name, "op": "experts", "tokens": tokens, "experts": experts, "k": k,
            "hidden": hidden, "ffn": ffn, "x": x, "pad": pad}


def _moe(name, tokens, experts, k, hidden, ffn, x="bf16", pad=0, score="softmax", bias=False,
         groups=1, top_groups=1, group_top=1, scale=1.0):
    return {"name": name, "op": "moe", "tokens": tokens, "experts": experts, "k": k,
            "hidden": hidden, "ffn": ffn, "x": x, "pad": pad, "score": score, "bias": bias,
            "groups": groups, "top_groups": top_groups, "group_top": group_top, "scale": scale}


def listed():
    return [
        # a batch of odd size and width in 32 bits: the last block of a row is a part of one
        _quantize("quantize-odd", 333, 5461, x="fp32"),
        # a matrix of a 70B layer brought to MXFP4
        _quantize("quantize-matrix", 28672, 8192),
        # one token through q, k and v of an 8B layer: the smallest product, bound by latency
        _linear("linear-token", 1, 4096, 4096, kv=1024),
        # a decode batch of odd size through an up projection of a 70B layer: bound by the weights
        _linear("linear-batch", 13, 8192, 28672, x="fp16", bias=True),
        # odd sizes throughout, 32-bit activations and results
        _linear("linear-odd", 333, 5461, 2047, x="fp32", bias=True),
        # a chunk of a prompt through a down projection of a 70B layer
        _linear("linear-chunk", 512, 28672, 8192, x="fp16", out="bf16"),
        # a batch of long prompts through an up projection of a 70B layer: bound by the arithmetic
        _linear("linear-prompt", 8192, 8192, 28672),
        # odd sizes, another type, a padded batch
        _experts("experts-odd", 203, 7, 3, 1537, 2051, x="fp16", pad=11),
        # a decode batch through a layer of eight large experts: all of their weights are read
        _experts("experts-batch", 32, 8, 2, 6144, 16384),
        # a prompt through the same layer: bound by the arithmetic
        _experts("experts-prompt", 4096, 8, 2, 6144, 16384),
        # one token through a layer of many small experts, from the router's logits
        _moe("moe-token", 1, 64, 6, 2048, 1408),
        # a small decode batch through many experts in groups, one place of the batch empty
        _moe("moe-few", 16, 128, 8, 4096, 1536, pad=1, score="sigmoid", bias=True, groups=8,
             top_groups=4, group_top=2, scale=2.5),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A width: mostly whole blocks of 128, at times odd."""
    v = _spread(rng, lo, hi)
    return v if rng.random() < 0.3 or v < 192 else v // 128 * 128


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "linear", "experts", "experts", "moe"])
    x = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "quantize":
        c = _quantize("", _spread(rng, 1, 28672), _size(rng, 64, 28672), x=x)
        while c["m"] * c["k"] > 28672 * 8192:
            c["m"] = max(1, c["m"] // 2)
    elif op == "linear":
        c = _linear("", _spread(rng, 1, 8192), _size(rng, 256, 28672), _size(rng, 256, 28672),
                    x=x, out=rng.choice([x, x, "bf16", "fp32"]), bias=rng.random() < 0.4)
        while c["k"] * c["n"] > 8192 * 28672:
            c["k"], c["n"] = max(256, c["k"] // 2), max(256, c["n"] // 2)
        if rng.random() < 0.3:
            c["kv"] = max(128, c["n"] // rng.choice([4, 5, 8]))
            c["n"] -= 2 * (c["kv"] // 2)  # no more work than without k and v
    else:
        few = op == "moe"
        groups = rng.choice([1, 1, 4, 8]) if few else 1
        e = rng.choice([8, 16, 32, 64, 128]) if groups > 1 else rng.choice([4, 7, 8, 16, 32, 61, 64])
        keep = rng.randint(1, groups)
        k = rng.randint(1, min(keep * e // groups, 8))
        hidden = _size(rng, 512, 6144)
        ffn = min(_size(rng, 512, 16384), 4 * hidden)
        while e * hidden * ffn > 8 * 6144 * 16384:
            hidden, ffn = hidden // 2, ffn // 2
        # 16-bit results: in 32 bits they would show the few of the hidden layer's values
        # that a sum's last bit moves to the next code
        x = rng.choice(["bf16", "bf16", "fp16"])
        if few:
            tokens = _spread(rng, 1, 16)
            score = rng.choice(["softmax", "sigmoid"])
            c = _moe("", tokens, e, k, hidden, ffn, x=x, score=score,
                     bias=score == "sigmoid" and rng.random() < 0.7, groups=groups, top_groups=keep,
                     group_top=2 if score == "sigmoid" and groups > 1 and rng.random() < 0.5 else 1,
                     scale=rng.choice([1.0, 2.5]))
            c["pad"] = rng.choice([0, 0, tokens // 5])
        else:
            tokens = min(_spread(rng, 1, 4096), max(1, 8192 * 6144 * 16384 // (k * hidden * ffn)))
            c = _experts("", tokens, e, k, hidden, ffn, x=x, pad=rng.choice([0, 0, tokens // 9]))
    del c["name"]
    return c


# --- inputs -------------------------------------------------------------------

def _gen(seed, j):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1009 + j)
    return g


def _activations(g, rows, width, dtype):
    """Normal values with a few columns 20 times larger, as a layer's inputs have them."""
    x = torch.randn((rows, width), generator=g, device=DEV)
    x[:, torch.randperm(width, generator=g, device=DEV)[:max(1, width // 1000)]] *= 20
    return x.to(DTYPES[dtype])


def _matrix(g, n, k):
    """Packed codes and scales of normal weights; a row is whole blocks, zeros past k."""
    codes, scale = _coded(torch.randn((n, k), generator=g, device=DEV).mul_(0.02))
    return codes[:, 0::2] | codes[:, 1::2] << 4, scale


def _bank(g, experts, n, k):
    """The same for a stack of experts."""
    blocks = (k + 31) // 32
    codes = torch.empty((experts, n, blocks * 16), dtype=torch.uint8, device=DEV)
    scales = torch.empty((experts, n, blocks), dtype=torch.uint8, device=DEV)
    for e in range(experts):
        codes[e], scales[e] = _matrix(g, n, k)
    return codes, scales


def prepare(case, seed):
    if case["op"] == "quantize":
        return {"case": case, "x": _activations(_gen(seed, 1), case["m"], case["k"], case["x"])}
    if case["op"] == "linear":
        mats = [_matrix(_gen(seed, 10 + j), n, case["k"])
                for j, n in enumerate([case["n"]] + [case["kv"]] * 2) if n]
        g = _gen(seed, 1)
        return {"case": case, "x": _activations(g, case["m"], case["k"], case["x"]),
                "w": [w for w, _ in mats], "scales": [s for _, s in mats],
                "bias": [torch.randn(w.shape[0], generator=g, device=DEV).to(DTYPES[case["x"]])
                         if case["bias"] else None for w, _ in mats]}
    t, e = case["tokens"], case["experts"]
    g = _gen(seed, 2)
    # some experts are more popular than others
    logits = torch.randn((t, e), generator=g, device=DEV) * 1.5 \
        + torch.randn(e, generator=g, device=DEV) * 0.5
    state = {"case": case, "x": _activations(g, t, case["hidden"], case["x"])}
    if case["op"] == "moe":
        logits[t - case["pad"]:] = -math.inf
        state["logits"] = logits
        state["bias"] = torch.randn(e, generator=g, device=DEV) * 0.1 if case["bias"] else None
    else:
        top, ids = torch.topk(logits, case["k"], dim=1)
        weights = torch.softmax(top, dim=1)
        ids = ids.to(torch.int32)
        ids[t - case["pad"]:] = -1
        weights[t - case["pad"]:] = 0
        # slots sorted by expert, those without one last, and where each expert starts
        flat = torch.where(ids < 0, e, ids).flatten()
        offsets = torch.zeros(e + 1, dtype=torch.int32, device=DEV)
        offsets[1:] = torch.cumsum((flat[:, None] == torch.arange(e, device=DEV)).sum(dim=0), 0)
        state |= {"ids": ids, "weights": weights, "offsets": offsets,
                  "order": torch.sort(flat, stable=True)[1].to(torch.int32)}
    for j, (part, n, k) in enumerate((("gate", case["ffn"], case["hidden"]),
                                      ("up", case["ffn"], case["hidden"]),
                                      ("down", case["hidden"], case["ffn"]))):
        state[part], state[part + "_scale"] = _bank(_gen(seed, 20 + j), e, n, k)
    return state


# --- the plain forms ----------------------------------------------------------

def _coded(x):
    """Codes 0..15 and scale bytes of x's rows, whole blocks of 32."""
    m, k = x.shape
    blocks = (k + 31) // 32
    if k % 32:
        x = torch.cat([x, torch.zeros((m, blocks * 32 - k), dtype=x.dtype, device=DEV)], dim=1)
    x = x.view(m, blocks, 32)
    # two below the exponent of a block's largest magnitude: 4 and 6 are e2m1's largest
    top = x.abs().amax(dim=2)
    field = torch.where(top > 0, torch.frexp(top)[1] + 124, 0).clamp_min_(0)
    a = x * (254 - field << 23).view(torch.float32)[..., None]  # times 2^(127 - field)
    mag = a.abs()
    # the midpoints between neighbours; a tie goes to the even code
    codes = (mag > 0.25).to(torch.uint8)
    codes += mag >= 0.75
    codes += mag > 1.25
    codes += mag >= 1.75
    codes += mag > 2.5
    codes += mag >= 3.5
    codes += mag > 5
    codes += (a < 0).to(torch.uint8) * 8
    return codes.view(m, blocks * 32), field.to(torch.uint8)


def _values(codes, scale):
    """32-bit values of codes (rows of whole blocks) and scales."""
    table = torch.tensor(VALUES + [-v for v in VALUES], device=DEV)
    field = scale.to(torch.int32)
    power = torch.where(field > 0, field << 23, 1 << 22).view(torch.float32)
    v = table[codes.to(torch.int32)].view(*scale.shape, 32) * power[..., None]
    return v.flatten(-2)


def _unpacked(w, scale):
    """The values of packed matrices."""
    return _values(torch.stack([w & 15, w >> 4], dim=-1).flatten(-2), scale)


def _product(x, w, scale):
    """x's rows, quantised, times the rows of packed matrices."""
    if x.dim() == 3:
        q = _values(*_coded(x.flatten(0, 1))).view(*x.shape[:2], -1)
    else:
        q = _values(*_coded(x))
    return q @ _unpacked(w, scale).transpose(-1, -2)


def _choose(case, logits, bias):
    """Experts and weights of the router's logits, in 64 bits: scores next to each other."""
    x = logits.double()
    off = x == -math.inf
    if case["score"] == "softmax":
        e = torch.where(off, 0.0, torch.exp(x - x.amax(dim=1, keepdim=True)))
        total = e.sum(dim=1, keepdim=True)
        s = torch.where(total > 0, e / total, 0.0)
        key = x  # grows with the score
    else:
        s = torch.where(off, 0.0, 1 / (1 + torch.exp(-x)))
        key = torch.where(off, -math.inf, s if bias is None else s + bias.double())
    if case["groups"] > 1:
        parts = key.view(len(key), case["groups"], -1)
        best = torch.sort(parts, dim=2, descending=True)[0][..., :case["group_top"]].sum(dim=2)
        kept = torch.sort(best, dim=1, descending=True, stable=True)[1][:, :case["top_groups"]]
        out = torch.ones_like(best, dtype=torch.bool).scatter_(1, kept, False)
        key = torch.where(out[..., None], -math.inf, parts).flatten(1)
    top, ids = torch.sort(key, dim=1, descending=True, stable=True)
    top, ids = top[:, :case["k"]], ids[:, :case["k"]]
    empty = top == -math.inf
    w = torch.where(empty, 0.0, s.gather(1, ids))
    total = w.sum(dim=1, keepdim=True)
    w = torch.where(total > 0, w / total, 0.0)
    return torch.where(empty, -1, ids), (w * case["scale"]).float()


def _plain(state):
    case = state["case"]
    if case["op"] == "quantize":
        return _values(*_coded(state["x"].float()))[:, :case["k"]].to(DTYPES[case["x"]])
    if case["op"] == "linear":
        ys = [_product(state["x"].float(), w, s) + (0.0 if b is None else b.float())
              for w, s, b in zip(state["w"], state["scales"], state["bias"])]
        return [y.to(DTYPES[case["out"]]) for y in ys]
    if case["op"] == "moe":
        ids, weights = _choose(case, state["logits"], state["bias"])
    else:
        ids, weights = state["ids"].long(), state["weights"]
    # every expert for every token, with weight 0 where it is not the token's
    t, e = case["tokens"], case["experts"]
    share = torch.zeros((t, e + 1), device=DEV).scatter_add_(1, torch.where(ids < 0, e, ids),
                                                           weights)[:, :e]
    gate = _product(state["x"].float(), state["gate"], state["gate_scale"])
    up = _product(state["x"].float(), state["up"], state["up_scale"])
    # in 64 bits: silu(g) next to g, and products of few bits, lie on a power of two or a tie
    # between codes in 32
    gate = gate.double()
    h = gate / (1 + torch.exp(-gate)) * up
    y = _product(h, state["down"], state["down_scale"])
    return (y * share.T[..., None]).sum(dim=0).to(DTYPES[case["x"]])


def run(state):
    if not own:
        return _plain(state)
    from paper_2606_15789_amd import wc
    case = state["case"]
    if case["op"] == "quantize":
        q, scale = wc.quantize_mx_torch(state["x"])
        return wc.dequantize_mx_torch(q, scale, case["k"], dtype=DTYPES[case["x"]])
    if case["op"] == "linear":
        return wc.linear_mx_torch(state["x"], state["w"], state["scales"], state["bias"],
                                  dtype=DTYPES[case["out"]])
    banks = (state["gate"], state["gate_scale"], state["up"], state["up_scale"], state["down"],
             state["down_scale"])
    if case["op"] == "moe":
        return wc.moe_mx_torch(state["x"], state["logits"], case["k"], *banks, score=case["score"],
                               bias=state["bias"], groups=case["groups"],
                               top_groups=case["top_groups"], group_top=case["group_top"],
                               scale=case["scale"])
    routing = wc.Routing(state["ids"], state["weights"], state["offsets"], state["order"])
    return wc.experts_mx_torch(state["x"], routing, *banks)


def work(case):
    size = SIZE[case["x"]]
    if case["op"] == "quantize":
        return {"bytes": 2 * case["m"] * case["k"] * size, "flops": 0}
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"] + 2 * case["kv"]
        return {"bytes": m * k * size + n * ((k + 31) // 32 * 17)
                + (n * size if case["bias"] else 0) + m * n * SIZE[case["out"]],
                "flops": 2 * m * n * k}
    t, e, k, hidden, ffn = (case[p] for p in ("tokens", "experts", "k", "hidden", "ffn"))
    t -= case["pad"]
    # the experts that k draws a token without replacement hit, were all alike
    hit = e * (1 - (1 - k / e) ** t)
    one = (2 * ffn * ((hidden + 31) // 32) + hidden * ((ffn + 31) // 32)) * 17
    way = case["tokens"] * (4 * e if case["op"] == "moe" else 12 * k)
    return {"bytes": hit * one + (t + case["tokens"]) * hidden * size + way,
            "flops": 6 * t * k * hidden * ffn}


# --- the definitions in 64 bits -----------------------------------------------

def _power64(n):
    """2^n from its bits: ldexp and exp2 of the GPU are off by their last bit."""
    return (n.long() + 1023 << 52).view(torch.float64)


def _blocks64(x):
    """x's rows with each 32 of them rounded to e2m1 times a power of two."""
    m, k = x.shape
    whole = torch.zeros((m, (k + 31) // 32 * 32), dtype=torch.float64, device=DEV)
    whole[:, :k] = x
    parts = whole.unflatten(1, (-1, 32))
    top = parts.abs().max(dim=2, keepdim=True)[0]
    _, power = torch.frexp(top)  # top = f 2^power, f from 1/2 to 1
    scale = _power64((power - 3).clamp_min(-127))
    v = parts / scale
    # one binade at a time: the step is 1/2 below 2, 1 below 4 and 2 from there on
    size = v.abs()
    step = 0.5 + 0.5 * (size >= 2).double() + (size >= 4).double()
    near = (torch.round(size / step) * step).clamp_max(6)
    return (near * v.sign() * scale).flatten(1)[:, :k]


def _weights64(w, scale, k):
    grid = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=DEV) / 2
    grid = torch.cat([grid, -grid])
    both = torch.empty((w.shape[0], w.shape[1], 2), dtype=torch.float64, device=DEV)
    both[..., 0] = grid[torch.remainder(w, 16).int()]
    both[..., 1] = grid[torch.div(w, 16, rounding_mode="floor").int()]
    power = _power64(scale.long() - 127).repeat_interleave(32, dim=1)
    return (both.flatten(1) * power)[:, :k]


def _chosen64(case, logits, bias):
    """A token's weight for every expert."""
    x = logits.double()
    on = x > -math.inf
    s = (torch.softmax(x.clamp_min(-1e300), dim=1) if case["score"] == "softmax"
         else torch.sigmoid(x)) * on
    key = s + (0 if bias is None else bias.double())
    key[~on] = -math.inf
    if case["groups"] > 1:
        per = case["experts"] // case["groups"]
        best = key.unflatten(1, (case["groups"], per)).topk(case["group_top"], dim=2)[0].sum(2)
        rank = best.argsort(dim=1, descending=True, stable=True).argsort(dim=1)
        key[(rank >= case["top_groups"]).repeat_interleave(per, dim=1)] = -math.inf
    rank = key.argsort(dim=1, descending=True, stable=True).argsort(dim=1)
    w = s * ((rank < case["k"]) & (key > -math.inf))
    return w / w.sum(dim=1, keepdim=True).clamp_min(1e-300) * case["scale"]


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quantize":
        return _blocks64(state["x"].double())
    if case["op"] == "linear":
        x = _blocks64(state["x"].double())
        ys = []
        for w, s, b in zip(state["w"], state["scales"], state["bias"]):
            y = torch.mm(x, _weights64(w, s, case["k"]).t())
            ys.append(y if b is None else y + b.double())
        return ys
    if case["op"] == "moe":
        share = _chosen64(case, state["logits"], state["bias"])
    else:
        share = torch.stack([(state["weights"].double() * (state["ids"] == e)).sum(dim=1)
                             for e in range(case["experts"])], dim=1)
    hidden, ffn = case["hidden"], case["ffn"]
    x = _blocks64(state["x"].double())
    y = torch.zeros_like(x)
    for e in range(case["experts"]):
        mine = share[:, e].nonzero()[:, 0]
        if not len(mine):
            continue
        g = torch.mm(x[mine], _weights64(state["gate"][e], state["gate_scale"][e], hidden).t())
        u = torch.mm(x[mine], _weights64(state["up"][e], state["up_scale"][e], hidden).t())
        h = _blocks64(g * torch.sigmoid(g) * u)
        y[mine] += torch.mm(h, _weights64(state["down"][e], state["down_scale"][e], ffn).t()) \
            * share[mine, e][:, None]
    return y
