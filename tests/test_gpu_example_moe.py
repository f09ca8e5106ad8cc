"""GPU: the mixture-layer example end to end: encode, decode, q/k/v, routing, experts,
against the layer computed in 64 bits from the uncompressed tensors."""
import pytest

from paper_2606_15789_amd import example_moe, wc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,hidden,ffn,kv,experts,k", [(1, 512, 768, 128, 8, 2),
                                                            (37, 384, 640, 96, 6, 3),
                                                            (300, 272, 336, 64, 4, 2)])
def test_layer_from_blob(tokens, hidden, ffn, kv, experts, k):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    tensors = example_moe.synthetic_layer(hidden, ffn, kv, experts, seed=tokens)
    index, blob = example_moe.compress(tensors)
    layer = example_moe.Int8MoELayer(index, blob, k)
    # decoding is lossless: the banks hold the codes
    for e in range(experts):
        for name in ("gate", "up", "down", "gate.scale", "down.scale"):
            assert torch.equal(layer.t[name][e], tensors[f"{e}.{name}"])
    x = torch.randn((tokens, hidden), device="cuda").bfloat16()
    q, kk, v, y, r = layer(x)

    def rows(a):  # quantised, as the values they stand for
        step = a.abs().amax(dim=1, keepdim=True) / 127
        return torch.round(a / step) * step

    def w(name):
        return tensors[name].double() * tensors[name + ".scale"].double()[:, None]
    xq = rows(x.double())
    # Against quantisation in 64 bits: a code next to a half may differ by one step, one
    # 127th of its row's largest value; y is rounded to bf16 (2^-8), twice.
    for got, name in ((q, "q"), (kk, "k"), (v, "v")):
        ref = xq @ w(name).T
        assert float((got.double() - ref).norm() / ref.norm()) < 2.0 ** -8
    ref = torch.zeros_like(xq)
    ids, weights = r.ids.long(), r.weights.double()
    for e in range(experts):
        t, j = (ids == e).nonzero(as_tuple=True)
        if len(t):
            g, u = xq[t] @ w(f"{e}.gate").T, xq[t] @ w(f"{e}.up").T
            h = rows(g * torch.sigmoid(g) * u)
            ref.index_add_(0, t, (h @ w(f"{e}.down").T) * weights[t, j][:, None])
    off = (y.double() - x.double() - ref).norm()
    assert float(off / (x.double() + ref).norm()) < 2.0 ** -7
    logits = (x @ tensors["router"].T).double()
    top, chosen = logits.topk(k + 1, dim=1)
    clear = (top[:, :-1] > top[:, 1:]).all(dim=1)  # no equal logits among the best
    assert torch.equal(ids[clear], chosen[clear][:, :k])
    assert isinstance(r, wc.Routing)
