"""The served replica's own routing."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_logits_keep_32_bits(monkeypatch):
    """What decides between experts is not rounded to the rows' type: logits are the products of the
    normed rows in 32 bits."""
    import paper_2609_29160_gb300 as tre
    from paper_2609_29160_gb300 import served
    rep = served.Replica(layers=2, q_heads=4, kv_heads=2, dim=64, pages=64, experts=8, top=2, chunk=48, seed=3)
    normed, seen = [], []
    norm, route = tre.tre_block_norm, tre.tre_route

    def own_norm(*a, **how):
        got = norm(*a, **how)
        normed.append(got[1])
        return got

    def own_route(x, *a, **how):
        seen.append((x.clone(), normed[-1].clone()))
        return route(x, *a, **how)

    monkeypatch.setattr(tre, "tre_block_norm", own_norm)
    monkeypatch.setattr(tre, "tre_route", own_route)
    rep.serve([(0, 70, 5), (1, 3, 9)], seed=1)
    assert seen
    for i, (x, n) in enumerate(seen):
        router = rep.layers[i % 2]["router"].double()
        want, size = n.double() @ router, n.double().abs() @ router.abs()
        assert x.dtype == torch.float32
        # a sum of products in 32 bits, in any order
        assert ((x - want).abs() <= 2.0 ** -24 * (n.shape[1] + 2) * size).all()
