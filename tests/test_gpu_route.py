"""Routing to experts: choices as the formulas make them, weights near them."""
import math

import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


def logits(rows, experts, dtype="f32", seed=1, std=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, experts, generator=g, device="cuda") * std).to(R.T[dtype])


def check(tre, x, top, **how):
    ids, w = tre.tre_route(x, top, **how)
    want, ww = R.route(x, top, **how)
    assert ids.dtype == torch.int32 and torch.equal(ids.cpu(), want)
    # an exponential, a sum of up to 1,024, a quotient and products in 32 bits
    assert ((w.double().cpu() - ww).abs() <= 2.0 ** -24 * 40 * ww.abs() + 1e-37).all()
    return ids, w


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top", [(1, 1), (2, 2), (8, 2), (33, 32), (60, 4), (64, 6), (160, 6), (256, 8), (1024, 32)])
def test_top(tre, experts, top, scores, dtype):
    for rows in (1, 5, 130):
        check(tre, logits(rows, experts, dtype), top, scores=scores, renorm=rows != 5, scale=1.0 if rows == 1 else 2.5)


@pytest.mark.parametrize("experts,groups,top_groups", [(16, 4, 2), (60, 4, 1), (64, 8, 4), (160, 8, 3), (256, 8, 4),
                                                       (256, 4, 2), (512, 8, 2), (512, 16, 5), (1024, 32, 7), (320, 5, 2)])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("bias", [False, True])
def test_groups(tre, experts, groups, top_groups, best, bias):
    b = 0.1 * torch.randn(experts, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") if bias else None
    top = min(8, top_groups * experts // groups)
    for scores in ("softmax", "sigmoid"):
        check(tre, logits(200, experts), top, scores=scores, bias=b, groups=groups, top_groups=top_groups, group_best=best)


def test_ties(tre):
    """Equal logits go by index, in the row and between groups."""
    x = logits(64, 96, "bf16").mul(2).round().div(2)
    check(tre, x, 8)
    check(tre, x, 8, scores="sigmoid")
    check(tre, x, 8, scores="sigmoid", groups=6, top_groups=3)
    b = torch.zeros(96, device="cuda")
    check(tre, x, 8, scores="sigmoid", bias=b)
    check(tre, x, 8, scores="softmax", bias=b, groups=3, top_groups=2, group_best=2)
    check(tre, torch.zeros(3, 96, device="cuda"), 32, scores="sigmoid", bias=b)
    check(tre, torch.zeros(3, 96, device="cuda"), 5, groups=4, top_groups=2)
    zero = torch.zeros(2, 64, device="cuda")
    zero[:, ::2] = -0.0
    check(tre, zero, 4)


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("gap", [1e-9, 1e-8, 6e-8, 3e-7, 2e-6])
def test_scores_closer_than_32_bits_tell(tre, scores, gap):
    """c = s + bias of many experts within a few gaps of each other."""
    for seed, (experts, groups) in enumerate([(64, 1), (64, 4), (256, 8), (40, 1)]):
        x = logits(150, experts, seed=seed)
        s = torch.softmax(x.double(), -1) if scores == "softmax" else torch.sigmoid(x.double())
        g = torch.Generator(device="cuda").manual_seed(seed)
        # (one row's scores set the biases: its sums are all near 0.7)
        b = (0.7 - s[0] + gap * torch.randn(experts, generator=g, device="cuda").double()).float()
        check(tre, x[:1].expand(3, experts), 6, scores=scores, bias=b, groups=groups, top_groups=max(1, groups // 2))
        check(tre, x, 6, scores=scores, bias=b, groups=groups, top_groups=max(1, groups // 2))


def test_experts_that_are_not_there(tre):
    x = logits(40, 64)
    x[:, 10:20] = -math.inf
    x[0] = -math.inf
    x[1] = float("nan")
    x[2, 3:] = -math.inf
    x[3, ::2] = float("nan")
    x[4, 5] = math.inf
    x[5, 5] = x[5, 60] = math.inf
    x[6] = math.inf
    x[7, 7] = 3.4e38
    x[7, 8] = math.inf
    x[8] = -3.4e38
    for scores in ("softmax", "sigmoid"):
        for renorm in (True, False):
            ids, w = tre.tre_route(x, 6, scores=scores, renorm=renorm, groups=4, top_groups=2, group_best=1)
            want, ww = R.route(x, 6, scores=scores, renorm=renorm, groups=4, top_groups=2, group_best=1)
            assert torch.equal(ids.cpu(), want)
            keep = [i for i in range(40) if i != 8]
            assert ((w.double().cpu() - ww).abs() <= 2.0 ** -18 * ww + 1e-37)[keep].all()
            assert (ids[:2] == -1).all() and (w[:2] == 0).all()
    b = torch.zeros(64, device="cuda")
    b[0], b[1], b[2] = -math.inf, float("nan"), math.inf
    check(tre, logits(20, 64), 5, scores="sigmoid", bias=b)
    check(tre, logits(20, 64), 5, scores="softmax", bias=b)


def test_small_scores_keep_their_ratios(tre):
    """Sigmoids whose scores 32 bits hold no more, renormed."""
    x = -90 - logits(20, 32).abs()
    ids, w = tre.tre_route(x, 4, scores="sigmoid")
    want, ww = R.route(x, 4, scores="sigmoid")
    assert torch.equal(ids.cpu(), want) and ((w.double().cpu() - ww).abs() <= 2.0 ** -18 * ww).all()


def test_strides_outputs_streams_graphs(tre):
    wide = logits(77, 200)
    x = wide[:, 3:131]
    base = check(tre, x, 4)
    check(tre, wide[::2, :64], 4)
    check(tre, wide[:1].expand(9, 200), 4)
    ids, w = torch.empty(77, 4, dtype=torch.int32, device="cuda"), torch.empty(77, 4, device="cuda")
    got = tre.tre_route(x, 4, ids=ids, weights=w)
    assert got[0] is ids and got[1] is w and torch.equal(ids, base[0]) and torch.equal(w, base[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = tre.tre_route(x, 4, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], base[0]) and torch.equal(got[1], base[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = tre.tre_route(x, 4)
    wide.neg_()
    g.replay()
    assert torch.equal(out[0], check(tre, x, 4)[0])
    assert tre.tre_route(logits(0, 64), 3)[0].shape == (0, 3)


def test_many_rows(tre):
    b = 0.05 * torch.randn(256, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    x = logits(9000, 256)
    ids, w = tre.tre_route(x, 8, scores="sigmoid", bias=b, groups=8, top_groups=4)
    pick = torch.arange(0, 9000, 31, device="cuda")
    want, _ = R.route(x[pick], 8, scores="sigmoid", bias=b, groups=8, top_groups=4)
    assert torch.equal(ids[pick].cpu(), want)
