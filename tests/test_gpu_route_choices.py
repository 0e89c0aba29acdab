"""Choices of experts where 32 bits cannot tell, beyond ordinary scores."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


def logits(rows, experts, seed=1, std=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, experts, generator=g, device="cuda") * std


def check(tre, x, top, **how):
    ids, w = tre.tre_route(x, top, **how)
    want, ww = R.route(x, top, **how)
    bad = (ids.cpu() != want).any(-1)
    assert not bad.any(), f"{int(bad.sum())} of {len(bad)} rows"
    # an exponential, a sum of up to 1,024, a quotient and products in 32 bits; and the difference d
    # of two logits is rounded by 2^-24 |d|, which is that much of its exponential: |d| is at most the
    # weight's own |log| and that of a sum of up to 1,024
    d = ww.clamp(1e-300).log().abs() + 7
    assert ((w.double().cpu() - ww).abs() <= 2.0 ** -24 * (40 + d) * ww.abs() + 1e-37).all()


def closest(x, scores, bias, groups, top_groups, n):
    """The n rows whose last kept group (by the sum of its two best) is closest to the next."""
    s = torch.softmax(x.double(), -1) if scores == "softmax" else torch.sigmoid(x.double())
    c = (s + bias.double()).unflatten(-1, (groups, -1))
    value = c.topk(2, -1).values.sum(-1).sort(-1, descending=True).values
    return x[(value[:, top_groups - 1] - value[:, top_groups]).argsort()[:n]]


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("most", [0.6, 30.0, 300.0, 1e5])
def test_groups_whose_biases_cancel(tre, scores, most):
    """A group's two best c are large and of opposite sign, their sum is small: each is off by
    half a unit of its own size."""
    for experts, groups, seed in ((8, 4, 1), (64, 8, 2), (256, 8, 3), (40, 4, 4)):
        x = logits(60_000, experts, seed)
        bias = torch.full((experts,), -most, device="cuda")
        bias[::experts // groups] = most
        if experts == 8:
            bias[0::2], bias[1::2] = most, 0.5 - most
        near = closest(x, scores, bias, groups, groups // 2, 400)
        check(tre, near, 2, scores=scores, bias=bias, groups=groups, top_groups=groups // 2, group_best=2)


def test_one_group_of_large_biases(tre):
    """Others than the last that stays are off too: one far larger in its parts, not in its sum."""
    x = logits(60_000, 32, 5)
    bias = torch.zeros(32, device="cuda")
    bias[0:8] = torch.tensor([5e4] + [-5e4] * 7, device="cuda")
    near = closest(x, "sigmoid", bias, 4, 2, 1500)
    check(tre, near, 3, scores="sigmoid", bias=bias, groups=4, top_groups=2, group_best=2)


@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("experts,groups", [(64, 8), (256, 8), (96, 4), (1024, 16)])
def test_choices_go_by_logits_without_a_bias(tre, scores, experts, groups):
    """Scores that 64 bits round to the same number are as different as their logits."""
    x = logits(60, experts, 6)
    x[:20] = x[:20].abs() * 9 + 38                        # sigmoids of 1, less than 2^-54
    x[20:40, ::3] += 60
    x[40:50] *= 700                                       # softmax scores of 0
    x[50:] = x[50:] * 40 - 200
    for top, best in ((4, 2), (8, 2), (8, 1), (24, 2)):
        check(tre, x, top, scores=scores, groups=groups, top_groups=groups // 2, group_best=best, renorm=False)
    check(tre, x[:40], 6, scores=scores, groups=groups, top_groups=groups // 2, group_best=2)


@pytest.mark.parametrize("top", [11, 16, 20, 24, 31, 32])
@pytest.mark.parametrize("experts", [33, 64, 200, 256, 512, 1024])
def test_many_of_them(tre, experts, top):
    """More candidates than lanes: every kind of choice, with logits that repeat and that do not."""
    bias = 0.1 * torch.randn(experts, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    x = logits(50, experts, top)
    x[20:30] = x[20:30].bfloat16().float()
    x[30:35] = (2 * x[30:35]).round() / 2
    x[35] = 0
    x[36, 5:] = -float("inf")
    x[37:40, ::2] = -float("inf")
    x[40:45] *= 30
    for scores in ("softmax", "sigmoid"):
        check(tre, x, top, scores=scores)
        check(tre, x, top, scores=scores, bias=bias)
        check(tre, x, top, scores=scores, bias=bias + 100)
        if experts % 8 == 0:
            for best in (1, 2):
                check(tre, x, top, scores=scores, bias=bias, groups=8, top_groups=4, group_best=best)
                check(tre, x, top, scores=scores, groups=8, top_groups=4, group_best=best)


@pytest.mark.parametrize("gap", [0.0, 1e-9, 3e-8, 1e-6])
def test_many_of_them_close_to_each_other(tre, gap):
    """As many equal or nearly equal c as there are lanes and more, around the last that is chosen."""
    g = torch.Generator(device="cuda").manual_seed(8)
    for experts in (64, 256, 1024):
        x = logits(12, experts, 9)
        s = torch.sigmoid(x.double())
        bias = (0.7 - s[0] + gap * torch.randn(experts, generator=g, device="cuda").double()).float()
        bias[::7] += 0.2
        for top in (12, 24, 32):
            check(tre, x[:1], top, scores="sigmoid", bias=bias)
            check(tre, x, top, scores="sigmoid", bias=bias)
