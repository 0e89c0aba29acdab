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
