"""The experts' products against the formula in 64 bits."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


class Case:
    """Random experts; `liked`: how much more some are chosen than others."""

    def __init__(self, tre, t, top, experts, dim, inner, group, dtype, zeros=False, liked=0.5, seed=2, out=None):
        self.dtype = R.T[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)
        c1, s1, z1, self.m1 = R.matrix4(experts, 2 * inner, dim, group, self.dtype, zeros, seed)
        c2, s2, z2, self.m2 = R.matrix4(experts, out or dim, inner, group, self.dtype, zeros, seed + 1)
        self.w1, self.w2 = tre.Weights4(c1, s1, z1, gated=True), tre.Weights4(c2, s2, z2)
        self.x = torch.randn(t, dim, generator=g, device="cuda").to(self.dtype)
        like = torch.randn(t, experts, generator=g, device="cuda") + liked * 4 * torch.randn(
            experts, generator=g, device="cuda")
        self.ids = like.topk(top, -1).indices.int().contiguous()
        self.weights = torch.rand(t, top, generator=g, device="cuda") - 0.2

    def check(self, tre):
        got = tre.tre_experts(self.x, self.ids, self.weights, self.w1, self.w2)
        R.near(got, *R.experts(self.x, self.ids, self.weights, self.m1, self.m2, self.dtype))
        assert torch.equal(got, tre.tre_experts(self.x, self.ids, self.weights, self.w1, self.w2))
        tre.check_replica()
        return got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("t,top,experts", [(1, 1, 1), (1, 4, 16), (2, 6, 64), (7, 2, 3), (33, 8, 128), (9, 32, 40)])
def test_few_tokens(tre, t, top, experts, dtype):
    Case(tre, t, top, experts, 256, 128, 64, dtype).check(tre)


@pytest.mark.parametrize("group,zeros,inner", [(32, False, 96), (32, True, 32), (64, True, 192), (128, False, 384)])
@pytest.mark.parametrize("t", [5, 40, 300])
def test_groups(tre, t, group, zeros, inner):
    Case(tre, t, 3, 8, 384, inner, group, "bf16", zeros).check(tre)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("t,top,experts", [(100, 2, 4), (700, 4, 8), (1000, 6, 16), (513, 1, 1), (600, 2, 60)])
def test_many_tokens(tre, t, top, experts, dtype):
    Case(tre, t, top, experts, 320, 160, 32, dtype).check(tre)


def test_one_expert_gets_all(tre):
    """Far more than the others, which get few or none."""
    for t in (50, 900):
        c = Case(tre, t, 2, 32, 256, 128, 128, "bf16")
        c.ids[:, 0] = 5
        c.ids[:, 1] = 31
        c.ids[3, 1] = 0
        c.check(tre)


def test_odd_widths(tre):
    for t in (3, 200):
        Case(tre, t, 2, 4, 160, 32, 32, "f16", out=45).check(tre)
        Case(tre, t, 2, 4, 160, 96, 32, "bf16", out=259).check(tre)


@pytest.mark.parametrize("t", [6, 300])
def test_ids_of_none(tre, t):
    """-1 adds nothing, an id past the last is counted, the same expert may come twice, a token
    without experts gives zeros; weights beside no expert do not count."""
    from paper_2609_29160_gb300 import replica
    c = Case(tre, t, 4, 8, 256, 128, 64, "bf16")
    c.ids[0] = -1
    c.ids[1, 2:] = -1
    c.ids[2, 0] = 8
    c.ids[3, 1] = 2 ** 31 - 1
    c.ids[3, 2] = -(2 ** 31)
    c.ids[4] = 3
    c.weights[0] = float("nan")
    c.weights[1, 2:] = float("inf")
    diag = replica.host_diag()
    got = tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2, diag=diag)
    torch.cuda.synchronize()
    assert tre.read_diag(diag)["dropped_range"] == 2
    w = torch.where((c.ids >= 0) & (c.ids < 8), c.weights, torch.zeros_like(c.weights))
    R.near(got, *R.experts(c.x, c.ids, w, c.m1, c.m2, c.dtype))
    assert (got[0] == 0).all()
    c.ids[:] = -1
    assert (tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2) == 0).all()


@pytest.mark.parametrize("t", [5, 400])
def test_tokens_do_not_reach_each_other(tre, t):
    c = Case(tre, t, 2, 4, 256, 128, 64, "f16")
    want = c.check(tre)
    c.x[1] = float("nan")
    c.x[3, 7] = float("inf")
    got = tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2)
    keep = [i for i in range(t) if i not in (1, 3)]
    assert torch.equal(got[keep], want[keep])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[3]).any()


@pytest.mark.parametrize("t", [4, 300])
def test_strides_streams_graphs(tre, t):
    c = Case(tre, t, 2, 8, 256, 128, 64, "bf16")
    want = tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2)
    wide = torch.zeros(t, 512, dtype=c.dtype, device="cuda")
    wide[:, 128:384] = c.x
    out = torch.full((t, 300), 7.0, dtype=c.dtype, device="cuda")
    assert torch.equal(tre.tre_experts(wide[:, 128:384], c.ids, c.weights, c.w1, c.w2, out=out[:, 9:265]), want)
    assert (out[:, :9] == 7).all() and (out[:, 265:] == 7).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2))
        graphs.append(g)
    c.x.neg_()
    c.ids.copy_(c.ids.flip(1))
    want = tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_no_rows(tre):
    c = Case(tre, 0, 2, 4, 256, 128, 64, "bf16")
    assert tre.tre_experts(c.x, c.ids, c.weights, c.w1, c.w2).shape == (0, 256)


@pytest.mark.parametrize("t,top,experts", [(500, 6, 200), (2000, 1, 1024), (300, 8, 512), (2100, 1, 3)])
def test_many_experts(tre, t, top, experts):
    """Plans of more pairs than a block sorts alone, for few and for many tokens an expert."""
    Case(tre, t, top, experts, 64, 32, 32, "bf16", liked=0.2).check(tre)
