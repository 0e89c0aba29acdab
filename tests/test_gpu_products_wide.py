"""Products along thousands of elements: experts of wide inner rows, long sums of both kernels."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


@pytest.mark.parametrize("dtype,group,zeros", [("bf16", 128, False), ("f16", 32, True)])
@pytest.mark.parametrize("t", [1, 9, 40, 300])
def test_experts_of_wide_inner_rows(tre, t, dtype, group, zeros):
    c1, s1, z1, m1 = R.matrix4(4, 2 * 4224, 256, group, R.T[dtype], zeros, 3)
    c2, s2, z2, m2 = R.matrix4(4, 200, 4224, group, R.T[dtype], zeros, 4)
    w1, w2 = tre.Weights4(c1, s1, z1, gated=True), tre.Weights4(c2, s2, z2)
    g = torch.Generator(device="cuda").manual_seed(t)
    x = torch.randn(t, 256, generator=g, device="cuda").to(R.T[dtype])
    ids = torch.rand(t, 4, generator=g, device="cuda").topk(2, -1).indices.int().contiguous()
    ids[0] = 3                                         # the same expert twice
    weights = torch.rand(t, 2, generator=g, device="cuda")
    got = tre.tre_experts(x, ids, weights, w1, w2)
    R.near(got, *R.experts(x, ids, weights, m1, m2, R.T[dtype]))
    assert torch.equal(got, tre.tre_experts(x, ids, weights, w1, w2))
    tre.check_replica()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("t", [2, 30, 130])
@pytest.mark.parametrize("k,group", [(14336, 128), (16416, 32), (32768, 64)])
def test_long_sums(tre, t, k, group, kind):
    codes, scales, z, m = R.matrix4(None, 70, k, group, torch.bfloat16, True, 5)
    w = tre.Weights4(codes, scales, z)
    g = torch.Generator(device="cuda").manual_seed(k)
    x = torch.randn(t, k, generator=g, device="cuda").to(R.T[kind])
    R.near(tre.tre_linear4(x, w, dtype="f32"), *R.product(x, m))
    tre.check_replica()
