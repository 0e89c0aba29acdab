"""Rows in 32 bits through 4-bit matrices: the whole range of their type."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


def small_matrix(n, k, group, dtype, most):
    """(codes, scales, the matrix in 64 bits) with elements up to 8 * most."""
    codes, scales, _, _ = R.matrix4(None, n, k, group, dtype, False, 5)
    scales = ((torch.rand(scales.shape, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda") + 0.5)
              * most / 1.5).to(dtype)
    q = torch.stack([codes & 15, codes >> 4], -1).double().view(n, k // group, group) - 8
    return codes, scales, (q * scales.double()[..., None]).view(n, k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t", [8, 120])
def test_rows_of_the_largest_numbers(tre, t, dtype):
    """Elements up to the largest float. 128 of them times at most 8 * 2^-12 stay below a quarter of it,
    so that every result is a number."""
    codes, scales, m = small_matrix(64, 128, 64, dtype, 2.0 ** -12)
    w = tre.Weights4(codes, scales)
    g = torch.Generator(device="cuda").manual_seed(7)
    most = torch.finfo(torch.float32).max
    x = (torch.rand(t, 128, generator=g, device="cuda") * 2 - 1).clamp(-0.99, 0.99)
    size = torch.tensor([3e37, 4.3e37, 1e38, 1.7e38, 2e38, 3e38, most, most], device="cuda").repeat(t // 8)
    x = x * size[:, None]
    x[torch.arange(t), torch.arange(t) % 128] = size
    got = tre.tre_linear4(x, w)
    assert torch.isfinite(got).all()
    R.near(got, *R.product(x, m))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("t", [8, 120])
def test_rows_of_the_smallest_numbers(tre, t, dtype):
    """Elements of up to 1e-30 .. 1e-42 (the last are below the normal numbers)."""
    codes, scales, z, m = R.matrix4(None, 64, 128, 64, dtype, True, 5)
    w = tre.Weights4(codes, scales, z)
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.rand(t, 128, generator=g, device="cuda") * 2 - 1
    x = x * torch.tensor([1e-30, 1e-34, 1e-36, 1e-37, 1e-38, 1e-39, 1e-40, 1e-42], device="cuda").repeat(t // 8)[:, None]
    got = tre.tre_linear4(x, w)
    R.near(got, *R.product(x, m))


@pytest.mark.parametrize("t", [6, 102])
@pytest.mark.parametrize("below", [12, 17, 20, 24, 27])
def test_small_elements_beside_a_large_one(tre, t, below):
    """Elements of 2^-below of a row's largest, whose code is its zero, keep 22 bits: the bound
    is of their own size, as the large one has no part in the result."""
    codes, scales, z, m = R.matrix4(None, 96, 256, 64, torch.bfloat16, False, 9)
    at = 37                                            # (the odd elements are the upper half bytes)
    codes[:, at // 2] = (codes[:, at // 2] & 15) | 8 << 4
    m[:, at] = 0
    w = tre.Weights4(codes, scales)
    g = torch.Generator(device="cuda").manual_seed(below)
    x = (torch.rand(t, 256, generator=g, device="cuda") + 1) * 2.0 ** -below
    x = x * (torch.randint(0, 2, x.shape, generator=g, device="cuda") * 2 - 1)
    x[:, at] = torch.rand(t, generator=g, device="cuda") * 0.99 + 1
    size = x.double().abs() @ m.abs().T
    # 2^-22 of each element; R.product's bound is of the same sizes
    y, off = R.product(x, m)
    R.near(tre.tre_linear4(x, w), y, off + 2.0 ** -22 * size)
    # one element alone: no sum hides its bits
    one = torch.zeros_like(x)
    one[:, at] = x[:, at]
    one[:, 5] = x[:, 5]
    want = one.double() @ m.T
    off = want.abs() * (2.0 ** -22 + 4 * 2.0 ** -24)      # its bits; product, scale, both halves' sum, the power
    R.near(tre.tre_linear4(one, w), want, off)
