"""Norms around a block of rows that no 16-byte access takes, at every width's way."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("dim", [255, 257, 511, 513, 777, 1023, 1025, 4095, 4097, 8191, 8193, 9001, 12289, 16383])
def test_odd_widths(tre, dim, dtype, stream):
    g = torch.Generator(device="cuda").manual_seed(dim)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")

    for rows in (1, 6):
        a = {"residual": normal(rows, dim).to(R.T[stream]), "y": normal(rows, dim).to(R.T[dtype]),
             "post_weight": (1 + 0.2 * normal(dim)).to(R.T[dtype]), "gate": normal(rows, dim).to(R.T[dtype]),
             "weight": (1 + 0.2 * normal(dim)).to(R.T[dtype])}
        r, off, n, offn = R.block_norm(a["residual"], a["y"], a["post_weight"], a["gate"], 1.0, a["weight"], 1e-6)
        got = tre.tre_block_norm(**a)
        R.near(got[0], r, off)
        R.near(got[1], n, offn)
        again = tre.tre_block_norm(**a, residual_out=a["residual"], out=a["y"])      # in place
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("dim", [1000, 1024, 8200, 16384])
def test_rows_on_any_element(tre, dim):
    """Widths that eight divides, on addresses that sixteen bytes do not."""
    g = torch.Generator(device="cuda").manual_seed(dim)
    wide = torch.randn(9, dim + 3, generator=g, device="cuda").bfloat16()
    y, w = torch.randn(9, dim, generator=g, device="cuda").bfloat16(), torch.ones(dim, device="cuda").bfloat16()
    x = wide[:, 1:dim + 1]
    out = torch.full((9, dim + 2), 7.0, device="cuda", dtype=torch.bfloat16)
    r, off, n, offn = R.block_norm(x, y, w, None, 1.0, w, 1e-6)
    got = tre.tre_block_norm(x, y, post_weight=w, weight=w, out=out[:, 1:dim + 1])
    R.near(got[0], r, off)
    R.near(got[1], n, offn)
    assert (out[:, 0] == 7).all() and (out[:, -1] == 7).all()
