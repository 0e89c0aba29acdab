"""The gate of gated products, silu(g) * u, at every size of g."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


def gate_and_up(tre, dtype):
    """A matrix of two rows whose product is (x[0], x[1])."""
    codes = torch.full((2, 16), 0x88, dtype=torch.uint8, device="cuda")
    codes[0, 0] = 0x89
    codes[1, 0] = 0x98
    return tre.Weights4(codes, torch.ones(2, 1, dtype=dtype, device="cuda"), gated=True)


def rows(g, u, dtype):
    x = torch.zeros(len(g), 32, dtype=dtype, device="cuda")
    x[:, 0], x[:, 1] = g, u
    return x


def silu_times(x):
    g, u = x[:, :1].double(), x[:, 1:2].double()
    return g * torch.sigmoid(g) * u


# quarters from -103.25 to 103.25: exact in the halves that rows in 32 bits are made of
GATES = torch.arange(-413, 414) / 4


@pytest.mark.parametrize("u", [3.0, -0.75, 1024.0])
def test_rows_in_32_bits(tre, u):
    """e = exp(-|g|) by two exponentials of its half (2 units of 2^-23 each, so 8 of 2^-24 together),
    which the denominator has by at most a half again (4), its sum, a reciprocal and four
    products (6)."""
    w = gate_and_up(tre, torch.bfloat16)
    x = rows(GATES.cuda(), u, torch.float32)
    want = silu_times(x)
    off = 18 * 2.0 ** -24 * want.abs() + R.LEAST[torch.float32]
    R.near(tre.tre_linear4(x, w), want, off, "many")
    for i in range(0, len(x), 101):
        R.near(tre.tre_linear4(x[i:i + 7], w), want[i:i + 7], off[i:i + 7], "few")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("u", [1.0, 2.0 ** 10, 2.0 ** 60, 2.0 ** 100])
def test_rows_in_16_bits(tre, dtype, u):
    """The quick exponential of half the gate is off by (2 + 0.6 |g|) units of 2^-23 and taken
    twice; everything else adds less than ten."""
    if dtype == "f16" and u > 2.0 ** 10:
        u = 60000.0                                        # (half's largest is 65504)
    w = gate_and_up(tre, R.T[dtype])
    g = GATES[::4].to(R.T[dtype]).cuda()
    if dtype == "f16":
        g = g[g < 1]                                       # (and so are the outputs)
    elif u > 2.0 ** 90:
        g = g[g < 80]
    x = rows(g, u, R.T[dtype])
    want = silu_times(x)
    off = (2 * (2 + 0.6 * x[:, :1].double().abs()) * 1.5 + 10) * 2.0 ** -23 * want.abs()
    # (the smallest results: what 32 bits hold of them)
    off = off + R.LEAST[torch.float32]
    for n in (1, 9, 40, len(x)):
        R.near(tre.tre_linear4(x[:n], w), want[:n], off[:n], f"first {n}")
        R.near(tre.tre_linear4(x[-n:], w), want[-n:], off[-n:], f"last {n}")


def test_infinities(tre):
    w = gate_and_up(tre, torch.bfloat16)
    inf, nan = float("inf"), float("nan")
    g = torch.tensor([inf, inf, 0.0, -0.0, nan, 1.0, -inf], device="cuda")
    u = torch.tensor([2.0, -2.0, 5.0, 5.0, 1.0, nan, 1.0], device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        # (an infinite element times the zeros of the other row is NaN: rows of infinities are not finite)
        y = tre.tre_linear4(rows(g, u, dtype), w)[:, 0]
        assert not torch.isfinite(y[[0, 1, 4, 5, 6]]).any() and (y[2:4] == 0).all()
