"""Norms around a block against the formulas in 64 bits."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


def make(rows, dim, dtype, stream=None, gate="", post=True, weight=None, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")

    t = R.T[dtype]
    a = {"residual": (normal(rows, dim) * 3).to(R.T[stream or dtype]), "y": normal(rows, dim).to(t),
         "weight": (1 + 0.2 * normal(dim)).to(R.T[weight or dtype]), "scale": 0.7, "eps": 1e-5}
    if post:
        a["post_weight"] = (1 + 0.2 * normal(dim)).to(R.T[weight or dtype])
    if gate:
        a["gate"] = normal(*{"channel": (dim,), "token": (rows, 1), "full": (rows, dim)}[gate]).to(t)
    return a


def want(a):
    return R.block_norm(a["residual"], a.get("y"), a.get("post_weight"), a.get("gate"), a.get("scale", 1.0),
                        a.get("weight"), a.get("eps", 1e-6))


def check(tre, a, **kw):
    r, off, n, offn = want(a)
    got = tre.tre_block_norm(**a, **kw)
    R.near(got[0], r, off, "residual")
    R.near(got[1], n, offn, "normed")
    return got


@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("dim", [1, 7, 64, 133, 256, 264, 1000, 1032, 4096, 5120, 8200, 16384])
def test_widths_and_types(tre, dim, dtype, stream):
    check(tre, make(5, dim, dtype, stream, "channel"))
    check(tre, make(3, dim, dtype, stream, "", False))


@pytest.mark.parametrize("gate", ["", "channel", "token", "full"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("weight", ["bf16", "f32"])
def test_forms(tre, gate, post, weight):
    for rows in (1, 2, 700):
        check(tre, make(rows, 520, "bf16", "f32", gate, post, weight))


def test_many_rows(tre):
    check(tre, make(20000, 72, "f16", "f16", "full"))
    check(tre, make(3001, 2048, "bf16", "f32", "token"))


def test_without_a_block_or_a_weight(tre):
    a = make(9, 300, "bf16", "f32")
    r, n = tre.tre_block_norm(a["residual"], weight=a["weight"], dtype="bf16")
    assert r is a["residual"] and n.dtype == torch.bfloat16
    w = R.block_norm(a["residual"], None, None, None, 1.0, a["weight"], 1e-6)
    R.near(n, w[2], w[3])
    r, n = tre.tre_block_norm(a["residual"], a["y"], scale=0.5)
    assert n is None
    w = R.block_norm(a["residual"], a["y"], None, None, 0.5, None, 1e-6)
    R.near(r, w[0], w[1])
    n = tre.tre_block_norm(a["residual"], weight=a["weight"].float())[1]
    assert n.dtype == torch.float32


def test_types_beside_each_other(tre):
    """Rows in 32 bits with the model's weights and gate, normed rows of either type."""
    a = make(11, 640, "f16", "f32", "channel")
    a["y"] = a["y"].float() * 1.0001
    for dtype in ("f16", "f32"):
        got = check(tre, a, dtype=dtype)
        assert got[1].dtype == R.T[dtype] and got[0].dtype == torch.float32


def test_in_place(tre):
    for dim in (512, 133):
        a = make(40, dim, "bf16", "bf16", "channel")
        r, off, n, offn = want(a)
        got = tre.tre_block_norm(**a, residual_out=a["residual"], out=a["y"])
        assert got[0] is a["residual"] and got[1] is a["y"]
        R.near(got[0], r, off)
        R.near(got[1], n, offn)


@pytest.mark.parametrize("shift", [0, 1, 8])
def test_strides(tre, shift):
    """Rows inside wider ones, on any element; what lies beside them stays."""
    a = make(30, 256, "bf16", "f32", "full")
    wide = {k: torch.zeros(30, 300 if shift == 1 else 304, dtype=a[k].dtype, device="cuda") for k in ("residual", "y", "gate")}
    for k, t in wide.items():
        t[:, shift:shift + 256] = a[k]
        a[k] = t[:, shift:shift + 256]
    r, off, n, offn = want(a)
    ro, out = (torch.full((30, 304), 7.0, dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16))
    got = tre.tre_block_norm(**a, residual_out=ro[:, shift:shift + 256], out=out[:, shift:shift + 256])
    R.near(got[0], r, off)
    R.near(got[1], n, offn)
    for t in (ro, out):
        assert (t[:, :shift] == 7).all() and (t[:, shift + 256:] == 7).all()
    every = make(60, 256, "bf16", "bf16")
    every["residual"], every["y"] = every["residual"][::2], every["y"][::2]
    check(tre, every)
    every["residual"] = every["residual"][:1].expand(30, 256)
    check(tre, every)


def test_rows_do_not_reach_each_other(tre):
    a = make(8, 264, "bf16")
    base = tre.tre_block_norm(**a)
    a["y"][1] = float("nan")
    a["residual"][4, 3] = float("inf")
    a["y"][6] = 0
    got = tre.tre_block_norm(**a)
    keep = [0, 2, 3, 5, 7]
    assert all(torch.equal(x[keep], y[keep]) for x, y in zip(got, base))
    assert torch.isnan(got[1][1]).all() and torch.isfinite(got[1][6]).all()
    assert got[0][4, 3] == float("inf") and torch.isnan(got[1][4, 3])


def test_sizes_of_numbers(tre):
    """Zeros, the smallest and large numbers."""
    a = make(4, 512, "f32")
    a["residual"] *= torch.tensor([0.0, 1e-20, 1.0, 1e15], device="cuda")[:, None]
    a["y"] *= torch.tensor([0.0, 1e-20, 1.0, 1e15], device="cuda")[:, None]
    check(tre, a)


def test_no_rows_streams_graphs(tre):
    a = make(0, 64, "bf16")
    assert tre.tre_block_norm(**a)[1].shape == (0, 64)
    a = make(70, 1024, "bf16", "f32", "channel")
    base = tre.tre_block_norm(**a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = tre.tre_block_norm(**a, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip(got, base))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = tre.tre_block_norm(**a)
    a["y"].neg_()
    g.replay()
    assert all(torch.equal(x, y) for x, y in zip(out, tre.tre_block_norm(**a)))
