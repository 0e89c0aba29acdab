"""Products with matrices in 4 bits against the formula in 64 bits."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


def rows(t, k, dtype, seed=1, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(t, k, generator=g, device="cuda") * std).to(dtype)


def check(tre, t, n, k, group, dtype, zeros=False, gated=False, seed=3, kind=None):
    codes, scales, z, m = R.matrix4(None, n, k, group, R.T[dtype], zeros, seed)
    w = tre.Weights4(codes, scales, z, gated=gated)
    x = rows(t, k, R.T[kind or dtype], seed)
    y, off = R.product(x, m)
    if gated:
        y, off = R.act(y, off)
    got = tre.tre_linear4(x, w)
    assert got.shape == y.shape and got.dtype == x.dtype
    R.near(got, y, off, f"{t} x {k} x {n}")
    assert torch.equal(got, tre.tre_linear4(x, w))
    tre.check_replica()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("t", [1, 2, 8, 9, 16, 17, 32])
def test_few_rows(tre, t, dtype):
    check(tre, t, 272, 384, 128, dtype)


@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, False), (64, True), (128, True)])
@pytest.mark.parametrize("t", [1, 11, 30])
def test_groups_and_zeros(tre, t, group, zeros):
    check(tre, t, 100, 3 * group, group, "bf16", zeros)
    check(tre, t, 100, 8 * group, group, "f16", zeros)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 127, 250])
@pytest.mark.parametrize("t", [3, 70])
def test_widths(tre, t, n):
    check(tre, t, n, 160, 32, "f16")


@pytest.mark.parametrize("n", [2, 30, 32, 34, 62, 256, 258, 500])
@pytest.mark.parametrize("t", [1, 20, 90])
def test_gated(tre, t, n):
    check(tre, t, n, 192, 64, "bf16", gated=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("t", [33, 64, 65, 255, 256, 257, 600])
def test_many_rows(tre, t, dtype):
    check(tre, t, 300, 256, 128, dtype)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("n,k", [(256, 128), (700, 1408), (4100, 640)])
def test_many_rows_groups(tre, n, k, group, zeros):
    check(tre, 150, n, k, group, "bf16", zeros)


def test_more_units_than_blocks(tre):
    check(tre, 1100, 9000, 320, 64, "f16")
    check(tre, 2100, 2050, 2048, 128, "bf16", gated=True)


@pytest.mark.parametrize("k", [32, 96, 224])
def test_odd_chunks(tre, k):
    for t in (2, 45):
        check(tre, t, 80, k, 32, "bf16", True)


@pytest.mark.parametrize("t", [1, 7, 16, 17, 130])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_in_32_bits(tre, t, dtype):
    check(tre, t, 130, 256, 64, dtype, True, kind="f32")
    check(tre, t, 130, 256, 128, dtype, gated=True, kind="f32")


def test_rows_in_32_bits_of_any_size(tre):
    """Sizes from the smallest to the largest numbers; infinities and NaN in their own rows."""
    codes, scales, z, m = R.matrix4(None, 64, 128, 64, torch.bfloat16, False, 5)
    w = tre.Weights4(codes, scales)
    x = rows(8, 128, torch.float32)
    for i, s in enumerate((1e-25, 1e-10, 1.0, 1e10, 1e30)):
        x[i] *= s
    x[5] = 0
    x[6, 3] = float("inf")
    x[7, 100] = float("nan")
    got = tre.tre_linear4(x, w)
    y, off = R.product(x[:6], m)
    R.near(got[:6], y, off)
    assert not torch.isfinite(got[6]).any() and torch.isnan(got[7]).all()


@pytest.mark.parametrize("t", [5, 100])
def test_rows_do_not_reach_each_other(tre, t):
    codes, scales, z, m = R.matrix4(None, 96, 128, 64, torch.bfloat16, True, 5)
    w = tre.Weights4(codes, scales, z)
    x = rows(t, 128, torch.bfloat16)
    want = tre.tre_linear4(x, w)
    y = x.clone()
    y[1] = float("nan")
    y[3, 5] = float("inf")
    got = tre.tre_linear4(y, w)
    keep = [i for i in range(t) if i not in (1, 3)]
    assert torch.equal(got[keep], want[keep])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[3]).any()


@pytest.mark.parametrize("t", [4, 80])
def test_strides(tre, t):
    codes, scales, z, m = R.matrix4(None, 50, 128, 32, torch.float16, False, 6)
    w = tre.Weights4(codes, scales)
    wide = rows(t, 300, torch.float16)
    x = wide[:, 40:168] if wide.stride(0) % 8 == 0 else rows(t, 304, torch.float16)[:, 40:168]
    out = torch.full((t, 77), 7.0, dtype=torch.float16, device="cuda")
    got = tre.tre_linear4(x, w, out=out[:, 3:53])
    R.near(got, *R.product(x, m))
    assert (out[:, :3] == 7).all() and (out[:, 53:] == 7).all()
    every = rows(2 * t, 128, torch.float16)
    R.near(tre.tre_linear4(every[::2], w), *R.product(every[::2], m))
    one = rows(1, 128, torch.float16).expand(t, 128)       # one row for all
    R.near(tre.tre_linear4(one, w), *R.product(one, m))


def test_no_rows(tre):
    codes, scales, z, m = R.matrix4(None, 50, 128, 32, torch.float16, False, 6)
    w = tre.Weights4(codes, scales)
    assert tre.tre_linear4(rows(0, 128, torch.float16), w).shape == (0, 50)
    assert tre.tre_linear4(rows(0, 128, torch.float32), w).shape == (0, 50)


@pytest.mark.parametrize("t,kind", [(3, "f16"), (200, "f16"), (40, "f32")])
def test_streams_and_graphs(tre, t, kind):
    codes, scales, z, m = R.matrix4(None, 128, 256, 64, torch.float16, False, 6)
    w = tre.Weights4(codes, scales)
    x = rows(t, 256, R.T[kind])
    want = tre.tre_linear4(x, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = tre.tre_linear4(x, w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    graphs, outs = [], []
    torch.cuda.synchronize()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(tre.tre_linear4(x, w))
        graphs.append(g)
    x.copy_(rows(t, 256, R.T[kind], seed=9))
    want = tre.tre_linear4(x, w)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    tre.check_replica()


@pytest.mark.parametrize("t,n,k,group", [(20, 20000, 512, 128), (40, 18000, 256, 64), (97, 300, 320, 64), (130, 520, 96, 32),
                                         (200, 6000, 256, 128), (333, 20000, 128, 128), (500, 9000, 192, 64)])
def test_units_of_every_width(tre, t, n, k, group):
    """Few and many rows on the tensor cores, by themselves and as a gated matrix in 32 bits."""
    check(tre, t, n, k, group, "bf16", group == 64)
    check(tre, t, n, k, group, "f16", gated=True)
    check(tre, t, n // 4 * 2, k, group, "f16", True, gated=True, kind="f32")


def test_outputs_on_any_element(tre):
    """Rows of y that 16 bytes do not divide, of both kernels' widest stores."""
    codes, scales, z, m = R.matrix4(None, 264, 128, 64, torch.bfloat16, False, 6)
    for gated in (False, True):
        w = tre.Weights4(codes, scales, gated=gated)
        for t in (5, 300):
            x = rows(t, 128, torch.bfloat16)
            want = tre.tre_linear4(x, w)
            for shift, wide in ((1, 270), (2, 270), (8, 272), (4, 269)):
                out = torch.full((t, wide), 7.0, dtype=torch.bfloat16, device="cuda")
                got = tre.tre_linear4(x, w, out=out[:, shift:shift + want.shape[1]])
                assert torch.equal(got, want)
                assert (out[:, :shift] == 7).all() and (out[:, shift + want.shape[1]:] == 7).all()


@pytest.mark.parametrize("t", [1, 20, 40, 300])
@pytest.mark.parametrize("n", [31, 264])
def test_rows_out_in_32_bits(tre, t, n):
    """Rows of 16 bits into rows of 32, which are then rounded no more."""
    codes, scales, z, m = R.matrix4(None, n, 192, 64, torch.bfloat16, True, 6)
    w = tre.Weights4(codes, scales, z)
    x = rows(t, 192, torch.bfloat16)
    got = tre.tre_linear4(x, w, dtype="f32")
    assert got.dtype == torch.float32
    R.near(got, *R.product(x, m))
    assert torch.equal(got.bfloat16(), tre.tre_linear4(x, w))
    out = torch.full((t, n + 3), 7.0, device="cuda")
    assert torch.equal(tre.tre_linear4(x, w, out=out[:, 2:n + 2]), got)
    assert (out[:, :2] == 7).all() and (out[:, n + 2:] == 7).all()
