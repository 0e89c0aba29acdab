"""tre_qk_norm_rope, tre_kv_append and tre_kv_read against their definitions in 64 bits."""
import math

import pytest
import torch

import paper_2609_29160_gb300 as tre
from tests import replica_ref as ref

pytestmark = pytest.mark.gpu


def bound_of(want, size, dim, dtype):
    """A norm is a 32-bit sum of dim squares and a handful of operations, a turned
    element two products and a sum; then one rounding to dtype."""
    return 2.0 ** -24 * (dim + 16) * size + ref.U[dtype] * want.abs() + 1e-7 * (dtype != torch.float32)


def heads(T, H, D, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(T, H, D, generator=g, device="cuda") * 1.5).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("dim,rot", [(64, 64), (64, 16), (128, 128), (128, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk", [(1, 1, 1), (7, 5, 3), (400, 32, 8)])
def test_norm_and_rotation(dtype, dim, rot, interleaved, T, Hq, Hk):
    q, k = heads(T, Hq, dim, dtype), heads(T, Hk, dim, dtype, 1)
    qw, kw = heads(1, 1, dim, dtype, 2)[0, 0], heads(1, 1, dim, dtype, 3)[0, 0]
    table = ref.rotation(500, rot)
    pos = torch.randint(0, 500, (T,), device="cuda", dtype=torch.int32)
    got = tre.tre_qk_norm_rope(q, k, pos, qw, kw, eps=1e-5, cos_sin=table, interleaved=interleaved)
    for x, w, y in ((q, qw, got[0]), (k, kw, got[1])):
        want, size = ref.norm_rope(x, w, 1e-5, table, pos, interleaved)
        assert y.dtype == dtype and y.shape == x.shape
        assert ((y.double() - want).abs() <= bound_of(want, size, dim, dtype)).all()


@pytest.mark.parametrize("what", ["norm", "rotate", "q only", "k only", "q normed", "f32 weights"])
def test_parts_of_the_pass(what):
    dt = torch.bfloat16
    q, k = heads(33, 6, 128, dt), heads(33, 2, 128, dt, 1)
    w = heads(1, 1, 128, torch.float32 if what == "f32 weights" else dt, 2)[0, 0]
    table = None if what == "norm" else ref.rotation(64, 64)
    pos = torch.arange(33, device="cuda", dtype=torch.int32)
    qw, kw = (None, None) if what == "rotate" else (w, None if what == "q normed" else w)
    qi, ki = None if what == "k only" else q, None if what == "q only" else k
    got = tre.tre_qk_norm_rope(qi, ki, pos, qw, kw, cos_sin=table)
    for x, wt, y in ((qi, qw, got[0]), (ki, kw, got[1])):
        if x is None:
            assert y is None
            continue
        want, size = ref.norm_rope(x, wt, 1e-6, table, pos, False)
        assert ((y.double() - want).abs() <= bound_of(want, size, 128, dt)).all()


def test_strides_and_in_place():
    qkv = heads(50, 12, 64, torch.bfloat16)
    q, k = qkv[:, :8], qkv[:, 8:10]
    w = heads(1, 1, 64, torch.bfloat16, 2)[0, 0]
    table, pos = ref.rotation(50, 64), torch.arange(50, device="cuda", dtype=torch.int32)
    want = tre.tre_qk_norm_rope(q.contiguous(), k.contiguous(), pos, w, w, cos_sin=table)
    tail = qkv[:, 10:].clone()
    heads_first = torch.empty(8, 50, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    got = tre.tre_qk_norm_rope(q, k, pos, w, w, cos_sin=table, q_out=heads_first, k_out=k)
    assert torch.equal(got[0], want[0]) and torch.equal(k, want[1])
    assert torch.equal(qkv[:, 10:], tail)


def test_positions_outside_the_table():
    q = heads(4, 2, 64, torch.float16)
    pos = torch.tensor([3, -1, 10, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    diag = tre.new_diag()
    y, _ = tre.tre_qk_norm_rope(q, None, pos, cos_sin=ref.rotation(10, 64), diag=diag)
    assert (y[1:] == 0).all() and (y[0] != 0).any()
    assert tre.read_diag(diag)["dropped_range"] == 3


def test_rows_of_zeros_and_of_large_values():
    q = torch.zeros(3, 1, 64, device="cuda")
    q[1] = 1e18
    q[2] = 1e-22
    w = torch.ones(64, device="cuda")
    y, _ = tre.tre_qk_norm_rope(q, None, None, w, None, eps=1e-6)
    assert (y[0] == 0).all()
    assert ((y[1] - 1).abs() < 1e-5).all()
    assert ((y[2] - 1e-19).abs() < 1e-24).all()


POOLS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3"), ("bf16", "i8"),
         ("f16", "i8")]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("order", ["nhd", "hnd", "paired"])
@pytest.mark.parametrize("page", [1, 16, 100])
def test_append_as_it_is(dim, dtype, pool, order, page):
    """Without norms and rotation codes and scales are those of the definition, bit
    for bit, and nothing else in the cache changes."""
    dt, pt = ref.T[dtype], ref.T[pool]
    bt = ref.Batch([(0, 1), (30, 40), (200, 0), (15, 1), (99, 130)], page, 3, dim, pt, order=order)
    k, v = heads(bt.rows, 3, dim, dt), heads(bt.rows, 3, dim, dt, 1)
    k[5, 1] = 0
    want = {n: t.clone() for n, t in (("k", bt.k), ("v", bt.v))}
    scales = {n: t.clone() for n, t in (("k", bt.ks), ("v", bt.vs)) if t is not None}
    for i, (b, n) in enumerate(bt.lens):
        j = torch.arange(b, b + n, device="cuda")
        pg, slot, _ = bt.held(i, j)
        for name, x in (("k", k), ("v", v)):
            x = x[bt.starts[i]:bt.starts[i] + n]
            if pt in ref.TOP:
                c, sc = ref.codes(x, pt)
                want[name].view(torch.uint8)[pg, slot] = c.view(torch.uint8)
                scales[name][pg, slot] = sc
            else:
                want[name][pg, slot] = x
    assert tre.tre_kv_append(bt.cache(tre), bt.batch(tre), k, v) is None
    for name, t in (("k", bt.k), ("v", bt.v)):
        assert torch.equal(t.view(torch.uint8), want[name].view(torch.uint8))
        if scales:
            assert torch.equal(bt.ks if name == "k" else bt.vs, scales[name])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("group,lens", [(1, [(0, 1), (31, 1)]), (4, [(0, 300), (7, 45), (1000, 1)])])
def test_append_with_norms_and_rotation(dim, dtype, pool, interleaved, group, lens):
    dt, pt = ref.T[dtype], ref.T[pool]
    bt = ref.Batch(lens, 16, 2, dim, pt)
    q, k, v = (heads(bt.rows, h, dim, dt, s) for s, h in enumerate((2 * group, 2, 2)))
    qw, kw = heads(1, 1, dim, dt, 5)[0, 0], heads(1, 1, dim, dt, 6)[0, 0]
    table = ref.rotation(2000, dim)
    cache, batch = bt.cache(tre), bt.batch(tre)
    got = tre.tre_kv_append(cache, batch, k, v, q=q, q_weight=qw, k_weight=kw, cos_sin=table,
                            interleaved=interleaved)
    pos = torch.cat([torch.arange(b, b + n, device="cuda") for b, n in lens])
    want, size = ref.norm_rope(q, qw, 1e-6, table, pos, interleaved)
    assert ((got.double() - want).abs() <= bound_of(want, size, dim, dt)).all()
    kk, vv = tre.tre_kv_read(cache, batch, dtype="f32")
    want, size = ref.norm_rope(k, kw, 1e-6, table, pos, interleaved)
    for y, x, near in ((kk, want, bound_of(want, size, dim, torch.float32)), (vv, v.double(), 0.0)):
        if pt in ref.TOP:
            sc = x.abs().amax(-1, keepdim=True) / ref.TOP[pt]
            # half a step of the code, of a value that is itself `near`
            step = sc if pt == torch.int8 else torch.maximum(x.abs() * 2.0 ** -3, sc * 2.0 ** -9)
            bound = step / 2 * (1 + 1e-4) + near
        else:
            bound = ref.U[dt] * x.abs() + near + 1e-7
        assert ((y.double() - x).abs() <= bound).all()


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pool", ["bf16", "f16", "e4m3", "i8"])
@pytest.mark.parametrize("dim,heads_n,page", [(64, 1, 16), (128, 3, 7), (128, 8, 64)])
def test_read_back(out, pool, dim, heads_n, page):
    lens = [(0, 1), (0, 250), (0, 0), (77, 30)]
    bt = ref.Batch(lens, page, heads_n, dim, ref.T[pool], fill=math.nan)
    k, v = tre.tre_kv_read(bt.cache(tre), bt.batch(tre), dtype=out)
    for i, (b, n) in enumerate(lens):
        pg, slot, _ = bt.held(i, torch.arange(b, b + n, device="cuda"))
        for got, t, s in ((k, bt.k, bt.ks), (v, bt.v, bt.vs)):
            x = (t.view(torch.uint8)[pg, slot].view(t.dtype) if s is not None else t[pg, slot]).float()
            x = x if s is None else x * s[pg, slot][..., None]
            assert torch.equal(got[bt.starts[i]:bt.starts[i] + n], x.to(ref.T[out]))


def test_places_that_hold_nothing():
    """Unmapped pages and positions before zero are neither written nor read."""
    bt = ref.Batch([(10, 30), (40, 8)], 16, 2, 64, torch.int8, drop=0.5, seed=2, pad=(2, 3))
    bt.ctx = torch.tensor([25, 48], dtype=torch.int32, device="cuda")
    bt.table[1, 2] = bt.n_pages          # positions 32 to 47 of the second sequence
    before = bt.k.clone()
    k, v = heads(bt.rows, 2, 64, torch.bfloat16), heads(bt.rows, 2, 64, torch.bfloat16, 1)
    q = heads(bt.rows, 4, 64, torch.bfloat16, 2)
    diag = tre.new_diag()
    got = tre.tre_kv_append(bt.cache(tre), bt.batch(tre), k, v, q=q, cos_sin=ref.rotation(100, 64),
                            diag=diag)
    rk, _ = tre.tre_kv_read(bt.cache(tre), bt.batch(tre), dtype="f32")
    lost, written = 0, torch.zeros(bt.n_pages, 16, dtype=torch.bool, device="cuda")
    for i, (b, n) in enumerate(bt.lens):
        c = int(bt.ctx[i])
        pg, slot, ok = bt.held(i, torch.arange(c - n, c, device="cuda"))
        rows = slice(bt.starts[i], bt.starts[i] + n)
        lost += int((~ok).sum())
        written[pg[ok], slot[ok]] = True
        assert (got[rows][~ok] == 0).all() and (rk[rows][~ok] == 0).all()
        assert (rk[rows][ok] != 0).any(-1).all()
    assert lost > 5 and tre.read_diag(diag)["dropped_range"] == lost
    assert torch.equal(bt.k[~written], before[~written])
    for rows in (slice(0, 2), slice(bt.rows - 3, bt.rows)):
        assert (got[rows] == 0).all() and (rk[rows] == 0).all()


@pytest.mark.parametrize("pool", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_rows_that_hold_no_number(pool, bad):
    bt = ref.Batch([(0, 3)], 16, 2, 64, pool)
    k = heads(3, 2, 64, torch.bfloat16)
    k[1, 1, 7] = bad
    tre.tre_kv_append(bt.cache(tre), bt.batch(tre), k, k)
    y, _ = tre.tre_kv_read(bt.cache(tre), bt.batch(tre), dtype="f32")
    assert torch.isnan(y[1, 1]).all()
    y[1, 1] = 0
    assert torch.isfinite(y).all()


def test_another_stream():
    bt = ref.Batch([(0, 300)], 16, 2, 64, torch.bfloat16)
    k, q = heads(300, 2, 64, torch.bfloat16), heads(300, 4, 64, torch.bfloat16, 1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = tre.tre_kv_append(bt.cache(tre), bt.batch(tre), k, k, q=q, stream=s)
    a, b = tre.tre_kv_read(bt.cache(tre), bt.batch(tre), stream=s)
    s.synchronize()
    assert torch.equal(got, q) and torch.equal(a, k) and torch.equal(b, k)


def test_refusals():
    bt = ref.Batch([(0, 3)], 16, 2, 64, torch.bfloat16)
    c, b = bt.cache(tre), bt.batch(tre)
    k = heads(3, 2, 64, torch.bfloat16)
    for bad, what in ((k[:2], "rows"), (k[:, :1], "heads"), (k.half(), "type|takes no")):
        with pytest.raises(ValueError, match=what):
            tre.tre_kv_append(c, b, bad, k)
        with pytest.raises(ValueError, match=what):
            tre.tre_kv_append(c, b, k, bad)
    with pytest.raises(ValueError, match="64"):
        tre.tre_kv_append(c, b, heads(3, 2, 128, torch.bfloat16), k)
    with pytest.raises(ValueError, match="elements"):
        tre.tre_kv_append(c, b, k, k, k_weight=torch.ones(32, device="cuda"))
    with pytest.raises(ValueError, match="cos_sin"):
        tre.tre_kv_append(c, b, k, k, cos_sin=torch.ones(3, 64, device="cuda").half())
    with pytest.raises(tre.TreError, match="invalid argument"):
        tre.tre_kv_append(c, b, k, k, cos_sin=torch.ones(3, 24, device="cuda"))
    with pytest.raises(tre.TreError, match="invalid argument"):
        tre.tre_qk_norm_rope(k, None, None, cos_sin=ref.rotation(9, 64))
    with pytest.raises(tre.TreError, match="invalid argument"):
        tre.tre_qk_norm_rope(heads(3, 2, 48, torch.bfloat16), None)
    with pytest.raises(tre.TreError, match="invalid argument"):
        tre.tre_qk_norm_rope(k, None, eps=-1.0)
    with pytest.raises(ValueError, match="at least one"):
        tre.tre_qk_norm_rope(None, None)
    with pytest.raises(ValueError, match="positions|int32"):
        tre.tre_qk_norm_rope(k, None, torch.zeros(3, device="cuda"), cos_sin=ref.rotation(9, 64))
    with pytest.raises(ValueError, match="both"):
        tre.tre_kv_read(c, b, k_out=k)
    with pytest.raises(ValueError, match="type"):
        tre.tre_kv_read(c, b, dtype="i8")
    with pytest.raises(ValueError, match="scale"):
        tre.KvCache(bt.k.to(torch.int8), bt.v.to(torch.int8))
    with pytest.raises(ValueError, match="strides"):
        tre.KvCache(bt.k, torch.zeros(*bt.k.shape[:3], 128, device="cuda").bfloat16()[..., :64])
    with pytest.raises(ValueError, match="ctx_len"):
        tre.KvBatch(bt.table, bt.ctx.repeat(2), bt.q_start, 3)
    with pytest.raises(ValueError, match="pages"):
        tre.KvBatch(bt.table.long(), bt.ctx, bt.q_start, 3)


def test_no_rows():
    bt = ref.Batch([(30, 0)], 16, 2, 64, torch.bfloat16)
    k = heads(0, 2, 64, torch.bfloat16)
    assert tre.tre_kv_append(bt.cache(tre), bt.batch(tre), k, k, q=k).shape == (0, 2, 64)
    assert tre.tre_kv_read(bt.cache(tre), bt.batch(tre))[0].shape == (0, 2, 64)
    assert tre.tre_qk_norm_rope(k, None)[0].shape == (0, 2, 64)
