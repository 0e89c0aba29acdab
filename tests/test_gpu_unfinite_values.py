"""Attention over values that are no finite numbers: they reach the rows that see them, in
their own columns, and nothing else: no other row, sequence or column."""
import math

import pytest
import torch

import paper_2609_29160_gb300 as tre
from tests import replica_ref as ref

pytestmark = pytest.mark.gpu


def classes(bt, window):
    """What rows see of values that are no finite numbers: booleans [rows][heads][dim] for
    plus and minus infinity and NaN."""
    shape = (bt.rows, bt.heads, bt.dim)
    plus, minus, nan = (torch.zeros(shape, dtype=torch.bool, device=bt.v.device) for _ in range(3))
    for i, (b, n) in enumerate(bt.lens):
        if n == 0:
            continue
        pos = torch.arange(b, b + n, device=bt.v.device)
        j = torch.arange(b + n, device=bt.v.device)
        page, slot, ok = bt.held(i, j)
        v = bt.values(bt.v, bt.vs, page, slot)
        bad = j[(~torch.isfinite(v)).flatten(1).any(1) & ok]
        for p in bad.tolist():
            see = pos >= p
            if window:
                see &= p > pos - window
            rows = torch.arange(bt.starts[i], bt.starts[i] + n, device=pos.device)[see]
            for t, of in ((plus, v[p] == math.inf), (minus, v[p] == -math.inf), (nan, torch.isnan(v[p]))):
                t[rows] |= of
    return plus, minus, nan


def check(bt, H, dtype="bf16", window=0):
    dt, G = ref.T[dtype], H // bt.heads
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(bt.rows, H, bt.dim, generator=g, device="cuda").to(dt)
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre), window=window)
    want, _, bound = ref.attention(bt, q, bt.dim ** -0.5, window)
    plus, minus, nan = (t.repeat_interleave(G, 1) for t in classes(bt, window))
    odd = plus | minus | nan
    assert odd.any() and not odd.all()
    off = (out.double() - want).abs()
    assert torch.isfinite(out[~odd]).all()
    assert (off <= bound)[~odd].all(), f"{(off / bound)[~odd].max().item():.2f} of the bound"
    none = nan | (plus & minus)
    assert torch.isnan(out[none]).all()
    assert (out[plus & ~none] == math.inf).all() and (out[minus & ~none] == -math.inf).all()
    again = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre), window=window)
    assert torch.equal(out.nan_to_num(7.0), again.nan_to_num(7.0))


def spoil(bt, i, p, value, head=0, column=5, columns=1):
    """`value` at position p of sequence i. A cache of codes takes a code that is no number
    (e4m3 has no infinity)."""
    pg, slot = int(bt.table[i, p // bt.page]), p % bt.page
    if bt.v.dtype == torch.float8_e4m3fn:
        bt.v.view(torch.uint8)[pg, slot, head, column:column + columns] = 0x7f if value > 0 else 0xff
    elif bt.v.dtype == torch.int8:
        bt.vs[pg, slot, head] = value
    else:
        bt.v[pg, slot, head, column:column + columns] = value


POOLS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3"), ("bf16", "i8")]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype,pool", POOLS)
@pytest.mark.parametrize("window", [0, 50, 200])
@pytest.mark.parametrize("group,lens", [(4, [(300, 260), (70, 1), (40, 9)]), (1, [(500, 300), (0, 200)]),
                                        (8, [(60, 7), (33, 16), (90, 1)])])
def test_in_the_middle_of_new_tokens(dim, dtype, pool, window, group, lens):
    """Several in one chunk, in other columns and heads, beside sequences that have none."""
    bt = ref.Batch(lens, 16, 2, dim, ref.T[pool], seed=41)
    b, n = lens[0]
    for k, p in enumerate((b + n // 2, b + n // 2 + 1, b + n - 1, b + 1)):
        spoil(bt, 0, p, (math.inf, -math.inf, math.nan, math.inf)[k], head=k % 2, column=7 * k,
              columns=1 if k < 3 else dim - 21)
    check(bt, 2 * group, dtype, window)


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("pool", ["bf16", "e4m3", "i8"])
def test_early_in_a_long_context_beside_a_healthy_one(pool, value):
    """The first rows' value is seen by all that follow, over far more positions than could
    be gone through one by one; sequences beside it are what they would be alone."""
    lens = [(60000, 300), (3000, 280), (500, 1)]
    bt = ref.Batch(lens, 64, 2, 128, ref.T[pool], seed=42)
    spoil(bt, 0, 3, value)
    check(bt, 8)


@pytest.mark.parametrize("pool", ["bf16", "f16", "e4m3"])
def test_last_of_a_long_context(pool):
    """All rows of a chunk but the last keep their 40,000 positions' sum."""
    bt = ref.Batch([(40000, 500), (700, 400)], 64, 2, 64, ref.T[pool], seed=43)
    spoil(bt, 0, 40499, math.inf)
    check(bt, 4, "f16" if pool == "f16" else "bf16")


@pytest.mark.parametrize("heads,group,dim", [(8, 1, 64), (4, 4, 128)])
@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
@pytest.mark.parametrize("every", [1, 5])
def test_in_many_sequences(pool, heads, group, dim, every):
    """More units to do again than a block holds at a time."""
    lens = [((37 * i) % 400, 40 + (389 * i) % 900) for i in range(24)] + [(70, 1), (0, 3)]
    bt = ref.Batch(lens, 32, heads, dim, ref.T[pool], seed=44)
    for i, (b, n) in enumerate(lens):
        if i % every == 0 and n > 1:
            for p in {b + n - 1, b + n // 3}:
                spoil(bt, i, p, math.nan if i % 2 else math.inf, head=i % heads, column=i)
    check(bt, heads * group)


@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [3, 24, 256])
@pytest.mark.parametrize("window", [0, 130])
def test_pages_of_other_sizes(page, pool, window):
    bt = ref.Batch([(9000, 300), (129, 140), (0, 20)], page, 2, 64, ref.T[pool], seed=45)
    for p in (9150, 9299, 8900):
        spoil(bt, 0, p, math.inf)
    spoil(bt, 2, 19, math.nan)
    check(bt, 4, window=window)


@pytest.mark.parametrize("dtype,pool", [("bf16", "e4m3"), ("f16", "i8")])
def test_rows_that_an_append_left_without_a_number(dtype, pool):
    """A new token's value holds an infinity: its codes and scale are no numbers, and only
    rows that see it are not."""
    lens = [(100, 150), (20, 5), (300, 1)]
    bt = ref.Batch(lens, 16, 2, 64, ref.T[pool], seed=46)
    k = torch.randn(bt.rows, 2, 64, device="cuda").to(ref.T[dtype])
    v = k.clone()
    v[90, 0, 3] = math.inf
    v[bt.starts[1] + 4, 1, 3] = math.nan
    tre.tre_kv_append(bt.cache(tre), bt.batch(tre), k, v)
    q = torch.randn(bt.rows, 8, 64, device="cuda").to(ref.T[dtype])
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    odd = torch.zeros(bt.rows, 8, dtype=torch.bool, device="cuda")
    odd[90:150, :4] = True
    odd[bt.starts[1] + 4, 4:] = True
    assert torch.isnan(out[odd]).all() and torch.isfinite(out[~odd]).all()


def test_more_units_than_a_block_keeps_in_mind():
    """Over 10,000 units, every one with a row that must not see its sequence's last value."""
    bt = ref.Batch([(i % 7, 66 + i % 5) for i in range(720)], 16, 16, 64, torch.float16, seed=47)
    q = torch.randn(bt.rows, 16, 64, device="cuda").half()
    want = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    last = torch.zeros(bt.rows, dtype=torch.bool, device="cuda")
    for i, (b, n) in enumerate(bt.lens):
        p = b + n - 1
        bt.v[int(bt.table[i, p // 16]), p % 16, :, i % 64] = math.inf
        last[bt.starts[i] + n - 1] = True
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    assert torch.equal(out[~last], want[~last])
    assert ((out[last] == math.inf).sum(-1) == 1).all() and not torch.isnan(out).any()
