"""tre_chunk_attention against its definition in 64 bits."""
import math

import pytest
import torch

import paper_2609_29160_gb300 as tre
from tests import replica_ref as ref

pytestmark = pytest.mark.gpu


def check(bt, H, dtype="bf16", window=0, scale=None, hints=True, seed=1, q=None):
    dt = ref.T[dtype]
    if q is None:
        g = torch.Generator(device="cuda").manual_seed(seed)
        q = torch.randn(bt.rows, H, bt.dim, generator=g, device="cuda").to(dt)
    sc = 1 / math.sqrt(bt.dim) if scale is None else scale
    out, lse = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre, hints), scale=scale,
                                       window=window, lse=True)
    want, want_lse, bound = ref.attention(bt, q, sc, window)
    off = (out.double() - want).abs()
    assert torch.isfinite(out.double()).all()
    assert (off <= bound).all(), f"{(off / bound).max().item():.2f} of the bound"
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert (out[empty] == 0).all()
    # a logarithm of a 32-bit sum of scores of this size
    assert (lse.double() - want_lse)[~empty].abs().amax().nan_to_num() < 2e-3 if (~empty).any() else True
    again = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre, hints), scale=scale,
                                    window=window)
    assert torch.equal(out, again)
    return out, lse


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype,pool", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"),
                                        ("f16", "e4m3"), ("bf16", "i8"), ("f16", "i8")])
@pytest.mark.parametrize("lens", [
    [(0, 1)], [(15, 1)], [(16, 1), (17, 1), (0, 0), (63, 1), (64, 1), (1000, 1)],
    [(0, 5), (3, 17), (130, 1), (40, 130)],
    [(0, 129), (127, 128), (128, 256), (300, 257)],
])
def test_types_and_lengths(dim, dtype, pool, lens):
    bt = ref.Batch(lens, 16, 2, dim, ref.T[pool], seed=3)
    check(bt, 8, dtype)


@pytest.mark.parametrize("heads,group", [(1, 1), (4, 1), (3, 5), (1, 7), (2, 16), (1, 33)])
@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
def test_head_layouts(heads, group, pool):
    bt = ref.Batch([(70, 1), (9, 3), (200, 40)], 16, heads, 64, ref.T[pool], seed=4)
    check(bt, heads * group)


@pytest.mark.parametrize("page", [1, 3, 8, 24, 100, 256])
@pytest.mark.parametrize("pool,dim", [("bf16", 128), ("i8", 64)])
def test_page_sizes(page, pool, dim):
    bt = ref.Batch([(300, 1), (129, 140), (0, 2), (511, 1)], page, 2, dim, ref.T[pool], seed=5)
    check(bt, 4)


@pytest.mark.parametrize("order", ["hnd", "paired"])
@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
def test_cache_layouts(order, pool):
    bt = ref.Batch([(100, 1), (50, 150)], 16, 4, 128, ref.T[pool], seed=6, order=order)
    check(bt, 8)


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 1000])
@pytest.mark.parametrize("pool", ["bf16", "i8"])
def test_window(window, pool):
    bt = ref.Batch([(700, 1), (20, 300), (0, 140), (300, 4)], 16, 2, 64, ref.T[pool], seed=7)
    check(bt, 4, window=window)


@pytest.mark.parametrize("drop", [0.3, 0.9, 1.0])
@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
def test_pages_that_hold_nothing(drop, pool):
    """Unmapped pages are seen by no row; rows that see nothing give zeros."""
    bt = ref.Batch([(90, 1), (33, 200), (500, 1), (0, 20)], 16, 2, 128, ref.T[pool], seed=8,
                   drop=drop)
    check(bt, 6)
    check(bt, 6, window=20)


def test_lengths_that_disagree():
    """Lengths below the new tokens (rows before position zero see nothing), of zero,
    and past the table."""
    bt = ref.Batch([(10, 30), (0, 1), (40, 150), (60, 1)], 16, 2, 64, torch.bfloat16, seed=9)
    bt.ctx = torch.tensor([12, 0, -5, 1000], dtype=torch.int32, device="cuda")
    check(bt, 4)


@pytest.mark.parametrize("pad", [(0, 5), (7, 0), (3, 150)])
@pytest.mark.parametrize("long", [False, True])
def test_rows_of_no_sequence(pad, long):
    bt = ref.Batch([(3000 if long else 30, 1), (20, 9)], 16, 2, 128, torch.bfloat16, seed=10, pad=pad)
    check(bt, 4)


@pytest.mark.parametrize("lens", [[(4000, 1)], [(9000, 3), (100, 1)], [(5000, 64)], [(20000, 1)],
                                  [(3000, 130)]])
@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
def test_long_contexts_in_parts(lens, pool):
    bt = ref.Batch(lens, 64, 2, 128, ref.T[pool], seed=11)
    check(bt, 8)
    check(bt, 8, hints=False)


def test_wrong_hints_cost_time_only():
    bt = ref.Batch([(3000, 1), (100, 200)], 16, 2, 128, torch.bfloat16, seed=12)
    q = torch.randn(bt.rows, 4, 128, device="cuda").bfloat16()
    want, _, bound = ref.attention(bt, q, 128 ** -0.5, 0)
    for new, ctx in ((1, 10), (7, 700), (1000, 10 ** 6)):
        b = tre.KvBatch(bt.table, bt.ctx, bt.q_start, bt.rows, max_new=new, max_ctx=ctx)
        out = tre.tre_chunk_attention(q, bt.cache(tre), b)
        assert ((out.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("pool", ["bf16", "f16", "e4m3", "i8"])
def test_unused_slots_may_hold_anything(value, pool):
    bt = ref.Batch([(37, 1), (5, 70), (250, 9)], 32, 2, 64, ref.T[pool], seed=13, fill=value)
    check(bt, 8, "f16" if pool == "f16" else "bf16")


@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(0, 40)], [(20, 300)], [(1000, 8)]])
def test_values_ahead_do_not_reach_earlier_rows(pool, lens):
    """The last new token's key and value are no number: only its own row sees them."""
    bt = ref.Batch(lens, 16, 2, 128, ref.T[pool], seed=14)
    last = sum(lens[0]) - 1
    pg = int(bt.table[0, last // 16])
    for t in ((bt.k, bt.v) if bt.ks is None else (bt.ks, bt.vs)):
        t[pg, last % 16] = math.inf if t is bt.v or t is bt.vs else math.nan
    q = torch.randn(bt.rows, 8, 128, device="cuda").bfloat16()
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    want, _, bound = ref.attention(bt, q, 128 ** -0.5, 0)
    assert ((out.double() - want).abs()[:-1] <= bound[:-1]).all()
    assert not torch.isfinite(out[-1].double()).any()


@pytest.mark.parametrize("lens", [[(40, 1)], [(4000, 1)], [(30, 200)]])
def test_keys_that_are_no_number(lens):
    bt = ref.Batch(lens, 16, 1, 64, torch.bfloat16, seed=20)
    bt.k[:] = math.nan
    q = torch.randn(bt.rows, 4, 64, device="cuda").bfloat16()
    out, lse = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre), lse=True)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("scale", [1e-6, 3.0])
def test_scales(scale):
    bt = ref.Batch([(400, 1), (100, 150)], 16, 2, 64, torch.bfloat16, seed=15)
    check(bt, 4, scale=scale)


def test_large_scores():
    """Scores in the thousands, rising along the context: the maximum moves often."""
    bt = ref.Batch([(600, 1), (100, 200)], 16, 1, 64, torch.float16, seed=16)
    for i in range(2):
        for p in range(int(bt.ctx[i])):
            bt.k[int(bt.table[i, p // 16]), p % 16] *= 0.05 * p
    q = torch.randn(bt.rows, 2, 64, device="cuda").half() * 4
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    want, _, bound = ref.attention(bt, q, 0.125, 0)
    assert ((out.double() - want).abs() <= bound).all()


def test_strided_queries_and_outputs():
    bt = ref.Batch([(90, 1), (20, 160)], 16, 2, 64, torch.bfloat16, seed=17)
    wide = torch.randn(bt.rows, 12, 64, device="cuda").bfloat16()
    q = wide[:, 2:6]
    buf = torch.full((bt.rows, 4, 96), 7.0, dtype=torch.bfloat16, device="cuda")
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre), out=buf[..., :64])
    dense = tre.tre_chunk_attention(q.contiguous(), bt.cache(tre), bt.batch(tre))
    assert torch.equal(out, dense)
    assert (buf[..., 64:] == 7).all()


def test_offsets_past_32_bits():
    """A cache of over 2^32 elements, read and seen at its far end."""
    pages, page = 1100, 4096
    k = torch.zeros(pages, page, 8, 128, dtype=torch.int8, device="cuda")
    v = torch.zeros_like(k)
    ks = torch.ones(pages, page, 8, device="cuda") / 64
    vs = torch.ones(pages, page, 8, device="cuda")
    ids = [1099, 3, 1098]
    for n, p in enumerate(ids):
        k[p].random_(-100, 100)
        v[p].random_(-100, 100)
    bt = ref.Batch([(9000, 1), (1, 1)], page, 8, 128, torch.int8, seed=18)
    bt.k, bt.v, bt.ks, bt.vs, bt.n_pages = k, v, ks, vs, pages
    bt.table = torch.tensor([ids, ids], dtype=torch.int32, device="cuda")
    check(bt, 8)
    kk, vv = tre.tre_kv_read(bt.cache(tre), bt.batch(tre), dtype="f32")
    assert torch.equal(kk[0], k[1098, 9000 - 8192].float() / 64)
    assert torch.equal(vv[0], v[1098, 9000 - 8192].float())


def test_another_stream():
    bt = ref.Batch([(3000, 1), (20, 160)], 16, 2, 64, torch.bfloat16, seed=19)
    q = torch.randn(bt.rows, 4, 64, device="cuda").bfloat16()
    want = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre), stream=s) for _ in range(5)]
    s.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_memory_still_in_use_on_the_current_stream():
    """What a call makes for another stream is no block that the current stream's work,
    queued before and already let go by its owner, has still to write."""
    bt = ref.Batch([(3000, 1), (20, 160)], 16, 2, 64, torch.bfloat16, seed=28)
    q = torch.randn(bt.rows, 4, 64, device="cuda").bfloat16()
    cache, batch = bt.cache(tre), bt.batch(tre)
    s = torch.cuda.Stream()
    want = tre.tre_chunk_attention(q, cache, batch, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    big = torch.zeros(1 << 28, device="cuda")
    for _ in range(20):
        big += 1
    gone = [torch.empty_like(q) for _ in range(4)] + [
        torch.empty(1 << 20, dtype=torch.uint8, device="cuda") for _ in range(2)]
    for t in gone:
        t.fill_(3)
    del gone, t
    got = tre.tre_chunk_attention(q, cache, batch, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    bt = ref.Batch([(30, 1)], 16, 2, 64, torch.bfloat16)
    c, b = bt.cache(tre), bt.batch(tre)
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="rows"):
        tre.tre_chunk_attention(torch.cat([q, q]), c, b)
    with pytest.raises(ValueError, match="multiple"):
        tre.tre_chunk_attention(q[:, :3], c, b)
    with pytest.raises(ValueError, match="dim"):
        tre.tre_chunk_attention(q[..., :32], c, b)
    with pytest.raises(ValueError, match="takes no"):
        tre.tre_chunk_attention(q.half(), c, b)
    with pytest.raises(ValueError, match="type"):
        tre.tre_chunk_attention(q.float(), c, b)
    with pytest.raises(ValueError, match="dense"):
        tre.tre_chunk_attention(q.repeat(1, 1, 2)[..., ::2], c, b)
    for bad in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(tre.TreError, match="invalid argument"):
            tre.tre_chunk_attention(q, c, b, scale=bad)
    with pytest.raises(tre.TreError, match="invalid argument"):
        tre.tre_chunk_attention(q, c, b, window=-1)
    off = torch.zeros(4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(1, 4, 64)
    with pytest.raises(tre.TreError, match="invalid argument"):
        tre.tre_chunk_attention(off, c, b)
    with pytest.raises(ValueError, match="CUDA"):
        tre.tre_chunk_attention(q.cpu(), c, b)


def test_no_rows():
    bt = ref.Batch([(30, 0)], 16, 2, 64, torch.bfloat16)
    q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre)).shape == (0, 4, 64)


@pytest.mark.parametrize("pool", ["bf16", "i8"])
@pytest.mark.parametrize("new", [1, 100])
def test_a_cache_of_no_pages(pool, new):
    dt = ref.T[pool]
    k = torch.zeros(0, 16, 2, 64, dtype=dt, device="cuda")
    sc = torch.zeros(0, 16, 2, device="cuda") if dt in ref.TOP else None
    c = tre.KvCache(k, k, sc, sc)
    b = tre.KvBatch(torch.zeros(1, 7, dtype=torch.int32, device="cuda"),
                    torch.tensor([new], dtype=torch.int32, device="cuda"),
                    torch.tensor([0, new], dtype=torch.int32, device="cuda"), new)
    out, lse = tre.tre_chunk_attention(torch.ones(new, 4, 64, device="cuda").bfloat16(), c, b, lse=True)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[(2500, 1), (40, 1)], [(300, 200), (20, 1)]])
def test_in_a_graph(pool, lens):
    """Captured once, replayed over other contents of the same tensors."""
    bt = ref.Batch(lens, 16, 2, 64, ref.T[pool], seed=21)
    q = torch.randn(bt.rows, 8, 64, device="cuda").bfloat16()
    k = torch.randn(bt.rows, 2, 64, device="cuda").bfloat16()
    c, b = bt.cache(tre), bt.batch(tre)

    def step():
        tre.tre_kv_append(c, b, k, k)
        return tre.tre_chunk_attention(q, c, b)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    q.copy_(torch.randn_like(q))
    k.copy_(torch.randn_like(k))
    bt.ctx.copy_(bt.ctx - 7)
    g.replay()
    torch.cuda.synchronize()
    got = out.clone()
    assert torch.equal(got, step())


@pytest.mark.parametrize("groups,lens", [(1, [(5, 600), (0, 65), (0, 64), (3000, 70)]),
                                         (8, [(0, 9), (0, 8), (100, 7), (4000, 33)]),
                                         (5, [(0, 13), (77, 12), (2000, 400)])])
@pytest.mark.parametrize("pool", ["f16", "e4m3", "i8"])
def test_few_and_many_rows_side_by_side(groups, lens, pool):
    """Sequences on both sides of the line between the two kernels, parts on either."""
    bt = ref.Batch(lens, 32, 2, 128, ref.T[pool], seed=22, drop=0.05)
    check(bt, 2 * groups, "f16")
    check(bt, 2 * groups, "f16", window=90)


@pytest.mark.parametrize("groups,lens", [
    (1, [(300, 16), (400, 17), (100, 300), (2000, 1)]),
    (4, [(300, 4), (300, 5), (2500, 1), (100, 100)]),
    (20, [(700, 1), (3000, 1), (50, 2), (10, 30)]),
    (70, [(700, 1), (3000, 1), (50, 2)])])
@pytest.mark.parametrize("pool", ["bf16", "i8"])
def test_a_few_rows_beside_chunks(groups, lens, pool):
    """Sequences of one token, of 16 and of 17 rows, next to longer ones."""
    check(ref.Batch(lens, 16, 2, 128, ref.T[pool], seed=26), 2 * groups)


@pytest.mark.parametrize("lens", [[(16000, 1280)], [(15000, 700), (9000, 600), (200, 1)]])
@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
def test_chunks_of_one_to_two_rounds_in_parts(lens, pool):
    check(ref.Batch(lens, 64, 8, 64, ref.T[pool], seed=27), 32)


@pytest.mark.parametrize("pool,heads,group,dim", [("bf16", 8, 1, 64), ("f16", 4, 4, 128),
                                                  ("i8", 4, 4, 64), ("e4m3", 4, 2, 128)])
def test_more_ragged_units_than_sms(pool, heads, group, dim):
    """Which block takes which sequence's rows changes nothing, call after call."""
    lens = [((37 * i) % 400, 40 + (389 * i) % 900) for i in range(24)] + [(70, 1), (0, 3)]
    bt = ref.Batch(lens, 32, heads, dim, ref.T[pool], seed=29)
    dt = "f16" if pool == "f16" else "bf16"
    out, _ = check(bt, heads * group, dt)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(bt.rows, heads * group, dim, generator=g, device="cuda").to(ref.T[dt])
    cache, batch = bt.cache(tre), bt.batch(tre)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = tre.tre_chunk_attention(q, cache, batch)
    for _ in range(3):
        got.zero_()
        graph.replay()
        assert torch.equal(got, out)


def test_many_sequences():
    """More sequences than a warp looks at in a step, most of them of no rows."""
    lens = [((7 * i) % 300, (i * i) % 5 if i % 9 else 40 + i % 100) for i in range(150)]
    bt = ref.Batch(lens, 16, 1, 64, torch.bfloat16, seed=23)
    check(bt, 4)
