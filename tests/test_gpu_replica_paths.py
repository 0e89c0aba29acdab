"""Paths of a replica's operators that ordinary inputs do not take: scales of very
different size, rows of zeros and of the smallest numbers, outputs off 32-byte
boundaries, the bits that weights keep, logarithms."""
import math

import pytest
import torch

import paper_2609_29160_gb300 as tre
from tests import replica_ref as ref

pytestmark = pytest.mark.gpu


def exact(bt, q, window=0, split=False):
    """64-bit (out, lse, bound, lse bound). Where a product takes weights in 16 bits they
    keep 11 over codes and 16-bit floats, 8 over bfloat16, 16 there with `split`; as
    halves those below 2^-14 of the largest weight (times its value's scale) are off by
    up to 2^-25 of that. bfloat16 queries over codes lose up to 2^-25 of a row's largest
    element. A logarithm: its scores' errors, a 32-bit sum of n exponentials that are
    good to 2^-22, and a few 32-bit operations on the result."""
    rows, H, D = q.shape
    G = H // bt.heads
    out = torch.zeros(rows, H, D, dtype=torch.float64, device=q.device)
    bound, lse_bound = torch.zeros_like(out), torch.zeros_like(out[..., 0])
    lse = torch.full((rows, H), -math.inf, dtype=torch.float64, device=q.device)
    coded = bt.ks is not None
    half = coded or q.dtype == torch.float16
    u_p = 2.0 ** -11 if half else 2.0 ** -16 if split else 2.0 ** -8
    for i, (b, n) in enumerate(bt.lens):
        if n == 0:
            continue
        pos = torch.arange(b, b + n, device=q.device)
        j = torch.arange(b + n, device=q.device)
        page, slot, ok = bt.held(i, j)
        k, v = bt.values(bt.k, bt.ks, page, slot), bt.values(bt.v, bt.vs, page, slot)
        raw = bt.values(bt.v, None, page, slot)
        vs = bt.vs[page, slot].double() if coded else torch.ones_like(v[..., 0])
        see = (j[None] <= pos[:, None]) & ok[None]
        if window:
            see &= j[None] > pos[:, None] - window
        at = slice(bt.starts[i], bt.starts[i] + n)
        for h in range(H):
            x, kk, vv = q[at, h].double(), k[:, h // G], v[:, h // G]
            s = (x @ kk.T / math.sqrt(D)).masked_fill(~see, -math.inf)
            eps = 2.0 ** -24 * (D + 8) * (x.abs() @ kk.abs().T)
            if coded and q.dtype == torch.bfloat16:
                eps = eps + 2.0 ** -25 * x.abs().amax(1, keepdim=True) * kk.abs().sum(1)
            eps = (eps / math.sqrt(D)).masked_fill(~see, 0).amax(1, keepdim=True)
            some = see.any(1, keepdim=True)
            m = torch.where(some, s.amax(1, keepdim=True), torch.zeros_like(eps))
            p = torch.exp(s - m)
            l = p.sum(1, keepdim=True)
            w = p / torch.where(some, l, torch.ones_like(l))
            out[at, h] = w @ vv
            bound[at, h] = (u_p + 2 * eps + 2e-6) * (w @ vv.abs()) + ref.U[q.dtype] * out[at, h].abs() + 1e-7
            if half:
                top = (w * vs[:, h // G]).amax(1, keepdim=True)
                bound[at, h] += 2.0 ** -25 * top * (see.double() @ raw[:, h // G].abs())
            y = torch.where(some, m + torch.log(l), torch.full_like(m, -math.inf))
            lse[at, h] = y[:, 0]
            lse_bound[at, h] = (eps + see.sum(1, keepdim=True) * 2.0 ** -24 + 2.0 ** -21
                                + 2.0 ** -21 * (y.abs() + m.abs()))[:, 0]
    return out, lse, bound, lse_bound


def check(bt, H, dtype="bf16", window=0, split=False, out=None):
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(bt.rows, H, bt.dim, generator=g, device="cuda").to(ref.T[dtype])
    got, lse = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre), window=window, lse=True, out=out)
    want, want_lse, bound, lse_bound = exact(bt, q, window, split)
    # a result past the output type's largest number is infinite
    most = torch.finfo(q.dtype).max
    past = want.abs() - bound > most
    assert torch.equal(got[past].double(), want[past].sign() * math.inf)
    off = (got.double() - want).abs().masked_fill(want.abs() + bound >= most, 0)
    assert (off <= bound).all(), f"{(off / bound).max().item():.2f} of the bound"
    there = want_lse > -math.inf
    assert torch.isfinite(lse[there]).all() and (lse[~there] == -math.inf).all()
    off = (lse.double() - want_lse).abs()[there]
    assert (off <= lse_bound[there]).all(), f"{(off / lse_bound[there]).max().item():.2f} of the bound (lse)"


LENS = [[(0, 1), (90, 1), (700, 1)], [(0, 40), (300, 16)], [(0, 300), (1500, 140)], [(6000, 1)]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dtype,pool,dim", [("bf16", "bf16", 128), ("f16", "f16", 64), ("f16", "e4m3", 128),
                                            ("bf16", "e4m3", 64), ("f16", "i8", 64), ("bf16", "i8", 128)])
def test_bits_of_weights_and_logarithms(dtype, pool, dim, lens):
    check(ref.Batch(lens, 16, 2, dim, ref.T[pool], seed=31, drop=0.05), 8, dtype)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [[(0, 1), (3, 1), (90, 1), (700, 1)], [(0, 2), (20, 9)], [(9000, 1)]])
def test_single_tokens_keep_sixteen_bits_of_a_weight(dim, lens):
    """Few rows over a bfloat16 cache are bound by its bytes: their weights are multiplied in
    two halves."""
    check(ref.Batch(lens, 16, 2, dim, torch.bfloat16, seed=32), 8, split=True)


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("pool", ["e4m3", "i8"])
def test_scales_of_very_different_size(dtype, pool, lens):
    """Values that differ by up to 2^60 from token to token, rows of zeros among them (scale
    0, as an append leaves them)."""
    bt = ref.Batch(lens, 16, 2, 64, ref.T[pool], seed=33)
    g = torch.Generator(device="cuda").manual_seed(2)
    e = torch.randint(-30, 31, bt.vs.shape, generator=g, device="cuda")
    bt.vs.mul_(torch.exp2(e.float()))
    none = torch.rand(bt.vs.shape, generator=g, device="cuda") < 0.1
    for t, s in ((bt.k, bt.ks), (bt.v, bt.vs)):
        t.view(torch.uint8)[none] = 0
        s[none] = 0
    check(bt, 8, dtype)


def test_codes_of_the_smallest_rows():
    """Rows whose largest element is a subnormal of few bits: its scale is off by far more
    than a rounding of a normal number, and the quotient passes the last code."""
    for pool in (torch.int8, torch.float8_e4m3fn):
        n = 400
        bt = ref.Batch([(0, n)], 16, 2, 64, pool)
        g = torch.Generator(device="cuda").manual_seed(3)
        x = torch.randn(n, 2, 64, generator=g, device="cuda").bfloat16()
        # cosines from 2^-149 to about 2^-80, no sines: rows of x times that, rounded once
        c = torch.exp2(torch.linspace(-149, -80, n, device="cuda").double()).float()
        table = torch.zeros(n, 64, device="cuda")
        table[:, :32] = c[:, None]
        tre.tre_kv_append(bt.cache(tre), bt.batch(tre), x, x, cos_sin=table)
        j = torch.arange(n, device="cuda")
        pg, slot, _ = bt.held(0, j)
        want, sc = ref.codes(x.float() * c[:, None, None], pool)
        assert (sc < 2.0 ** -126).any() and (sc > 0).any()
        assert torch.equal(bt.ks[pg, slot], sc)
        got = bt.k.view(torch.uint8)[pg, slot]
        # (a zero keeps its sign in neither definition)
        same = (got == want.view(torch.uint8)) | ((got & 0x7f) == 0) & ((want.view(torch.uint8) & 0x7f) == 0)
        assert same.all(), (~same).sum()


@pytest.mark.parametrize("pool", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("lens", [[(90, 1), (20, 160)], [(20000, 1)], [(0, 300), (40, 20)]])
def test_outputs_on_16_byte_boundaries(pool, lens):
    bt = ref.Batch(lens, 16, 2, 64, ref.T[pool], seed=34)
    q = torch.randn(bt.rows, 8, 64, device="cuda").bfloat16()
    buf = torch.full((bt.rows, 8, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    dense = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre), out=buf[..., :64])
    assert out.data_ptr() == buf.data_ptr() and torch.equal(out, dense)
    assert (buf[..., 64:] == 7).all()


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pool", ["bf16", "e4m3", "i8"])
@pytest.mark.parametrize("width", [64, 72, 80])
def test_read_into_the_callers_rows(out, pool, width):
    bt = ref.Batch([(0, 130), (77, 30)], 16, 3, 64, ref.T[pool], seed=35)
    want = tre.tre_kv_read(bt.cache(tre), bt.batch(tre), dtype=out)
    buf = [torch.full((bt.rows, 3, width), 7.0, dtype=ref.T[out], device="cuda") for _ in range(2)]
    got = tre.tre_kv_read(bt.cache(tre), bt.batch(tre), dtype=out, k_out=buf[0][..., :64], v_out=buf[1][..., :64])
    for g, w, b in zip(got, want, buf):
        assert g.data_ptr() == b.data_ptr() and torch.equal(g, w)
        assert (b[..., 64:] == 7).all()
    with pytest.raises(ValueError, match="strides"):
        tre.tre_kv_read(bt.cache(tre), bt.batch(tre), dtype=out, k_out=buf[0][..., :64],
                        v_out=torch.empty_like(want[1]) if width != 64 else torch.empty(
                            bt.rows, 3, 72, dtype=ref.T[out], device="cuda")[..., :64])


@pytest.mark.parametrize("lens", [[(0, 1), (700, 1)], [(20, 9)], [(0, 300)]])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_value_without_end_stays_so(dtype, lens):
    """Rows that see an infinite value are infinite in its column and nowhere else."""
    bt = ref.Batch(lens, 16, 2, 64, ref.T[dtype], seed=36)
    for i in range(len(lens)):
        bt.v[int(bt.table[i, 0]), 0, :, 3] = math.inf
        bt.v[int(bt.table[i, 0]), 0, :, 9] = -math.inf
    q = torch.randn(bt.rows, 8, 64, device="cuda").to(ref.T[dtype])
    out = tre.tre_chunk_attention(q, bt.cache(tre), bt.batch(tre))
    assert (out[..., 3] == math.inf).all() and (out[..., 9] == -math.inf).all()
    out[..., [3, 9]] = 0
    assert torch.isfinite(out).all()


def test_calls_without_a_diag_have_their_own():
    """Dropped rows are counted in pinned host memory, and an error there is raised by the
    next call (once), or by check_replica. The error is written here by the host."""
    bt = ref.Batch([(30, 3)], 16, 2, 64, torch.bfloat16)
    c, b = bt.cache(tre), bt.batch(tre)
    k = torch.randn(3, 2, 64, device="cuda").bfloat16()
    tre.tre_kv_append(c, b, k, k)
    torch.cuda.synchronize()
    before = tre.read_diag(tre.replica_diag())["dropped_range"]
    bt.table[0, 2] = -1                     # of position 32
    tre.tre_kv_append(c, b, k, k)
    torch.cuda.synchronize()
    assert tre.read_diag(tre.replica_diag())["dropped_range"] == before + 1
    own = tre.Diag.from_address(tre.replica_diag().data_ptr())
    calls = [lambda: tre.tre_kv_append(c, b, k, k), lambda: tre.tre_kv_read(c, b),
             lambda: tre.tre_chunk_attention(k, c, b), lambda: tre.tre_qk_norm_rope(k, None),
             tre.check_replica]
    for call in calls:
        own.err = 5
        with pytest.raises(tre.TreError, match="timed out") as e:
            call()
        assert e.value.code == 5
        call()
    # a call with a diag of its own does not look
    own.err = 5
    tre.tre_kv_append(c, b, k, k, diag=tre.new_diag())
    own.err = 0
    d = tre.replica.host_diag()
    tre.tre_kv_append(c, b, k, k, diag=d)
    torch.cuda.synchronize()
    assert tre.read_diag(d)["dropped_range"] == 1


def test_a_replica_looks_at_its_diag():
    from paper_2609_29160_gb300 import served
    rep = served.Replica()
    d = tre.Diag.from_address(rep.diag.data_ptr())
    for field, error in (("err", tre.TreError), ("dropped_range", RuntimeError)):
        setattr(d, field, 5)
        with pytest.raises(error, match="step"):
            rep.serve([(0, 10, 2)])
        setattr(d, field, 0)


def test_inputs_let_go_while_another_stream_reads_them():
    """A query tensor that is dropped right after the call is not handed out again while the
    other stream has still to read it."""
    bt = ref.Batch([(3000, 1), (20, 160)], 16, 2, 64, torch.bfloat16, seed=37)
    keep = torch.randn(bt.rows, 4, 64, device="cuda").bfloat16()
    cache, batch = bt.cache(tre), bt.batch(tre)
    want = tre.tre_chunk_attention(keep, cache, batch)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    big = torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):                 # `s` is busy for some milliseconds
            big += 1
    q = keep.clone()
    torch.cuda.current_stream().synchronize()
    got = tre.tre_chunk_attention(q, cache, batch, stream=s)
    del q
    others = [torch.full_like(keep, 3.0) for _ in range(8)]
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(others) == 8


def test_first_call_on_a_stream_of_its_own():
    """A process whose first call names a stream."""
    import subprocess
    import sys
    code = ("import torch, paper_2609_29160_gb300 as tre; s = torch.cuda.Stream(); "
            "q = torch.ones(3, 2, 64, device='cuda'); torch.cuda.synchronize(); "
            "y, _ = tre.tre_qk_norm_rope(q, None, stream=s); s.synchronize(); "
            "assert torch.equal(y, q)")
    subprocess.run([sys.executable, "-c", code], check=True, timeout=300)
