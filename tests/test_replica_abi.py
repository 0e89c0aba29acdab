"""Host side of a replica's operators: struct sizes and argument checks that answer
without a GPU (no call here enqueues anything)."""
import ctypes as C

import pytest

import paper_2609_29160_gb300 as tre
from paper_2609_29160_gb300 import replica as R

A = 4096                       # an aligned address; never dereferenced


def cache(dtype=R.BF16, pages=4, page=16, heads=2, dim=64, k=A, v=A, st=(2048, 128, 64), ks=0,
          vs=0, ss=(0, 0, 0)):
    return R.CACHE.pack(dtype, pages, page, heads, dim, k, v, *st, ks, vs, *ss)


def batch(n_seq=1, rows=3, max_new=0, max_ctx=0, max_pages=2, pages=A, row=2, ctx=A, start=A):
    return R.BATCH.pack(n_seq, rows, max_new, max_ctx, max_pages, pages, row, ctx, start)


def heads(dtype=R.BF16, rows=3, hq=4, hk=2, dim=64, q=A, k=A, qs=(256, 64), ks=(128, 64), qo=A,
          ko=A, wt=R.BF16, qw=0, kw=0, eps=1e-6, cs=0, cr=0, n_pos=0, rot=0, inter=0):
    return R.HEADS.pack(dtype, rows, hq, hk, dim, q, k, *qs, *ks, qo, ko, *qs, *ks, wt, qw, kw,
                        eps, cs, cr, n_pos, rot, inter)


def attend(dtype=R.BF16, h=4, window=0, scale=0.125, q=A, qs=(256, 64), out=A, os=(256, 64), lse=0):
    return R.ATTEND.pack(dtype, h, window, scale, q, *qs, out, *os, lse)


def test_struct_sizes():
    """The sizes that the header's fields give on LP64."""
    assert (R.CACHE.size, R.BATCH.size, R.HEADS.size, R.ATTEND.size) == (104, 56, 184, 72)


@pytest.mark.parametrize("bad", [
    dict(dim=32), dict(dim=80), dict(dtype=R.E4M3), dict(dtype=1), dict(dtype=9), dict(rows=-1),
    dict(hq=-1), dict(q=A + 2), dict(q=0), dict(qs=(250, 64)), dict(ks=(128, 60)), dict(qo=0),
    dict(ko=A + 8), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(qw=A, wt=R.F16), dict(kw=A + 4), dict(cs=A, cr=64, n_pos=5, rot=24),
    dict(cs=A, cr=64, n_pos=5, rot=128), dict(cs=A, cr=64, n_pos=0, rot=64),
    dict(cs=A, cr=63, n_pos=5, rot=64), dict(cs=A + 4, cr=64, n_pos=5, rot=64)])
def test_heads_are_checked(bad):
    assert tre.load().tre_qk_norm_rope(heads(**bad), A, None, None) == 1


def test_positions_are_needed_to_turn():
    lib = tre.load()
    assert lib.tre_qk_norm_rope(heads(cs=A, cr=64, n_pos=5, rot=64), None, None, None) == 1
    assert lib.tre_qk_norm_rope(None, None, None, None) == 1
    assert lib.tre_qk_norm_rope(heads(rows=0, q=0, k=0, qo=0, ko=0), None, None, None) == 0


BAD_CACHES = [dict(dtype=R.F32), dict(dtype=1), dict(dim=96), dict(page=0), dict(heads=0),
              dict(pages=-1), dict(k=0), dict(v=A + 2), dict(st=(2048, 130, 64)),
              dict(dtype=R.I8), dict(dtype=R.E4M3, ks=A)]
BAD_BATCHES = [dict(n_seq=-1), dict(rows=-1), dict(max_pages=-1), dict(pages=0), dict(ctx=0),
               dict(start=0), dict(max_new=-1), dict(max_ctx=-2), dict(n_seq=0)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_are_checked(bad):
    lib, c = tre.load(), cache(**bad)
    n = C.c_size_t(0)
    assert lib.tre_kv_append(c, batch(), heads(), A, 128, 64, None, None) == 1
    assert lib.tre_kv_read(c, batch(), R.BF16, A, A, 128, 64, None, None) == 1
    assert lib.tre_chunk_attention(c, batch(), attend(), None, C.byref(n), None, None) == 1


@pytest.mark.parametrize("bad", BAD_BATCHES)
def test_batches_are_checked(bad):
    lib, b = tre.load(), batch(**bad)
    n = C.c_size_t(1 << 40)
    assert lib.tre_kv_append(cache(), b, heads(), A, 128, 64, None, None) == 1
    assert lib.tre_kv_read(cache(), b, R.BF16, A, A, 128, 64, None, None) == 1
    assert lib.tre_chunk_attention(cache(), b, attend(), A, C.byref(n), None, None) == 1


def test_append_and_read_arguments():
    lib = tre.load()
    for h in (dict(dtype=R.F32), dict(dtype=R.F16), dict(hk=1), dict(dim=128), dict(rows=2)):
        assert lib.tre_kv_append(cache(), batch(), heads(**h), A, 128, 64, None, None) == 1
    for v in ((0, 128, 64), (A + 2, 128, 64), (A, 129, 64), (A, 128, 4)):
        assert lib.tre_kv_append(cache(), batch(), heads(), *v, None, None) == 1
    assert lib.tre_kv_append(cache(), batch(rows=0), heads(rows=0), 0, 0, 0, None, None) == 0
    for r in ((R.I8, A, A, 128, 64), (1, A, A, 128, 64), (R.BF16, 0, A, 128, 64),
              (R.F32, A, A + 4, 128, 64), (R.BF16, A, A, 127, 64)):
        assert lib.tre_kv_read(cache(), batch(), *r, None, None) == 1
    assert lib.tre_kv_read(cache(), batch(rows=0), R.BF16, 0, 0, 128, 64, None, None) == 0


@pytest.mark.parametrize("bad", [
    dict(dtype=R.F32), dict(dtype=R.F16), dict(h=3), dict(h=0), dict(window=-1), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(qs=(252, 64)),
    dict(os=(256, 60)), dict(q=A + 8), dict(out=A + 2)])
def test_attention_arguments(bad):
    n = C.c_size_t(0)
    assert tre.load().tre_chunk_attention(cache(), batch(), attend(**bad), None, C.byref(n),
                                          None, None) == 1


def test_attention_workspace():
    lib = tre.load()
    n = C.c_size_t(0)
    b = batch(max_new=3, max_ctx=100_000, max_pages=7000, row=7000)
    assert lib.tre_chunk_attention(cache(), b, attend(), None, C.byref(n), None, None) == 0
    assert n.value > 0
    small = C.c_size_t(n.value - 1)
    assert lib.tre_chunk_attention(cache(), b, attend(), A, C.byref(small), None, None) == 2
    assert lib.tre_chunk_attention(cache(), b, attend(), None, None, None, None) == 1
    assert lib.tre_chunk_attention(cache(), batch(rows=0), attend(q=0, out=0), A, C.byref(n),
                                   None, None) == 0
