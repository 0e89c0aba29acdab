"""Host side of the operators around a replica's attention: struct sizes and argument checks
that answer without a GPU (no call here enqueues anything)."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2609_29160_gb300 as tre
from paper_2609_29160_gb300 import layer as L
from paper_2609_29160_gb300 import replica as R

A = 4096                       # an aligned address; never dereferenced


def block(dtype=R.BF16, y_dtype=R.BF16, stream=R.BF16, wt=R.BF16, out_dtype=R.BF16, rows=3, dim=64, residual=A,
          r_row=64, y=A, y_row=64, post=0, gate=0, g_row=0, g_col=1, scale=1.0, eps=1e-6, weight=A, ro=A, ro_row=64,
          out=A, out_row=64):
    return L.BLOCK.pack(dtype, y_dtype, stream, wt, out_dtype, rows, dim, residual, r_row, y, y_row, post, gate,
                        g_row, g_col, scale, eps, weight, ro, ro_row, out, out_row)


def router(dtype=R.F32, rows=3, experts=64, top=6, logits=A, row=64, scores=0, bias=0, groups=1, top_groups=1, best=1,
           renorm=1, scale=1.0, ids=A, weights=A):
    return L.ROUTER.pack(dtype, rows, experts, top, logits, row, scores, bias, groups, top_groups, best, renorm, scale,
                         ids, weights)


def source(dtype=R.BF16, experts=1, n=64, k=128, group=64, gated=0, codes=A, scales=A, zeros=0):
    return L.SOURCE.pack(dtype, experts, n, k, group, gated, codes, scales, zeros)


def w4(dtype=R.BF16, experts=1, n=64, k=128, group=64, gated=0, zeros=0, packed=A):
    return L.W4.pack(dtype, experts, n, k, group, gated, zeros, packed)


def linear(dtype=R.BF16, rows=3, x=A, x_row=128, y=A, y_row=64, y_dtype=None):
    return L.LINEAR.pack(dtype, dtype if y_dtype is None else y_dtype, rows, x, x_row, y, y_row)


def tokens(dtype=R.BF16, rows=3, top=2, x=A, x_row=128, ids=A, weights=A, y=A, y_row=128):
    return L.TOKENS.pack(dtype, rows, top, x, x_row, ids, weights, y, y_row)


def test_struct_sizes(tmp_path):
    """The sizes that the header's fields have for a C compiler."""
    names = ("tre_block_rows", "tre_router", "tre_w4_source", "tre_w4", "tre_linear", "tre_tokens")
    sizes = (L.BLOCK.size, L.ROUTER.size, L.SOURCE.size, L.W4.size, L.LINEAR.size, L.TOKENS.size)
    assert sizes == (144, 88, 48, 40, 48, 64)
    text = '#include "tre.h"\n' + "".join(f"_Static_assert(sizeof({n}) == {s}, \"{n}\");\n" for n, s in zip(names, sizes))
    src = tmp_path / "sizes.c"
    src.write_text(text)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert subprocess.run(["gcc", "-std=c11", "-fsyntax-only", "-I", os.path.join(root, "include"), str(src)]).returncode == 0


@pytest.mark.parametrize("bad", [
    dict(dtype=R.I8), dict(dtype=1), dict(y_dtype=R.F16), dict(stream=R.F16), dict(wt=R.F16), dict(out_dtype=R.F16),
    dict(dtype=R.F32), dict(rows=-1), dict(dim=0), dict(dim=16385), dict(residual=0), dict(residual=A + 1),
    dict(stream=R.F32, residual=A + 2), dict(y=A + 1), dict(out=A + 1), dict(ro=A + 1), dict(weight=A + 1),
    dict(weight=0), dict(out=0, ro=0, weight=0), dict(y=0, post=A), dict(y=0, gate=A), dict(gate=A, g_col=2),
    dict(gate=A + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("inf")), dict(scale=float("nan"))])
def test_block_norm_is_checked(bad):
    assert tre.load().tre_block_norm(block(**bad), None) == 1


def test_block_norm_of_no_rows():
    lib = tre.load()
    assert lib.tre_block_norm(block(rows=0, residual=0), None) == 0
    assert lib.tre_block_norm(None, None) == 1


@pytest.mark.parametrize("bad", [
    dict(dtype=R.I8), dict(dtype=1), dict(rows=-1), dict(experts=0), dict(experts=1025), dict(top=0), dict(top=33),
    dict(experts=4, top=5), dict(logits=0), dict(logits=A + 2), dict(scores=2), dict(bias=A + 2), dict(groups=0),
    dict(groups=3), dict(groups=64), dict(groups=4, top_groups=5), dict(groups=4, top_groups=0), dict(best=0),
    dict(best=3), dict(scale=float("nan")), dict(ids=0), dict(weights=0), dict(ids=A + 2), dict(weights=A + 1)])
def test_route_is_checked(bad):
    assert tre.load().tre_route(router(**bad), None) == 1


def test_route_of_no_rows():
    lib = tre.load()
    assert lib.tre_route(router(rows=0, logits=0, ids=0, weights=0), None) == 0
    assert lib.tre_route(None, None) == 1


BAD_MATRICES = [dict(dtype=R.F32), dict(dtype=R.I8), dict(experts=0), dict(experts=1025), dict(n=0), dict(k=0),
                dict(k=96), dict(group=16), dict(group=256), dict(group=48), dict(n=63, gated=1), dict(n=1 << 21),
                dict(k=1 << 21)]


@pytest.mark.parametrize("bad", BAD_MATRICES)
def test_matrices_are_checked(bad):
    lib, n = tre.load(), C.c_size_t(1 << 40)
    assert lib.tre_w4_pack(source(**bad), None, n, None) == 1
    assert lib.tre_linear4(w4(**bad), linear(), A, n, None, None) == 1
    assert lib.tre_experts(w4(**dict(dict(gated=1), **bad)), w4(k=32, group=32), tokens(), None, n, None, None) == 1


def test_pack():
    lib, n = tre.load(), C.c_size_t(0)
    assert lib.tre_w4_pack(source(), None, n, None) == 0 and n.value >= 64 * 128 // 2 + 2 * 64 * 2
    need = n.value
    assert lib.tre_w4_pack(source(zeros=A), None, n, None) == 0 and n.value > need
    n.value = need - 1
    assert lib.tre_w4_pack(source(), A, n, None) == 2
    n.value = need
    for bad in (dict(codes=0), dict(scales=0), dict(scales=A + 1)):
        assert lib.tre_w4_pack(source(**bad), A, n, None) == 1
    assert lib.tre_w4_pack(source(), A + 16, n, None) == 1
    assert lib.tre_w4_pack(source(), None, None, None) == 1 and lib.tre_w4_pack(None, None, n, None) == 1


@pytest.mark.parametrize("bad", [
    dict(dtype=R.F16), dict(dtype=1), dict(rows=-1), dict(x=0), dict(y=0), dict(x=A + 8), dict(y=A + 1),
    dict(x_row=127), dict(x_row=-8), dict(y_row=-1), dict(dtype=R.F32, x=A + 2), dict(dtype=R.F32, y=A + 2),
    dict(rows=2 ** 30 + 1), dict(dtype=R.F32, rows=2 ** 29 + 1), dict(y_dtype=R.F16), dict(y_dtype=1), dict(y_dtype=R.F32, y=A + 2), dict(dtype=R.F32, y_dtype=R.BF16)])
def test_linear_is_checked(bad):
    n = C.c_size_t(1 << 40)
    assert tre.load().tre_linear4(w4(gated=1), linear(y_dtype=R.F32), A, n, None, None) == 1
    assert tre.load().tre_linear4(w4(), linear(**bad), A, n, None, None) == 1


def test_linear_workspace():
    lib, n = tre.load(), C.c_size_t(7)
    assert lib.tre_linear4(w4(), linear(), None, n, None, None) == 0 and n.value == 0
    assert lib.tre_linear4(w4(), linear(dtype=R.F32), None, n, None, None) == 0 and n.value >= 6 * (128 * 2 + 64 * 4)
    n.value -= 1
    assert lib.tre_linear4(w4(), linear(dtype=R.F32), A, n, None, None) == 2
    assert lib.tre_linear4(w4(), linear(rows=0, x=0, y=0), A, n, None, None) == 0
    assert lib.tre_linear4(w4(experts=2), linear(), A, n, None, None) == 1
    assert lib.tre_linear4(w4(packed=0), linear(), A, n, None, None) == 1
    assert lib.tre_linear4(w4(packed=A + 16), linear(), A, n, None, None) == 1
    assert lib.tre_linear4(w4(), linear(), A, None, None, None) == 1


def pair(experts=4, gated=1, k2=32, n2=128, gated2=0, dtype2=R.BF16, experts2=4):
    return w4(experts=experts, gated=gated), w4(dtype=dtype2, experts=experts2, n=n2, k=k2, group=32, gated=gated2)


@pytest.mark.parametrize("bad", [
    dict(dtype=R.F16), dict(dtype=R.F32), dict(rows=-1), dict(top=0), dict(top=33), dict(x=0), dict(y=0), dict(ids=0),
    dict(weights=0), dict(x=A + 8), dict(x_row=120 + 4), dict(x_row=-8), dict(y=A + 1), dict(y_row=-1), dict(ids=A + 2),
    dict(weights=A + 2), dict(rows=2 ** 30, top=32)])
def test_experts_are_checked(bad):
    n = C.c_size_t(1 << 60)
    assert tre.load().tre_experts(*pair(), tokens(**bad), A, n, None, None) == 1


@pytest.mark.parametrize("bad", [dict(gated=0), dict(gated2=1), dict(k2=64), dict(dtype2=R.F16), dict(experts2=3)])
def test_experts_matrices_fit(bad):
    n = C.c_size_t(1 << 60)
    assert tre.load().tre_experts(*pair(**bad), tokens(), A, n, None, None) == 1


def test_experts_workspace():
    lib, n = tre.load(), C.c_size_t(0)
    assert lib.tre_experts(*pair(), tokens(), None, n, None, None) == 0 and n.value >= 6 * (32 * 2 + 128 * 4)
    n.value -= 1
    assert lib.tre_experts(*pair(), tokens(), A, n, None, None) == 2
    assert lib.tre_experts(*pair(), tokens(rows=0, x=0, y=0, ids=0, weights=0), A, n, None, None) == 0
    assert lib.tre_experts(*pair(), tokens(), A, None, None, None) == 1


def test_calls_want_cuda_tensors():
    import torch
    x = torch.zeros(3, 64)
    for call in (lambda: tre.tre_block_norm(x, weight=x[0]), lambda: tre.tre_route(x, 2),
                 lambda: tre.Weights4(torch.zeros(4, 32, dtype=torch.uint8), torch.ones(4, 2).bfloat16())):
        with pytest.raises(ValueError):
            call()
