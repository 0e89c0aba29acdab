"""The rest of a replica's layer: norms around blocks, products with matrices in 4 bits,
routing to experts, the experts' products.

Same names and manner as the rest of the binding (argument checks and marshalling
only; include/tre.h states the contracts). Weights4 holds a matrix, or one for each
expert, laid out for the products.
"""
from __future__ import annotations

import ctypes as C
import struct

import paper_2609_29160_gb300 as tre
from . import replica
from .replica import F32, _codes, _diag

# The structs of include/tre.h by their fields (see replica).
BLOCK = struct.Struct("@7iPqPqPPqqffPPqPq0q")      # tre_block_rows
ROUTER = struct.Struct("@4iPqiP4ifPP0q")           # tre_router
SOURCE = struct.Struct("@6iPPP0q")                 # tre_w4_source
W4 = struct.Struct("@7iP0q")                       # tre_w4
LINEAR = struct.Struct("@3iPqPq0q")                  # tre_linear
TOKENS = struct.Struct("@3iPqPPPq0q")              # tre_tokens

SCORES = {"softmax": 0, "sigmoid": 1}
_torch = None


def declare(lib):
    """Argument types of the entry points (called when the library is loaded)."""
    P = C.c_void_p
    size = C.POINTER(C.c_size_t)
    lib.tre_block_norm.argtypes = [P, P]
    lib.tre_route.argtypes = [P, P]
    lib.tre_w4_pack.argtypes = [P, P, size, P]
    lib.tre_linear4.argtypes = [P, P, P, size, P, P]
    lib.tre_experts.argtypes = [P, P, P, P, size, P, P]
    for f in ("tre_block_norm", "tre_route", "tre_w4_pack", "tre_linear4", "tre_experts"):
        getattr(lib, f).restype = C.c_int


_device = _stream = None      # torch's quickest ways to the current device, and to its stream


def _ready():
    """The library, with what calls look up filled in."""
    global _torch, _device, _stream
    if _torch is None:
        replica._types()
        _torch = tre._torch()
        _device = getattr(_torch._C, "_cuda_getDevice", _torch.cuda.current_device)
        _stream = getattr(_torch._C, "_cuda_getCurrentRawStream",
                          lambda dev: _torch.cuda.current_stream(dev).cuda_stream)
    return tre._lib or tre.load()


def _like(t):
    """A dense tensor of t's shape (torch's quickest way to one)."""
    return _torch.empty_like(t, memory_format=_torch.contiguous_format)


def _here(t, what):
    """Device of a CUDA tensor, which has to be the current one."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{what}: must be a CUDA tensor")
    if dev != _device():
        raise ValueError(f"{what}: must be on the current device")
    return dev


def _rows(t, what, dtype, dev, shape=None):
    """Row stride of a [rows][elements] tensor with a dense last axis."""
    if t.dtype is not dtype:
        raise ValueError(f"{what}: expected type {dtype}, got {t.dtype}")
    size, st = t.shape, t.stride()
    if len(size) != 2 or (shape is not None and size != shape):
        want = "[rows][elements]" if shape is None else list(shape)
        raise ValueError(f"{what}: expected {want}, got {tuple(size)}")
    if st[1] != 1 and size[1] > 1:
        raise ValueError(f"{what}: the last axis must be dense")
    if t.get_device() != dev:
        raise ValueError(f"{what}: must be on the device of the other tensors")
    return st[0]


def _weight(t, what, dim, dev):
    """Type of `dim` dense weights."""
    if t.shape != (dim,) or (t.stride(0) != 1 and dim > 1):
        raise ValueError(f"{what}: expected {dim} dense elements")
    if t.get_device() != dev:
        raise ValueError(f"{what}: must be on the device of the other tensors")
    return t.dtype


def _model_type(kinds):
    """The one type of 16 bits among them (float32 where there is none)."""
    kind = _torch.float32
    for k in kinds:
        if k is not _torch.float32 and k is not kind:
            if kind is not _torch.float32:
                raise ValueError(f"types: expected float32 and one of 16 bits, got {kind} and {k}")
            replica._code(k, replica._FLOATS, "types")
            kind = k
    return kind


def tre_block_norm(residual, y=None, post_weight=None, gate=None, scale=1.0, weight=None, eps=1e-6,
                   residual_out=None, out=None, dtype=None, stream=None):
    """A block's output y [rows][dim] into the residual stream, r = residual + scale * gate *
    norm(y) (post_weight None: y as it is; gate: [dim], [rows][1] or [rows][dim], None: 1; y
    None: residual as it is), and the stream normed for the next block (weight None: not).
    Returns (r, normed): r is `residual` itself where there is no y and no residual_out, normed
    is None without a weight. Types: one of 16 bits or float32 throughout, or both (a gate
    is of the former); dtype: that of the normed rows (None: y's, without one the residual's).
    residual_out may be residual, out may be y."""
    if stream is not None:
        return replica._on(stream, tre_block_norm, residual, y, post_weight, gate, scale, weight, eps,
                           residual_out, out, dtype)
    lib = _ready()
    dev = _here(residual, "residual")
    kind = r_kind = residual.dtype
    r_row = _rows(residual, "residual", r_kind, dev)
    shape = residual.shape
    rows, dim = shape
    if not 1 <= dim <= 16384:
        raise ValueError(f"residual: expected rows of 1 to 16384 elements, got {dim}")
    yp = y_row = gp = g_row = g_col = pp = wp = ro_row = rp = o_row = op = 0
    y_kind = w_kind = o_kind = r_kind          # (of what is not there: any of them)
    g_kind = None
    if y is not None:
        y_kind = y.dtype
        y_row = _rows(y, "y", y_kind, dev, shape)
        yp = y.data_ptr()
        if residual_out is None:
            residual_out = _like(residual)
            ro_row = dim
        if gate is not None:
            g_kind = gate.dtype
            if gate.dim() == 1:
                gate = gate[None]
            if gate.dim() != 2 or gate.shape[0] not in (1, rows) or gate.shape[1] not in (1, dim):
                raise ValueError(
                    f"gate: expected [{dim}], [{rows}][1] or [{rows}][{dim}], got {tuple(gate.shape)}")
            g_row = _rows(gate, "gate", g_kind, dev)
            if gate.shape[0] == 1:
                g_row = 0
            g_col = 1 if gate.shape[1] == dim and dim > 1 else 0
            gp = gate.data_ptr()
        if post_weight is not None:
            w_kind = _weight(post_weight, "post_weight", dim, dev)
            pp = post_weight.data_ptr()
    elif post_weight is not None or gate is not None:
        raise ValueError("post_weight, gate: only with a block's output y")
    elif weight is None and residual_out is None:
        raise ValueError("y, weight: expected at least one of them")
    if weight is not None:
        o_kind = _weight(weight, "weight", dim, dev)
        if post_weight is not None and w_kind is not o_kind:
            raise ValueError("post_weight, weight: expected one type")
        w_kind = o_kind
        wp = weight.data_ptr()
        if out is not None:
            o_kind = out.dtype
            o_row = _rows(out, "out", o_kind, dev, shape)
        else:
            o_kind = y_kind if dtype is None else replica._torch_type(
                replica._code(dtype, replica._FLOATS, "dtype"))
            out = _like(residual) if o_kind is r_kind else _torch.empty(shape, dtype=o_kind, device=residual.device)
            o_row = dim
        op = out.data_ptr()
    elif out is not None:
        raise ValueError("out: expected a weight")
    if residual_out is not None:
        if ro_row == 0:
            ro_row = _rows(residual_out, "residual_out", r_kind, dev, shape)
        rp = residual_out.data_ptr()
    if not (y_kind is kind and w_kind is kind and o_kind is kind and g_kind in (None, kind)):
        kind = _model_type((r_kind, y_kind, w_kind, o_kind) if g_kind is None else
                           (r_kind, y_kind, w_kind, o_kind, g_kind))
        if g_kind not in (None, kind):
            raise ValueError(f"gate: expected {kind}, got {g_kind}")
    codes = _codes
    if codes.get(kind) not in replica._FLOATS:
        raise ValueError(f"residual: type {kind} is not one of those it takes")
    if rows:
        err = lib.tre_block_norm(
            BLOCK.pack(codes[kind], codes[y_kind], codes[r_kind], codes[w_kind], codes[o_kind], rows, dim,
                       residual.data_ptr(), r_row, yp, y_row, pp, gp, g_row, g_col, scale, eps, wp, rp,
                       ro_row, op, o_row),
            _stream(dev))
        if err:
            tre._check("tre_block_norm", err)
    return residual if residual_out is None else residual_out, out


def tre_route(logits, top, scores="softmax", bias=None, groups=1, top_groups=1, group_best=None,
              renorm=True, scale=1.0, ids=None, weights=None, stream=None):
    """The `top` experts of each token by logits [rows][experts]: (ids [rows][top] int32,
    weights [rows][top] float32), -1 and 0 where fewer are there. scores: "softmax" or
    "sigmoid"; bias [experts] float32 counts in the choice alone; of `groups` groups of
    neighbouring experts the top_groups best stay, each by the sum of its group_best largest
    (None: 1 of a softmax, 2 of sigmoids)."""
    if stream is not None:
        return replica._on(stream, tre_route, logits, top, scores, bias, groups, top_groups, group_best,
                           renorm, scale, ids, weights)
    lib = _ready()
    dev = _here(logits, "logits")
    code = replica._code(logits.dtype, replica._FLOATS, "logits")
    row = _rows(logits, "logits", logits.dtype, dev)
    if scores not in SCORES:
        raise ValueError(f"scores: expected softmax or sigmoid, got {scores}")
    rows, experts = logits.shape
    bp = 0
    if bias is not None:
        if _weight(bias, "bias", experts, dev) is not _torch.float32:
            raise ValueError("bias: expected float32")
        bp = bias.data_ptr()
    if group_best is None:
        group_best = 2 if scores == "sigmoid" else 1
    if experts < 1 or experts > 1024 or not 1 <= top <= min(32, experts):
        raise ValueError(f"top: expected 1 to 32 of at most 1024 experts, got {top} of {experts}")
    if not 1 <= groups <= 32 or experts % groups or not 1 <= top_groups <= groups or group_best not in (1, 2):
        raise ValueError("groups: expected at most 32 that divide the experts, top_groups of them, group_best 1 or 2")
    shape = (rows, top)
    if ids is None:
        ids = _torch.empty(shape, dtype=_torch.int32, device=logits.device)
    elif _rows(ids, "ids", _torch.int32, dev, shape) != top and rows > 1 or not ids.is_contiguous():
        raise ValueError("ids: must be contiguous")
    if weights is None:
        weights = _torch.empty(shape, dtype=_torch.float32, device=logits.device)
    elif _rows(weights, "weights", _torch.float32, dev, shape) != top and rows > 1 or not weights.is_contiguous():
        raise ValueError("weights: must be contiguous")
    if rows:
        err = lib.tre_route(
            ROUTER.pack(code, rows, experts, top, logits.data_ptr(), row, SCORES[scores], bp, groups, top_groups,
                        group_best, 1 if renorm else 0, scale, ids.data_ptr(), weights.data_ptr()),
            _stream(dev))
        if err:
            tre._check("tre_route", err)
    return ids, weights


class Weights4:
    """A matrix in 4 bits, or one for each expert, laid out for the products (on the current
    stream): codes [n][k/2] or [experts][n][k/2] uint8, two a byte, the lower half first;
    scales [..][n][k/group] of bfloat16 or float16, the type of the rows that it will be
    multiplied with; zeros [..][n][k/group] uint8, None: 8. An element is (code - zero) *
    scale. gated: the first half of the rows are a gate's, the others what it multiplies.
    What it is made of is not kept."""

    def __init__(self, codes, scales, zeros=None, gated=False):
        lib = _ready()
        code = replica._code(scales.dtype, replica._HALVES, "scales")
        dev = _here(codes, "codes")
        if codes.dtype is not _torch.uint8 or codes.dim() not in (2, 3):
            raise ValueError("codes: expected uint8 [n][k/2] or [experts][n][k/2]")
        if scales.dim() != codes.dim() or scales.shape[:-1] != codes.shape[:-1]:
            raise ValueError(f"scales: expected {list(codes.shape[:-1])} rows, got {tuple(scales.shape)}")
        if zeros is not None and (zeros.dtype is not _torch.uint8 or zeros.shape != scales.shape):
            raise ValueError("zeros: expected uint8 of the scales' shape")
        for t, what in ((codes, "codes"), (scales, "scales"), (zeros, "zeros")):
            if t is None:
                continue
            if not t.is_contiguous():
                raise ValueError(f"{what}: must be contiguous")
            if t.get_device() != dev:
                raise ValueError(f"{what}: must be on the device of the other tensors")
        experts = codes.shape[0] if codes.dim() == 3 else 1
        n, k = codes.shape[-2], codes.shape[-1] * 2
        groups = scales.shape[-1]
        if n < 1 or experts < 1 or groups < 1 or k % groups or k // groups not in (32, 64, 128):
            raise ValueError(f"scales: expected one for every 32, 64 or 128 of {k} elements, got {groups}")
        if gated and n % 2:
            raise ValueError(f"codes: a gated matrix has two halves, got {n} rows")
        self.n, self.k, self.group, self.gated, self.experts = n, k, k // groups, bool(gated), experts
        self.dtype, self.code = scales.dtype, code
        self.out = n // 2 if gated else n                 # elements of a row of the product
        self.plain = codes.dim() == 2
        source = SOURCE.pack(code, experts, n, k, self.group, self.gated, codes.data_ptr(), scales.data_ptr(),
                             0 if zeros is None else zeros.data_ptr())
        size = C.c_size_t(0)
        tre._check("tre_w4_pack", lib.tre_w4_pack(source, None, size, None))
        self.packed = _torch.empty(size.value, dtype=_torch.uint8, device=codes.device)
        tre._check("tre_w4_pack", lib.tre_w4_pack(source, self.packed.data_ptr(), size, _stream(dev)))
        self.handle = W4.pack(code, experts, n, k, self.group, self.gated, zeros is not None,
                              self.packed.data_ptr())
        self.tensors = (self.packed,)


def _operand(x, what, w, dev, dtype):
    """Row stride of rows of dtype that w is multiplied with."""
    row = _rows(x, what, dtype, dev)
    if x.shape[1] != w.k:
        raise ValueError(f"{what}: expected rows of {w.k} elements, got {x.shape[1]}")
    if w.packed.get_device() != dev:
        raise ValueError(f"{what}: must be on the device of the weights")
    return w.k if x.shape[0] < 2 else row                 # (no other row is looked at)


def tre_linear4(x, w, out=None, dtype=None, diag=None, stream=None):
    """x [rows][k] times the transpose of w (Weights4 of one matrix): [rows][n]; of a gated w
    silu(its first half) * its second half, [rows][n/2]. x of w's type, or float32, which out
    is then too; dtype "f32": out is in any case (not of a gated w)."""
    if stream is not None:
        return replica._on(stream, tre_linear4, x, w, out, dtype, diag)
    lib = _ready()
    dev = _here(x, "x")
    f32 = x.dtype is _torch.float32
    kind = _torch.float32 if f32 else w.dtype
    row = _operand(x, "x", w, dev, kind)
    if w.experts != 1:
        raise ValueError(f"w: expected one matrix, got {w.experts}")
    code = y_code = F32 if f32 else w.code
    if dtype is not None:
        y_code = replica._code(dtype, replica._FLOATS, "dtype")
    elif out is not None and out.dtype is _torch.float32:
        y_code = F32
    if y_code != code:
        if y_code != F32 or w.gated:
            raise ValueError(f"dtype: expected {kind}, or float32 of a matrix that is not gated")
        kind = _torch.float32
    rows = x.shape[0]
    shape = (rows, w.out)
    if out is None:
        out = _torch.empty(shape, dtype=kind, device=x.device)
        o_row = w.out
    else:
        o_row = _rows(out, "out", kind, dev, shape)
    at = LINEAR.pack(code, y_code, rows, x.data_ptr(), row, out.data_ptr(), o_row)
    size, s, dg = C.c_size_t(0), _stream(dev), _diag(diag)
    ws = out                       # (a call that needs none still wants an address)
    if f32:
        err = lib.tre_linear4(w.handle, at, None, size, dg, s)
        if err:
            tre._check("tre_linear4", err)
        ws = _torch.empty(size.value, dtype=_torch.uint8, device=x.device)
    err = lib.tre_linear4(w.handle, at, ws.data_ptr() or 256, size, dg, s)
    if err:
        tre._check("tre_linear4", err)
    return out


def tre_experts(x, ids, weights, w1, w2, out=None, diag=None, stream=None):
    """Each token's experts: sum over j of weights[t][j] * w2[e] act(w1[e] x[t]), e = ids[t][j]
    (below zero: none). x [rows][k]; ids [rows][top] int32 and weights [rows][top] float32 as
    tre_route gives them; w1 gated, w2 not. Returns [rows][n of w2]."""
    if stream is not None:
        return replica._on(stream, tre_experts, x, ids, weights, w1, w2, out, diag)
    lib = _ready()
    dev = _here(x, "x")
    row = _operand(x, "x", w1, dev, w1.dtype)
    if not w1.gated or w2.gated:
        raise ValueError("w1, w2: expected a gated and a plain set of matrices")
    if w1.dtype is not w2.dtype or w1.experts != w2.experts or w2.k != w1.out or w2.packed.get_device() != dev:
        raise ValueError(f"w2: expected {w1.experts} matrices of {w1.dtype} with rows of {w1.out} elements")
    rows = x.shape[0]
    if ids.dim() != 2 or not 1 <= ids.shape[1] <= 32:
        raise ValueError(f"ids: expected [{rows}][1 to 32], got {tuple(ids.shape)}")
    shape = (rows, ids.shape[1])
    for t, what, dtype in ((ids, "ids", _torch.int32), (weights, "weights", _torch.float32)):
        _rows(t, what, dtype, dev, shape)
        if not t.is_contiguous():
            raise ValueError(f"{what}: must be contiguous")
    if out is None:
        out = _torch.empty((rows, w2.n), dtype=w1.dtype, device=x.device)
        o_row = w2.n
    else:
        o_row = _rows(out, "out", w1.dtype, dev, (rows, w2.n))
    tokens = TOKENS.pack(w1.code, rows, shape[1], x.data_ptr(), row, ids.data_ptr(), weights.data_ptr(),
                         out.data_ptr(), o_row)
    size, s, dg = C.c_size_t(0), _stream(dev), _diag(diag)
    err = lib.tre_experts(w1.handle, w2.handle, tokens, None, size, dg, s)
    if err:
        tre._check("tre_experts", err)
    ws = _torch.empty(size.value, dtype=_torch.uint8, device=x.device)
    err = lib.tre_experts(w1.handle, w2.handle, tokens, ws.data_ptr() or 256, size, dg, s)
    if err:
        tre._check("tre_experts", err)
    return out
