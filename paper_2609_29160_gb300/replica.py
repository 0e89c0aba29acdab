"""A replica's step: norms and rotation of heads, a paged cache, attention over it.

Same names and manner as the rest of the binding (argument checks and marshalling
only; include/tre.h states the contracts). KvCache and KvBatch hold the marshalled
form of tensors that a serving loop keeps; the tensors' contents may change between
calls, their places may not.
"""
from __future__ import annotations

import ctypes as C
import math
import struct

import paper_2609_29160_gb300 as tre

F32, BF16, F16, E4M3, I8 = 0, 2, 3, 4, 5

# The structs of include/tre.h by their fields, packed in one go: a step makes a few
# calls per layer, and setting twenty fields one by one takes longer than its
# smallest kernels.
CACHE = struct.Struct("@5i2P3q2P3q0q")     # tre_kv_cache
BATCH = struct.Struct("@5iPq2P0q")         # tre_kv_batch
HEADS = struct.Struct("@5i2P4q2P4qi2PfPq3i0q")   # tre_heads
ATTEND = struct.Struct("@3ifP2qP2qP0q")    # tre_attend


def declare(lib):
    """Argument types of the entry points (called when the library is loaded)."""
    P, L = C.c_void_p, C.c_int64
    lib.tre_qk_norm_rope.argtypes = [P, P, P, P]
    lib.tre_kv_append.argtypes = [P, P, P, P, L, L, P, P]
    lib.tre_kv_read.argtypes = [P, P, C.c_int, P, P, L, L, P, P]
    lib.tre_chunk_attention.argtypes = [P, P, P, P, C.POINTER(C.c_size_t), P, P]
    for f in ("tre_qk_norm_rope", "tre_kv_append", "tre_kv_read", "tre_chunk_attention"):
        getattr(lib, f).restype = C.c_int


_codes = {}
_torch = None
_HALVES, _FLOATS, _CODES = (BF16, F16), (F32, BF16, F16), (E4M3, I8)


def _types():
    """torch types (and names) of heads and caches, and their codes."""
    global _torch
    if not _codes:
        t = _torch = tre._torch()
        _codes.update({t.float32: F32, t.bfloat16: BF16, t.float16: F16, t.float8_e4m3fn: E4M3,
                       t.int8: I8})
        _codes.update({"f32": F32, "bf16": BF16, "f16": F16, "e4m3": E4M3, "i8": I8})
    return _codes


def _torch_type(code):
    t = tre._torch()
    return {F32: t.float32, BF16: t.bfloat16, F16: t.float16, E4M3: t.float8_e4m3fn, I8: t.int8}[code]


def _code(dtype, allowed, what):
    c = (_codes or _types()).get(dtype)
    if c not in allowed:
        raise ValueError(f"{what}: type {dtype} is not one of those it takes")
    return c


def _like(t):
    """A dense tensor of t's shape (torch's quickest way to one)."""
    return _torch.empty_like(t, memory_format=_torch.contiguous_format)


def _gpu(t, what):
    if not t.is_cuda:
        raise ValueError(f"{what}: must be a CUDA tensor")


def _rows(t, what, dtype, rows=None, heads=None, dim=None):
    """(shape, row stride, head stride) of a [rows][heads][dim] tensor of dtype with a
    dense last axis."""
    shape, st = t.shape, t.stride()
    if len(shape) != 3:
        raise ValueError(f"{what}: expected [rows][heads][dim], got {tuple(shape)}")
    if rows is not None and shape[0] != rows:
        raise ValueError(f"{what}: expected {rows} rows, got {shape[0]}")
    if heads is not None and shape[1] != heads:
        raise ValueError(f"{what}: expected {heads} heads, got {shape[1]}")
    if dim is not None and shape[2] != dim:
        raise ValueError(f"{what}: expected heads of dim {dim}, got {shape[2]}")
    if st[2] != 1:
        raise ValueError(f"{what}: the last axis must be dense")
    if t.dtype is not dtype:
        raise ValueError(f"{what}: expected type {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what}: must be a CUDA tensor")
    return shape, st[0], st[1]


def _index(t, what, n):
    """Address of a dense int32 tensor of n elements."""
    if not (t.is_cuda and t.dtype is _torch.int32 and t.is_contiguous() and t.numel() == n):
        tre._need(t, "int32", n, what)
        _gpu(t, what)
    return t.data_ptr()


def _on(stream, fn, *args):
    """fn(*args) on `stream`: the memory that it makes is that stream's own (a block of the
    current stream's may still be in use there), what it returns is kept for the current
    stream's work as well, and what it is given for that of `stream`, whose owner may let go
    of it right after the call. (Waiting for what the current stream has still to write to
    the inputs is the caller's, as everywhere in torch.)"""
    torch = tre._torch()
    here = torch.cuda.current_stream(stream.device)
    for x in args:
        for t in (x.k, x.v, x.k_scale, x.v_scale) if isinstance(x, KvCache) else (
                x.pages, x.ctx_len, x.q_start) if isinstance(x, KvBatch) else (x,):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(stream)
    with torch.cuda.stream(stream):
        made = fn(*args)
    for t in made if isinstance(made, tuple) else (made,):
        if t is not None and t.is_cuda:
            t.record_stream(here)
    return made


def host_diag():
    """A zeroed tre_diag in pinned host memory: kernels write to it there, and the host reads
    it (tre.read_diag) once the calls are done, without a copy."""
    return tre._torch().zeros(tre.DIAG_BYTES, dtype=tre._torch().uint8).pin_memory()


_own = None         # the tre_diag of calls that are given none, and its struct


def replica_diag():
    """The tre_diag (pinned host memory, accumulated) of the calls here that were given none.
    An error in it (a wait on the device that gave up, whose outputs are undefined) is raised
    by the next such call, or by check_replica."""
    global _own
    if _own is None:
        t = host_diag()
        _own = (t, tre.Diag.from_address(t.data_ptr()))
    return _own[0]


def _raise_error(fn):
    d = _own[1]
    code, d.err = d.err, 0
    raise tre.TreError(fn, code)


def check_replica():
    """Waits for the device and raises what a call that was given no diag left behind."""
    tre._torch().cuda.synchronize()
    if _own is not None and _own[1].err:
        _raise_error("an earlier call of a replica's step")


def _diag(diag):
    """Address of the caller's tre_diag, or of the calls' own."""
    if diag is not None:
        return diag.data_ptr()
    if _own is None:
        if tre._torch().cuda.is_current_stream_capturing():     # (no memory is made there)
            return None
        replica_diag()
    if _own[1].err:
        _raise_error("an earlier call of a replica's step")
    return _own[0].data_ptr()


class KvCache:
    """A paged cache over the caller's tensors: k, v [pages][page][heads][dim] (any
    strides with a dense last axis, the same for both) of bfloat16 or float16, or of
    float8_e4m3fn or int8 with k_scale, v_scale [pages][page][heads] float32."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        code = _code(k.dtype, (BF16, F16, E4M3, I8), "k")
        shape, st = k.shape, k.stride()
        if len(shape) != 4 or shape != v.shape:
            raise ValueError("k, v: expected two [pages][page][heads][dim] tensors")
        if v.dtype is not k.dtype:
            raise ValueError("k, v: expected one type")
        if st != v.stride() or st[3] != 1:
            raise ValueError("k, v: expected the same strides and a dense last axis")
        _gpu(k, "k")
        _gpu(v, "v")
        pages, page, heads, dim = shape
        ks = vs = 0
        ss = (0, 0, 0)
        if code in _CODES:
            if k_scale is None or v_scale is None:
                raise ValueError("k_scale, v_scale: a cache of 8-bit codes needs both")
            for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
                if t.shape != shape[:3] or t.dtype is not _torch.float32:
                    raise ValueError(f"{what}: expected float32 [pages][page][heads]")
                _gpu(t, what)
            ss = k_scale.stride()
            if v_scale.stride() != ss:
                raise ValueError("k_scale, v_scale: expected the same strides")
            ks, vs = k_scale.data_ptr(), v_scale.data_ptr()
        elif k_scale is not None or v_scale is not None:
            raise ValueError("k_scale, v_scale: only a cache of 8-bit codes has them")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.code, self.dtype, self.heads, self.dim = code, k.dtype, heads, dim
        self.packed = CACHE.pack(code, pages, page, heads, dim, k.data_ptr(), v.data_ptr(), st[0],
                                 st[1], st[2], ks, vs, *ss)

    @classmethod
    def empty(cls, pages, page, heads, dim, dtype="bf16", device="cuda"):
        """A cache of its own tensors (zeros)."""
        torch = tre._torch()
        code = _code(dtype, (BF16, F16, E4M3, I8), "dtype")
        k, v = (torch.zeros(pages, page, heads, dim, dtype=_torch_type(code), device=device)
                for _ in range(2))
        if code in _HALVES:
            return cls(k, v)
        return cls(k, v, *(torch.zeros(pages, page, heads, device=device) for _ in range(2)))


class KvBatch:
    """New tokens of a batch of sequences: pages [n_seq][max_pages], ctx_len [n_seq]
    (lengths with the new tokens), q_start [n_seq + 1], all int32 CUDA tensors, and
    the number of rows. max_new, max_ctx: the longest sequence's new tokens and
    length as far as the host knows them, 0 where it does not (work is split by
    them)."""

    def __init__(self, pages, ctx_len, q_start, n_rows, max_new=0, max_ctx=0):
        if not _codes:
            _types()
        shape, st = pages.shape, pages.stride()
        if len(shape) != 2 or st[1] != 1 or pages.dtype is not _torch.int32:
            raise ValueError("pages: expected int32 [n_seq][max_pages] with dense rows")
        _gpu(pages, "pages")
        n_seq, max_pages = shape
        if n_rows < 0:
            raise ValueError("n_rows: must not be negative")
        self.pages, self.ctx_len, self.q_start, self.n_rows = pages, ctx_len, q_start, n_rows
        self.packed = BATCH.pack(n_seq, n_rows, max_new, max_ctx, max_pages, pages.data_ptr(),
                                 st[0], _index(ctx_len, "ctx_len", n_seq),
                                 _index(q_start, "q_start", n_seq + 1))


def _weight(t, what, dim, dtype):
    if t.shape != (dim,) or (dim > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: expected {dim} dense elements")
    if t.dtype is not dtype and t.dtype is not _torch.float32:
        raise ValueError(f"{what}: expected float32 or {dtype}, got {t.dtype}")
    _gpu(t, what)
    return t.data_ptr()


def _heads(q, k, q_weight, k_weight, eps, cos_sin, interleaved, q_out, k_out, keys_out):
    """(tre_heads, q_out, k_out) of the two inputs."""
    one = q if q is not None else k
    if one is None:
        raise ValueError("q, k: expected at least one of them")
    dtype = one.dtype
    code = _code(dtype, _FLOATS, "q, k")
    rows = dim = None
    qp = qr = qh = hq = op = oor = oh = 0
    if q is not None:
        shape, qr, qh = _rows(q, "q", dtype)
        rows, hq, dim = shape
        if q_out is None:
            q_out = _like(q)
            oor, oh = hq * dim, dim
        else:
            _, oor, oh = _rows(q_out, "q_out", dtype, *shape)
        qp, op = q.data_ptr(), q_out.data_ptr()
    kp = kr = kh = hk = up = ur = uh = 0
    if k is not None:
        shape, kr, kh = _rows(k, "k", dtype, rows, None, dim)
        rows, hk, dim = shape
        kp = k.data_ptr()
        if keys_out:
            if k_out is None:
                k_out = _like(k)
                ur, uh = hk * dim, dim
            else:
                _, ur, uh = _rows(k_out, "k_out", dtype, *shape)
            up = k_out.data_ptr()
    wt = F32
    qw = kw = 0
    if q_weight is not None:
        qw = _weight(q_weight, "q_weight", dim, dtype)
        wt = _codes[q_weight.dtype]
    if k_weight is not None:
        kw = _weight(k_weight, "k_weight", dim, dtype)
        if q_weight is not None and _codes[k_weight.dtype] != wt:
            raise ValueError("q_weight, k_weight: expected one type")
        wt = _codes[k_weight.dtype]
    cs = cr = n_pos = rot = 0
    if cos_sin is not None:
        shape, st = cos_sin.shape, cos_sin.stride()
        if len(shape) != 2 or st[1] != 1 or cos_sin.dtype is not _torch.float32:
            raise ValueError("cos_sin: expected float32 [positions][rot] with dense rows")
        _gpu(cos_sin, "cos_sin")
        n_pos, rot = shape
        cs, cr = cos_sin.data_ptr(), st[0]
    return (HEADS.pack(code, rows, hq, hk, dim, qp, kp, qr, qh, kr, kh, op, up, oor, oh, ur, uh,
                       wt, qw, kw, eps, cs, cr, n_pos, rot, 1 if interleaved else 0),
            q_out, k_out)


def tre_qk_norm_rope(q, k, positions=None, q_weight=None, k_weight=None, eps=1e-6, cos_sin=None,
                     interleaved=False, q_out=None, k_out=None, diag=None, stream=None):
    """Per-head norms and position rotation of q [rows][q heads][dim] and
    k [rows][k heads][dim] (either may be None) in one pass. Weights None: not
    normed; cos_sin None: not turned. Returns (q_out, k_out)."""
    if stream is not None:
        return _on(stream, tre_qk_norm_rope, q, k, positions, q_weight, k_weight, eps, cos_sin,
                   interleaved, q_out, k_out, diag)
    lib = tre._lib or tre.load()
    packed, q_out, k_out = _heads(q, k, q_weight, k_weight, eps, cos_sin, interleaved, q_out,
                                  k_out, True)
    at = None
    if positions is not None:
        at = _index(positions, "positions", (q if q is not None else k).shape[0])
    code = lib.tre_qk_norm_rope(packed, at, _diag(diag), tre._stream(None))
    if code:
        tre._check("tre_qk_norm_rope", code)
    return q_out, k_out


def tre_kv_append(cache, batch, k, v, q=None, q_weight=None, k_weight=None, eps=1e-6,
                  cos_sin=None, interleaved=False, q_out=None, diag=None, stream=None):
    """Writes the batch's new keys and values [rows][heads][dim] into the cache, keys
    normed and turned on the way; with q also returns the queries normed and
    turned (else None)."""
    if stream is not None:
        return _on(stream, tre_kv_append, cache, batch, k, v, q, q_weight, k_weight, eps, cos_sin,
                   interleaved, q_out, diag)
    lib = tre._lib or tre.load()
    if k is None:
        raise ValueError("k: expected keys")
    packed, q_out, _ = _heads(q, k, q_weight, k_weight, eps, cos_sin, interleaved, q_out, None,
                              False)
    dtype = k.dtype
    want = (batch.n_rows, cache.heads, cache.dim)
    if k.shape != want:
        _rows(k, "k", dtype, *want)
    _, vr, vh = _rows(v, "v", dtype, *want)
    if cache.dtype is not dtype and cache.code not in _CODES:
        raise ValueError(f"k: a cache of {cache.dtype} takes no type {dtype}")
    code = lib.tre_kv_append(cache.packed, batch.packed, packed, v.data_ptr(), vr, vh, _diag(diag),
                             tre._stream(None))
    if code:
        tre._check("tre_kv_append", code)
    return q_out


def tre_kv_read(cache, batch, dtype="bf16", k_out=None, v_out=None, diag=None, stream=None):
    """The batch's rows out of the cache: (k, v) [rows][heads][dim] of dtype."""
    if stream is not None:
        return _on(stream, tre_kv_read, cache, batch, dtype, k_out, v_out, diag)
    lib = tre._lib or tre.load()
    code = _code(dtype, _FLOATS, "dtype")
    shape = (batch.n_rows, cache.heads, cache.dim)
    if (k_out is None) != (v_out is None):
        raise ValueError("k_out, v_out: expected both or neither")
    row, head = shape[1] * shape[2], shape[2]
    if k_out is None:
        tt = _torch_type(code)
        k_out = _torch.empty(shape, dtype=tt, device=cache.k.device)
        v_out = _like(k_out)
    else:
        tt = _torch_type(code)
        _, row, head = _rows(k_out, "k_out", tt, *shape)
        if _rows(v_out, "v_out", tt, *shape)[1:] != (row, head):
            raise ValueError("k_out, v_out: expected the same strides")
    code = lib.tre_kv_read(cache.packed, batch.packed, code, k_out.data_ptr(), v_out.data_ptr(),
                           row, head, _diag(diag), tre._stream(None))
    if code:
        tre._check("tre_kv_read", code)
    return k_out, v_out


def tre_chunk_attention(q, cache, batch, scale=None, window=0, lse=False, out=None, diag=None,
                        stream=None):
    """Attention of the batch's rows q [rows][heads][dim] over the cache, each row up
    to its own position (its last `window` positions only, with a window). Returns
    out [rows][heads][dim]; with lse also float32 [rows][heads]."""
    if stream is not None:
        return _on(stream, tre_chunk_attention, q, cache, batch, scale, window, lse, out, diag)
    lib = tre._lib or tre.load()
    dtype = q.dtype
    code = _code(dtype, _HALVES, "q")
    shape, qr, qh = _rows(q, "q", dtype, batch.n_rows, None, cache.dim)
    if cache.dtype is not dtype and cache.code not in _CODES:
        raise ValueError(f"q: a cache of {cache.dtype} takes no type {dtype}")
    heads = shape[1]
    if heads == 0 or heads % cache.heads:
        raise ValueError(f"q: expected a multiple of {cache.heads} heads, got {heads}")
    if out is None:
        out = _like(q)
        o_row, oh = heads * cache.dim, cache.dim
    else:
        _, o_row, oh = _rows(out, "out", dtype, *shape)
    ls = _torch.empty(shape[:2], dtype=_torch.float32, device=q.device) if lse else None
    at = ATTEND.pack(code, heads, window, 1.0 / math.sqrt(cache.dim) if scale is None else scale,
                     q.data_ptr(), qr, qh, out.data_ptr(), o_row, oh,
                     0 if ls is None else ls.data_ptr())
    size, s = C.c_size_t(0), tre._stream(None)
    dg = _diag(diag)
    code = lib.tre_chunk_attention(cache.packed, batch.packed, at, None, size, dg, s)
    if code:
        tre._check("tre_chunk_attention", code)
    # (a call that needs none still wants an address: it then only hands it back)
    ws = _torch.empty(size.value, dtype=_torch.uint8, device=q.device) if size.value else out
    code = lib.tre_chunk_attention(cache.packed, batch.packed, at, ws.data_ptr() or 256, size, dg, s)
    if code:
        tre._check("tre_chunk_attention", code)
    return (out, ls) if lse else out
