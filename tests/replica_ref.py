"""Plain 64-bit statements of a replica's operators, and inputs for their tests."""
import math
import random

import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
# unit roundoffs (8, 11 and 24 significant bits, to nearest)
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
T = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
     "e4m3": torch.float8_e4m3fn, "i8": torch.int8}


def rotation(n, rot, device="cuda"):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(n, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def norm_rope(x, weight, eps, table, pos, interleaved):
    """(y, size): the result, and per element the sum of the absolute values of the
    terms it is made of (what its rounding errors are relative to)."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()
    size = x.abs()
    if table is None:
        return x, size
    half = table.shape[1] // 2
    inside = (pos >= 0) & (pos < table.shape[0])
    row = table[pos.clamp(0, table.shape[0] - 1)].double()[:, None]
    c, s = row[..., :half], row[..., half:]
    ia = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    ib = ia + (1 if interleaved else half)
    a, b = x[..., ia], x[..., ib]
    y, size = x.clone(), size.clone()
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = (a * c).abs() + (b * s).abs()
    size[..., ib] = (b * c).abs() + (a * s).abs()
    y[~inside] = 0
    return y, size


def codes(x, dtype):
    """Codes and scales of 32-bit rows, in the 32-bit arithmetic of the contract."""
    sc = x.float().abs().amax(-1)
    sc = sc / torch.full_like(sc, TOP[dtype])      # by a plain number it is a product
    y = x.float() / torch.where(sc == 0, torch.ones_like(sc), sc)[..., None]
    if dtype == torch.int8:
        return y.round().clamp(-127, 127).to(torch.int8), sc
    return y.clamp(-448, 448).to(dtype), sc


class Batch:
    """Sequences of given (cached, new) lengths in pages of a shuffled pool; `drop`
    takes that share of the pages out of the tables."""

    def __init__(self, lens, page, heads, dim, dtype, seed=0, spare=3, drop=0.0, order="nhd",
                 pad=(0, 0), device="cuda", fill=None, room=0):
        rng = random.Random(seed)
        g = torch.Generator(device=device).manual_seed(seed)
        self.lens, self.page, self.dim, self.heads = lens, page, dim, heads
        total = [b + n for b, n in lens]
        need = [-(-t // page) for t in total]
        n_pages = sum(need) + spare
        ids = list(range(n_pages))
        rng.shuffle(ids)
        width = max(need + [1]) + room
        table = torch.full((len(lens), width), -1, dtype=torch.int32)
        at = 0
        for i, k in enumerate(need):
            for j in range(k):
                table[i, j] = rng.choice((-1, n_pages, 2 ** 31 - 1)) if rng.random() < drop else ids[at + j]
            at += k
        self.n_pages = n_pages
        self.table = table.to(device)
        self.ctx = torch.tensor(total, dtype=torch.int32, device=device)
        starts = [pad[0]]
        for _, n in lens:
            starts.append(starts[-1] + n)
        self.starts = starts
        self.q_start = torch.tensor(starts, dtype=torch.int32, device=device)
        self.rows = starts[-1] + pad[1]

        def pool(dt, *tail):
            if order == "nhd":
                t = torch.zeros(n_pages, page, heads, *tail, dtype=dt, device=device)
            elif order == "hnd":
                t = torch.zeros(n_pages, heads, page, *tail, dtype=dt, device=device).transpose(1, 2)
            else:                                     # keys and values side by side
                t = torch.zeros(n_pages, 2, page, heads, *tail, dtype=dt, device=device)[:, 0]
            return t

        def rows():
            return torch.randn(n_pages, page, heads, dim, generator=g, device=device)

        self.k, self.v = pool(dtype, dim), pool(dtype, dim)
        self.ks = self.vs = None
        if dtype in TOP:
            self.ks, self.vs = pool(torch.float32), pool(torch.float32)
            for t, s in ((self.k, self.ks), (self.v, self.vs)):
                c, sc = codes(rows(), dtype)
                t.view(torch.uint8).copy_(c.view(torch.uint8))
                s.copy_(sc)
        else:
            self.k.copy_(rows())
            self.v.copy_(rows())
        if fill is not None:
            self._fill_outside(fill)

    def _fill_outside(self, value):
        """`value` in every slot that no sequence's position uses."""
        used = torch.zeros(self.n_pages, self.page, dtype=torch.bool)
        for i, (b, n) in enumerate(self.lens):
            for p in range(b + n):
                pg = int(self.table[i, p // self.page])
                if 0 <= pg < self.n_pages:
                    used[pg, p % self.page] = True
        out = ~used.to(self.k.device)
        for t in ((self.k, self.v) if self.ks is None else (self.ks, self.vs)):
            t[out] = value

    def cache(self, tre):
        return tre.KvCache(self.k, self.v, self.ks, self.vs)

    def batch(self, tre, hints=True):
        h = dict(max_new=max([n for _, n in self.lens] + [0]),
                 max_ctx=max([b + n for b, n in self.lens] + [0])) if hints else {}
        return tre.KvBatch(self.table, self.ctx, self.q_start, self.rows, **h)

    def held(self, i, j):
        """(page, slot, mapped) of positions j of sequence i."""
        pg = torch.div(j, self.page, rounding_mode="floor")
        ok = (j >= 0) & (pg < self.table.shape[1])
        ids = self.table[i, pg.clamp(0, self.table.shape[1] - 1)].long()
        ok &= (ids >= 0) & (ids < self.n_pages)
        return ids.clamp(0, self.n_pages - 1), j % self.page, ok

    def values(self, t, scale, page, slot):
        x = t.view(torch.uint8)[page, slot].view(t.dtype) if t.dtype in TOP else t[page, slot]
        x = x.double()
        return x if scale is None else x * scale[page, slot].double()[..., None]


def attention(bt, q, scale, window):
    """64-bit (out, lse, bound): bound is what the kernels' roundings can move each
    output by. Probabilities are rounded to the type of the value product (u_p),
    scores are sums of dim 32-bit products (eps_s), the output is rounded once."""
    rows, H, D = q.shape
    G = H // bt.heads
    out = torch.zeros(rows, H, D, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    lse = torch.full((rows, H), -math.inf, dtype=torch.float64, device=q.device)
    u_p = 2.0 ** -8 if bt.ks is not None else U[q.dtype]
    for i, (b, n) in enumerate(bt.lens):
        if n == 0:
            continue
        ctx = int(bt.ctx[i])
        pos = torch.arange(ctx - n, ctx, device=q.device)
        j = torch.arange(max(ctx, 1), device=q.device)
        page, slot, ok = bt.held(i, j)
        k, v = bt.values(bt.k, bt.ks, page, slot), bt.values(bt.v, bt.vs, page, slot)
        see = (j[None] <= pos[:, None]) & ok[None]
        if window:
            see &= j[None] > pos[:, None] - window
        x = q[bt.starts[i]:bt.starts[i] + n].double()
        for h in range(H):
            kk = torch.where(ok[:, None], k[:, h // G], torch.zeros_like(k[:, 0]))
            s = x[:, h] @ kk.T * scale
            eps = 2.0 ** -24 * (D + 8) * (x[:, h].abs() @ kk.abs().T * scale)
            s = torch.where(see, s, torch.full_like(s, -math.inf))
            m = s.amax(1, keepdim=True)
            some = m > -math.inf
            m = torch.where(some, m, torch.zeros_like(m))
            p = torch.where(see, torch.exp(s - m), torch.zeros_like(s))
            l = p.sum(1, keepdim=True)
            w = p / torch.where(l > 0, l, torch.ones_like(l))
            # masked values do not count, whatever they hold
            vv = torch.where(torch.isfinite(v[:, h // G]), v[:, h // G], torch.zeros_like(v[:, 0]))
            rows_i = slice(bt.starts[i], bt.starts[i] + n)
            out[rows_i, h] = w @ vv
            eps = torch.where(see & torch.isfinite(eps), eps, torch.zeros_like(eps)).amax(1, keepdim=True)
            size = w @ vv.abs()
            bound[rows_i, h] = (u_p + 2 * eps + 2e-6) * size + U[q.dtype] * (w @ vv).abs() + 1e-7
            lse[rows_i, h] = torch.where(some, m + torch.log(l), torch.full_like(m, -math.inf))[:, 0]
    return out, lse, bound
