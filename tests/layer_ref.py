"""Plain 64-bit statements of the operators around a replica's attention, and inputs for
their tests. Each gives the result and how far the kernels' roundings can move it."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
T = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LEAST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}


def rounding(y, dtype):
    """Half a step of dtype at y (and of the smallest numbers)."""
    return U[dtype] * y.abs() + LEAST[dtype]


def norm(x, weight, eps):
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()


def block_norm(residual, y, post_weight, gate, scale, weight, eps):
    """(r, its error, normed, its error) before the last rounding. 32-bit steps: a mean's error
    is at most dim / 32 + 40 roundings of a positive sum, a root halves it; products and the
    device's reciprocal root (2 units) add a few."""
    dim = residual.shape[-1]
    few = 2.0 ** -24 * (dim / 32 + 60)
    r = residual.double()
    off = torch.zeros_like(r)
    if y is not None:
        v = y.double()
        if post_weight is not None:
            v = norm(v, post_weight, eps)
        if gate is not None:
            v = v * gate.double()
        v = v * scale
        r = r + v
        off = few * v.abs() + 2.0 ** -24 * r.abs()
    if weight is None:
        return r, off, None, None
    n = norm(r, weight, eps)
    # r's own errors reach n in its element, and all of them through the root
    root = torch.sqrt(r.square().mean(-1, keepdim=True) + eps)
    mean_off = (off * r.abs()).mean(-1, keepdim=True) / root.square()
    return r, off, n, off / root * weight.double().abs() + n.abs() * (mean_off + few)


def route(logits, top, scores="softmax", bias=None, groups=1, top_groups=1, group_best=None, renorm=True,
          scale=1.0):
    """(ids, weights) by the formulas in 64 bits, on the CPU, a row at a time."""
    if group_best is None:
        group_best = 2 if scores == "sigmoid" else 1
    rows, experts = logits.shape
    ids = torch.full((rows, top), -1, dtype=torch.int32)
    weights = torch.zeros(rows, top, dtype=torch.float64)
    b = [0.0] * experts if bias is None else bias.double().cpu().tolist()
    most = torch.finfo(torch.float32).max
    for t, row in enumerate(logits.double().cpu().tolist()):
        there = [e for e, x in enumerate(row) if x == x and x > -math.inf]
        x = {e: min(row[e], most) for e in there}
        if scores == "softmax":
            peak = max(x.values(), default=0.0)
            total = sum(math.exp(v - peak) for v in x.values())
            s = {e: math.exp(v - peak) / total for e, v in x.items()}
        else:
            s = {e: 1 / (1 + math.exp(-v)) if v > -700 else math.exp(v) for e, v in x.items()}
        c = {e: s[e] + b[e] for e in there}
        c = {e: v for e, v in c.items() if v == v and v > -math.inf}
        # (without a bias the logit decides as the score does, further than 64 bits tell)
        key = (lambda e: (-x[e], e)) if bias is None else (lambda e: (-c[e], e))
        per = experts // groups
        rank = []
        for g in range(groups):
            mine = sorted((e for e in c if e // per == g), key=key)[:group_best]
            value = -math.inf
            if mine:
                value = x[mine[0]] if bias is None and group_best == 1 else sum(c[e] for e in mine)
            rank.append((-value, g))
        keep = {g for _, g in sorted(rank)[:top_groups]}
        best = sorted((e for e in c if e // per in keep), key=key)[:top]
        w = [s[e] for e in best]
        if renorm and best:
            total = sum(w)
            w = [v / total if total > 0 else 0.0 for v in w]
        for j, (e, v) in enumerate(zip(best, w)):
            ids[t, j] = e
            weights[t, j] = v * scale
    return ids, weights


def matrix4(experts, n, k, group, dtype, zeros, seed, device="cuda"):
    """(codes, scales, zeros, the matrix in 64 bits), of one matrix without the first axis
    where experts is None."""
    g = torch.Generator(device=device).manual_seed(seed)
    e = experts or 1
    codes = torch.randint(0, 256, (e, n, k // 2), generator=g, device=device, dtype=torch.uint8)
    scales = (torch.rand(e, n, k // group, generator=g, device=device) * 2 - 0.5) / math.sqrt(k)
    scales = scales.to(dtype)
    z = torch.randint(0, 16, scales.shape, generator=g, device=device, dtype=torch.uint8) if zeros else None
    q = torch.stack([codes & 15, codes >> 4], -1).double().view(e, n, k // group, group)
    q = (q - (8 if z is None else z.double()[..., None])) * scales.double()[..., None]
    out = [codes, scales, z, q.reshape(e, n, k)]
    if experts is None:
        out = [t[0] if t is not None else None for t in out]
    return out


def product(x, m):
    """(x m^T, error): every 16 products are one step of a 32-bit sum (two units each, for
    hardware that cuts instead of rounding), and a group's scale adds a few."""
    x = x.double()
    size = x.abs() @ m.abs().T
    return x @ m.T, 2.0 ** -23 * (2 * x.shape[-1] / 16 + 64) * size


def act(y, off):
    """silu(g) * u of the halves, and its error: silu's slope stays below 1.1; the device's
    exponential is within 2^-20 of itself for the sizes here."""
    g, u = y.chunk(2, -1)
    og, ou = off.chunk(2, -1)
    s = g * torch.sigmoid(g)
    return s * u, 1.1 * og * u.abs() + s.abs() * ou + 1.1 * og * ou + 2.0 ** -19 * (s * u).abs()


def experts(x, ids, weights, m1, m2, dtype):
    """(y, error) with m1, m2 [experts][..]; the error counts the rounding of the inner rows
    and of each expert's output (where there are many tokens)."""
    y = torch.zeros(x.shape[0], m2.shape[1], dtype=torch.float64, device=x.device)
    off = torch.zeros_like(y)
    for e in range(m1.shape[0]):
        token, slot = torch.nonzero(ids == e, as_tuple=True)
        if len(token) == 0:
            continue
        h, oh = act(*product(x[token], m1[e]))
        oh = oh + rounding(h, dtype) * 1.01
        z, oz = product(h, m2[e])
        oz = oz + oh @ m2[e].abs().T
        w = weights[token, slot].double()[:, None]
        y.index_add_(0, token, w * z)
        off.index_add_(0, token, w.abs() * oz + 2.0 ** -22 * (w * z).abs())
    return y, off


def near(got, want, off, what=""):
    """Asserts |got - want| <= off + got's own rounding."""
    d = (got.double() - want).abs()
    bound = off + rounding(want.abs() + off, got.dtype)
    bad = ~(d <= bound)
    assert not bool(bad.any()), (
        f"{what}: {int(bad.sum())} of {d.numel()} off, worst {float((d / bound).nan_to_num(1e9).max()):.3g} bounds")
