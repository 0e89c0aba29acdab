"""The rest of a replica's layer around its attention, as measurable cases.

  norm     a block's output normed, gated, scaled and added to the residual stream, and the
           stream normed for the next block, one pass
  route    experts of each token: scores, a bias for the choice, groups, top k, weights
  linear   rows times a matrix held in 4 bits with a scale (and a zero) for each group of
           a row's elements, alone or as the gated half of a feed-forward layer
  experts  a gated feed-forward layer of many experts held in 4 bits, each token through its own
  routed   route, then experts
  block    norm, gated linear, linear, norm: the dense half of a layer

Sizes come from the case alone, values from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # three running requests between two blocks: the smallest call, all latency
        {"name": "norm_3x4096_bf16", "op": "norm", "T": 3, "C": 4096, "dtype": "bf16",
         "stream": "bf16", "post": False, "gate": "", "scale": 1.0},
        # prompts of a large batch, residual stream in 32 bits, block normed on both sides
        # and gated by channel
        {"name": "norm_20011x5120_bf16_f32", "op": "norm", "T": 20011, "C": 5120, "dtype": "bf16",
         "stream": "f32", "post": True, "gate": "channel", "scale": 0.5},
        # five running requests, few experts
        {"name": "route_5x64_softmax", "op": "route", "T": 5, "E": 64, "k": 6, "logits": "f32",
         "scores": "softmax", "bias": False, "groups": 1, "top_groups": 1, "renorm": True,
         "scale": 1.0, "holes": False},
        # prompts of a large batch, many experts in groups, choice balanced by a bias;
        # some rows are padding, some experts are off
        {"name": "route_16384x256_sigmoid", "op": "route", "T": 16384, "E": 256, "k": 8,
         "logits": "f32", "scores": "sigmoid", "bias": True, "groups": 8, "top_groups": 4,
         "renorm": True, "scale": 2.5, "holes": True},
        # one token of one request through a projection
        {"name": "linear_1x4096x4096_bf16", "op": "linear", "T": 1, "K": 4096, "N": 4096,
         "dtype": "bf16", "group": 128, "zeros": False, "gated": False},
        # a few requests, small groups with zeros, a width that no tile divides
        {"name": "linear_13x2816x7001_f16", "op": "linear", "T": 13, "K": 2816, "N": 7001,
         "dtype": "f16", "group": 32, "zeros": True, "gated": False},
        # a short prompt's chunk through the gated half of a feed-forward layer
        {"name": "linear_333x4096x10240_bf16", "op": "linear", "T": 333, "K": 4096, "N": 10240,
         "dtype": "bf16", "group": 64, "zeros": False, "gated": True},
        # a long prompt's chunk
        {"name": "linear_4096x4096x8192_bf16", "op": "linear", "T": 4096, "K": 4096, "N": 8192,
         "dtype": "bf16", "group": 128, "zeros": False, "gated": False},
        # two running requests, six experts each
        {"name": "experts_2x2048_bf16", "op": "experts", "T": 2, "C": 2048, "I": 1024, "E": 64,
         "k": 6, "dtype": "bf16", "group": 128, "zeros": False},
        # a batch of running requests that meets nearly every expert with a few tokens
        {"name": "experts_61x2048_f16", "op": "experts", "T": 61, "C": 2048, "I": 768, "E": 128,
         "k": 8, "dtype": "f16", "group": 64, "zeros": True},
        # prompts' chunks: hundreds of tokens for each expert, padding among them
        {"name": "routed_4096x2048_bf16", "op": "routed", "T": 4096, "C": 2048, "I": 1024, "E": 64,
         "k": 6, "dtype": "bf16", "group": 128, "zeros": False, "logits": "f32",
         "scores": "softmax", "bias": False, "groups": 1, "top_groups": 1, "renorm": True,
         "scale": 1.0, "holes": True},
        # the dense half of a layer for a batch of running requests
        {"name": "block_24x4096_bf16", "op": "block", "T": 24, "C": 4096, "I": 8192, "dtype": "bf16",
         "stream": "bf16", "post": True, "gate": "", "scale": 1.0, "group": 128, "zeros": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _router(rng, c):
    c["E"] = rng.choice((8, 16, 60, 64, 128, 160, 256, 512))
    c["k"] = min(rng.choice((1, 2, 4, 6, 8, 8, 10)), c["E"] // 2)
    c["scores"] = rng.choice(("softmax", "sigmoid"))
    c["groups"] = rng.choice([g for g in (1, 1, 4, 8) if c["E"] % g == 0 and c["E"] // g >= 4])
    c["top_groups"] = max(1, c["groups"] // rng.choice((1, 2)))
    while c["top_groups"] * (c["E"] // c["groups"]) < c["k"]:
        c["top_groups"] += 1
    c.update(bias=c["scores"] == "sigmoid" and rng.random() < 0.7, renorm=rng.random() < 0.7,
             scale=rng.choice((1.0, 2.5)), holes=rng.random() < 0.4)
    return c


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, odd ones among them."""
    op = rng.choice(("norm", "route", "linear", "linear", "linear", "experts", "experts", "routed",
                     "block"))
    dtype = rng.choice(("bf16", "f16"))
    c = {"op": op}
    if op == "route":
        c["logits"] = rng.choice(("f32", "bf16", "f16"))
        _router(rng, c)
        c["T"] = _log(rng, 1, min(30_000, 4_000_000 // c["E"]))
        return c
    c["dtype"] = dtype
    if op in ("norm", "block"):
        c.update(stream=rng.choice((dtype, "f32")), post=rng.random() < 0.5,
                 gate=rng.choice(("", "channel", "token", "full")), scale=rng.choice((1.0, 0.5)))
    if op == "norm":
        c["C"] = rng.choice((_log(rng, 64, 16384), 8 * _log(rng, 8, 2048)))
        c["T"] = _log(rng, 1, 80_000_000 // c["C"])
        return c
    c.update(group=rng.choice((32, 64, 128, 128)), zeros=rng.random() < 0.4)
    g = c["group"]
    if op == "linear":
        c["gated"] = rng.random() < 0.3
        c["K"] = g * _log(rng, 2, 8192 // g)
        c["N"] = 2 * _log(rng, 32, 6000) + (0 if c["gated"] else rng.randint(0, 1))
        c["T"] = _log(rng, 1, min(8192, 130_000_000_000 // (c["K"] * c["N"])))
        return c
    c["C"] = 128 * rng.randint(2, 22)
    if op == "block":
        c["I"] = g * _log(rng, 2, 8192 // g)
        c["T"] = _log(rng, 1, 2048)
        return c
    c["I"] = 128 * rng.randint(1, 8)
    _router(rng, c)
    # what plain and exact forms hold of all experts stays small
    c["E"], c["groups"], c["top_groups"] = min(c["E"], 128), 1, 1
    c["k"] = min(c["k"], 8)
    while c["E"] * c["C"] * c["I"] > 200_000_000:
        c["I"] -= 128
    c["T"] = _log(rng, 1, min(4096, 50_000_000_000 // (c["k"] * c["C"] * c["I"])))
    if op == "routed":
        c["logits"] = rng.choice(("f32", "bf16"))
    else:
        for name in ("scores", "groups", "top_groups", "bias", "renorm", "scale", "holes"):
            del c[name]
    return c


def weight_bytes(c, rows, k):
    return rows * k // 2 + rows * (k // c["group"]) * (3 if c["zeros"] else 2)


def route_work(c):
    return {"bytes": c["T"] * (c["E"] * BYTES[c["logits"]] + 8 * c["k"]),
            "flops": 4 * c["T"] * c["E"]}


def experts_work(c):
    # (every expert that some token goes to is read: as many as an even draw meets)
    met = c["E"] * (1 - (1 - c["k"] / c["E"]) ** c["T"])
    one = weight_bytes(c, 2 * c["I"], c["C"]) + weight_bytes(c, c["C"], c["I"])
    return {"bytes": int(met * one) + 2 * c["T"] * c["C"] * BYTES[c["dtype"]] + 8 * c["T"] * c["k"],
            "flops": 6 * c["T"] * c["k"] * c["C"] * c["I"]}


def norm_work(c):
    el, st = BYTES[c["dtype"]], BYTES[c["stream"]]
    gate = {"": 0, "channel": c["C"], "token": c["T"], "full": c["T"] * c["C"]}[c["gate"]]
    return {"bytes": c["T"] * c["C"] * (2 * el + 2 * st) + gate * el, "flops": 10 * c["T"] * c["C"]}


def work(c):
    if c["op"] == "norm":
        return norm_work(c)
    if c["op"] == "route":
        return route_work(c)
    if c["op"] == "experts":
        return experts_work(c)
    if c["op"] == "routed":
        a, b = route_work(c), experts_work(c)
        return {n: a[n] + b[n] for n in a}
    el, T = BYTES[c["dtype"]], c["T"]
    if c["op"] == "linear":
        out = c["N"] // 2 if c["gated"] else c["N"]
        return {"bytes": weight_bytes(c, c["N"], c["K"]) + T * (c["K"] + out) * el,
                "flops": 2 * T * c["N"] * c["K"]}
    C, I = c["C"], c["I"]
    return {"bytes": weight_bytes(c, 2 * I, C) + weight_bytes(c, C, I)
            + T * C * (2 * el + 2 * BYTES[c["stream"]]), "flops": 6 * T * C * I}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def quantised(normal, c, experts, rows, k):
    """Codes [experts][rows][k/2] (two a byte, the lower half first), scales and zeros
    [experts][rows][k/group] of a random matrix of size about 1/sqrt(k)."""
    dt, g = DT[c["dtype"]], c["group"]
    codes = torch.empty(experts, rows, k // 2, dtype=torch.uint8, device=DEV)
    scales = torch.empty(experts, rows, k // g, dtype=dt, device=DEV)
    zeros = torch.empty(experts, rows, k // g, dtype=torch.uint8, device=DEV) if c["zeros"] else None
    per = max(1, 50_000_000 // (rows * k))
    for e in range(0, experts, per):
        w = normal(min(per, experts - e), rows, k // g, g) / math.sqrt(k)
        if zeros is None:
            sc = (w.abs().amax(-1) / 7).to(dt)
            z = torch.full_like(sc, 8.0).float()
        else:
            lo, hi = w.amin(-1).clamp(max=0), w.amax(-1).clamp(min=0)
            sc = ((hi - lo) / 15).to(dt)
            z = torch.round(-lo / sc.float()).clamp(0, 15)
            zeros[e:e + per] = z.to(torch.uint8)
        q = torch.round(w / sc.float()[..., None] + z[..., None]).clamp(0, 15).to(torch.uint8)
        q = q.view(q.shape[0], rows, k // 2, 2)
        codes[e:e + per] = q[..., 0] | q[..., 1] << 4
        scales[e:e + per] = sc
    return codes, scales, zeros


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    s = {"case": c}
    op, T = c["op"], c["T"]
    if op in ("norm", "block"):
        dt, C = DT[c["dtype"]], c["C"]
        s["residual"] = (normal(T, C) * 3).to(DT[c["stream"]])
        s["y"] = normal(T, C).to(dt)
        s["weight"] = (1 + 0.2 * normal(C)).to(dt)
        if c["post"]:
            s["post_weight"] = (0.7 + 0.2 * normal(C)).to(dt)
        if c["gate"]:
            s["gate"] = torch.sigmoid(normal(*{"channel": (C,), "token": (T, 1), "full": (T, C)}[c["gate"]])).to(dt)
    if op in ("route", "routed"):
        # some experts are liked by all tokens
        x = normal(T, c["E"]) * 1.5 + 0.7 * normal(c["E"])
        if c["holes"]:
            x[:, uniform(c["E"]) < 0.03] = -math.inf          # experts that are off
            x[uniform(T) < 0.05] = -math.inf                  # padding
        s["logits"] = x.to(DT[c["logits"]])
        if c["bias"]:
            s["bias"] = 0.05 * normal(c["E"])
    if op in ("experts", "routed"):
        s["x"] = normal(T, c["C"]).to(DT[c["dtype"]])
    if op == "experts":
        liked = normal(T, c["E"]) + 0.5 * normal(c["E"])
        top = torch.sort(liked, dim=-1, descending=True, stable=True)
        s["ids"] = top.indices[:, :c["k"]].int().contiguous()
        s["weights"] = torch.softmax(top.values[:, :c["k"]], -1)
    if op == "linear":
        s["x"] = normal(T, c["K"]).to(DT[c["dtype"]])
        s["w"] = [t[0] if t is not None else None for t in quantised(normal, c, 1, c["N"], c["K"])]
    elif op in ("experts", "routed"):
        s["w1"] = quantised(normal, c, c["E"], 2 * c["I"], c["C"])
        s["w2"] = quantised(normal, c, c["E"], c["C"], c["I"])
    elif op == "block":
        s["w1"] = [t[0] if t is not None else None for t in quantised(normal, c, 1, 2 * c["I"], c["C"])]
        s["w2"] = [t[0] if t is not None else None for t in quantised(normal, c, 1, c["C"], c["I"])]
    if own:
        import paper_2609_29160_gb300 as tre
        for n, gated in (("w", c.get("gated", False)), ("w1", True), ("w2", False)):
            if n in s:
                codes, scales, zeros = s[n]
                s[n + "_own"] = tre.Weights4(codes, scales, zeros, gated=gated)
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def run_own(s):
    import paper_2609_29160_gb300 as tre
    c = s["case"]
    op = c["op"]
    if op in ("norm", "block"):
        how = dict(post_weight=s.get("post_weight"), gate=s.get("gate"), scale=c["scale"],
                   weight=s["weight"], eps=EPS)
        if op == "norm":
            r, n = tre.tre_block_norm(s["residual"], s["y"], **how)
            return {"residual": r, "out": n}
        # (a residual stream in 32 bits has its block's rows in 32 bits too; what goes into it
        # is rounded there alone)
        r, n = tre.tre_block_norm(s["residual"], s["y"], dtype=c["stream"], **how)
        h = tre.tre_linear4(n, s["w1_own"])
        y = tre.tre_linear4(h, s["w2_own"], dtype="f32")
        r, n = tre.tre_block_norm(r, y, dtype=c["dtype"], **how)
        return {"residual": r, "out": n}
    if op == "linear":
        return {"out": tre.tre_linear4(s["x"], s["w_own"])}
    if op in ("route", "routed"):
        ids, weights = tre.tre_route(s["logits"], c["k"], scores=c["scores"], bias=s.get("bias"),
                                     groups=c["groups"], top_groups=c["top_groups"],
                                     renorm=c["renorm"], scale=c["scale"])
        if op == "route":
            return {"ids": ids, "weights": weights}
        out = tre.tre_experts(s["x"], ids, weights, s["w1_own"], s["w2_own"])
        return {"ids": ids, "weights": weights, "out": out}
    return {"out": tre.tre_experts(s["x"], s["ids"], s["weights"], s["w1_own"], s["w2_own"])}


# ---------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits
# ---------------------------------------------------------------------------
def plain_matrix(w, group):
    """The matrix in 32 bits of codes, scales and zeros (of one expert)."""
    codes, scales, zeros = w
    q = torch.stack([codes & 15, codes >> 4], -1).float().view(codes.shape[0], -1, group)
    z = 8.0 if zeros is None else zeros.float()[..., None]
    return ((q - z) * scales.float()[..., None]).view(codes.shape[0], -1)


def plain_gated(a):
    gate, up = a.chunk(2, -1)
    return gate / (1 + torch.exp(-gate)) * up


def plain_norm(x, weight):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()


def plain_block_norm(s, residual, y):
    y = y.float()
    if "post_weight" in s:
        y = plain_norm(y, s["post_weight"])
    if "gate" in s:
        y = y * s["gate"].float()
    r = residual.float() + s["case"]["scale"] * y
    return r, plain_norm(r, s["weight"])


def plain_route(s):
    """(ids, weights) in 64 bits: scores of two experts may be next to each other."""
    c = s["case"]
    x = s["logits"].double()
    there = x > -math.inf
    if c["scores"] == "softmax":
        top = x.amax(-1, keepdim=True)
        e = torch.exp(x - torch.where(there.any(-1, keepdim=True), top, torch.zeros_like(top)))
        total = e.sum(-1, keepdim=True)
        score = e / torch.where(total > 0, total, torch.ones_like(total))
    else:
        score = 1 / (1 + torch.exp(-x))
    by = score + s["bias"].double() if "bias" in s else score
    by = torch.where(there, by, torch.full_like(by, -math.inf))
    if c["groups"] > 1:
        # a group counts as its best expert, with sigmoid scores as its two best
        g = by.view(c["T"], c["groups"], -1)
        best = torch.sort(g, dim=-1, descending=True).values[..., :2 if c["scores"] == "sigmoid" else 1]
        some = best[..., 0] > -math.inf
        best = torch.where(best > -math.inf, best, torch.zeros_like(best)).sum(-1)
        best = torch.where(some, best, torch.full_like(best, -math.inf))
        keep = torch.sort(best, dim=-1, descending=True, stable=True).indices[:, :c["top_groups"]]
        kept = torch.zeros_like(best, dtype=torch.bool).scatter_(1, keep, True)
        by = torch.where(kept[..., None].expand_as(g).reshape_as(by), by, torch.full_like(by, -math.inf))
    top = torch.sort(by, dim=-1, descending=True, stable=True)
    ids, some = top.indices[:, :c["k"]], top.values[:, :c["k"]] > -math.inf
    w = torch.where(some, score.gather(1, ids), torch.zeros_like(score[:, :1]))
    if c["renorm"]:
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
    return torch.where(some, ids, torch.full_like(ids, -1)).int(), (w * c["scale"]).float()


def plain_experts(s, ids, weights):
    c = s["case"]
    x = s["x"].float()
    out = torch.zeros_like(x)
    for e in range(c["E"]):
        token, slot = torch.nonzero(ids == e, as_tuple=True)
        if len(token) == 0:
            continue
        w1, w2 = ([t[e] if t is not None else None for t in s[n]] for n in ("w1", "w2"))
        h = plain_gated(x[token] @ plain_matrix(w1, c["group"]).T)
        out.index_add_(0, token, (h @ plain_matrix(w2, c["group"]).T) * weights[token, slot][:, None])
    return out.to(DT[c["dtype"]])


def run_plain(s):
    c = s["case"]
    op = c["op"]
    if op in ("norm", "block"):
        r, n = plain_block_norm(s, s["residual"], s["y"])
        if op == "block":
            h = plain_gated(n @ plain_matrix(s["w1"], c["group"]).T)
            r, n = plain_block_norm(s, r, h @ plain_matrix(s["w2"], c["group"]).T)
        return {"residual": r.to(DT[c["stream"]]), "out": n.to(DT[c["dtype"]])}
    if op == "linear":
        y = s["x"].float() @ plain_matrix(s["w"], c["group"]).T
        return {"out": (plain_gated(y) if c["gated"] else y).to(DT[c["dtype"]])}
    if op in ("route", "routed"):
        ids, weights = plain_route(s)
        got = {"ids": ids, "weights": weights}
        if op == "routed":
            got["out"] = plain_experts(s, ids, weights)
        return got
    return {"out": plain_experts(s, s["ids"], s["weights"])}


def run(s):
    return run_own(s) if own else run_plain(s)


# ---------------------------------------------------------------------------
# the same from the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact_matrix(codes, scales, zeros):
    """Of one expert."""
    w = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=DEV)
    w[:, 0::2] = (codes % 16).double()
    w[:, 1::2] = torch.div(codes, 16, rounding_mode="floor").double()
    per = w.shape[1] // scales.shape[1]
    w -= 8 if zeros is None else zeros.double().repeat_interleave(per, 1)
    return w * scales.double().repeat_interleave(per, 1)


def exact_feed_forward(x, w1, w2):
    a = torch.einsum("tc,nc->tn", x, exact_matrix(*w1))
    half = a.shape[1] // 2
    return torch.einsum("ti,ni->tn", a[:, :half] * torch.sigmoid(a[:, :half]) * a[:, half:], exact_matrix(*w2))


def exact_block_norm(s, r, y):
    def normed(v, weight):
        return v / torch.sqrt((v * v).sum(-1, keepdim=True) / v.shape[-1] + EPS) * weight.double()

    y = y.double()
    if s.get("post_weight") is not None:
        y = normed(y, s["post_weight"])
    if s.get("gate") is not None:
        y = y * s["gate"].double()
    r = r.double() + y * s["case"]["scale"]
    return r, normed(r, s["weight"])


def exact_route(s):
    """By repeated maxima, the first place that has one."""
    c = s["case"]
    x = s["logits"].double()
    T, E = x.shape
    score = torch.softmax(x, -1).nan_to_num(0.0) if c["scores"] == "softmax" else torch.sigmoid(x)
    left = torch.where(x == -math.inf, -math.inf, score + (s["bias"].double() if c["bias"] else 0.0))
    rows = torch.arange(T, device=DEV)

    def take(a):
        """Largest of each row and the first place that has it, which is then taken out."""
        top = a.max(-1).values
        at = (a == top[:, None]).int().argmax(-1)
        a[rows, at] = -math.inf
        return top, at

    if c["groups"] > 1:
        per = E // c["groups"]
        total = torch.full((T, c["groups"]), -math.inf, dtype=torch.float64, device=DEV)
        for g in range(c["groups"]):
            a = left[:, g * per:(g + 1) * per].clone()
            first, _ = take(a)
            second, _ = take(a)
            if c["scores"] == "sigmoid":
                first = torch.where(second > -math.inf, first + second, first)
            total[:, g] = first
        keep = torch.zeros(T, c["groups"], dtype=torch.bool, device=DEV)
        for _ in range(c["top_groups"]):
            top, at = take(total)
            keep[rows, at] |= top > -math.inf
        left = left.masked_fill(~keep.repeat_interleave(per, 1), -math.inf)
    ids, w = [], []
    for _ in range(c["k"]):
        top, at = take(left)
        ids.append(torch.where(top > -math.inf, at, -1))
        w.append(torch.where(top > -math.inf, score[rows, at], 0.0))
    ids, w = torch.stack(ids, 1), torch.stack(w, 1)
    if c["renorm"]:
        w = (w / w.sum(-1, keepdim=True)).nan_to_num(0.0)
    return ids.int(), w * c["scale"]


def exact_experts(s, ids, weights):
    c = s["case"]
    x = s["x"].double()
    out = torch.zeros_like(x)
    for e in range(c["E"]):
        mine = ids == e
        rows = mine.any(-1)
        if not bool(rows.any()):
            continue
        w = torch.where(mine, weights.double(), 0.0).sum(-1)[rows, None]
        y = exact_feed_forward(x[rows], *([t[e] if t is not None else None for t in s[n]] for n in ("w1", "w2")))
        out[rows] += w * y
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        r, n = exact_block_norm(s, s["residual"], s["y"])
        return {"residual": r, "out": n}
    if op == "block":
        r, n = exact_block_norm(s, s["residual"], s["y"])
        r, n = exact_block_norm(s, r, exact_feed_forward(n, s["w1"], s["w2"]))
        return {"residual": r, "out": n}
    if op == "linear":
        a = s["x"].double() @ exact_matrix(*s["w"]).T
        if case["gated"]:
            half = a.shape[1] // 2
            a = a[:, :half] * torch.sigmoid(a[:, :half]) * a[:, half:]
        return {"out": a}
    if op in ("route", "routed"):
        ids, weights = exact_route(s)
        got = {"ids": ids, "weights": weights}
        if op == "routed":
            got["out"] = exact_experts(s, ids, weights)
        return got
    return {"out": exact_experts(s, s["ids"], s["weights"])}
