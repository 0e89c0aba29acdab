"""What a replica of a served model runs for each batch of new tokens, as measurable cases.

  rope    per-head norms of queries and keys with the position rotation, one pass
  write   new keys and values into a paged cache (normed, rotated, quantised on the
          way where the case says so), then those rows read back as the model sees them
  read    whole contexts read back from a quantised cache
  attend  attention of new tokens over the paged cache: single tokens, chunks of a
          prompt, both in one batch
  step    write (queries normed and rotated in the same pass), then attend

Lengths come from the case alone (its `pattern`), values from the seed. A batch has
`n` sequences with `lo`..`hi` cached tokens (spread over the logarithm); the first
`chunks` of them bring up to `chunk` new tokens, the others one each. Pages are
handed out in random order.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
      "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1, "i8": 1}
TOP = {"e4m3": 448.0, "i8": 127.0}     # largest code of a quantised cache


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # four tokens of running requests: the smallest call, all latency
        {"name": "rope_4x32+8x128_bf16", "op": "rope", "T": 4, "Hq": 32, "Hkv": 8, "D": 128,
         "dtype": "bf16", "rot": 128, "interleaved": False, "norm": True},
        # a large batch of prompts in 32 bits, half of each head rotated in adjacent pairs
        {"name": "rope_40013x16+16x64_f32", "op": "rope", "T": 40013, "Hq": 16, "Hkv": 16,
         "D": 64, "dtype": "f32", "rot": 32, "interleaved": True, "norm": True},
        # one new token for each of 64 running requests, 8-bit floating cache
        {"name": "write_64x1_e4m3", "op": "write", "Hq": 32, "Hkv": 8, "D": 128, "dtype": "bf16",
         "pool": "e4m3", "page": 16, "n": 64, "lo": 30, "hi": 4000, "chunks": 0, "chunk": 1,
         "pattern": 1, "rot": 128, "interleaved": False, "norm": True},
        # ragged chunks of a dozen prompts, 8-bit integer cache
        {"name": "write_12x4001_i8", "op": "write", "Hq": 16, "Hkv": 16, "D": 64, "dtype": "f16",
         "pool": "i8", "page": 48, "n": 12, "lo": 1, "hi": 9000, "chunks": 12, "chunk": 4001,
         "pattern": 2, "rot": 64, "interleaved": False, "norm": True},
        # sixteen long contexts read back to move them to another replica
        {"name": "read_16x50000_e4m3", "op": "read", "Hkv": 8, "D": 128, "dtype": "bf16",
         "pool": "e4m3", "page": 64, "n": 16, "lo": 500, "hi": 50000, "pattern": 3},
        # two short requests, one token each: the smallest attention, all latency
        {"name": "attend_2x700_bf16_64", "op": "attend", "Hq": 16, "Hkv": 16, "D": 64,
         "dtype": "bf16", "pool": "bf16", "page": 16, "n": 2, "lo": 200, "hi": 700, "chunks": 0,
         "chunk": 1, "pattern": 4, "window": 0},
        # 96 running requests of all lengths, one token each
        {"name": "attend_96x16000_bf16", "op": "attend", "Hq": 32, "Hkv": 8, "D": 128,
         "dtype": "bf16", "pool": "bf16", "page": 16, "n": 96, "lo": 500, "hi": 16000,
         "chunks": 0, "chunk": 1, "pattern": 5, "window": 0},
        # eight requests over very long documents, 8-bit cache
        {"name": "attend_8x120000_e4m3", "op": "attend", "Hq": 64, "Hkv": 8, "D": 128,
         "dtype": "f16", "pool": "e4m3", "page": 64, "n": 8, "lo": 30000, "hi": 120000,
         "chunks": 0, "chunk": 1, "pattern": 6, "window": 0},
        # a chunk of a long prompt over what is cached of it
        {"name": "attend_1x4096_32000_bf16", "op": "attend", "Hq": 32, "Hkv": 8, "D": 128,
         "dtype": "bf16", "pool": "bf16", "page": 32, "n": 1, "lo": 32000, "hi": 32000,
         "chunks": 1, "chunk": 4096, "pattern": 7, "window": 0},
        # prompts from their first token on, every query head with keys of its own
        {"name": "attend_24x2000_f16_64", "op": "attend", "Hq": 16, "Hkv": 16, "D": 64,
         "dtype": "f16", "pool": "f16", "page": 24, "n": 24, "lo": 0, "hi": 0, "chunks": 24,
         "chunk": 2000, "pattern": 8, "window": 0},
        # chunks of two prompts beside 62 running requests, 8-bit integer cache, local layers
        {"name": "attend_2x1024+62_i8_local", "op": "attend", "Hq": 32, "Hkv": 8, "D": 128,
         "dtype": "bf16", "pool": "i8", "page": 16, "n": 64, "lo": 300, "hi": 8000, "chunks": 2,
         "chunk": 1024, "pattern": 9, "window": 4096},
        # the whole step of a batch: one prompt's chunk and 47 running requests
        {"name": "step_1x512+47_bf16", "op": "step", "Hq": 32, "Hkv": 4, "D": 128,
         "dtype": "bf16", "pool": "bf16", "page": 16, "n": 48, "lo": 100, "hi": 6000,
         "chunks": 1, "chunk": 512, "pattern": 10, "window": 0, "rot": 128,
         "interleaved": False, "norm": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, mostly odd."""
    op = rng.choice(("rope", "write", "write", "read", "attend", "attend", "attend", "attend",
                     "step"))
    D = rng.choice((64, 128))
    Hkv = rng.choice((1, 2, 4, 8, 8, 16))
    G = rng.choice((1, 2, 4, 4, 5, 8))
    dtype = rng.choice(("bf16", "f16"))
    c = {"op": op, "Hkv": Hkv, "D": D, "dtype": dtype}
    if op != "read":
        c["Hq"] = Hkv * G
    if op in ("rope", "write", "step"):
        c.update(rot=rng.choice((D, D, D // 2)), interleaved=rng.random() < 0.3,
                 norm=rng.random() < 0.8)
    if op == "rope":
        c["dtype"] = rng.choice(("bf16", "f16", "f32"))
        top = 80_000_000 // ((Hkv * G + Hkv) * D)
        c["T"] = _log(rng, 1, min(top, 60_000))
        return c
    c.update(page=rng.choice((16, 16, 24, 32, 48, 64, 128)), pattern=rng.randrange(1 << 20),
             pool=rng.choice((dtype, "e4m3", "i8")))
    if op == "read":
        c["pool"] = rng.choice(("e4m3", "i8"))
        c.update(n=_log(rng, 1, 64), lo=1)
        c["hi"] = _log(rng, 16, max(16, min(50_000, 400_000_000 // (c["n"] * Hkv * D))))
        return c
    if op == "step":
        c["pool"] = dtype
    if op != "write":
        c["window"] = rng.choice((0, 0, 0, 128, 1000, 4096))
    kind = rng.choice(("steps", "chunks", "mixed"))
    if kind == "steps":                # one token for each of n requests
        c.update(n=_log(rng, 1, 200), chunks=0, chunk=1)
        c["hi"] = _log(rng, 16, max(16, min(100_000, 1_000_000_000 // (c["n"] * Hkv * D))))
        c["lo"] = max(1, c["hi"] // rng.choice((1, 4, 30)))
    else:
        chunks = _log(rng, 1, 16)
        chunk = _log(rng, 2, 4096 // chunks if chunks < 8 else 1000)
        n = chunks + (_log(rng, 1, 100) if kind == "mixed" else 0)
        # scores of the padded chunks, and keys of the padded batch, stay below the listed ones'
        hi = min(32_000, 3_000_000_000 // (chunks * chunk * Hkv * G) - chunk,
                 1_000_000_000 // (n * Hkv * D) - chunk)
        hi = _log(rng, 1, max(2, hi))
        c.update(n=n, chunks=chunks, chunk=chunk, lo=max(0, hi // 8 - 1), hi=hi)
    return c


def lengths(c):
    """(cached tokens, new tokens) of each sequence of a case."""
    rng = random.Random(c["pattern"])
    before, new = [], []
    for i in range(c["n"]):
        b = _log(rng, c["lo"], c["hi"]) if c["lo"] > 0 else rng.randint(0, c["hi"])
        if c["op"] == "read":
            before.append(0)
            new.append(b)
            continue
        before.append(b)
        if i < c["chunks"]:
            new.append(c["chunk"] if i == 0 else _log(rng, max(1, c["chunk"] // 8), c["chunk"]))
        else:
            new.append(1)
    return before, new


def seen(c):
    """Visible (row, position) pairs, and cached tokens that some row sees, over all sequences."""
    pairs = tokens = 0
    for b, n in zip(*lengths(c)):
        w = c["window"] or b + n
        # row t sees min(b + t + 1, w) positions
        full = max(0, min(n, w - b))             # rows whose window is not yet full
        pairs += full * b + full * (full + 1) // 2 + (n - full) * w
        tokens += min(b + n, w + n - 1)
    return pairs, tokens


def work(c):
    D, Hkv, el = c["D"], c["Hkv"], BYTES[c["dtype"]]
    if c["op"] == "rope":
        rows = c["T"] * (c["Hq"] + Hkv)
        return {"bytes": 2 * rows * D * el + c["T"] * (8 + c["rot"] * 4), "flops": rows * (4 * D + 3 * c["rot"])}
    T = sum(lengths(c)[1])
    stored = D * BYTES[c["pool"]] + (4 if c["pool"] in TOP else 0)     # of one key or value
    if c["op"] == "read":
        return {"bytes": 2 * T * Hkv * (stored + D * el), "flops": 2 * T * Hkv * D}
    b = f = 0
    if c["op"] in ("write", "step"):
        b += T * D * el * (2 * c["Hq"] + 2 * Hkv) + 2 * T * Hkv * stored
        f += T * (c["Hq"] + Hkv) * (4 * D + 3 * c["rot"])
    if c["op"] == "write":
        b += 2 * T * Hkv * (stored + D * el)
    if c["op"] in ("attend", "step"):
        pairs, tokens = seen(c)
        b += 2 * tokens * Hkv * stored + (2 if c["op"] == "attend" else 1) * T * c["Hq"] * D * el
        f += 4 * pairs * c["Hq"] * D
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def quantise(x, pool):
    """(codes, scales) of rows of x (32 bits): one scale for each row of the last axis."""
    sc = x.abs().amax(-1) / TOP[pool]
    y = x / torch.where(sc > 0, sc, torch.ones_like(sc))[..., None]
    if pool == "i8":
        return torch.round(y).clamp_(-127, 127).to(torch.int8), sc
    return y.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn), sc


def rotation(positions, rot):
    """[positions][rot]: cosines, then sines, of the angles of adjacent frequencies."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    a = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, D, Hkv = DT[c["dtype"]], c["D"], c["Hkv"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    s = {"case": c}
    if c["op"] in ("rope", "write", "step"):
        if c["norm"]:
            s["q_weight"] = (1 + 0.2 * normal(D)).to(dt)
            s["k_weight"] = (1 + 0.2 * normal(D)).to(dt)
    if c["op"] == "rope":
        T = c["T"]
        # queries, keys and values come out of one projection, side by side
        qkv = (normal(T, c["Hq"] + 2 * Hkv, D) * 1.5).to(dt)
        s["q"], s["k"] = qkv[:, :c["Hq"]], qkv[:, c["Hq"]:c["Hq"] + Hkv]
        s["cos_sin"] = rotation(32768, c["rot"])
        s["positions"] = torch.randint(0, 32768, (T,), generator=g, device=DEV, dtype=torch.int32)
        return s
    before, new = lengths(c)
    total = [b + n for b, n in zip(before, new)]
    page = c["page"]
    need = [-(-t // page) for t in total]
    n_pages = sum(need) + 8
    ids = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int32)
    table = torch.full((c["n"], max(need)), -1, dtype=torch.int32)
    at = torch.tensor([0] + need).cumsum(0).tolist()
    ids = ids.cpu()
    for i, k in enumerate(need):
        table[i, :k] = ids[at[i]:at[i] + k]
    s["table"] = table.to(DEV)
    s["ctx_len"] = torch.tensor(total, dtype=torch.int32, device=DEV)
    s["q_start"] = torch.tensor([0] + new).cumsum(0).to(torch.int32).to(DEV)
    s["max_new"], s["max_ctx"] = max(new), max(total)
    T = s["T"] = sum(new)
    # keys have a few channels far larger than the others
    lift = torch.ones(D, device=DEV)
    lift[torch.randint(0, D, (3,), generator=g, device=DEV)] = 4.0
    for name, by in (("k", lift), ("v", None)):
        if c["pool"] in TOP:
            codes = torch.empty(n_pages, page, Hkv, D, dtype=DT[c["pool"]], device=DEV)
            scales = torch.empty(n_pages, page, Hkv, device=DEV)
            per = max(1, 100_000_000 // (page * Hkv * D))
            for p in range(0, n_pages, per):
                x = normal(min(per, n_pages - p), page, Hkv, D)
                codes[p:p + per], scales[p:p + per] = quantise(x if by is None else x.mul_(by), c["pool"])
            s[name + "_pool"], s[name + "_scale"] = codes, scales
        else:
            x = torch.empty(n_pages, page, Hkv, D, dtype=dt, device=DEV).normal_(generator=g)
            s[name + "_pool"], s[name + "_scale"] = x if by is None else x.mul_(by.to(dt)), None
    if c["op"] in ("write", "step"):
        qkv = (normal(T, c["Hq"] + 2 * Hkv, D) * 1.5).to(dt)
        s["q"], s["k"], s["v"] = qkv.split([c["Hq"], Hkv, Hkv], 1)
        s["cos_sin"] = rotation(s["max_ctx"], c["rot"])
    elif c["op"] == "attend":
        s["q"] = normal(T, c["Hq"], D).to(dt)
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def run_own(s):
    import paper_2609_29160_gb300 as tre
    c = s["case"]
    how = {}
    if c["op"] in ("rope", "write", "step"):
        how = dict(q_weight=s.get("q_weight"), k_weight=s.get("k_weight"), eps=EPS,
                   cos_sin=s["cos_sin"], interleaved=c["interleaved"])
    if c["op"] == "rope":
        q, k = tre.tre_qk_norm_rope(s["q"], s["k"], s["positions"], **how)
        return {"q": q, "k": k}
    cache = tre.KvCache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
    batch = tre.KvBatch(s["table"], s["ctx_len"], s["q_start"], s["T"], max_new=s["max_new"], max_ctx=s["max_ctx"])
    if c["op"] == "read":
        k, v = tre.tre_kv_read(cache, batch, dtype=c["dtype"])
        return {"k": k, "v": v}
    if c["op"] == "attend":
        return {"out": tre.tre_chunk_attention(s["q"], cache, batch, window=c["window"])}
    q = tre.tre_kv_append(cache, batch, s["k"], s["v"], q=s["q"], **how)
    if c["op"] == "write":
        k, v = tre.tre_kv_read(cache, batch, dtype=c["dtype"])
        return {"q": q, "k": k, "v": v}
    out = tre.tre_chunk_attention(q, cache, batch, window=c["window"])
    return {"out": out, "k": s["k_pool"], "v": s["v_pool"]}


# ---------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits
# ---------------------------------------------------------------------------
def plain_norm_rope(x, weight, cs, interleaved):
    """x [T][H][D], cs [T][rot]: the normed and rotated rows in 32 bits."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    rot = cs.shape[1]
    cos, sin = cs[:, None, :rot // 2], cs[:, None, rot // 2:]
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else r.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([r, x[..., rot:]], -1)


def plain_places(s):
    """Page and slot of every new token, and its position."""
    row = torch.arange(s["T"], device=DEV)
    seq = torch.searchsorted(s["q_start"], row.int(), right=True) - 1
    pos = row - s["q_start"][seq + 1] + s["ctx_len"][seq]
    page = s["case"]["page"]
    return s["table"][seq, pos // page].long(), pos % page, pos


def plain_write(s):
    c = s["case"]
    page, slot, pos = plain_places(s)
    cs = s["cos_sin"][pos]
    q = plain_norm_rope(s["q"], s.get("q_weight"), cs, c["interleaved"]).to(DT[c["dtype"]])
    k, v = plain_norm_rope(s["k"], s.get("k_weight"), cs, c["interleaved"]), s["v"].float()
    if c["pool"] in TOP:
        (k, s["k_scale"][page, slot]), (v, s["v_scale"][page, slot]) = quantise(k, c["pool"]), quantise(v, c["pool"])
        s["k_pool"].view(torch.uint8)[page, slot] = k.view(torch.uint8)
        s["v_pool"].view(torch.uint8)[page, slot] = v.view(torch.uint8)
    else:
        s["k_pool"][page, slot], s["v_pool"][page, slot] = k.to(DT[c["pool"]]), v.to(DT[c["pool"]])
    return q


def plain_rows(s, name, page, slot):
    """Rows of a cache in 32 bits."""
    p = s[name + "_pool"]
    if s[name + "_scale"] is None:
        return p[page, slot].float()
    return p.view(torch.uint8)[page, slot].view(p.dtype).float() * s[name + "_scale"][page, slot][..., None]


def plain_attend(s, q, first, last, longest):
    """Rows of sequences first..last-1, padded to the `longest` chunk among them."""
    c = s["case"]
    ctx, start = s["ctx_len"][first:last].long(), s["q_start"][first:last + 1].long()
    n, Hkv, D, G = last - first, c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    t = torch.arange(longest, device=DEV)
    new = start.diff()
    there = t < new[:, None]                                       # [n][t]
    rows = (start[:-1, None] + t).clamp(max=s["T"] - 1)
    j = torch.arange(s["max_ctx"], device=DEV)
    held = j < ctx[:, None]                                        # [n][j]
    page = s["table"][first:last, j // c["page"]].clamp(min=0).long()
    k = plain_rows(s, "k", page, j % c["page"])                    # [n][j][Hkv][D]
    x = q[rows].float().view(n, longest, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * longest, D)
    score = torch.matmul(x, k.permute(0, 2, 3, 1)).view(n, Hkv, G, longest, -1)
    del k
    pos = (ctx - new)[:, None] + t                                 # [n][t]
    visible = (j <= pos[..., None]) & held[:, None]
    if c["window"]:
        visible &= j > pos[..., None] - c["window"]
    score.mul_(1 / math.sqrt(D)).masked_fill_(~visible[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top.isfinite(), top, torch.zeros_like(top))).exp_()
    total = score.sum(-1, keepdim=True)
    score.div_(torch.where(total > 0, total, torch.ones_like(total)))
    v = plain_rows(s, "v", page, j % c["page"]) * held[..., None, None]
    out = torch.matmul(score.view(n, Hkv, G * longest, -1), v.permute(0, 2, 1, 3))
    out = out.view(n, Hkv, G, longest, D).permute(0, 3, 1, 2, 4).reshape(n, longest, Hkv * G, D)
    return out[there].to(DT[c["dtype"]])


def plain_attention(s, q):
    """Chunks and single tokens apart, so that neither is padded to the other."""
    c = s["case"]
    parts = []
    if c["chunks"]:
        parts.append(plain_attend(s, q, 0, c["chunks"], s["max_new"]))
    if c["chunks"] < c["n"]:
        parts.append(plain_attend(s, q, c["chunks"], c["n"], 1))
    return torch.cat(parts)


def run_plain(s):
    c = s["case"]
    if c["op"] == "rope":
        cs = s["cos_sin"][s["positions"]]
        return {n: plain_norm_rope(s[n], s.get(n + "_weight"), cs, c["interleaved"]).to(DT[c["dtype"]]) for n in ("q", "k")}
    if c["op"] == "attend":
        return {"out": plain_attention(s, s["q"])}
    got = {}
    if c["op"] in ("write", "step"):
        got["q"] = plain_write(s)
    if c["op"] == "step":
        return {"out": plain_attention(s, got["q"]), "k": s["k_pool"], "v": s["v_pool"]}
    page, slot, _ = plain_places(s)
    for n in ("k", "v"):
        got[n] = plain_rows(s, n, page, slot).to(DT[c["dtype"]])
    return got


def run(s):
    return run_own(s) if own else run_plain(s)


# ---------------------------------------------------------------------------
# the same from the definitions in 64 bits, a sequence at a time
# ---------------------------------------------------------------------------
def exact_heads(x, weight, table, pos, interleaved):
    x = x.double().clone()
    if weight is not None:
        x /= torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
        x *= weight.double()
    half = table.shape[1] // 2
    first = torch.arange(half, device=DEV) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    z = torch.complex(x[..., first], x[..., second])
    z *= torch.complex(table[pos, :half].double(), table[pos, half:].double())[:, None]
    x[..., first], x[..., second] = z.real.clone(), z.imag.clone()
    return x


def exact_stored(x, pool):
    """What a cache of type `pool` holds of x."""
    if pool not in TOP:
        return x.to(DT[pool]).double()
    sc = x.abs().max(-1, keepdim=True).values / TOP[pool]
    y = x / sc.clamp(min=1e-300)
    if pool == "i8":
        return torch.round(y) * sc
    # three bits after the leading one, steps no finer than 2^-9
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * sc


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        return {n: exact_heads(s[n], s.get(n + "_weight"), s["cos_sin"], s["positions"].long(), c["interleaved"]) for n in ("q", "k")}
    before, new = lengths(c)
    at = [0]
    for n in new:
        at.append(at[-1] + n)
    q = s.get("q")
    pools = {n: s[n + "_pool"] for n in ("k", "v")}
    fresh = {}
    pos = torch.cat([torch.arange(b, b + n, device=DEV) for b, n in zip(before, new)])
    if c["op"] in ("write", "step"):
        q, k = (exact_heads(s[n], s.get(n + "_weight"), s["cos_sin"], pos, c["interleaved"]) for n in ("q", "k"))
        fresh = {"k": exact_stored(k, c["pool"]), "v": exact_stored(s["v"].double(), c["pool"])}
        if c["op"] == "write":
            return {"q": q, **fresh}

    def context(name, i):
        """Sequence i's rows, the new ones included."""
        total = before[i] + new[i]
        pages = s["table"][i, :-(-total // c["page"])].long()
        x = pools[name].view(torch.uint8)[pages].view(pools[name].dtype) if c["pool"] in TOP else pools[name][pages]
        x = x.double()
        if s[name + "_scale"] is not None:
            x = x * s[name + "_scale"][pages].double()[..., None]
        x = x.reshape(-1, c["Hkv"], c["D"])[:total].clone()
        if fresh:
            x[before[i]:] = fresh[name][at[i]:at[i + 1]]
        return x

    if c["op"] == "read":
        return {n: torch.cat([context(n, i) for i in range(c["n"])]) for n in ("k", "v")}
    G = c["Hq"] // c["Hkv"]
    out = torch.empty(s["T"], c["Hq"], c["D"], dtype=torch.float64, device=DEV)
    for i in range(c["n"]):
        k, v = context("k", i), context("v", i)
        x = q[at[i]:at[i + 1]].double()
        p = torch.arange(before[i], before[i] + new[i], device=DEV)[:, None]
        j = torch.arange(before[i] + new[i], device=DEV)[None]
        hidden = j > p
        if c["window"]:
            hidden = hidden | (p - j >= c["window"])
        for h in range(c["Hkv"]):
            for m in range(h * G, (h + 1) * G):
                a = x[:, m] @ k[:, h].T
                a = torch.softmax((a / math.sqrt(c["D"])).masked_fill_(hidden, -math.inf), -1)
                out[at[i]:at[i + 1], m] = a @ v[:, h]
    if c["op"] == "attend":
        return {"out": out}
    got = {"out": out}
    for n in ("k", "v"):
        x = pools[n].double()
        for i in range(c["n"]):
            p = torch.arange(before[i], before[i] + new[i], device=DEV)
            x[s["table"][i].long()[p // c["page"]], p % c["page"]] = fresh[n][at[i]:at[i + 1]]
        got[n] = x
    return got
