"""A served replica: where the library's request records and service times come from.

A small decoder with random weights serves requests on this GPU by continuous
batching: every step takes one token of each running request and a chunk of one
prompt, through tre_kv_append and tre_chunk_attention over a paged cache, layer by
layer; with experts also through tre_block_norm, tre_linear4, tre_route and tre_experts, its
matrices in 4 bits. The clock is the measured time of the steps, so that what a prompt token and a
decode token cost here, against each other (Eq. 1's w_p) and in milliseconds, is what
this machine takes. The outcome is the library's own inputs: request records for
tss_window_reduce and PipelinePlan, and latent service times for tre_replay.

    python -m paper_2609_29160_gb300.served
"""
from __future__ import annotations

import paper_2609_29160_gb300 as tre
from paper_2609_29160_gb300 import replica


def in_four_bits(w, group=32, gated=False):
    """Weights4 of w [n][k] or [experts][n][k]: the nearest of sixteen steps, zero among them,
    to each group's element farthest from zero."""
    torch = tre._torch()
    g = w.float().unflatten(-1, (-1, group))
    scales = (g.abs().amax(-1) / 7).to(w.dtype)
    step = torch.where(scales > 0, scales, torch.ones_like(scales)).float()[..., None]
    codes = (torch.round(g / step).clamp(-8, 7) + 8).to(torch.uint8).flatten(-2)
    return tre.Weights4(codes[..., 0::2] | codes[..., 1::2] << 4, scales, gated=gated)


class Replica:
    """A decoder of `layers` layers with its paged caches, and the requests it runs.

    cache: type of the caches ("bf16", "e4m3", "i8"). chunk: most prompt tokens a step.
    time_scale: milliseconds of the clock for each millisecond measured (a model with so
    many more layers). experts: with some, layers have norms around their blocks, matrices in
    4 bits and a feed-forward block of so many experts, `top` of them for a token."""

    def __init__(self, layers=2, q_heads=8, kv_heads=2, dim=64, vocab=256, pages=512, page=16,
                 chunk=128, cache="bf16", max_positions=4096, time_scale=1.0, seed=0,
                 experts=0, top=2):
        torch = self.torch = tre._torch()
        g = torch.Generator(device="cuda").manual_seed(seed)
        width = q_heads * dim

        def weight(*shape, scale):
            return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()

        self.heads = (q_heads, kv_heads, dim)
        self.embed = weight(vocab, width, scale=1.0)
        self.layers = [{
            "qkv": weight(width, (q_heads + 2 * kv_heads) * dim, scale=width ** -0.5),
            "out": weight(width, width, scale=width ** -0.5),
            "q_weight": (1 + weight(dim, scale=0.1)), "k_weight": (1 + weight(dim, scale=0.1)),
            "cache": tre.KvCache.empty(pages, page, kv_heads, dim, cache)} for _ in range(layers)]
        self.experts, self.top = experts, top
        if experts:
            for w in self.layers:
                w["qkv"], w["out"] = in_four_bits(w["qkv"].T.contiguous()), in_four_bits(w["out"].T.contiguous())
                w["norm"], w["ff_norm"] = 1 + weight(width, scale=0.1), 1 + weight(width, scale=0.1)
                w["router"] = weight(width, experts, scale=width ** -0.5).float()
                w["up"] = in_four_bits(weight(experts, 2 * width, width, scale=width ** -0.5), gated=True)
                w["down"] = in_four_bits(weight(experts, width, width, scale=width ** -0.5))
            self.norm = 1 + weight(width, scale=0.1)
        f = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
        angle = torch.arange(max_positions, dtype=torch.float64, device="cuda")[:, None] * f
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()
        self.page, self.free, self.chunk = page, list(range(pages)), chunk
        self.time_scale, self.max_positions = time_scale, max_positions
        self.max_pages = -(-max_positions // page)
        self.steps = []                       # (prompt tokens, decode tokens, ms) of each
        self.diag = replica.host_diag()

    def attention(self, w, qkv, batch):
        """A layer's attention of the batch's new tokens."""
        hq, hk, dim = self.heads
        q, k, v = qkv.view(-1, hq + 2 * hk, dim).split([hq, hk, hk], 1)
        q = tre.tre_kv_append(w["cache"], batch, k, v, q=q, q_weight=w["q_weight"],
                              k_weight=w["k_weight"], cos_sin=self.cos_sin, diag=self.diag)
        return tre.tre_chunk_attention(q, w["cache"], batch, diag=self.diag).flatten(1)

    def forward(self, tokens, batch):
        """Last-layer rows of the batch's new tokens."""
        x = self.embed[tokens]
        if not self.experts:
            for w in self.layers:
                x = x + self.attention(w, x @ w["qkv"], batch) @ w["out"]
            return x
        y = None
        for w in self.layers:
            x, n = tre.tre_block_norm(x, y, weight=w["norm"])
            y = self.attention(w, tre.tre_linear4(n, w["qkv"], diag=self.diag), batch)
            x, n = tre.tre_block_norm(x, tre.tre_linear4(y, w["out"], diag=self.diag), weight=w["ff_norm"])
            # (in 32 bits: with logits of 16, experts that differ would tie and go by their number)
            ids, weights = tre.tre_route(n.float() @ w["router"], self.top)
            y = tre.tre_experts(n, ids, weights, w["up"], w["down"], diag=self.diag)
        return tre.tre_block_norm(x, y, weight=self.norm)[1]

    def _batch(self, work):
        """KvBatch of [(request, tokens in the cache, new tokens)]."""
        torch = self.torch
        table = torch.full((len(work), self.max_pages), -1, dtype=torch.int32)
        for i, (r, held, new) in enumerate(work):
            while len(r["pages"]) * self.page < held + new:
                r["pages"].append(self.free.pop())
            table[i, :len(r["pages"])] = torch.tensor(r["pages"], dtype=torch.int32)
        total = [held + new for _, held, new in work]
        starts = [0]
        for _, _, new in work:
            starts.append(starts[-1] + new)
        return tre.KvBatch(table.cuda(), torch.tensor(total, dtype=torch.int32).cuda(),
                           torch.tensor(starts, dtype=torch.int32).cuda(), starts[-1],
                           max_new=max(n for _, _, n in work), max_ctx=max(total))

    def _check(self):
        """What the kernels left in diag (the device has been waited for)."""
        d = tre.read_diag(self.diag)
        if d["err"]:
            raise tre.TreError("served step", d["err"])
        if d["dropped_range"]:
            raise RuntimeError(f"served step: {d['dropped_range']} rows had no place")

    def _step(self, work):
        """Runs one step; the next token of each sequence."""
        torch = self.torch
        tokens = torch.cat([r["tokens"][held:held + new] for r, held, new in work])
        batch = self._batch(work)
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        x = self.forward(tokens, batch)
        ends = batch.q_start[1:].long() - 1
        best = (x[ends] @ self.embed.T).float().argmax(1)
        b.record()
        b.synchronize()
        self._check()
        ms = a.elapsed_time(b)
        prompt = sum(n for r, held, n in work if held < r["L_in"])
        self.steps.append((prompt, sum(n for _, _, n in work) - prompt, ms))
        return best, ms * self.time_scale

    def serve(self, arrivals, seed=0):
        """arrivals: [(arrival ms, prompt tokens, output tokens)] in order of arrival.
        Returns the requests as dicts: their times in ms and their tokens."""
        torch = self.torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        vocab = self.embed.shape[0]
        waiting = []
        for t, n_in, n_out in arrivals:
            if n_in < 1 or n_out < 1 or n_in + n_out > self.max_positions:
                raise ValueError("arrivals: a request needs a token in and out, and its place")
            waiting.append({"t_arr": t, "L_in": n_in, "L_out": n_out, "pages": [], "held": 0,
                            "tokens": torch.randint(0, vocab, (n_in,), generator=g, device="cuda")})
        # (the first launches are not the clock's: a token's, and those of a prompt's chunk as
        # long as there is room for)
        for n in (1, self.chunk):
            n = min(n, self.max_positions, len(self.free) * self.page)
            if n == 0:
                break
            first = {"pages": [], "L_in": n, "tokens": torch.zeros(n, dtype=torch.int64, device="cuda")}
            try:
                self._step([(first, 0, n)])
                self.steps.pop()
            finally:
                self.free += first["pages"]
        done, running, clock = [], [], 0.0
        need = lambda r: -(-(r["L_in"] + r["L_out"]) // self.page)      # noqa: E731
        room = len(self.free)
        while waiting or running:
            if not running and waiting and waiting[0]["t_arr"] > clock:
                clock = float(waiting[0]["t_arr"])
            # a request starts when pages for all of it are left
            while waiting and waiting[0]["t_arr"] <= clock:
                if need(waiting[0]) > room:
                    if not running:
                        raise ValueError("pages: too few for one request")
                    break
                r = waiting.pop(0)
                room -= need(r)
                r["t_start"] = clock
                running.append(r)
            work, prompt = [], None
            for r in running:
                left = len(r["tokens"]) - r["held"]
                if r["held"] >= r["L_in"]:
                    work.append((r, r["held"], left))
                elif prompt is None:                   # one prompt's chunk a step
                    prompt = (r, r["held"], min(left, self.chunk))
            work += [prompt] if prompt else []
            best, ms = self._step(work)
            clock += ms
            for (r, held, new), token in zip(work, best):
                r["held"] = held + new
                if r["held"] < r["L_in"]:
                    continue
                r.setdefault("t_first", clock)
                r["tokens"] = torch.cat([r["tokens"], token[None]])
                if len(r["tokens"]) == r["L_in"] + r["L_out"]:
                    r["t_end"] = clock
                    self.free += r.pop("pages")
                    room += need(r)
                    done.append(r)
            running = [r for r in running if "t_end" not in r]
        return done

    def prompt_weight(self, requests=16, context=256, times=10):
        """What a prompt token costs against a decode token (Eq. 1's w_p): a step of a
        prompt's chunk and one of a token each of `requests` requests, timed, all with
        `context` tokens in the cache (for all of which there has to be room)."""
        torch = self.torch
        ms = []
        for n, new in ((1, self.chunk), (requests, 1)):
            if context + new > self.max_positions:
                raise ValueError(f"prompt_weight: {context} + {new} tokens, the replica takes {self.max_positions}")
            if n * -(-(context + new) // self.page) > len(self.free):
                raise ValueError(f"prompt_weight: too few free pages for {n} x {context + new} tokens")
            tokens = torch.zeros(n * new, dtype=torch.int64, device="cuda")
            work = [({"pages": []}, context, new) for _ in range(n)]
            try:
                batch = self._batch(work)
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                for k in range(times + 3):
                    if k == 3:
                        a.record()
                    self.forward(tokens, batch)
                b.record()
                b.synchronize()
                self._check()
            finally:
                for r, _, _ in work:
                    self.free += r["pages"]
            ms.append(a.elapsed_time(b) / times / len(tokens))
        return ms[0] / ms[1]


def records(served, torch_device="cuda"):
    """Request records of served requests of several models ([requests of model 0, ..]),
    as tss_window_reduce takes them: int32 CUDA columns in order of arrival."""
    torch = tre._torch()
    rows = [(m, int(r["t_arr"]), int(r["t_start"]), int(r["t_first"]), int(r["t_end"]), r["L_in"],
             r["L_out"]) for m, reqs in enumerate(served) for r in reqs]
    rows.sort(key=lambda x: x[1])
    cols = torch.tensor(rows, dtype=torch.int32).reshape(-1, 7).T.contiguous()
    names = ("model", "t_arr_ms", "t_start_ms", "t_first_ms", "t_end_ms", "L_in", "L_out")
    return {n: c.contiguous().to(torch_device) for n, c in zip(names, cols)}


def latent(rec):
    """The latent trace of these records for tre_replay: service times instead of times."""
    return {"model": rec["model"], "t_arr_ms": rec["t_arr_ms"],
            "d_first_ms": rec["t_first_ms"] - rec["t_start_ms"],
            "d_total_ms": rec["t_end_ms"] - rec["t_start_ms"],
            "L_in": rec["L_in"], "L_out": rec["L_out"]}


def main():
    import random
    rng = random.Random(1)
    served, weights = [], []
    for m, cache in enumerate(("bf16", "e4m3", "i8")):
        rep = Replica(layers=4, q_heads=16, kv_heads=4, dim=128, pages=2048, cache=cache,
                      time_scale=8.0, seed=m)
        t, arrivals = 0, []
        for _ in range(60):
            t += int(rng.expovariate(1 / (40 + 20 * m)))
            arrivals.append((t, 1 + int(rng.lognormvariate(4.5, 0.8)), 1 + int(rng.expovariate(1 / 24))))
        served.append(rep.serve(arrivals))
        weights.append(rep.prompt_weight())
        tokens = sum(p + d for p, d, _ in rep.steps)
        print(f"model {m} ({cache} cache): {len(rep.steps)} steps, {tokens} tokens, "
              f"w_p {weights[-1]:.3f}")
    rec = records(served)
    window = 250
    K = int(rec["t_end_ms"].max()) // window + 1
    counts = tre.tss_window_reduce(3, window, K, requests=rec)
    prof = {"w_p": weights, "w_q": 2.0, "alpha": 0.3, "tau_crit": 0.8, "tau_surplus": 1.2}
    theta = tre.tss_calibrate(counts, prof, window, [400] * 3, requests=rec)
    scored = tre.tss_score(counts, dict(prof, theta=theta), window)
    names = ("critical", "nominal", "surplus", "idle")
    for m in range(3):
        seen = [int((scored["cls"][:, m] == c).sum()) for c in range(4)]
        print(f"model {m}: theta {float(theta[m]):.1f}, windows "
              + ", ".join(f"{n} {k}" for n, k in zip(names, seen)))


if __name__ == "__main__":
    main()
