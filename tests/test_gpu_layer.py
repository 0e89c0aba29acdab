"""A layer's operators one after the other as they are used, and their refusals in Python."""
import pytest
import torch

import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tre():
    import paper_2609_29160_gb300 as t
    t.load()
    return t


class Layer:
    def __init__(self, tre, dim, inner, experts, dtype="bf16", seed=4):
        self.dtype = R.T[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n1, self.n2, self.n3 = ((1 + 0.1 * torch.randn(dim, generator=g, device="cuda")).to(self.dtype) for _ in range(3))
        self.router = torch.randn(dim, experts, generator=g, device="cuda").to(self.dtype) / dim ** 0.5
        mats = [R.matrix4(None, dim, dim, 64, self.dtype, True, seed), R.matrix4(experts, 2 * inner, dim, 32, self.dtype, False, seed + 1),
                R.matrix4(experts, dim, inner, 32, self.dtype, False, seed + 2)]
        self.m = [x[3] for x in mats]
        self.w = [tre.Weights4(*x[:3], gated=i == 1) for i, x in enumerate(mats)]

    def run(self, tre, x, y):
        r, n = tre.tre_block_norm(x, y, weight=self.n1)
        a = tre.tre_linear4(n, self.w[0])
        r, n = tre.tre_block_norm(r, a, post_weight=self.n3, weight=self.n2)
        ids, weights = tre.tre_route((n @ self.router).float(), 2)
        e = tre.tre_experts(n, ids, weights, self.w[1], self.w[2])
        return n, ids, weights, e, tre.tre_block_norm(r, e, scale=0.5)[0]


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_layer(tre, rows):
    """Each step against the formula on the step's own inputs."""
    layer = Layer(tre, 256, 96, 8)
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, y = (torch.randn(rows, 256, generator=g, device="cuda").bfloat16() for _ in range(2))
    n, ids, weights, e, last = layer.run(tre, x, y)
    r, off, n1, off1 = R.block_norm(x, y, None, None, 1.0, layer.n1, 1e-6)
    r_own, n_own = tre.tre_block_norm(x, y, weight=layer.n1)
    R.near(r_own, r, off)
    R.near(n_own, n1, off1)
    a = tre.tre_linear4(n_own, layer.w[0])
    R.near(a, *R.product(n_own, layer.m[0]))
    r2, off2, n2, offn2 = R.block_norm(r_own, a, layer.n3, None, 1.0, layer.n2, 1e-6)
    R.near(n, n2, offn2)
    want, _ = R.route((n @ layer.router).float(), 2)
    assert torch.equal(ids.cpu(), want)
    R.near(e, *R.experts(n, ids, weights, layer.m[1], layer.m[2], layer.dtype))
    again = layer.run(tre, x, y)
    assert all(torch.equal(p, q) for p, q in zip(again, (n, ids, weights, e, last)))
    tre.check_replica()


@pytest.mark.parametrize("rows", [3, 300])
def test_layer_in_graphs(tre, rows):
    """Two captured runs that share no workspace, replayed with other inputs, one after the other
    and from two streams at once."""
    layer = Layer(tre, 256, 96, 8)
    g = torch.Generator(device="cuda").manual_seed(rows)
    xs = [torch.randn(2, rows, 256, generator=g, device="cuda").bfloat16() for _ in range(2)]
    layer.run(tre, xs[0][0], xs[0][1])
    tre.replica_diag()
    graphs, outs = [], []
    torch.cuda.synchronize()
    for x in xs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(layer.run(tre, x[0], x[1]))
        graphs.append(graph)
    for x in xs:
        x.neg_()
    want = [layer.run(tre, x[0], x[1]) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_calls_on_two_streams_at_once(tre):
    layer = Layer(tre, 256, 96, 8)
    g = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.randn(2, n, 256, generator=g, device="cuda").bfloat16() for n in (2, 40, 700)]
    want = [layer.run(tre, x[0], x[1]) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(4):
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append(layer.run(tre, x[0], x[1]))
    torch.cuda.synchronize()
    for i, a in enumerate(got):
        assert all(torch.equal(p, q) for p, q in zip(a, want[i % 3]))


def test_served_replica_of_experts():
    """Requests through layers of experts: each gets its tokens, and runs again give the same."""
    from paper_2609_29160_gb300 import served
    out = []
    for _ in range(2):
        rep = served.Replica(layers=2, q_heads=4, kv_heads=2, dim=64, pages=64, experts=8, top=2, chunk=48, seed=3)
        done = rep.serve([(0, 70, 5), (1, 3, 9), (1, 120, 2)], seed=1)
        assert len(done) == 3 and all(len(r["tokens"]) == r["L_in"] + r["L_out"] for r in done)
        out.append({r["L_in"]: r["tokens"].tolist() for r in done})
    assert out[0].keys() == out[1].keys()
    assert rep.prompt_weight(requests=4, context=64, times=2) > 0


def bad_calls(tre):
    t, u8 = torch, torch.uint8

    def z(*s, dtype=t.bfloat16, device="cuda"):
        return t.zeros(*s, dtype=dtype, device=device)

    x, w = z(3, 128), z(128)
    codes, sc = z(64, 64, dtype=u8), z(64, 2)
    m = tre.Weights4(codes, sc)
    up, down = tre.Weights4(z(4, 64, 64, dtype=u8), z(4, 64, 4), gated=True), tre.Weights4(z(4, 128, 16, dtype=u8), z(4, 128, 1))
    ids, ws = z(3, 2, dtype=t.int32), z(3, 2, dtype=t.float32)
    return [
        lambda: tre.tre_block_norm(x), lambda: tre.tre_block_norm(x, x.half(), weight=w),
        lambda: tre.tre_block_norm(x, x[:2], weight=w), lambda: tre.tre_block_norm(x, x, weight=w[:64]),
        lambda: tre.tre_block_norm(x, x, gate=z(5), weight=w), lambda: tre.tre_block_norm(x, x, gate=w.float(), weight=w),
        lambda: tre.tre_block_norm(x, gate=w, weight=w), lambda: tre.tre_block_norm(x, x, out=x),
        lambda: tre.tre_block_norm(x, x, weight=w, post_weight=w.float()), lambda: tre.tre_block_norm(x.cpu(), weight=w),
        lambda: tre.tre_block_norm(x, x.cpu(), weight=w), lambda: tre.tre_block_norm(x.t(), weight=z(3)),
        lambda: tre.tre_block_norm(z(3, 16385), weight=z(16385)), lambda: tre.tre_block_norm(x.double(), weight=w),
        lambda: tre.tre_block_norm(z(3, 8, dtype=t.int8), weight=z(8)), lambda: tre.tre_block_norm(x, weight=w, dtype="f16"),
        lambda: tre.tre_route(x, 0), lambda: tre.tre_route(x, 33), lambda: tre.tre_route(x, 2, scores="linear"),
        lambda: tre.tre_route(x, 2, bias=w), lambda: tre.tre_route(x, 2, groups=3), lambda: tre.tre_route(x, 2, groups=4, top_groups=5),
        lambda: tre.tre_route(x, 2, group_best=3), lambda: tre.tre_route(x.double(), 2), lambda: tre.tre_route(x[0], 2),
        lambda: tre.tre_route(x, 2, ids=z(3, 2, dtype=t.int64)), lambda: tre.tre_route(x, 2, weights=z(3, 4, dtype=t.float32)[:, ::2]),
        lambda: tre.Weights4(codes, sc.float()), lambda: tre.Weights4(codes.int(), sc), lambda: tre.Weights4(codes, z(64, 3)),
        lambda: tre.Weights4(codes, z(63, 2)), lambda: tre.Weights4(codes[:, ::2], z(64, 2)), lambda: tre.Weights4(codes, sc, z(64, 2)),
        lambda: tre.Weights4(z(63, 64, dtype=u8), z(63, 2), gated=True), lambda: tre.Weights4(codes, sc.cpu()),
        lambda: tre.tre_linear4(x.half(), m), lambda: tre.tre_linear4(x[:, :64], m), lambda: tre.tre_linear4(x, up),
        lambda: tre.tre_linear4(x.cpu(), m), lambda: tre.tre_linear4(x, m, out=z(3, 63)), lambda: tre.tre_linear4(x, m, out=z(3, 64).half()),
        lambda: tre.tre_linear4(x, m, dtype="f16"), lambda: tre.tre_linear4(x, tre.Weights4(codes, sc, gated=True), dtype="f32"),
        lambda: tre.tre_linear4(x.float(), m, dtype="bf16"),
        lambda: tre.tre_experts(x, ids.long(), ws, up, down), lambda: tre.tre_experts(x, ids, ws.half(), up, down),
        lambda: tre.tre_experts(x, ids[:2], ws, up, down), lambda: tre.tre_experts(x, ids, ws, down, up),
        lambda: tre.tre_experts(x, ids, ws, up, up), lambda: tre.tre_experts(x, ids, ws, up, m),
        lambda: tre.tre_experts(x.float(), ids, ws, up, down), lambda: tre.tre_experts(x, ids.t().contiguous().t(), ws, up, down),
        lambda: tre.tre_experts(x, z(3, 33, dtype=t.int32), z(3, 33, dtype=t.float32), up, down),
    ]


def test_refusals(tre):
    for i, call in enumerate(bad_calls(tre)):
        with pytest.raises((ValueError, tre.TreError)):
            call()
            raise AssertionError(f"call {i} was taken")
    # rows that 16 bytes do not divide have no way into the products
    x = torch.zeros(4, 132, dtype=torch.bfloat16, device="cuda")[:, :128]
    m = tre.Weights4(torch.zeros(64, 64, dtype=torch.uint8, device="cuda"), torch.zeros(64, 2, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(tre.TreError):
        tre.tre_linear4(x, m)
