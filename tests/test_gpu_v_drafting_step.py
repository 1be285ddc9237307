"""A serving step with drafted tokens as it is used: projection with bias, append to the cache, attention of the tree, output projection
added to the residual; then the accepted path moves to its place and decoding goes on."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from tests.cache_util import pack_bits

pytestmark = pytest.mark.gpu

HQ, HK, DIM, GROUP, PAGE, HIDDEN = 8, 2, 128, 64, 16, 512


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


class Layer:
    def __init__(self, ctx, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.ctx = ctx
        self.w = (rnd((HQ + 2 * HK) * DIM, HIDDEN) * HIDDEN ** -0.5).bfloat16()
        self.b = (rnd((HQ + 2 * HK) * DIM) * 0.3).bfloat16()
        self.wo = (rnd(HIDDEN, HQ * DIM) * (HQ * DIM) ** -0.5).bfloat16()
        self.bo = (rnd(HIDDEN) * 0.3).bfloat16()
        self.inv = torch.tensor([10000.0 ** (-2 * i / DIM) for i in range(DIM // 2)], dtype=torch.float64, device="cuda")

    def project(self, x):
        from paper_2607_28418_b200 import binding
        qkv = binding.wide_linear(self.ctx, x, self.w, bias=self.b)
        a, b = HQ * DIM, HK * DIM
        return qkv[:, :a], qkv[:, a:a + b], qkv[:, a + b:]

    def step(self, cache, seqs, x, pos, tree, mask=None):
        """The layer's attention half for the nodes x [rows, HIDDEN] of the sequences' trees."""
        from paper_2607_28418_b200 import binding
        q, k, v = self.project(x)
        q = binding.wide_cache_append(self.ctx, cache, seqs, q, k, v, pos, self.inv)
        o = binding.wide_attn_tree(self.ctx, q, cache, seqs, HQ, HQ // HK, tree, mask_bits=mask)
        return binding.wide_linear(self.ctx, o, self.wo, bias=self.bo, residual=x)

    def turned(self, x, heads, pos):
        """The rotation of rows x in 64 bits, rounded to bf16."""
        y = x.double().view(len(x), heads, DIM)
        a = pos.double()[:, None, None] * self.inv
        u, w = y[..., :DIM // 2], y[..., DIM // 2:]
        return torch.cat([u * a.cos() - w * a.sin(), u * a.sin() + w * a.cos()], -1).bfloat16()


def places(n_seqs, pages_each, seed):
    order = torch.randperm(n_seqs * pages_each, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    return order.view(n_seqs, pages_each).cuda()


def fill(ctx, layer, cache, table, lens, seed):
    """A prompt in the cache: its hidden states' keys and values, rotated."""
    from paper_2607_28418_b200 import binding
    x = torch.randn((sum(lens), HIDDEN), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()
    starts = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    seqs = binding.Sequences(table, torch.tensor(lens, dtype=torch.int32, device="cuda"), starts)
    _, k, v = layer.project(x)
    pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    binding.wide_cache_append(ctx, cache, seqs, None, k, v, pos, layer.inv)
    return x


def test_a_step_against_64_bits(ctx):
    """Each stage is taken from its inputs as the GPU has them, so that a rounding is counted once: the projection (2^-8 of its result and the
    sums' 2^-23 a step), the cache's levels as it holds them, the attention (its probabilities' 2^-8), the output projection."""
    from paper_2607_28418_b200 import binding
    layer = Layer(ctx, 1)
    lens, parents = [70, 33], [[-1, 0, 0, 1, 2, 2, -1], [-1, 0, 1]]
    n = [len(p) for p in parents]
    table = places(2, 8, 2)
    cache = binding.Cache.empty(16, HK, DIM, GROUP, PAGE)
    fill(ctx, layer, cache, table, lens, 3)
    starts = torch.tensor([0, n[0], n[0] + n[1]], dtype=torch.int32, device="cuda")
    seqs = binding.Sequences(table, torch.tensor([a + b for a, b in zip(lens, n)], dtype=torch.int32, device="cuda"), starts)
    tree = torch.cat([binding.tree_ancestors(p, 1) for p in parents]).cuda()
    depth = []
    for p in parents:
        d = []
        for i in p:
            d.append(0 if i < 0 else d[i] + 1)
        depth.append(d)
    pos = torch.tensor([a + d for a, ds in zip(lens, depth) for d in ds], dtype=torch.int32, device="cuda")
    x = torch.randn((sum(n), HIDDEN), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").bfloat16()
    on = np.random.default_rng(5).random((sum(n), HK)) < 0.6
    got = layer.step(cache, seqs, x, pos, tree, torch.from_numpy(pack_bits(on)).cuda())

    qkv = x.double() @ layer.w.double().t() + layer.b.double()
    q, k, v = layer.project(x)
    for part, ref in ((q, qkv[:, :HQ * DIM]), (k, qkv[:, HQ * DIM:(HQ + HK) * DIM]), (v, qkv[:, (HQ + HK) * DIM:])):
        assert ((part.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -23 * (HIDDEN / 16 + 2) * 40).all()
    turned = layer.turned(q, HQ, pos)
    all_starts = torch.tensor([0, lens[0] + n[0], sum(lens) + sum(n)], dtype=torch.int32, device="cuda")
    whole = binding.Sequences(table, seqs.kv_lens, all_starts)
    kk, vv = binding.wide_cache_read(ctx, cache, whole, sum(lens) + sum(n), dtype=torch.float32)
    # the new keys are held within half a step (the range of a sub-group / 15, at most 1 here) of the rotated ones
    new_k = torch.cat([kk[lens[0]:lens[0] + n[0]], kk[sum(lens) + n[0]:]]).double().view(-1, HK, DIM)
    assert ((new_k - layer.turned(k, HK, pos).double()).abs() <= 0.5 + 2.0 ** -6).all()
    o, at, row = torch.zeros((sum(n), HQ, DIM), dtype=torch.float64, device="cuda"), 0, 0
    slack = torch.zeros_like(o)
    for a, m, p in zip(lens, n, parents):
        keys, values = (z[at:at + a + m].double().view(-1, HK, DIM) for z in (kk, vv))
        see = torch.ones((m, a + m), dtype=torch.bool)
        for i, up in enumerate(p):
            see[i, a:] = see[up, a:] if up >= 0 else False
            see[i, a + i] = True
        z = turned[row:row + m].double().view(m, HK, HQ // HK, DIM)
        s = torch.einsum("mhsd,nhd->mhsn", z, keys) * DIM ** -0.5
        pr = torch.softmax(s.masked_fill(~see[:, None, None].cuda(), -torch.inf), -1)
        o[row:row + m] = torch.einsum("mhsn,nhd->mhsd", pr, values).reshape(m, HQ, DIM)
        # a logit's products are off by 2^-11 of the key (and by 2^-8 where a rotated query is the neighbouring bf16 number: one in thousands),
        # probabilities and values by 2^-11
        weighed = torch.einsum("mhsn,nhd->mhsd", pr, values.abs()).reshape(m, HQ, DIM)
        size = torch.einsum("mhsd,nhd->mhsn", z.abs(), keys.abs()).amax(-1).reshape(m, HQ, 1) * DIM ** -0.5
        slack[row:row + m] = weighed * (2.0 ** -10 + 2.0 ** -9 * size) + 2.0 ** -8 * o[row:row + m].abs()
        at, row = at + a + m, row + m
    live = torch.from_numpy(np.repeat(on, HQ // HK, axis=1)).cuda()[..., None]
    o, slack = (o * live).flatten(1), (slack * live).flatten(1)
    ref = o @ layer.wo.double().t() + layer.bo.double() + x.double()
    tol = slack @ layer.wo.double().abs().t() + 2.0 ** -8 * ref.abs() + 2.0 ** -23 * 64 * 10
    assert ((got.double() - ref).abs() <= tol).all()


def test_the_accepted_path_goes_on(ctx):
    """Nodes 0, 2, 5 of a tree are accepted: their keys and values are written again at the positions of the answer, and the next token sees the
    bytes that a decoder without drafts would have."""
    from paper_2607_28418_b200 import binding
    layer = Layer(ctx, 11)
    table = places(1, 8, 12)
    drafted, plain = (binding.Cache.empty(8, HK, DIM, GROUP, PAGE) for _ in range(2))
    for c in (drafted, plain):
        c.pages.zero_()
        fill(ctx, layer, c, table, [61], 13)
    parents, path = [-1, -1, 0, 0, 2, 2, 5], [0, 2, 5]
    depth = [0, 0, 1, 1, 2, 2, 3]
    x = torch.randn((7, HIDDEN), generator=torch.Generator(device="cuda").manual_seed(14), device="cuda").bfloat16()
    one = torch.tensor([0, 7], dtype=torch.int32, device="cuda")
    seqs = binding.Sequences(table, torch.tensor([68], dtype=torch.int32, device="cuda"), one)
    pos = torch.tensor([61 + d for d in depth], dtype=torch.int32, device="cuda")
    tree = binding.tree_ancestors(parents).cuda()
    out = layer.step(drafted, seqs, x, pos, tree)
    # a decoder without drafts: the path token by token, each seeing those before it
    for i, node in enumerate(path):
        s = binding.Sequences(table, torch.tensor([62 + i], dtype=torch.int32, device="cuda"))
        y = layer.step(plain, s, x[node:node + 1], pos[node:node + 1], torch.ones((1, 1), dtype=torch.int32, device="cuda"))
        # (another number of rows sums in another order: the products' and the probabilities' roundings, each once more)
        assert ((y - out[node:node + 1]).abs().float() <= 2.0 ** -5 * (1 + out[node].abs().float())).all()
    _, k, v = layer.project(x)
    moved = binding.Sequences(table, torch.tensor([64], dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda"))
    binding.wide_cache_append(ctx, drafted, moved, None, k[path].contiguous(), v[path].contiguous(), pos[path].contiguous(), layer.inv)
    a, b = (binding.wide_cache_read(ctx, c, binding.Sequences(table, moved.kv_lens, torch.tensor([0, 64], dtype=torch.int32, device="cuda")), 64) for c in (drafted, plain))
    held = [z.float() for z in a], [z.float() for z in b]
    # prompt and values' levels from the same projections are the same bytes; the path's projections of one row and of seven agree to a rounding, so levels may be neighbours
    assert torch.equal(held[0][0][:61], held[1][0][:61]) and torch.equal(held[0][1][:61], held[1][1][:61])
    for p, q in zip(*held):
        assert ((p[61:] - q[61:]).abs() <= 1.0).all()


def test_the_whole_step_in_one_graph(ctx):
    """Captured once, replayed while lengths, tokens and trees change in place."""
    from paper_2607_28418_b200 import binding
    layer = Layer(ctx, 21)
    table = places(2, 16, 22)
    caches = [binding.Cache.empty(32, HK, DIM, GROUP, PAGE) for _ in range(2)]
    for c in caches:
        c.pages.zero_()
        fill(ctx, layer, c, table, [100, 40], 23)
    x = torch.randn((9, HIDDEN), device="cuda").bfloat16()
    starts = torch.tensor([0, 5, 9], dtype=torch.int32, device="cuda")
    lens = torch.tensor([105, 44], dtype=torch.int32, device="cuda")
    seqs = binding.Sequences(table, lens, starts)
    pos = torch.tensor([100, 101, 101, 102, 102, 40, 41, 41, 42], dtype=torch.int32, device="cuda")
    tree = torch.cat([binding.tree_ancestors([-1, 0, 0, 1, 2], 1), binding.tree_ancestors([-1, 0, 0, 2], 1)]).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        layer.step(caches[0], seqs, x, pos, tree)
        with torch.cuda.graph(graph, stream=side):
            out = layer.step(caches[0], seqs, x, pos, tree)
    torch.cuda.synchronize()
    for turn in range(3):
        x.mul_(-0.9)
        lens.add_(turn)
        pos.add_(turn)
        tree.copy_(torch.cat([binding.tree_ancestors([-1, 0, 1, 2, turn], 1), binding.tree_ancestors([-1, -1, 0, 1], 1)]))
        graph.replay()
        torch.cuda.synchronize()
        ref = layer.step(caches[1], seqs, x, pos, tree)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        assert torch.equal(caches[0].pages, caches[1].pages)


def test_what_the_binding_refuses(ctx):
    from paper_2607_28418_b200 import binding
    layer = Layer(ctx, 31)
    x = torch.randn((4, HIDDEN), device="cuda").bfloat16()
    table = places(1, 4, 32)
    cache = binding.Cache.empty(4, HK, DIM, GROUP, PAGE)
    seqs = binding.Sequences(table, torch.tensor([4], dtype=torch.int32, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda"))
    q, k, v = layer.project(x)
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    bits = binding.tree_ancestors([-1, 0, 1, 2]).cuda()
    lin, app, tree = binding.wide_linear, binding.wide_cache_append, binding.wide_attn_tree
    bad = [
        lambda: lin(ctx, x, layer.w[:, :64]), lambda: lin(ctx, x.float(), layer.w), lambda: lin(ctx, x.t(), layer.w), lambda: lin(ctx, x, layer.w, activation="tanh"),
        lambda: lin(ctx, x, layer.w, bias=layer.b[:8]), lambda: lin(ctx, x, layer.w, bias=layer.b.float()), lambda: lin(ctx, x, layer.w, bias=layer.b.cpu()),
        lambda: lin(ctx, x, layer.w, residual=x), lambda: lin(ctx, x, layer.wo.t()[:HIDDEN]), lambda: lin(ctx, x, layer.w, y=q), lambda: lin(ctx, x, layer.w, out_dtype=torch.float16),
        lambda: app(ctx, cache, seqs, q, k, v.float(), pos, layer.inv), lambda: app(ctx, cache, seqs, q[:3], k, v, pos, layer.inv),
        lambda: app(ctx, cache, seqs, q, k, v, pos[:3], layer.inv), lambda: app(ctx, cache, seqs, q, k, v, pos.long(), layer.inv),
        lambda: app(ctx, cache, seqs, q, k, v, pos, layer.inv.float()), lambda: app(ctx, cache, seqs, None, k, v, pos, layer.inv, q_out=q),
        lambda: app(ctx, cache, seqs, q, k, v, pos, layer.inv, q_out=q[:, :64]), lambda: app(ctx, cache, seqs, q, k[:, :64], v[:, :64], pos, layer.inv),
        lambda: app(ctx, cache, seqs, q, k, v, pos, layer.inv, axis=pos), lambda: app(ctx, cache, seqs, q, k, v, pos.cpu(), layer.inv),
        lambda: tree(ctx, q, cache, seqs, HQ, 4, bits[:3]), lambda: tree(ctx, q, cache, seqs, HQ, 4, bits.long()), lambda: tree(ctx, q, cache, seqs, HQ, 4, bits.cpu()),
        lambda: tree(ctx, q, cache, seqs, HQ, 4, bits, mask_bits=bits[:2]), lambda: tree(ctx, q[:, :128], cache, seqs, HQ, 4, bits),
        lambda: tree(ctx, q, cache, seqs, HQ, 4, bits, o=torch.empty_like(q.contiguous()).float()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was let through")
    for call in (lambda: lin(ctx, x[:, :60].contiguous(), layer.w[:, :60].contiguous()), lambda: tree(ctx, q, cache, seqs, HQ, 3, bits),
                 lambda: tree(ctx, q, cache, seqs, HQ, 4, bits, workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
                 lambda: lin(ctx, x, layer.w, y=layer.w[:4, :8].reshape(-1)[:0].new_empty((4, layer.w.shape[0] + 4))[:, :-4])):
        with pytest.raises(binding.WideError):
            call()
    assert ctx.status() == 0
