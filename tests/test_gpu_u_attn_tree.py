"""wide_attn_tree against the softmax in 64 bits over the values that the cache holds."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from tests.cache_util import CacheCase, pack_bits, to_device

pytestmark = pytest.mark.gpu

SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


def random_trees(c, seed, words=None):
    """(tree_bits [rows, words], what each row sees of the new rows: a list of bool [n, n])."""
    from paper_2607_28418_b200 import binding
    rng = np.random.default_rng(seed)
    words = words or max(1, (max(c.news) + 31) // 32)
    bits, sees = [], []
    for n in c.news:
        parents = [int(rng.integers(-1, i)) if i else -1 for i in range(n)]
        b = binding.tree_ancestors(parents, words) if n else torch.zeros((0, words), dtype=torch.int32)
        bits.append(b)
        sees.append(seen_by(b.numpy(), n))
    return torch.cat(bits), sees


def seen_by(bits, n):
    j = np.arange(n)
    return ((bits.view(np.uint32)[:, j // 32] >> (j % 32).astype(np.uint32)) & 1).astype(bool).reshape(n, n)


def reference(c, q, on, per, sees, scale=0.0, missing=()):
    """(reference, tolerance) [rows, hq, dim], 64 bits.  A key's number is rounded to fp16, 2^-11 of itself and 2^-18 of the key's largest, a query's
    to 2^-16 of its row's largest, or, where some of the item's queries do not fit that type, keys to 2^-8; a logit sums dim / 16 steps of products
    in fp32 (2^-23 of their magnitudes a step, as does its scaling).  A probability is off by that, by the exponential (2^-21) and by its rounding
    to fp16 (2^-11, and 2^-32 of the largest), a value by 2^-11; both by 2^-8 in blocks whose values fp16 does not hold well.  An output adds
    len / 16 steps of weighed values; its own rounding is 2^-8.  missing: positions without a page."""
    dim, hq = c.dim, q.shape[1]
    share = hq // c.heads
    scale = scale if scale > 0 else dim ** -0.5
    ref, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s, n in enumerate(c.news):
        if n == 0 or c.lens[s] == 0:
            continue
        a = slice(c.row_start[s], c.row_start[s] + n)
        k, v = (torch.from_numpy(np.asarray(x, dtype=np.float64)).cuda() for x in c.held(s))
        z = torch.from_numpy(q[a].astype(np.float64)).cuda().view(n, c.heads, share, dim)
        logits = torch.einsum("mhsd,nhd->mhsn", z, k) * scale
        size = torch.einsum("mhsd,nhd->mhsn", z.abs(), k.abs()).amax(-1) * scale
        see = torch.ones((n, c.lens[s]), dtype=torch.bool)
        see[:, c.lens[s] - n:] = torch.from_numpy(sees[s])
        for lost in missing[s] if missing else ():
            see[:, lost] = False
        logits.masked_fill_(~see[:, None, None].cuda(), -torch.inf)
        p = torch.nan_to_num(torch.softmax(logits, -1), nan=0.0)
        o = torch.einsum("mhsn,nhd->mhsd", p, v)
        weighed = torch.einsum("mhsn,nhd->mhsd", p, v.abs())
        small = (z.abs().sum(-1) * k.abs().amax() * 2.0 ** -18 + z.abs().amax(-1) * k.abs().sum(-1).amax() * 2.0 ** -16) * scale
        tops = z.reshape(-1, 8).abs().amax(-1)
        fits = bool(((tops == 0) | (tops >= 2.0 ** -9) & (tops <= 2.0 ** 14)).all())
        parts = v.reshape(c.lens[s], c.heads, -1, c.group)
        low, high = parts.amin(-1), parts.amax(-1)
        narrow = bool((((high - low) / 15 >= 2.0 ** -12) & (torch.maximum(high, -low) <= 30000)).all())
        each = (2.0 ** -10 if narrow else 2.0 ** -7) + 2.0 ** -20 + 2 * (size * ((2.0 ** -11 if fits else 2.0 ** -8) + 2.0 ** -23 * (dim / 16 + 3)) + small)
        t = 2.0 ** -8 * o.abs() + weighed * (each[..., None] + 2.0 ** -23 * (c.lens[s] / 16 + 8)) + v.abs().amax() * c.lens[s] * 2.0 ** -32 + 1e-37
        live = np.ones((n, hq), dtype=bool) if on is None else np.repeat(on[a], per, axis=1)
        ref[a] = o.reshape(n, hq, dim).cpu().numpy() * live[..., None]
        tol[a] = t.reshape(n, hq, dim).cpu().numpy()
    return ref, tol


def run(ctx, c, q, on, per, bits, pages=None, **kw):
    from paper_2607_28418_b200 import binding
    mask = None if on is None else torch.from_numpy(pack_bits(on)).cuda()
    cache = c.cache(c.full_pages() if pages is None else pages)
    return binding.wide_attn_tree(ctx, to_device(q.reshape(c.rows, -1)), cache, c.seqs(), q.shape[1], per, bits.cuda(), mask_bits=mask, **kw)


def check(got, ref, tol):
    got = got.float().cpu().numpy().reshape(ref.shape).astype(np.float64)
    assert np.isfinite(got).all()
    off = np.abs(got - ref) - tol
    assert (off <= 0).all(), f"off by {np.abs(got - ref).max():.3e}, {off.max():.3e} over the tolerance, at {np.unravel_index(off.argmax(), off.shape)}"
    assert (got[ref == 0] == 0).all()


def queries(c, hq, seed, amplitude=1.0):
    return co.round_bf16(np.random.default_rng(seed).standard_normal((c.rows, hq, c.dim)) * amplitude)


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("lens,news", [([200], [8]), ([1], [1]), ([5], [5]), ([127, 128, 129, 300, 16], [16, 3, 1, 30, 16])])
def test_one_pass(ctx, dim, group, lens, news):
    c = CacheCase(lens, news, 2, dim, group, 32, seed=dim + group)
    q = queries(c, 2, 1)
    bits, sees = random_trees(c, 2)
    ref, tol = reference(c, q, None, 1, sees)
    check(run(ctx, c, q, None, 1, bits), ref, tol)


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("heads,share", [(3, 1), (2, 4), (1, 7), (2, 8), (1, 16)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_ragged_batches_and_routed_heads(ctx, dim, group, heads, share, page):
    c = CacheCase([61, 200, 67, 33, 1, 90, 0, 700, 513], [61, 3, 17, 0, 1, 64, 0, 40, 5], heads, dim, group, page, seed=share + dim + page)
    q = queries(c, heads * share, 3)
    on = np.random.default_rng(4).random((c.rows, heads)) < 0.6
    bits, sees = random_trees(c, 5)
    ref, tol = reference(c, q, on, share, sees)
    check(run(ctx, c, q, on, share, bits), ref, tol)


@pytest.mark.parametrize("new", [1, 2, 15, 31, 32, 33, 64, 100, 256])
@pytest.mark.parametrize("share", [1, 4])
def test_sizes_of_trees(ctx, new, share):
    c = CacheCase([300, new], [new, new], 2, 128, 64, 16, seed=new)
    q = queries(c, 2 * share, 6)
    bits, sees = random_trees(c, 7)
    ref, tol = reference(c, q, None, share, sees)
    check(run(ctx, c, q, None, share, bits), ref, tol)


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("lens", [[9000], [5000, 1, 3000], [2500] * 9])
def test_items_cut_between_ctas(ctx, dim, group, lens):
    c = CacheCase(lens, [min(n, 20) for n in lens], 2, dim, group, 64, seed=8)
    q = queries(c, 8, 9)
    bits, sees = random_trees(c, 10)
    ref, tol = reference(c, q, None, 4, sees)
    check(run(ctx, c, q, None, 4, bits), ref, tol)


@pytest.mark.parametrize("new", [9, 30])
def test_any_relation_and_rows_that_see_nothing(ctx, new):
    """Bits need not be a tree; a row without bits in a sequence without a prefix gives zeros; bits behind the last row mean nothing."""
    c = CacheCase([new, 150], [new, new], 2, 128, 64, 16, seed=11)
    q = queries(c, 8, 12)
    rng = np.random.default_rng(13)
    bits = torch.from_numpy(rng.integers(0, 2 ** 32, (c.rows, 2), dtype=np.uint64).astype(np.uint32).view(np.int32).copy())
    bits[0], bits[3], bits[new] = 0, 0, 0
    sees = [seen_by(bits[:new].numpy().copy(), new), seen_by(bits[new:].numpy().copy(), new)]
    ref, tol = reference(c, q, None, 4, sees)
    assert (ref[0] == 0).all() and (ref[3] == 0).all() and (ref[new] != 0).any()
    check(run(ctx, c, q, None, 4, bits), ref, tol)


@pytest.mark.parametrize("amplitude,scale", [(8.0, 0.0), (30.0, 0.0), (1.0, 2.0), (2.0 ** -20, 0.0), (1.0, 1e-4)])
def test_peaked_and_flat_softmaxes(ctx, amplitude, scale):
    c = CacheCase([1500, 700], [30, 12], 2, 128, 64, 64, seed=14, scale_k=2.0)
    q = queries(c, 8, 15, amplitude)
    bits, sees = random_trees(c, 16)
    ref, tol = reference(c, q, None, 4, sees, scale)
    check(run(ctx, c, q, None, 4, bits, scale=scale), ref, tol)


def test_logits_that_rise_from_tile_to_tile(ctx):
    """Every tile passes the reference of the one before: sums and outputs are scaled again and again."""
    c = CacheCase([2000], [24], 1, 128, 64, 64, seed=17)
    ramp = np.linspace(0, 60, 2000)[:, None, None]
    c.k = [co.round_bf16((np.ones((2000, 1, 128)) * ramp / 128 ** 0.5 + 0.1 * np.random.default_rng(1).standard_normal((2000, 1, 128))).astype(np.float32))]
    q = co.round_bf16(np.ones((c.rows, 4, 128), dtype=np.float32) * np.array([1, -1, 0.5, 2])[:, None].astype(np.float32))
    bits, sees = random_trees(c, 18)
    ref, tol = reference(c, q, None, 4, sees)
    check(run(ctx, c, q, None, 4, bits), ref, tol)


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_missing_numbers_stay_with_the_rows_that_see_them(ctx, dim, group, bad):
    c = CacheCase([150], [20], 2, dim, group, 32, seed=19)
    bits, sees = random_trees(c, 20)
    node, far = 4, 9
    c.v[0][130 + node, 0, dim - 1] = bad      # the last sub-group of head 0
    c.k[0][130 + far, 1, 0] = bad             # any channel: the logit
    q = queries(c, 4, 21)
    got = run(ctx, c, q, None, 2, bits).float().cpu().numpy().reshape(20, 4, dim)
    v_seen, k_seen = sees[0][:, node], sees[0][:, far]
    assert v_seen.any() and not v_seen.all() and k_seen.any() and not k_seen.all()
    assert np.isnan(got[v_seen][:, :2, dim - group:]).all() and np.isnan(got[k_seen][:, 2:]).all()
    if dim > group:
        assert np.isfinite(got[:, :2, :dim - group]).all()
    for hidden, heads in ((~v_seen, slice(0, 2)), (~k_seen, slice(2, 4))):
        assert np.isfinite(got[hidden][:, heads]).all()
    clean = CacheCase([150], [20], 2, dim, group, 32, seed=19)
    ref, tol = reference(clean, q, None, 2, sees)
    assert (np.abs(got - ref)[~v_seen][:, :2] <= tol[~v_seen][:, :2]).all()
    assert (np.abs(got - ref)[~k_seen][:, 2:] <= tol[~k_seen][:, 2:]).all()


def test_garbage_behind_the_end_is_not_read(ctx):
    """Positions behind the length, in the last block and in the page, hold bytes that decode to NaN and infinities."""
    c = CacheCase([37, 130], [9, 30], 2, 128, 64, 64, seed=22)
    c.garbage[:] = 0xFF
    q = queries(c, 8, 23)
    bits, sees = random_trees(c, 24)
    ref, tol = reference(c, q, None, 4, sees)
    check(run(ctx, c, q, None, 4, bits), ref, tol)


def test_bad_places(ctx):
    """A page out of range is not seen; a sequence that is left out, or has more rows than bits, gives zeros; rows of nobody stay."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([200, 90, 60, 80], [10, 10, 10, 40], 2, 128, 64, 32, seed=25)
    q = queries(c, 8, 26)
    bits, sees = random_trees(c, 27, words=1) if max(c.news) <= 32 else (None, None)
    if bits is None:
        rng = np.random.default_rng(27)
        bits = torch.from_numpy(rng.integers(0, 2 ** 31, (c.rows, 1)).astype(np.int32))
        sees = [seen_by(bits[c.row_start[s]:c.row_start[s + 1]].numpy().copy(), n) if n <= 32 else np.zeros((n, n), bool) for s, n in enumerate(c.news)]
    ref, tol = reference(c, q, None, 4, sees, missing=[range(32, 64), (), (), ()])
    table, lens = c.table.copy(), list(c.lens)
    table[0, 1] = c.n_pages
    lens[2] = 10 ** 6
    starts = c.row_start.copy()
    seqs = binding.Sequences(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), torch.from_numpy(starts).cuda())
    wide = torch.full((c.rows + 3, 8 * 128), 3.0, device="cuda").to(torch.bfloat16)
    qq = torch.cat([to_device(q.reshape(c.rows, -1)), wide[:3]])
    out = binding.wide_attn_tree(ctx, qq, c.cache(c.full_pages()), seqs, 8, 4, torch.cat([bits, bits[:3]]).cuda(), o=wide)
    assert ctx.status() == binding.ERR_BAD_INDEX and ctx.status() == 0
    assert (out[c.rows:] == 3).all()
    got = out[:c.rows].float().cpu().numpy().reshape(ref.shape)
    assert (got[20:] == 0).all()                       # sequence 2 is left out, sequence 3 has 40 rows and 32 bits
    assert (np.abs(got[:20] - ref[:20]) <= tol[:20]).all()


def test_many_sequences(ctx):
    """More than the plan holds in shared memory."""
    n = 1500
    c = CacheCase([20 + i % 40 for i in range(n)], [1 + i % 4 for i in range(n)], 1, 64, 64, 16, seed=28)
    q = queries(c, 2, 29)
    bits, sees = random_trees(c, 30)
    ref, tol = reference(c, q, None, 2, sees)
    check(run(ctx, c, q, None, 2, bits), ref, tol)


def test_a_chain_is_causal_attention(ctx):
    """Every node the child of the one before: wide_attn_cache, within what both leave to rounding."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([400, 90], [12, 6], 2, 128, 64, 64, seed=31)
    q = queries(c, 8, 32)
    bits = torch.cat([binding.tree_ancestors(list(range(-1, n - 1)), 1) for n in c.news])
    sees = [np.tril(np.ones((n, n), dtype=bool)) for n in c.news]
    _, tol = reference(c, q, None, 4, sees)
    tree = run(ctx, c, q, None, 4, bits).float().cpu().numpy().reshape(tol.shape)
    chain = binding.wide_attn_cache(ctx, to_device(q.reshape(c.rows, -1)), c.cache(c.full_pages()), c.seqs(), 8, 4).float().cpu().numpy().reshape(tol.shape)
    assert (np.abs(tree - chain) <= 3 * tol).all()


def test_same_bits_replayed_on_another_stream_with_a_workspace(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([3000, 77, 500], [30, 20, 9], 2, 128, 128, 64, seed=33)
    q = to_device(queries(c, 8, 34).reshape(c.rows, -1))
    bits = random_trees(c, 35)[0].cuda()
    cache, seqs = c.cache(c.full_pages()), c.seqs()
    ref = binding.wide_attn_tree(ctx, q, cache, seqs, 8, 4, bits)
    ws = torch.empty(binding.attn_tree_workspace_bytes(), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty_like(ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            binding.wide_attn_tree(ctx, q, cache, seqs, 8, 4, bits, o=out, workspace=ws)
    for _ in range(4):
        out.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


def test_strided_queries_and_nothing_to_do(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([100], [12], 2, 64, 64, 16, seed=36)
    q = to_device(queries(c, 4, 37).reshape(c.rows, -1))
    bits = random_trees(c, 38)[0].cuda()
    cache, seqs = c.cache(c.full_pages()), c.seqs()
    fused = torch.randn((c.rows, 512), device="cuda").to(torch.bfloat16)
    fused[:, 128:384] = q
    assert torch.equal(binding.wide_attn_tree(ctx, fused[:, 128:384], cache, seqs, 4, 2, bits), binding.wide_attn_tree(ctx, q, cache, seqs, 4, 2, bits))
    assert binding.wide_attn_tree(ctx, q[:0], cache, seqs, 4, 2, bits[:0]).shape == (0, 256)


@pytest.mark.parametrize("dim,group", SHAPES)
def test_how_near_it_comes(ctx, dim, group):
    """On ordinary values the root mean square of all errors together is hardly more than that of the output's rounding to bf16 (at most 2^-9 / sqrt(3)
    of a number in [1, 2) and half that below the next power: 0.41 to 0.85 of 2^-9).  What else there is adds in squares: probabilities and values
    2^-12 each, keys 2^-12 a logit of size 1."""
    c = CacheCase([700, 90], [24, 8], 2, dim, group, 32, seed=3)
    q = queries(c, 8, 4)
    bits, sees = random_trees(c, 5)
    ref, _ = reference(c, q, None, 4, sees)
    got = run(ctx, c, q, None, 4, bits).float().cpu().numpy().reshape(ref.shape)
    assert np.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum()) < 2.0 ** -9


@pytest.mark.parametrize("scale_q,scale_k,scale_v", [(2.0 ** -40, 2.0 ** 40, 1.0), (2.0 ** 30, 2.0 ** -30, 2.0 ** -30), (1.0, 1.0, 2.0 ** 60), (2.0 ** 100, 2.0 ** -100, 2.0 ** -100), (2.0 ** -7, 2.0 ** 7, 2.0 ** -9)])
def test_sizes_that_fp16_does_not_hold(ctx, scale_q, scale_k, scale_v):
    """Queries, keys and values of any size, each alone and rows of different sizes together: only their products have to be sensible."""
    c = CacheCase([300, 40, 150], [20, 8, 3], 2, 128, 64, 32, seed=6)
    c.k = [co.round_bf16(x * np.float32(scale_k)) for x in c.k]
    c.v = [co.round_bf16(x * np.float32(scale_v)) for x in c.v]
    q = queries(c, 8, 7) * np.float32(scale_q)
    q[::3] *= 2.0 ** -12
    q[5] = 0
    bits, sees = random_trees(c, 8)
    ref, tol = reference(c, q, None, 4, sees)
    check(run(ctx, c, q, None, 4, bits), ref, tol)


def test_values_of_both_kinds_in_a_tile(ctx):
    """A tile with blocks of ordinary values, of tiny and of large ones, in turn; a row's output is the sum of all."""
    c = CacheCase([520], [12], 2, 128, 32, 32, seed=9)
    factor = np.repeat(np.array([1.0, 2.0 ** -20, 2.0 ** 17, 1.0, 2.0 ** -14], dtype=np.float32), 16)
    c.v = [co.round_bf16(x * np.resize(factor, len(x))[:, None, None]) for x in c.v]
    q = queries(c, 8, 10)
    bits, sees = random_trees(c, 11)
    ref, tol = reference(c, q, None, 4, sees)
    check(run(ctx, c, q, None, 4, bits), ref, tol)


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("new", [12, 40])
def test_keys_of_many_sizes(ctx, dim, group, new):
    """Keys that fp16 does not hold as they are, each with a power of two of its own, beside ordinary ones and zeros; queries that fit."""
    c = CacheCase([530, 77], [new, 5], 2, dim, group, 32, seed=12)
    factor = np.array([1.0, 2.0 ** -14, 0.0, 2.0 ** -40, 2.0 ** 4, 2.0 ** -9, 2.0 ** -100], dtype=np.float32)
    c.k = [co.round_bf16(x * np.resize(factor, len(x))[:, None, None]) for x in c.k]
    q = queries(c, 8, 13)
    bits, sees = random_trees(c, 14)
    ref, tol = reference(c, q, None, 4, sees)
    check(run(ctx, c, q, None, 4, bits), ref, tol)


def test_calls_on_two_streams(ctx):
    """Trees of two streams at once, each with a workspace of its own, beside a linear layer: the bits of each call alone."""
    from paper_2607_28418_b200 import binding
    cases = [CacheCase([3000, 900], [30, 7], 4, 128, 64, 32, seed=21), CacheCase([700] * 12, [9] * 12, 4, 128, 64, 32, seed=22)]
    x, w = torch.randn((40, 4096), device="cuda").bfloat16(), torch.randn((4096, 4096), device="cuda").bfloat16()
    y = binding.wide_linear(ctx, x, w)
    sets = []
    for i, c in enumerate(cases):
        q = to_device(queries(c, 16, 23 + i).reshape(c.rows, -1))
        bits, _ = random_trees(c, 25 + i)
        args = (ctx, q, c.cache(c.full_pages()), c.seqs(), 16, 4, bits.cuda())
        work = torch.empty(binding.attn_tree_workspace_bytes(), dtype=torch.uint8, device="cuda")
        sets.append((args, work, binding.wide_attn_tree(*args), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for args, work, _, stream in sets:
            with torch.cuda.stream(stream):
                got.append((binding.wide_attn_tree(*args, workspace=work), binding.wide_linear(ctx, x, w)))
        torch.cuda.synchronize()
        for (o, z), (_, _, alone, _) in zip(got, sets):
            assert torch.equal(o, alone) and torch.equal(z, y)
