"""wide_attn_cache against the 64-bit oracle over the values the cache holds."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from tests.cache_util import CacheCase, pack_bits, to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


def queries(c, hq, seed, amplitude=1.0):
    rng = np.random.default_rng(seed)
    return co.round_bf16(rng.standard_normal((c.rows, hq, c.dim)) * amplitude)


def reference(c, q, on, per, causal=True, scale=0.0, held=None, lost=None):
    """(reference, tolerance) [rows, hq, dim]."""
    scale = scale if scale > 0 else c.dim ** -0.5
    ref, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s, n in enumerate(c.news):
        a = slice(c.row_start[s], c.row_start[s] + n)
        if n == 0 or c.lens[s] == 0:
            continue
        k, v = held[s] if held else c.held(s)
        ref[a] = co.attention(q[a], k, v, on[a], per, causal, scale, lost[s] if lost else ())
        tol[a] = co.attention_tolerance(ref[a], q[a], k, v, scale)
    return ref, tol


def check(got, ref, tol, what=""):
    got = got.float().cpu().numpy().reshape(ref.shape).astype(np.float64)
    assert np.isfinite(got).all(), what
    off = np.abs(got - ref) - tol
    assert (off <= 0).all(), f"{what}: off by {np.abs(got - ref).max():.3e}, {off.max():.3e} over the tolerance, at {np.unravel_index(off.argmax(), off.shape)}"
    assert (got[ref == 0] == 0).all(), what      # inactive pairs and empty rows are exact zeros


def run(ctx, c, q, on, per, row_start=True, **kw):
    from paper_2607_28418_b200 import binding
    bits = None if on is None else torch.from_numpy(pack_bits(on)).cuda()
    return binding.wide_attn_cache(ctx, to_device(q.reshape(c.rows, -1)), c.cache(c.full_pages()), c.seqs(row_start), q.shape[1], per,
                                   mask_bits=bits, **kw)


SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("heads,share", [(3, 1), (2, 4), (1, 8), (2, 5), (1, 16)])
def test_one_new_row(ctx, dim, group, heads, share):
    lens = [1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 127, 128, 129, 300]
    c = CacheCase(lens, [1] * len(lens), heads, dim, group, 16, seed=share + dim)
    hq = heads * share
    q = queries(c, hq, 1)
    on = np.random.default_rng(2).random((c.rows, heads)) < 0.7
    ref, tol = reference(c, q, on, share)
    check(run(ctx, c, q, on, share, row_start=False), ref, tol)
    check(run(ctx, c, q, on, share), ref, tol)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_several_new_rows_and_pages(ctx, page, causal):
    c = CacheCase([5, 200, 67, 33, 1, 90, 0, 257], [5, 3, 7, 0, 1, 17, 0, 2], 2, 128, 64, page, seed=page)
    q = queries(c, 8, 3)
    on = np.random.default_rng(4).random((c.rows, 4)) < 0.5     # two groups of two heads on a KV head
    ref, tol = reference(c, q, on, 2, causal)
    check(run(ctx, c, q, on, 2, causal=causal), ref, tol)
    ref, tol = reference(c, q, np.ones_like(on), 2, causal)
    check(run(ctx, c, q, None, 2, causal=causal), ref, tol)


@pytest.mark.parametrize("dim,group", SHAPES)
def test_long_chunks(ctx, dim, group):
    """More rows than one pass over a KV head takes, starting inside the sequence and at its beginning."""
    c = CacheCase([120, 77], [45, 77], 2, dim, group, 32, seed=5)
    q = queries(c, 6, 6)
    on = np.random.default_rng(7).random((c.rows, 2)) < 0.6
    ref, tol = reference(c, q, on, 3)
    check(run(ctx, c, q, on, 3), ref, tol)


@pytest.mark.parametrize("share", [1, 4])
def test_long_sequences_are_split_and_joined(ctx, share):
    c = CacheCase([5000, 3, 1777], [1, 1, 1], 2, 128, 64, 64, seed=8)
    q = queries(c, 2 * share, 9)
    on = np.array([[True, True], [False, True], [True, False]])
    ref, tol = reference(c, q, on, share)
    got = run(ctx, c, q, on, share)
    check(got, ref, tol)
    for _ in range(3):
        assert torch.equal(run(ctx, c, q, on, share), got)      # the same bits in every run


@pytest.mark.parametrize("seqs", [1, 40, 300])
def test_batches_of_any_size(ctx, seqs):
    rng = np.random.default_rng(seqs)
    lens = rng.integers(1, 60, seqs).tolist()
    c = CacheCase(lens, [1] * seqs, 5, 64, 64, 16, seed=10)
    q = queries(c, 5, 11)
    on = rng.random((seqs, 5)) < 0.5
    on[0] = False
    ref, tol = reference(c, q, on, 1)
    check(run(ctx, c, q, on, 1, row_start=False), ref, tol)


@pytest.mark.parametrize("share", [9, 12, 16, 17, 24, 25, 40])
@pytest.mark.parametrize("dim,group", [(64, 32), (128, 128)])
def test_many_query_heads_on_a_kv_head(ctx, share, dim, group):
    """Row counts on both sides of what one pass holds (8, 16, 24)."""
    c = CacheCase([70, 1, 33], [1, 1, 1], 2, dim, group, 16, seed=share)
    q = queries(c, 2 * share, 1)
    on = np.random.default_rng(2).random((c.rows, 2)) < 0.7
    ref, tol = reference(c, q, on, share)
    check(run(ctx, c, q, on, share, row_start=False), ref, tol)
    check(run(ctx, c, q, on, share), ref, tol)


@pytest.mark.parametrize("longest", [1535, 1536, 1537, 1600])
@pytest.mark.parametrize("seqs", [36, 37, 38, 75])
def test_around_one_item_a_cta(ctx, longest, seqs):
    """Few short items get a CTA each; one block or one item more, and they are cut evenly."""
    lens = [longest] + [1 + 7 * i % 40 for i in range(seqs - 1)]
    c = CacheCase(lens, [1] * seqs, 4, 64, 64, 16, seed=seqs)
    q = queries(c, 4, 3)
    ref, tol = reference(c, q, np.ones((seqs, 4), bool), 1)
    check(run(ctx, c, q, None, 1, row_start=False), ref, tol)


def test_more_sequences_than_the_plan_has_room_for(ctx):
    """The plan goes to the workspace; some sequences are empty, some have several new rows."""
    rng = np.random.default_rng(40)
    seqs = 1500
    lens = rng.integers(0, 25, seqs)
    news = np.minimum(lens, rng.integers(0, 4, seqs))
    c = CacheCase(lens.tolist(), news.tolist(), 3, 64, 32, 16, seed=41)
    q = queries(c, 6, 42)
    on = rng.random((c.rows, 3)) < 0.5
    ref, tol = reference(c, q, on, 2)
    check(run(ctx, c, q, on, 2), ref, tol)


def test_chunk_whose_rows_leave_a_head_unused(ctx):
    """More new rows than are looked at for unused heads: the head's rows are zeros all the same."""
    c = CacheCase([60], [25], 2, 64, 64, 16, seed=43)
    q = queries(c, 4, 44)
    on = np.zeros((25, 2), bool)
    on[:, 0] = np.arange(25) % 3 > 0
    check(run(ctx, c, q, on, 2), *reference(c, q, on, 2))
    on[:] = False
    got = run(ctx, c, q, on, 2)
    assert (got == 0).all()


def test_workspace_needs_no_initial_value(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([3000, 5, 700], [1, 2, 1], 2, 128, 64, 64, seed=45)
    q = queries(c, 4, 46)
    on = np.ones((c.rows, 2), bool)
    ref, tol = reference(c, q, on, 2)
    for fill in (0x00, 0xFF, 0x01):
        ws = torch.full((binding.attn_cache_workspace_bytes(c.rows, 4, 2, 128),), fill, dtype=torch.uint8, device="cuda")
        check(run(ctx, c, q, on, 2, workspace=ws), ref, tol)


def test_long_flat_average_keeps_its_digits(ctx):
    """131072 keys of nearly equal weight: the average is some 300 times smaller than the values, whose 4-bit parts
    cancel.  Rounding the output to bf16 is off by at most 2^-8 of each element, hence of the norm; the bound leaves half
    as much again for everything else."""
    from paper_2607_28418_b200 import binding
    n, dim = 131072, 128
    g = torch.Generator(device="cuda").manual_seed(47)
    k = torch.randn((n, dim), generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn((n, dim), generator=g, device="cuda").to(torch.bfloat16)
    cache = binding.Cache.empty(n // 64, 1, dim, 128, 64)
    seqs = binding.Sequences(torch.arange(n // 64, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda"),
                             torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    binding.wide_cache_write(ctx, cache, seqs, k, v)
    kd, vd = binding.wide_cache_read(ctx, cache, seqs, n, dtype=torch.float32)
    one = binding.Sequences(seqs.page_table, seqs.kv_lens)
    q = (torch.randn((1, 4 * dim), generator=g, device="cuda") * 0.3).to(torch.bfloat16)
    got = binding.wide_attn_cache(ctx, q, cache, one, 4, 4).double().view(4, dim)
    p = torch.softmax(q.double().view(4, dim) @ kd.double().t() / dim ** 0.5, -1)
    ref = p @ vd.double()
    assert (got - ref).norm() <= 1.5 * 2.0 ** -8 * ref.norm(), ((got - ref).norm() / ref.norm()).item()


def test_many_groups_and_heads_that_span_groups(ctx):
    """40 groups (two mask words) of one head, and a group that covers heads of two KV heads."""
    c = CacheCase([50, 81, 7], [1, 2, 1], 20, 64, 32, 16, seed=12)
    q = queries(c, 40, 13)
    on = np.random.default_rng(14).random((c.rows, 40)) < 0.3
    check(run(ctx, c, q, on, 1), *reference(c, q, on, 1))
    on = np.random.default_rng(15).random((c.rows, 10)) < 0.5
    check(run(ctx, c, q, on, 4), *reference(c, q, on, 4))


def test_sharp_and_flat_softmax(ctx):
    c = CacheCase([700, 700], [1, 1], 2, 128, 64, 16, seed=16, scale_k=3.0)
    on = np.ones((2, 2), bool)
    q = queries(c, 8, 17, amplitude=8.0)       # logits in the hundreds: one key takes all
    check(run(ctx, c, q, on, 4), *reference(c, q, on, 4), "sharp")
    q = queries(c, 8, 18) * 0.0                # every key the same
    check(run(ctx, c, q, on, 4), *reference(c, q, on, 4), "flat")
    q = queries(c, 8, 19)
    check(run(ctx, c, q, on, 4, scale=0.3), *reference(c, q, on, 4, scale=0.3), "scale")


@pytest.mark.parametrize("scale_v", [1e-30, 1e-6, 1e5, 1e30])
def test_magnitudes_of_values(ctx, scale_v):
    """Values far outside fp16; one sequence whose steps differ by many orders between tokens."""
    c = CacheCase([90, 200], [1, 3], 2, 128, 32, 16, seed=20)
    c.v[0] = co.round_bf16(c.v[0] * scale_v)
    c.v[1] = co.round_bf16(c.v[1] * np.exp2(np.random.default_rng(21).integers(-12, 13, (200, 1, 1))) * scale_v)
    q = queries(c, 4, 22)
    on = np.ones((c.rows, 2), bool)
    check(run(ctx, c, q, on, 2), *reference(c, q, on, 2))


def test_small_and_large_queries(ctx):
    """Query rows of one call whose magnitudes differ by 2^40; keys shrunk and grown to match."""
    c = CacheCase([60, 60], [2, 2], 2, 64, 64, 16, seed=23)
    q = queries(c, 4, 24)
    mag = np.exp2([[[-20.0]], [[0.0]], [[20.0]], [[3.0]]])
    q = co.round_bf16(q * mag)
    c.k[0] = co.round_bf16(c.k[0])
    on = np.ones((c.rows, 2), bool)
    for row, factor in ((0, 2.0 ** 20), (2, 2.0 ** -20)):
        one = np.zeros_like(on)
        one[row] = True
        s = row // 2
        keep = c.k[s]
        c.k[s] = co.round_bf16(keep * factor)
        check(run(ctx, c, q, one, 2), *reference(c, q, one, 2), f"row {row}")
        c.k[s] = keep


def test_garbage_behind_the_last_position_and_behind_the_mask(ctx):
    """Infinities and NaN in positions nobody sees: behind the end, after the row (causal), on pages of others."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([21, 40], [1, 4], 2, 128, 64, 16, seed=25)
    pages = np.full_like(c.garbage, 0xFF)      # codes 15, scale and minimum NaN
    for s in range(2):
        co.store(pages, 16, 64, c.table[s], c.lens[s], c.k[s], c.v[s])
    q = queries(c, 4, 26)
    on = np.ones((c.rows, 2), bool)
    held = [c.held(0), c.held(1)]
    ref, tol = reference(c, q, on, 2, held=held)
    args = (to_device(q.reshape(c.rows, -1)), c.cache(pages), c.seqs(), 4, 2)
    check(binding.wide_attn_cache(ctx, *args), ref, tol)
    # the last two positions of sequence 1 are NaN: the rows before them must not notice
    bad = c.k[1].copy()
    bad[38:] = np.nan
    badv = c.v[1].copy()
    badv[38:] = np.inf
    co.store(pages, 16, 64, c.table[1], 40, bad, badv)
    got = binding.wide_attn_cache(ctx, to_device(q.reshape(c.rows, -1)), c.cache(pages), c.seqs(), 4, 2)
    check(got[:3], ref[:3], tol[:3])
    assert torch.isnan(got[3:].float()).all()


def test_nan_queries_stay_in_their_rows(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([70], [3], 2, 64, 64, 16, seed=27)
    q = queries(c, 8, 28)
    on = np.ones((3, 2), bool)
    ref, tol = reference(c, q, on, 4)
    q[1, 2, 5] = np.nan
    q[2, 6, :] = np.inf
    got = run(ctx, c, q, on, 4).float().cpu().numpy().reshape(3, 8, 64)
    assert np.isnan(got[1, 2]).all() and np.isnan(got[2, 6]).all()
    got[1, 2], got[2, 6] = ref[1, 2], ref[2, 6]
    check(torch.from_numpy(got), ref, tol)


def test_strided_queries_and_rows_behind_the_last_sequence(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([30, 18], [2, 1], 2, 128, 64, 16, seed=29)
    q = queries(c, 4, 30)
    fused = torch.full((c.rows + 3, 1024), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:c.rows, 256:768] = to_device(q.reshape(c.rows, -1))
    on = np.ones((c.rows + 3, 2), bool)
    o = torch.full((c.rows + 3, 512), 5.0, dtype=torch.bfloat16, device="cuda")
    binding.wide_attn_cache(ctx, fused[:, 256:768], c.cache(c.full_pages()), c.seqs(), 4, 2,
                            mask_bits=torch.from_numpy(pack_bits(on)).cuda(), o=o)
    check(o[:c.rows], *reference(c, q, on, 2))
    assert (o[c.rows:] == 5).all()


def test_lengths_at_the_end_of_the_integers(ctx):
    """A length that cannot be rounded up to whole blocks is left out and reported; its row is zero, its neighbour's is not."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([40, 200], [1, 1], 2, 64, 64, 256, seed=35)
    q = queries(c, 4, 36)
    table = torch.full((2, 1 << 23), int(c.table[0, 0]), dtype=torch.int32, device="cuda")    # 2^31 positions
    table[1, 0] = int(c.table[1, 0])
    seqs = binding.Sequences(table, torch.tensor([2 ** 31 - 1, 200], dtype=torch.int32, device="cuda"))
    ref, tol = reference(c, q, np.ones((2, 2), bool), 2)
    ref[0], tol[0] = 0, 0
    cache = c.cache(c.full_pages())
    o = torch.full((2, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    binding.wide_attn_cache(ctx, to_device(q.reshape(2, -1)), cache, seqs, 4, 2, o=o)
    assert ctx.status() == binding.ERR_BAD_INDEX
    check(o, ref, tol)
    before = cache.pages.cpu().numpy()
    one = torch.ones((2, 128), dtype=torch.bfloat16, device="cuda")
    binding.wide_cache_write(ctx, cache, binding.Sequences(table[:1], seqs.kv_lens[:1]), one[:1], one[:1])
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert np.array_equal(cache.pages.cpu().numpy(), before)


def test_indices_out_of_range(ctx):
    """Keys on pages that are none are seen by nobody; sequences with a bad length give zeros; all is reported."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([40, 40, 40, 16], [1, 2, 1, 1], 2, 64, 64, 16, seed=31)
    q = queries(c, 4, 32)
    on = np.ones((c.rows, 2), bool)
    seqs = c.seqs()
    seqs.page_table[1, 1] = 1 << 30
    seqs.kv_lens[2] = 1000
    seqs.page_table[3, 0] = -1
    ref, tol = reference(c, q, on, 2, lost=[(), range(16, 32), (), range(16)])
    ref[3], tol[3] = 0, 0
    got = binding.wide_attn_cache(ctx, to_device(q.reshape(c.rows, -1)), c.cache(c.full_pages()), seqs, 4, 2)
    assert ctx.status() == binding.ERR_BAD_INDEX
    check(got, ref, tol)
    # rows that are no range: left as they were
    seqs = c.seqs()
    seqs.row_start[:] = torch.tensor([0, 1, 3, 2, 100], dtype=torch.int32)
    o = torch.full((c.rows, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    binding.wide_attn_cache(ctx, to_device(q.reshape(c.rows, -1)), c.cache(c.full_pages()), seqs, 4, 2, o=o)
    assert ctx.status() == binding.ERR_BAD_INDEX
    ref, tol = reference(c, q, on, 2)
    check(o[:3], ref[:3], tol[:3])
    assert (o[3:] == 5).all()


def test_shared_pages(ctx):
    """Two sequences with a common beginning on the same pages."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([50, 50], [1, 1], 2, 128, 128, 16, seed=33)
    c.k[1][:32], c.v[1][:32] = c.k[0][:32], c.v[0][:32]
    pages = c.full_pages()
    seqs = c.seqs()
    seqs.page_table[1, :2] = seqs.page_table[0, :2]
    q = queries(c, 4, 34)
    on = np.ones((2, 2), bool)
    check(binding.wide_attn_cache(ctx, to_device(q.reshape(2, -1)), c.cache(pages), seqs, 4, 2), *reference(c, q, on, 2))


def test_cache_beyond_four_gigabytes(ctx):
    from paper_2607_28418_b200 import binding
    size = binding.cache_page_bytes(256, 2, 128, 64)
    n_pages = (5 << 30) // size + 1
    c = CacheCase([400], [1], 2, 128, 64, 256, seed=35)
    small = c.full_pages()
    cache = binding.Cache.empty(n_pages, 2, 128, 64, 256)
    table = torch.tensor([[n_pages - 1, n_pages - 5]], dtype=torch.int32, device="cuda")
    for i in range(2):
        cache.pages[table[0, i].item()] = torch.from_numpy(small[c.table[0, i]]).cuda().view(-1)
    seqs = binding.Sequences(table, torch.tensor([400], dtype=torch.int32, device="cuda"))
    q = queries(c, 8, 36)
    on = np.ones((1, 2), bool)
    check(binding.wide_attn_cache(ctx, to_device(q.reshape(1, -1)), cache, seqs, 8, 4), *reference(c, q, on, 4))


def test_captured_and_replayed_as_the_cache_grows(ctx):
    """One graph of store and attend, replayed with longer sequences than it was captured with; two graphs
    with a workspace each on two streams at once."""
    from paper_2607_28418_b200 import binding
    n, heads, dim = 6, 2, 64
    lens = [100, 3, 77, 1, 250, 40]
    c = CacheCase([x + 200 for x in lens], [1] * n, heads, dim, 64, 16, seed=37)
    cache = c.cache(c.full_pages())
    q = queries(c, 4, 38)
    qd, on = to_device(q.reshape(n, -1)), np.ones((n, heads), bool)
    graphs, outs, seqss = [], [], []
    for i in range(2):
        seqs = c.seqs(row_start=False)
        seqs.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        ws = torch.empty(binding.attn_cache_workspace_bytes(n, 4, heads, dim), dtype=torch.uint8, device="cuda")
        o = torch.empty((n, 4 * dim), dtype=torch.bfloat16, device="cuda")
        binding.wide_attn_cache(ctx, qd, cache, seqs, 4, 2, o=o, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.wide_attn_cache(ctx, qd, cache, seqs, 4, 2, o=o, workspace=ws)
        graphs.append((g, ws))
        outs.append(o)
        seqss.append(seqs)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for more in (0, 13, 200):
        for i in range(2):
            seqss[i].kv_lens.copy_(torch.tensor([x + more for x in lens], dtype=torch.int32))
        torch.cuda.synchronize()
        for _ in range(5):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i][0].replay()
        torch.cuda.synchronize()
        now = CacheCase.__new__(CacheCase)
        now.__dict__.update(c.__dict__)
        now.lens = [x + more for x in lens]
        now.k = [k[:m] for k, m in zip(c.k, now.lens)]
        now.v = [v[:m] for v, m in zip(c.v, now.lens)]
        ref, tol = reference(now, q, on, 2)
        for o in outs:
            check(o, ref, tol, f"{more} more")


def test_together_with_the_routed_layer(ctx):
    """rope -> store -> attention over the cache -> masked output projection, token by token, against
    wide_attn over the keys and values read back."""
    from paper_2607_28418_b200 import binding
    T, hq, hkv, dim, hidden = 80, 8, 2, 128, 256
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v = rand(T, hq * dim), rand(T, hkv * dim), rand(T, hkv * dim)
    w_o = (rand(hidden, hq * dim).float() * 0.03).to(torch.bfloat16)
    inv = torch.tensor([10000.0 ** (-i / 64) for i in range(64)], dtype=torch.float64, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    cache = binding.Cache.empty(8, hkv, dim, 64, 16)
    table = torch.tensor([[3, 1, 7, 0, 5]], dtype=torch.int32, device="cuda")
    on = np.random.default_rng(1).random((T, 2)) < 0.6
    bits = torch.from_numpy(pack_bits(on)).cuda()
    # the prompt in one call, the answer token by token
    step_o = torch.empty((T, hq * dim), dtype=torch.bfloat16, device="cuda")
    for a, b in [(0, 40)] + [(i, i + 1) for i in range(40, T)]:
        qr, kr = binding.wide_rope(ctx, q[a:b], k[a:b], pos[a:b].contiguous(), inv, head_dim=dim)
        seqs = binding.Sequences(table, torch.tensor([b], dtype=torch.int32, device="cuda"), torch.tensor([0, b - a], dtype=torch.int32, device="cuda"))
        binding.wide_cache_write(ctx, cache, seqs, kr, v[a:b])
        step_o[a:b] = binding.wide_attn_cache(ctx, qr, cache, seqs, hq, 4, mask_bits=bits[a:b].contiguous())
    seqs = binding.Sequences(table, torch.tensor([T], dtype=torch.int32, device="cuda"), torch.tensor([0, T], dtype=torch.int32, device="cuda"))
    kd, vd = binding.wide_cache_read(ctx, cache, seqs, T)
    qr, kr = binding.wide_rope(ctx, q, k, pos, inv, head_dim=dim)
    ref_k = co.round_bf16(co.held(kr.float().cpu().numpy().reshape(T, hkv, dim), 64).reshape(T, -1))
    assert np.array_equal(kd.float().cpu().numpy(), ref_k)
    meta = binding.wide_reorder(ctx, bits, 2, 128)
    dense = binding.wide_attn(ctx, qr, kd, vd, hq, hkv, 4, meta)
    # both are within their own tolerance of the same attention; wide_attn sees keys and values rounded to
    # bf16 (2^-8 of |k|, |v|) and rounds probabilities to bf16 (2^-8): 2e-2 of the largest value, as its own tests
    scale = dense.float().abs().max().item()
    assert (step_o.float() - dense.float()).abs().max().item() <= 2e-2 * scale
    y1 = binding.wide_oproj(ctx, step_o, w_o, 512, bits, meta, flags=binding.FLAG_INPUT_MASKED)
    y2 = binding.wide_oproj(ctx, dense, w_o, 512, bits, meta, flags=binding.FLAG_INPUT_MASKED)
    assert (y1.float() - y2.float()).abs().max().item() <= 4e-2 * y2.float().abs().max().item()


def test_binding_refuses(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([20], [1], 2, 64, 64, 16)
    cache, seqs, q = c.cache(c.full_pages()), c.seqs(), to_device(queries(c, 4, 1).reshape(1, -1))
    for bad in (dict(o=torch.empty((1, 256), device="cuda")), dict(o=torch.empty((2, 256), dtype=torch.bfloat16, device="cuda")),
                dict(mask_bits=torch.zeros((1, 2), dtype=torch.int32, device="cuda")), dict(mask_bits=torch.zeros((1, 1), device="cuda")),
                dict(workspace=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            binding.wide_attn_cache(ctx, q, cache, seqs, 4, 2, **bad)
    with pytest.raises(binding.WideError) as e:
        binding.wide_attn_cache(ctx, q, cache, seqs, 4, 2, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.ERR_WORKSPACE
    with pytest.raises(binding.WideError) as e:
        binding.wide_attn_cache(ctx, q.float(), cache, seqs, 4, 2)
    assert e.value.code == binding.ERR_UNSUPPORTED_SHAPE
    with pytest.raises(ValueError):
        binding.wide_attn_cache(ctx, q, cache, seqs, 8, 2)
    assert binding.wide_attn_cache(ctx, q[:0], cache, seqs, 4, 2).shape == (0, 256)
