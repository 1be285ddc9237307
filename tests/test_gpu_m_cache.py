"""The 4-bit cache on the GPU: bytes written and values read back, bit for bit against the oracle."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from tests.cache_util import CacheCase, to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


def written(ctx, c, row_start=True):
    from paper_2607_28418_b200 import binding
    cache = c.cache(c.garbage.copy())
    binding.wide_cache_write(ctx, cache, c.seqs(row_start), to_device(c.new("k"), c.dtype), to_device(c.new("v"), c.dtype))
    return cache


def expected_pages(c):
    pages = c.garbage.copy()
    for s, n in enumerate(c.news):
        if n:
            co.store(pages, c.page, c.group, c.table[s], c.lens[s], c.k[s][c.lens[s] - n:], c.v[s][c.lens[s] - n:])
    return pages


SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64])
def test_write_is_the_oracle_byte_for_byte(ctx, dim, group, dtype, page):
    # one token, a whole block, starts and ends inside blocks and pages, no new rows, all rows new
    c = CacheCase([1, 16, 37, 70, 5, 0, 131, 33], [1, 16, 20, 1, 0, 0, 131, 15], 3, dim, group, page, seed=dim + group + page, dtype=dtype)
    cache = written(ctx, c)
    assert np.array_equal(cache.pages.cpu().numpy(), expected_pages(c))


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("page", [32, 128, 256])
def test_one_row_a_sequence_without_row_start(ctx, dim, group, page):
    lens = list(range(1, 40)) + [200, 256, 257]
    c = CacheCase(lens, [1] * len(lens), 2, dim, group, page, seed=page)
    cache = written(ctx, c, row_start=False)
    assert np.array_equal(cache.pages.cpu().numpy(), expected_pages(c))


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_read_is_the_oracle_value_for_value(ctx, dim, group, dtype):
    from paper_2607_28418_b200 import binding
    c = CacheCase([1, 16, 37, 70, 5, 0, 131, 33], [1, 16, 20, 1, 0, 0, 131, 15], 3, dim, group, 32, seed=1, dtype=dtype)
    k, v = binding.wide_cache_read(ctx, c.cache(c.full_pages()), c.seqs(), c.rows, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    for got, which in ((k, "k"), (v, "v")):
        ref = co.held(c.new(which).reshape(c.rows, c.heads, dim), group).reshape(c.rows, -1)
        ref = co.round_bf16(ref) if dtype == "bf16" else ref
        assert np.array_equal(got.float().cpu().numpy(), ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_values_near_borders(ctx, dtype):
    """Whole multiples of half a step, and their neighbours: a rounding in the wrong place changes a code."""
    rng = np.random.default_rng(5)
    n, dim = 512, 128
    x = (rng.integers(0, 31, (n, 1, dim)) / 2.0 * np.exp2(rng.integers(-3, 4, (n, 1, 1)))).astype(np.float32) + rng.integers(-8, 9, (n, 1, 1)).astype(np.float32)
    x = co.round_bf16(x)
    if dtype == "f32":
        x = np.nextafter(x, np.where(rng.random(x.shape) < 0.5, -np.inf, np.inf).astype(np.float32), dtype=np.float32)
    c = CacheCase([n], [n], 1, dim, 64, 64, dtype=dtype)
    c.k, c.v = [x], [x[::-1].copy()]
    assert np.array_equal(written(ctx, c).pages.cpu().numpy(), expected_pages(c))


def test_extreme_magnitudes_and_non_finite_values(ctx):
    rng = np.random.default_rng(6)
    n, dim = 96, 64
    x = rng.standard_normal((n, 2, dim)).astype(np.float32)
    x[0:16] *= np.float32(8e37)
    x[16, 0, :] = np.where(np.arange(dim) % 2, 3.3e38, -3.3e38)
    x[17:32] *= 1e-38
    x[32:40] *= 1e-42
    x[40] = 0.0
    x[41] = -0.0
    x[42] = 7.5
    x[43:48, :, ::3] *= 1e-30          # large and vanishing values side by side
    x[48:56] += 1e6
    x = co.round_bf16(x)
    x[60, 0, 3] = np.nan
    x[61, 1, 40] = np.inf
    x[62, 0, 5] = -np.inf
    c = CacheCase([n], [n], 2, dim, 32, 16)
    c.k, c.v = [x], [x[::-1].copy()]
    cache = written(ctx, c)
    assert np.array_equal(cache.pages.cpu().numpy(), expected_pages(c))
    from paper_2607_28418_b200 import binding
    k, _ = binding.wide_cache_read(ctx, cache, c.seqs(), n, dtype=torch.float32)
    assert np.array_equal(k.cpu().numpy(), co.held(x, 32).reshape(n, -1), equal_nan=True)
    assert torch.isnan(k).sum().item() == 32 * (~np.isfinite(x)).reshape(-1, 32).any(1).sum()


def test_rows_of_a_fused_projection_and_rows_behind_the_last_sequence(ctx):
    """k and v as slices of one matrix; the rows behind the last sequence are neither stored nor overwritten."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([50, 20], [9, 20], 2, 128, 64, 16, seed=8)
    width = 2 * 128
    fused = torch.full((c.rows + 5, 3 * width + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    k, v = fused[:, width:2 * width], fused[:, 2 * width + 64:]
    k[:c.rows] = to_device(c.new("k"))
    v[:c.rows] = to_device(c.new("v"))
    cache = c.cache(c.garbage.copy())
    binding.wide_cache_write(ctx, cache, c.seqs(), k, v)
    assert np.array_equal(cache.pages.cpu().numpy(), expected_pages(c))
    out = torch.full((c.rows + 5, 3 * width), 7.0, dtype=torch.bfloat16, device="cuda")
    binding.wide_cache_read(ctx, cache, c.seqs(), c.rows + 5, k=out[:, width:2 * width], v=out[:, 2 * width:])
    assert (out[c.rows:] == 7).all() and (out[:, :width] == 7).all()
    ref = co.round_bf16(co.held(c.new("k").reshape(c.rows, 2, 128), 64).reshape(c.rows, -1))
    assert np.array_equal(out[:c.rows, width:2 * width].float().cpu().numpy(), ref)


@pytest.mark.parametrize("offset,extra", [(0, 0), (4, 0), (0, 4), (4, 4), (8, 8)])
def test_f32_rows_at_every_16_bytes(ctx, offset, extra):
    """Rows on 16-byte but not on 32-byte boundaries are the same values, and nothing beside them is touched."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([50, 20], [9, 20], 2, 64, 32, 16, seed=8, dtype="f32")
    flat = torch.full((offset + c.rows * (256 + extra) + 8,), 7.0, device="cuda")
    both = flat[offset:offset + c.rows * (256 + extra)].view(c.rows, 256 + extra)
    k, v = both[:, :128], both[:, 128:256]
    k.copy_(to_device(c.new("k"), "f32"))
    v.copy_(to_device(c.new("v"), "f32"))
    cache = c.cache(c.garbage.copy())
    binding.wide_cache_write(ctx, cache, c.seqs(), k, v)
    assert np.array_equal(cache.pages.cpu().numpy(), expected_pages(c))
    binding.wide_cache_read(ctx, cache, c.seqs(), c.rows, k=k, v=v)
    for got, which in ((k, "k"), (v, "v")):
        assert np.array_equal(got.cpu().numpy(), co.held(c.new(which).reshape(c.rows, 2, 64), 32).reshape(c.rows, -1).astype(np.float32))
    assert (both[:, 256:] == 7).all() and (flat[:offset] == 7).all() and (flat[-8:] == 7).all()


def test_indices_out_of_range_are_dropped_and_reported(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([40, 40, 40, 40, 40], [40, 40, 40, 40, 40], 2, 64, 64, 16, seed=9)
    good = expected_pages(c)
    seqs = c.seqs()
    seqs.page_table[1, 1] = c.n_pages            # one page of sequence 1
    seqs.page_table[2, 0] = -7
    seqs.kv_lens[3] = 49                         # longer than its table: 3 pages of 16
    seqs.kv_lens[4] = 39                         # fewer positions than new rows
    cache = c.cache(c.garbage.copy())
    binding.wide_cache_write(ctx, cache, seqs, to_device(c.new("k")), to_device(c.new("v")))
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert ctx.status() == 0
    want = c.garbage.copy()
    for s, pages in ((0, (0, 1, 2)), (1, (0, 2)), (2, (1, 2))):
        for p in pages:
            want[c.table[s, p]] = good[c.table[s, p]]
    assert np.array_equal(cache.pages.cpu().numpy(), want)
    k, _ = binding.wide_cache_read(ctx, c.cache(good), seqs, c.rows, k=torch.full((c.rows, 128), 9.0, device="cuda"),
                                   v=torch.full((c.rows, 128), 9.0, device="cuda"))
    assert ctx.status() == binding.ERR_BAD_INDEX
    ref = co.held(c.new("k").reshape(c.rows, 2, 64), 64).reshape(c.rows, -1).astype(np.float32)
    ref[40 + 16:40 + 32] = 0
    ref[80:96] = 0
    ref[120:] = 9
    assert np.array_equal(k.cpu().numpy(), ref)
    # row ranges that are no ranges
    seqs = c.seqs()
    seqs.row_start[:] = torch.tensor([0, 40, 30, 70, 70, 1000], dtype=torch.int32)
    cache = c.cache(c.garbage.copy())
    binding.wide_cache_write(ctx, cache, seqs, to_device(c.new("k")), to_device(c.new("v")))
    assert ctx.status() == binding.ERR_BAD_INDEX
    got = cache.pages.cpu().numpy()
    for s in (1, 3, 4):
        for p in c.table[s]:
            assert np.array_equal(got[p], c.garbage[p])
    for p in c.table[0]:
        assert np.array_equal(got[p], good[p])
    # not one good row
    binding.wide_cache_write(ctx, cache, binding.Sequences(seqs.page_table, seqs.kv_lens, torch.full_like(seqs.row_start, -1)),
                             to_device(c.new("k")), to_device(c.new("v")))
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert np.array_equal(cache.pages.cpu().numpy(), got)


@pytest.mark.parametrize("rows", [48, 640])
def test_row_start_that_does_not_ascend_is_reported(ctx, rows):
    """Which rows are then left out is open, but nothing that is not theirs is touched."""
    from paper_2607_28418_b200 import binding
    n = 64
    c = CacheCase([48] * n, [1] * n, 2, 64, 64, 16, seed=33)
    x = torch.ones((rows + 8, 128), dtype=torch.bfloat16, device="cuda")
    for start in ([48 * (s & 1) for s in range(n + 1)], [rows - 10 * s for s in range(n + 1)], [-5] + [2 ** 31 - 1] * n, [-2 ** 31] * n + [rows]):
        seqs = binding.Sequences(torch.from_numpy(c.table).cuda(), torch.full((n,), 48, dtype=torch.int32, device="cuda"),
                                 torch.tensor(start, dtype=torch.int32, device="cuda"))
        cache = c.cache(c.garbage.copy())
        binding.wide_cache_write(ctx, cache, seqs, x[:rows], x[:rows])
        assert ctx.status() == binding.ERR_BAD_INDEX
        got = cache.pages.cpu().numpy()
        spare = np.setdiff1d(np.arange(c.n_pages), c.table.ravel())
        assert len(spare) and np.array_equal(got[spare], c.garbage[spare])
        k, v = torch.full((rows + 8, 128), 9.0, device="cuda"), torch.full((rows + 8, 128), 9.0, device="cuda")
        binding.wide_cache_read(ctx, cache, seqs, rows, k=k[:rows], v=v[:rows])
        assert ctx.status() == binding.ERR_BAD_INDEX
        assert (k[rows:] == 9).all() and (v[rows:] == 9).all()


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 1023, 1025, 2100])
@pytest.mark.parametrize("most", [1, 3, 40])
def test_every_sequence_is_found(ctx, n, most):
    """Sequences of no, few and many new rows (and rows before the first and behind the last): written and read back are all
    of theirs and only those."""
    from paper_2607_28418_b200 import binding
    rng = np.random.default_rng(1000 * n + most)
    news = rng.integers(0, most + 1, n)
    lens = news + rng.integers(0, 40, n)
    start = 7 + np.concatenate([[0], np.cumsum(news)])
    rows, pages = int(start[-1]) + 9, 5                      # five pages of 16 for up to 79 positions
    table = rng.permutation(pages * n).astype(np.int32).reshape(n, pages)
    cache = binding.Cache(torch.zeros((pages * n, binding.cache_page_bytes(16, 1, 64, 64)), dtype=torch.uint8, device="cuda"), 1, 64, 64, 16)
    seqs = binding.Sequences(*(torch.from_numpy(a.astype(np.int32)).cuda() for a in (table, lens, start)))
    x = (torch.arange(rows, dtype=torch.float32, device="cuda") % 251 + 1)[:, None].expand(rows, 64).contiguous()     # held exactly
    binding.wide_cache_write(ctx, cache, seqs, x, -x)
    k, v = torch.full((rows, 64), 0.5, device="cuda"), torch.full((rows, 64), 0.5, device="cuda")
    binding.wide_cache_read(ctx, cache, seqs, rows, k=k, v=v)
    assert ctx.status() == 0
    own = slice(7, rows - 9)
    assert torch.equal(k[own], x[own]) and torch.equal(v[own], -x[own])
    for y in (k, v):
        assert (y[:7] == 0.5).all() and (y[rows - 9:] == 0.5).all()


@pytest.mark.parametrize("seqs", [600, 4096])
def test_many_sequences(ctx, seqs):
    from paper_2607_28418_b200 import binding
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, 40, seqs)
    news = np.minimum(lens, rng.integers(0, 20, seqs))
    c = CacheCase(lens.tolist(), news.tolist(), 1, 64, 64, 16, seed=13)
    cache = written(ctx, c)
    assert np.array_equal(cache.pages.cpu().numpy(), expected_pages(c))
    k, v = binding.wide_cache_read(ctx, cache, c.seqs(), c.rows, dtype=torch.float32)
    assert np.array_equal(k.cpu().numpy(), co.held(c.new("k").reshape(c.rows, 1, 64), 64).reshape(c.rows, -1))


def test_minima_beside_vanishing_numbers(ctx):
    """Sub-groups whose minimum lies far below the scale, where m - s / 2 is no fp32 number (bf16 and fp32 inputs)."""
    rng = np.random.default_rng(14)
    for dtype in ("bf16", "f32"):
        x = np.abs(rng.standard_normal((200, 2, 64))).astype(np.float32) + 0.5
        x[:, :, 0] = np.exp2(rng.integers(-60, -5, (200, 2)).astype(np.float32))
        x[100:, :, 1] = -np.exp2(rng.integers(-60, -5, (100, 2)).astype(np.float32))
        x = co.round_bf16(x) if dtype == "bf16" else x
        c = CacheCase([200], [200], 2, 64, 32, 32, dtype=dtype)
        c.k, c.v = [x], [x[::-1].copy()]
        assert np.array_equal(written(ctx, c).pages.cpu().numpy(), expected_pages(c))


def test_places_beyond_four_gigabytes(ctx):
    from paper_2607_28418_b200 import binding
    page_bytes = binding.cache_page_bytes(256, 8, 128, 64)
    n_pages = (5 << 30) // page_bytes + 1
    cache = binding.Cache.empty(n_pages, 8, 128, 64, 256)
    table = torch.tensor([[n_pages - 1, 0], [n_pages - 2, 1]], dtype=torch.int32, device="cuda")
    seqs = binding.Sequences(table, torch.tensor([300, 256], dtype=torch.int32, device="cuda"), torch.tensor([0, 300, 556], dtype=torch.int32, device="cuda"))
    g = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn((556, 8 * 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    binding.wide_cache_write(ctx, cache, seqs, k, v)
    k2, v2 = binding.wide_cache_read(ctx, cache, seqs, 556)
    for a, b in ((k, k2), (v, v2)):
        ref = co.round_bf16(co.held(a.float().cpu().numpy().reshape(556, 8, 128), 64).reshape(556, -1))
        assert np.array_equal(b.float().cpu().numpy(), ref)


def test_on_another_stream_and_captured(ctx):
    """A step of write and read back, captured once and replayed on new rows of a growing cache."""
    from paper_2607_28418_b200 import binding
    c = CacheCase([30, 7], [1, 1], 2, 128, 128, 16, seed=11)
    cache = c.cache(c.garbage.copy())
    seqs = c.seqs()
    k, v = to_device(c.new("k")), to_device(c.new("v"))
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.wide_cache_write(ctx, cache, seqs, k, v)
        binding.wide_cache_read(ctx, cache, seqs, 2, k=ko, v=vo)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.wide_cache_write(ctx, cache, seqs, k, v)
        binding.wide_cache_read(ctx, cache, seqs, 2, k=ko, v=vo)
    want = c.garbage.copy()
    for q in range(2):   # the call before the capture
        co.store(want, 16, 128, c.table[q], c.lens[q], c.k[q][-1:], c.v[q][-1:])
    rng = np.random.default_rng(12)
    for step in range(2):
        new = [co.round_bf16(rng.standard_normal((2, 2, 128))) for _ in range(2)]
        k.copy_(to_device(new[0].reshape(2, -1)))
        v.copy_(to_device(new[1].reshape(2, -1)))
        lens = [31 + step, 8 + step]
        seqs.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        for q in range(2):
            co.store(want, 16, 128, c.table[q], lens[q], new[0][q:q + 1], new[1][q:q + 1])
        assert np.array_equal(ko.float().cpu().numpy(), co.round_bf16(co.held(new[0], 128)).reshape(2, -1))
    assert np.array_equal(cache.pages.cpu().numpy(), want)


def test_binding_refuses(ctx):
    from paper_2607_28418_b200 import binding
    c = CacheCase([20], [20], 2, 64, 64, 16)
    cache, seqs = c.cache(c.full_pages()), c.seqs()
    k = to_device(c.new("k"))
    with pytest.raises(ValueError):
        binding.wide_cache_write(ctx, cache, seqs, k, k.float())
    with pytest.raises(ValueError):
        binding.wide_cache_write(ctx, cache, seqs, k[:, :64], k[:, :64])
    with pytest.raises(ValueError):
        binding.wide_cache_write(ctx, cache, seqs, k.cpu(), k.cpu())
    with pytest.raises(ValueError):
        binding.wide_cache_write(ctx, cache, seqs, k.t().contiguous().t(), k)
    with pytest.raises(ValueError):
        binding.Sequences(seqs.page_table.long(), seqs.kv_lens)
    with pytest.raises(ValueError):
        binding.Sequences(seqs.page_table, seqs.kv_lens, seqs.kv_lens)
    with pytest.raises(ValueError):
        binding.Cache(cache.pages, 2, 64, 32, 16)
    with pytest.raises(binding.WideError):
        binding.Cache.empty(4, 2, 96)
    # nothing to do is no error
    binding.wide_cache_write(ctx, cache, seqs, k[:0], k[:0])
    none = binding.Sequences(seqs.page_table[:0], seqs.kv_lens[:0])
    binding.wide_cache_write(ctx, cache, none, k, k)
