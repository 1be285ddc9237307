"""wide_cache_append: the bits of wide_rope followed by wide_cache_write, and against the rotation in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from tests.cache_util import CacheCase, to_device

pytestmark = pytest.mark.gpu

SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


class Append:
    """Seeded inputs of a call: a fused projection [rows, (hq + 2 hk) * dim], positions, frequencies."""

    def __init__(self, lens, news, hk, dim, group, page, hq, rot, axes=1, dtype="bf16", seed=0, far=131072):
        self.c = CacheCase(lens, news, hk, dim, group, page, seed=seed, dtype=dtype)
        rng = np.random.default_rng(seed + 1)
        self.hq, self.hk, self.dim, self.rot, self.rows = hq, hk, dim, rot, self.c.rows
        self.fused = to_device(rng.standard_normal((self.rows, (hq + 2 * hk) * dim)) * (1 + 9 * (rng.random((hq + 2 * hk) * dim) < 0.1)), dtype)
        a, b = hq * dim, hk * dim
        self.q, self.k, self.v = (self.fused[:, :a] if hq else None), self.fused[:, a:a + b], self.fused[:, a + b:]
        self.pos = torch.from_numpy(rng.integers(0, far, (axes, self.rows)).astype(np.int32)).cuda()
        self.inv = torch.tensor([500000.0 ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")
        self.axis = torch.from_numpy(rng.integers(0, axes, rot // 2).astype(np.int32)).cuda() if axes > 1 else None

    def cache(self):
        return self.c.cache(self.c.garbage.copy())

    def run(self, ctx, cache, seqs, interleaved=False, **kw):
        from paper_2607_28418_b200 import binding
        return binding.wide_cache_append(ctx, cache, seqs, self.q, self.k, self.v, self.pos, self.inv, axis=self.axis, interleaved=interleaved, **kw)

    def two_calls(self, ctx, cache, seqs, interleaved=False):
        from paper_2607_28418_b200 import binding
        kw = dict(axis=self.axis, head_dim=self.dim, interleaved=interleaved)
        q = None if self.q is None else binding.wide_rope(ctx, self.q, None, self.pos, self.inv, **kw)[0]
        k, _ = binding.wide_rope(ctx, self.k, None, self.pos, self.inv, **kw)
        binding.wide_cache_write(ctx, cache, seqs, k, self.v)
        return q


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def check(ctx, x, interleaved=False, row_start=True):
    one, two, seqs = x.cache(), x.cache(), x.c.seqs(row_start)
    before = x.fused.clone()
    q = x.run(ctx, one, seqs, interleaved)
    q2 = x.two_calls(ctx, two, seqs, interleaved)
    assert torch.equal(one.pages, two.pages)
    assert (q is None and q2 is None) or same_bits(q, q2)
    assert same_bits(before, x.fused)


LENS, NEWS = [1, 16, 37, 70, 5, 0, 131, 33], [1, 16, 20, 1, 0, 0, 131, 15]


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [16, 48, 64, 128])
def test_bits_of_the_two_calls(ctx, dim, group, dtype, interleaved, rot):
    if rot > dim:
        rot = 32
    check(ctx, Append(LENS, NEWS, 3, dim, group, 16 if group == 32 else 64, 6, rot, axes=3, dtype=dtype, seed=dim + rot), interleaved)


@pytest.mark.parametrize("hq,hk", [(0, 1), (1, 1), (7, 1), (32, 8), (40, 40), (256, 256)])
@pytest.mark.parametrize("dim", [64, 128])
def test_numbers_of_heads(ctx, hq, hk, dim):
    check(ctx, Append([40, 3], [19, 2], hk, dim, 64, 32, hq, dim, seed=hq))


@pytest.mark.parametrize("lens", [list(range(1, 40)) + [200, 256, 257], [1], [4000]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_a_sequence_without_row_start(ctx, lens, dtype):
    check(ctx, Append(lens, [1] * len(lens), 2, 128, 64, 64, 8, 128, dtype=dtype), row_start=False)


def test_many_sequences_and_long_chunks(ctx):
    check(ctx, Append([17 + i % 50 for i in range(700)], [i % 3 for i in range(700)], 2, 64, 32, 16, 4, 64, seed=1))
    check(ctx, Append([2100, 900, 1], [2047, 300, 1], 4, 128, 128, 64, 8, 128, seed=2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_against_the_rotation_in_64_bits(ctx, dtype, interleaved):
    """The angle's rounding, sine, cosine and the products: 8 * 2^-24 of |u| + |w| (as for wide_rope), then the rounding to the type.  A key is
    held within half a step of that; a step is the range / 15 and the rounding of minimum (2^-7 of itself, as a range of the group may
    grow by it) and step (2^-7) to bf16."""
    from paper_2607_28418_b200 import binding
    x = Append(LENS, NEWS, 2, 128, 64, 64, 4, 96, axes=2, dtype=dtype, seed=9)
    cache, seqs = x.cache(), x.c.seqs()
    q = x.run(ctx, cache, seqs, interleaved)
    k, v = binding.wide_cache_read(ctx, cache, seqs, x.rows, dtype=torch.float32)
    pos, inv, axis = x.pos.cpu().numpy(), x.inv.tolist(), x.axis.cpu().numpy()
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    host = lambda t, h: t.float().cpu().numpy().astype(np.float64).reshape(x.rows, h, 128)  # noqa: E731
    for got, src, h in ((q, x.q, 4), (k, x.k, 2)):
        y = host(src, h)
        ref = co.rope(y.astype(np.float32), pos, inv, axis, interleaved, False)
        tol = 16 * 2.0 ** -24 * np.abs(y).max() + unit * np.abs(ref)
        if got is k:
            sub = ref.reshape(x.rows, h, 2, 64)
            low, high = sub.min(-1) - tol.max(), sub.max(-1) + tol.max()
            step = ((high - low) + 2.0 ** -7 * np.abs(low)) / 15 * (1 + 2.0 ** -7)
            tol = tol + np.repeat(step / 2, 64, axis=-1).reshape(ref.shape) + 2.0 ** -22 * np.abs(y).max()
        assert (np.abs(host(got, h) - ref) <= tol).all()
    ref = np.concatenate([co.held(p.reshape(1, 2, 128).astype(np.float32), 64) for p in host(x.v, 2)]).reshape(x.rows, 2, 128)
    assert np.array_equal(host(v, 2).astype(np.float32), ref.astype(np.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_have_no_levels(ctx, dtype):
    """Infinities, NaN, zeros, constants, values near the ends of the type: the slow way of the levels."""
    x = Append([90, 35], [70, 33], 2, 128, 32, 16, 2, 64, dtype=dtype, seed=3)
    f = x.fused.view(x.rows, -1, 128)
    f[3, :, 7], f[4, :, 70], f[5, :, 100], f[6], f[7] = float("inf"), float("nan"), -float("inf"), 0.0, -0.0
    f[8], f[9, :, 5], f[10], f[11] = 2.5, 3e38, 1e-38, f[11] * 1e-20
    check(ctx, x)
    check(ctx, x, interleaved=True)


def test_in_place_and_16_byte_rows(ctx):
    from paper_2607_28418_b200 import binding
    x = Append(LENS, NEWS, 2, 64, 64, 16, 3, 64, dtype="f32", seed=5)
    ref = x.two_calls(ctx, x.cache(), x.c.seqs())
    q = torch.full((x.rows, 3 * 64 + 12), 7.0, device="cuda")           # rows on 16-byte, not on 32-byte borders
    q[:, 4:196] = x.q
    view = q[:, 4:196]
    out = binding.wide_cache_append(ctx, x.cache(), x.c.seqs(), view, x.k, x.v, x.pos, x.inv, q_out=view)
    assert out is view and same_bits(view, ref)
    assert (q[:, :4] == 7).all() and (q[:, 196:] == 7).all()


def test_rows_of_no_sequence_and_bad_places(ctx):
    """Rows in front of, between and behind the sequences stay; so do those of a sequence that is left out; a missing page drops keys and
    values and nothing else."""
    from paper_2607_28418_b200 import binding
    x = Append([40, 50, 60, 20], [4, 4, 4, 4], 2, 128, 64, 16, 4, 128, seed=6)
    c = x.c
    table, lens = c.table.copy(), list(c.lens)
    table[1, 3] = 10 ** 6            # the page of the last positions, 46 .. 49 -> 48, 49 only
    lens[2] = 10 ** 6                # left out
    starts = np.array([1, 5, 9, 13, 15], dtype=np.int32)       # rows 0 and 15 belong to nobody
    seqs = binding.Sequences(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), torch.from_numpy(starts).cuda())
    one, two = x.cache(), x.cache()
    q = torch.full_like(x.q.contiguous(), 5.0)
    x.run(ctx, one, seqs, q_out=q)
    assert ctx.status() == binding.ERR_BAD_INDEX and ctx.status() == 0
    ref = x.two_calls(ctx, two, seqs)
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert torch.equal(one.pages, two.pages)
    stay = torch.zeros(x.rows, dtype=torch.bool)
    stay[[0, 9, 10, 11, 12, 15]] = True
    assert (q[stay.cuda()] == 5).all() and same_bits(q[~stay.cuda()], ref[~stay.cuda()])


def test_an_axis_out_of_range_leaves_its_pair(ctx):
    from paper_2607_28418_b200 import binding
    x = Append([20], [9], 1, 64, 64, 16, 1, 64, axes=2, seed=7)
    x.axis[3], x.axis[5] = -1, 2
    one, two = x.cache(), x.cache()
    q = x.run(ctx, one, x.c.seqs())
    assert ctx.status() == binding.ERR_BAD_INDEX
    ref = x.two_calls(ctx, two, x.c.seqs())
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert torch.equal(one.pages, two.pages) and same_bits(q, ref)


def test_captured_and_replayed_on_another_stream(ctx):
    x = Append([100, 37, 61], [1, 1, 1], 8, 128, 64, 64, 32, 128, seed=8)
    cache, seqs, q = x.cache(), x.c.seqs(False), torch.empty_like(x.q.contiguous())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            x.run(ctx, cache, seqs, q_out=q)
    for step in range(3):            # lengths and rows move on in place
        x.fused.mul_(-0.5 - step)
        seqs.kv_lens.copy_(torch.tensor([100 - step, 37 + step, 1 + step], dtype=torch.int32))
        x.pos.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        again = x.cache()
        again.pages.copy_(cache.pages)
        assert same_bits(q, x.two_calls(ctx, again, seqs))
        assert torch.equal(again.pages, cache.pages)


def test_nothing_to_do(ctx):
    from paper_2607_28418_b200 import binding
    x = Append([0, 5], [0, 0], 2, 64, 64, 16, 2, 64)
    cache = x.cache()
    assert x.run(ctx, cache, x.c.seqs()).shape == (0, 128)
    assert np.array_equal(cache.pages.cpu().numpy(), x.c.garbage)
    with pytest.raises(ValueError):
        binding.wide_cache_append(ctx, cache, x.c.seqs(), x.q, x.k, x.v, x.pos[:, :0], x.inv.float())
