"""wide_attn_cache where values differ by many powers of two: what a row does not weigh costs it no digits.  Every output is
held against a bound made of what its own row weighs (oracle.cache_oracle.attention_with_bound)."""
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


def run(ctx, c, q, on, per, **kw):
    from paper_2607_28418_b200 import binding
    bits = None if on is None else torch.from_numpy(pack_bits(on)).cuda()
    o = binding.wide_attn_cache(ctx, to_device(q.reshape(c.rows, -1)), c.cache(c.full_pages()), c.seqs(), q.shape[1], per, mask_bits=bits, **kw)
    return o.float().cpu().numpy().reshape(q.shape).astype(np.float64)


def reference(c, q, on, per, causal=True, blocks=2):
    parts = [co.attention_with_bound(q[a:a + n], c.k[s], c.v[s], c.group, on[a:a + n], per, causal, blocks=blocks)
             for s, (a, n) in enumerate(zip(c.row_start, c.news))]
    return tuple(np.concatenate(x) for x in zip(*parts))


def check(got, ref, bound, what=""):
    off = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    worst = np.unravel_index((off - bound).argmax(), off.shape)
    assert (off <= bound).all(), f"{what}: {off[worst]:.3e} off {ref[worst]:.3e}, bound {bound[worst]:.3e}, at {worst}; {(off > bound).mean():.1%} of all"
    assert (got[ref == 0] == 0).all(), what


def facing(c, hq, seed):
    """Queries that all point the same way per KV head, and that direction [heads, dim] (of -1 and 1)."""
    rng = np.random.default_rng(seed)
    u = np.where(rng.random((c.heads, c.dim)) < 0.5, -1.0, 1.0)
    q = np.repeat(u, hq // c.heads, 0)[None] * (0.5 + rng.random((c.rows, hq, c.dim)))
    return co.round_bf16(q), u


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("power", [10, 20, 24, 28, 30, 60])
@pytest.mark.parametrize("at", [0, 17, 100, 198])
def test_a_large_value_without_weight(ctx, dim, group, power, at):
    """The token is finite, visible, and has a probability of 2^-130 or less."""
    c = CacheCase([199], [1], 2, dim, group, 16, seed=power)
    q, u = facing(c, 8, 1)
    c.k[0][at] = -12 * u
    c.v[0][at] = co.round_bf16(c.v[0][at] * 2.0 ** power)
    on = np.ones((1, 2), bool)
    check(run(ctx, c, q, on, 4), *reference(c, q, on, 4))


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("power", [24, 30, 60])
@pytest.mark.parametrize("news", [2, 3, 5])
def test_a_large_value_of_a_later_token(ctx, dim, group, power, news):
    """Only the last of the new rows sees it (4, 8, ... rows a KV head: every number of rows a pass)."""
    c = CacheCase([75], [news], 2, dim, group, 16, seed=power + news)
    q = co.round_bf16(np.random.default_rng(2).standard_normal((news, 8, dim)))
    c.v[0][-1] = co.round_bf16(c.v[0][-1] * 2.0 ** power)
    on = np.ones((news, 2), bool)
    check(run(ctx, c, q, on, 4), *reference(c, q, on, 4))


@pytest.mark.parametrize("dim,group", [(64, 32), (128, 32), (128, 64)])
@pytest.mark.parametrize("power", [-60, -30, 20, 30, 60])
def test_one_sub_group_of_all_tokens_larger(ctx, dim, group, power):
    c = CacheCase([130, 40], [1, 3], 2, dim, group, 16, seed=3)
    for s in range(2):
        c.v[s][:, :, group:2 * group] *= 2.0 ** power
    q = co.round_bf16(np.random.default_rng(4).standard_normal((4, 8, dim)))
    on = np.ones((4, 2), bool)
    check(run(ctx, c, q, on, 4), *reference(c, q, on, 4))


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("power", [-40, 30])
@pytest.mark.parametrize("news,share", [(1, 4), (1, 12), (3, 8)])
def test_rows_that_look_at_different_tokens(ctx, dim, group, power, news, share):
    """Of the heads that share a pass, every second one looks at nothing but the token that the others leave out."""
    c = CacheCase([150], [news], 1, dim, group, 16, seed=5)
    q, u = facing(c, share, 6)
    q[:, ::2] *= -1
    c.k[0][60] = -12 * u
    c.v[0][60] = co.round_bf16(c.v[0][60] * 2.0 ** power)
    on = np.ones((news, 1), bool)
    check(run(ctx, c, q, on, share), *reference(c, q, on, share))


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("news,share,lens", [(1, 1, (900, 31)), (1, 8, (333, 900)), (2, 8, (333, 64)), (5, 4, (777, 20))])
@pytest.mark.parametrize("amplitude", [1.0, 6.0])
def test_steps_of_any_size_everywhere(ctx, dim, group, news, share, lens, amplitude):
    """Every sub-group of every token has its own power of two; logits rise along the sequence, and values fall."""
    c = CacheCase(lens, [news] * 2, 2, dim, group, 16, seed=7, scale_k=1.5)
    rng = np.random.default_rng(8)
    q = co.round_bf16(rng.standard_normal((c.rows, 2 * share, dim)) * amplitude)
    for s, n in enumerate(lens):
        e = rng.integers(-20, 21, (n, 2, dim // group)) - (60 * np.arange(n) // n)[:, None, None]
        c.v[s] = co.round_bf16(c.v[s] * np.exp2(np.repeat(e, group, -1)))
        c.k[s] = co.round_bf16(c.k[s] + q[-1, :1].mean(0) * (np.arange(n) / n)[:, None, None])
    on = np.ones((c.rows, 2), bool)
    check(run(ctx, c, q, on, share), *reference(c, q, on, share, blocks=8))      # 57 blocks for 8 or 12 warps


def test_vanishing_and_constant_values(ctx):
    """Steps among the smallest bf16 numbers, steps of zero (all channels alike), and both beside ordinary ones."""
    c = CacheCase([64, 64, 64], [1, 1, 1], 1, 64, 32, 16, seed=9)
    c.v[0] = co.round_bf16(c.v[0] * 1e-37)
    c.v[1][:, :, :32] = 3.5
    c.v[2][10:40] = 0.0
    c.v[2][40:] = co.round_bf16(c.v[2][40:] * 1e-36)
    q = co.round_bf16(np.random.default_rng(10).standard_normal((3, 4, 64)))
    on = np.ones((3, 1), bool)
    ref, bound = reference(c, q, on, 4)
    check(run(ctx, c, q, on, 4), ref, bound + 2.0 ** -130)     # 8 units of the smallest bf16 number, where outputs are that small


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("rise", [7.0, 8.0, 9.0])
def test_constant_values_under_rising_logits(ctx, dim, group, rise):
    """Steps of zero give the power of two nothing to follow, and logits rise by up to 2^8 without a new reference: their product must
    stay a number.  All channels of a key are alike (0 or `rise`) and queries are a single 1, so with this scale logits are whole powers."""
    scale = float(np.float32(np.log(2)))
    assert np.float32(scale) * np.float32(1.4426950408889634) == 1
    c = CacheCase([1536, 1536, 700], [1, 1, 1], 1, dim, group, 16, seed=11)
    rng = np.random.default_rng(12)
    for s, n in enumerate(c.lens):
        high = np.repeat(rng.random(-(-n // 16)) < 0.15, 16)[:n]
        c.k[s][:] = np.where(high, np.float32(rise), np.float32(0))[:, None, None]
        c.v[s][:] = co.round_bf16(rng.standard_normal((n, 1, 1)))
    q = np.zeros((3, 4, dim), np.float32)
    q[:, :, 5] = 1
    on = np.ones((3, 1), bool)
    parts = [co.attention_with_bound(q[s:s + 1], c.k[s], c.v[s], group, on[s:s + 1], 4, True, scale, blocks=13) for s in range(3)]
    ref, bound = (np.concatenate(x) for x in zip(*parts))
    check(run(ctx, c, q, on, 4, scale=scale), ref, bound)
