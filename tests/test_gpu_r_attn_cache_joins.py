"""wide_attn_cache where an item is cut between warps and CTAs, for every number of rows a pass: every output against a bound
that sees a lost block of keys (test_oracle_cache_bound.py), and a sequence alone against itself in a batch."""
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


def queries(c, hq, seed):
    return co.round_bf16(np.random.default_rng(seed).standard_normal((c.rows, hq, c.dim)))


def blocks_of_a_warp(c, share):
    """At most: where no sequence is longer than 96 blocks an item may be one CTA's, of 8 warps at least; else its piece of all units,
    four more an item than blocks, with the fewest rows a pass, on 148 CTAs of 8 warps."""
    longest = max(-(-x // 16) for x in c.lens)
    units = sum(c.heads * -(-n * share // 8) * (-(-x // 16) + 4) for x, n in zip(c.lens, c.news) if n)
    return max(units // (148 * 8) + 2, longest // 8 + 1 if longest <= 96 else 0)


def reference(c, q, on, per, causal=True, blocks=0):
    blocks = blocks or blocks_of_a_warp(c, q.shape[1] // c.heads)
    parts = [co.attention_with_bound(q[a:a + n], c.k[s], c.v[s], c.group, on[a:a + n], per, causal, blocks=blocks)
             for s, (a, n) in enumerate(zip(c.row_start, c.news))]
    return tuple(np.concatenate(x) for x in zip(*parts))


def run(ctx, c, q, on, per, **kw):
    from paper_2607_28418_b200 import binding
    bits = torch.from_numpy(pack_bits(on)).cuda()
    return binding.wide_attn_cache(ctx, to_device(q.reshape(c.rows, -1)), c.cache(c.full_pages()), c.seqs(), q.shape[1], per, mask_bits=bits, **kw)


def host(o, like):
    return o.float().cpu().numpy().reshape(like.shape).astype(np.float64)


def check(got, ref, bound):
    off = np.abs(got - ref)
    assert np.isfinite(got).all()
    worst = np.unravel_index((off - bound).argmax(), off.shape)
    assert (off <= bound).all(), f"{off[worst]:.3e} off {ref[worst]:.3e}, bound {bound[worst]:.3e}, at {worst}; {(off > bound).mean():.1%} of all"
    assert (got[ref == 0] == 0).all()


# (heads, query heads on each, lengths, new rows): one to three sequences, items over several CTAs
CUTS = [(2, 4, (5000, 3, 1777), (1, 1, 1)),           # 8 rows a pass
        (1, 8, (2600,), (1,)),
        (1, 16, (4000, 17), (1, 1)),                  # 16
        (2, 3, (1600, 1900), (5, 4)),
        (1, 24, (3100,), (1,)),                       # 24
        (2, 4, (1700, 2000, 40), (6, 5, 7)),
        (1, 4, (2500,), (30,)),                       # five passes of 24 rows
        (1, 5, (1700, 900), (40, 3))]


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("heads,share,lens,news", CUTS)
def test_pieces_of_an_item_are_joined(ctx, dim, group, heads, share, lens, news):
    c = CacheCase(lens, news, heads, dim, group, 64, seed=1)
    q = queries(c, heads * share, 2)
    on = np.ones((c.rows, heads), bool)
    got = run(ctx, c, q, on, share)
    check(host(got, q), *reference(c, q, on, share))
    assert torch.equal(run(ctx, c, q, on, share), got)


@pytest.mark.parametrize("share,news", [(4, 1), (12, 1), (4, 6)])
@pytest.mark.parametrize("causal", [True, False])
def test_masks_on_items_that_are_cut(ctx, share, news, causal):
    """Heads that no row uses, rows that use none, and the end of a sequence inside a piece."""
    c = CacheCase((3001, 1500, 2222), (news,) * 3, 4, 128, 64, 32, seed=3)
    q = queries(c, 4 * share, 4)
    on = np.random.default_rng(5).random((c.rows, 4)) < 0.4
    on[:news] = [True, False, True, False]
    on[-1] = False
    check(host(run(ctx, c, q, on, share, causal=causal), q), *reference(c, q, on, share, causal))


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("share,news", [(1, 1), (4, 1), (4, 3), (4, 6)])
def test_a_sequence_alone_and_in_batches(ctx, dim, group, share, news):
    """The others decide where its items are cut, and (by the average of new rows) how many rows share a pass: its outputs differ
    by no more than the bounds of both."""
    heads = 2
    lens, many = (700, 65, 2100, 1, 16, 333, 900), (news, 1, news, 1, 12, 2, 1)
    c = CacheCase(lens, many, heads, dim, group, 16, seed=6)
    q = queries(c, heads * share, 7)
    on = np.random.default_rng(8).random((c.rows, heads)) < 0.8
    ref, bound = reference(c, q, on, share, blocks=8)     # 900 tokens on a CTA of their own
    whole = host(run(ctx, c, q, on, share), q)
    check(whole, ref, bound)
    for pick in ([0], [2], [2, 3], [0, 4], [5, 0, 1, 6]):
        part = CacheCase.__new__(CacheCase)
        part.__dict__.update(c.__dict__)
        part.lens, part.news, part.table = [lens[s] for s in pick], [many[s] for s in pick], c.table[pick]
        part.k, part.v, part.n_seqs = [c.k[s] for s in pick], [c.v[s] for s in pick], len(pick)
        part.row_start = np.concatenate([[0], np.cumsum(part.news)]).astype(np.int32)
        part.rows = int(part.row_start[-1])
        rows = np.concatenate([np.arange(c.row_start[s], c.row_start[s + 1]) for s in pick])
        got = host(run(ctx, part, q[rows], on[rows], share), q[rows])
        check(got, ref[rows], bound[rows])
        assert (np.abs(got - whole[rows]) <= 2 * bound[rows]).all()
