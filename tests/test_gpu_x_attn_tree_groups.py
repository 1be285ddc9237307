"""wide_attn_tree where routing groups are not the query heads of a KV head, and with many KV heads."""
import numpy as np
import pytest
import torch

from tests.cache_util import CacheCase
from tests.test_gpu_u_attn_tree import check, ctx, queries, random_trees, reference, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,share,per", [(4, 4, 1), (4, 4, 2), (4, 4, 8), (4, 4, 16), (4, 6, 4), (6, 3, 2), (4, 2, 1), (8, 1, 4), (6, 4, 3)])
@pytest.mark.parametrize("news", [[3, 16, 1], [17, 5, 40]])
@pytest.mark.parametrize("dim,group", [(64, 32), (128, 64)])
def test_groups_wider_and_narrower_than_a_kv_head(ctx, heads, share, per, news, dim, group):  # noqa: F811
    """A group spans several KV heads, a part of one, or parts of two; up to 16 new rows the unused KV heads are left out, of more all are read."""
    c = CacheCase([n + 60 * i for i, n in enumerate(news)], news, heads, dim, group, 32, seed=per + share)
    hq = heads * share
    q = queries(c, hq, 41)
    on = np.random.default_rng(42).random((c.rows, hq // per)) < 0.3
    on[0], on[1] = False, True
    bits, sees = random_trees(c, 43)
    ref, tol = reference(c, q, on, per, sees)
    check(run(ctx, c, q, on, per, bits), ref, tol)


@pytest.mark.parametrize("heads,share,per", [(33, 1, 1), (40, 1, 1), (40, 2, 1), (40, 2, 5), (70, 1, 2), (64, 4, 1), (256, 1, 1), (256, 1, 32)])
@pytest.mark.parametrize("news", [[3, 7], [18, 2]])
def test_more_heads_and_groups_than_a_word_has_bits(ctx, heads, share, per, news):  # noqa: F811
    c = CacheCase([100, 45], news, heads, 64, 32, 16, seed=heads)
    hq = heads * share
    q = queries(c, hq, 44)
    on = np.random.default_rng(45).random((c.rows, hq // per)) < 0.2
    bits, sees = random_trees(c, 46)
    ref, tol = reference(c, q, on, per, sees)
    check(run(ctx, c, q, on, per, bits), ref, tol)


@pytest.mark.parametrize("heads,share,per", [(2, 2, 1), (34, 1, 2)])
def test_many_sequences_with_such_groups(ctx, heads, share, per):  # noqa: F811
    """The plan lies in the workspace (from 16384 bytes on; a sequence has 32 or 36)."""
    n = 600
    c = CacheCase([3 + i % 20 for i in range(n)], [1 + i % 3 for i in range(n)], heads, 64, 64, 16, seed=47)
    q = queries(c, heads * share, 48)
    on = np.random.default_rng(49).random((c.rows, heads * share // per)) < 0.4
    bits, sees = random_trees(c, 50)
    ref, tol = reference(c, q, on, per, sees)
    check(run(ctx, c, q, on, per, bits), ref, tol)


@pytest.mark.parametrize("share,news", [(4, [30]), (1, [30]), (1, [3])])
def test_items_cut_between_ctas_with_such_groups(ctx, share, news):  # noqa: F811
    c = CacheCase([6000], news, 4, 128, 64, 64, seed=51)
    hq = 4 * share
    per = hq // 2
    q = queries(c, hq, 52)
    on = np.random.default_rng(53).random((c.rows, 2)) < 0.5
    on[:, 1] = False
    bits, sees = random_trees(c, 54)
    ref, tol = reference(c, q, on, per, sees)
    check(run(ctx, c, q, on, per, bits), ref, tol)


@pytest.mark.parametrize("heads,seqs", [(1, 1), (2, 4), (8, 5)])
@pytest.mark.parametrize("tokens", [200, 384, 400, 1540])
@pytest.mark.parametrize("room", [0, 300])
def test_short_items_alone_or_cut(ctx, heads, seqs, tokens, room):  # noqa: F811
    """Few short items, around the lengths from which they are cut, with page tables that just fit and with wide ones: whatever is cut is joined."""
    from paper_2607_28418_b200 import binding
    from tests.cache_util import to_device
    c = CacheCase([tokens - 3 * i for i in range(seqs)], [9] * seqs, heads, 64, 64, 16, seed=tokens)
    q = queries(c, 4 * heads, 55)
    bits, sees = random_trees(c, 56)
    ref, tol = reference(c, q, None, 4, sees)
    wide = np.pad(c.table, ((0, 0), (0, room)), constant_values=-1)
    places = binding.Sequences(torch.from_numpy(wide).cuda(), torch.tensor(c.lens, dtype=torch.int32).cuda(), torch.from_numpy(c.row_start).cuda())
    o = torch.full((c.rows, 4 * heads * 64), float("nan"), device="cuda").bfloat16()
    check(binding.wide_attn_tree(ctx, to_device(q.reshape(c.rows, -1)), c.cache(c.full_pages()), places, 4 * heads, 4, bits.cuda(), o=o), ref, tol)
