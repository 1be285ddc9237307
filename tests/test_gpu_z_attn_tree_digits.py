"""Digits of wide_attn_tree: sub-groups of values without a step, sums over very long sequences."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests.cache_util import CacheCase
from tests.test_gpu_u_attn_tree import check, ctx, queries, random_trees, reference, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,group", [(64, 32), (128, 32), (128, 64)])
def test_constant_sub_groups_of_values_keep_the_digits(ctx, dim, group):  # noqa: F811
    """A sub-group of equal numbers has step 0 and a minimum that fp16 holds as it is (bf16's 8 digits, 2^-14 to 2^14): its block stays in fp16, so the errors are those of
    ordinary values (in bf16 they would be twice as many)."""
    c = CacheCase([700, 90], [24, 8], 2, dim, group, 32, seed=55)
    rng = np.random.default_rng(56)
    for v in c.v:                       # in every block a token with a constant sub-group, of either sign and many sizes
        flat = v.reshape(len(v), 2, dim // group, group)
        for i in range(0, len(v), 16):
            flat[min(i + int(rng.integers(16)), len(v) - 1), :, int(rng.integers(dim // group))] = co.round_bf16(np.float32(rng.choice([-1, 1]) * 2.0 ** rng.integers(-13, 2) * 1.3))
    q = queries(c, 8, 57)
    bits, sees = random_trees(c, 58)
    ref, _ = reference(c, q, None, 4, sees)
    got = run(ctx, c, q, None, 4, bits).float().cpu().numpy().reshape(ref.shape)
    assert np.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum()) < 2.0 ** -9


@pytest.mark.parametrize("size", [1e-6, 3e4, 1e30, 0.75])
def test_constant_sub_groups_of_any_size(ctx, size):  # noqa: F811
    """All sub-groups constant: a value is its minimum, in fp16 or bf16."""
    c = CacheCase([300], [12], 2, 128, 64, 32, seed=59)
    c.v = [co.round_bf16(np.broadcast_to(v.reshape(len(v), 2, 2, 64)[..., :1] * np.float32(size), (len(v), 2, 2, 64)).reshape(len(v), 2, 128).copy()) for v in c.v]
    q = queries(c, 8, 60)
    bits, sees = random_trees(c, 61)
    ref, tol = reference(c, q, None, 4, sees)
    check(run(ctx, c, q, None, 4, bits), ref, tol)
