"""Digits of wide_attn_tree: sub-groups of values without a step, sums over very long sequences."""
import numpy as np
import pytest
import torch

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


def long_case(ctx, lens, new, dim, seed, values):  # noqa: F811
    """Sequences of the given lengths that all have the same pages, and what the cache holds of the longest: keys and values [n, dim] in 64 bits."""
    from paper_2607_28418_b200 import binding
    n, page = max(lens), 256
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = binding.Cache.empty(-(-n // page), 1, dim, dim, page)
    table = torch.randperm(-(-n // page), generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()[None]
    k = torch.randn((n, dim), generator=g, device="cuda").bfloat16()
    v = values(torch.randn((n, dim), generator=g, device="cuda")).bfloat16()
    all_of_it = binding.Sequences(table, torch.tensor([n], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    binding.wide_cache_write(ctx, cache, all_of_it, k, v)
    k, v = (x.double() for x in binding.wide_cache_read(ctx, cache, all_of_it, n, dtype=torch.float32))
    seqs = binding.Sequences(table.expand(len(lens), -1).contiguous(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                             torch.arange(len(lens) + 1, dtype=torch.int32, device="cuda") * new)
    q = (torch.randn((new * len(lens), 4 * dim), generator=g, device="cuda") * 0.3).bfloat16()
    return cache, seqs, q, k, v


def error(q, k, v, o, n, new, dim):
    """The 2-norm of the error of one sequence's outputs (a chain of new rows) beside that of the outputs."""
    logits = q.double().view(4 * new, dim) @ k[:n].t() * dim ** -0.5
    chain = torch.tril(torch.ones((new, new), dtype=torch.bool, device="cuda")).repeat_interleave(4, 0)
    logits[:, n - new:].masked_fill_(~chain, -torch.inf)
    ref = torch.softmax(logits, -1) @ v[:n]
    return ((o.double().view(4 * new, dim) - ref).norm() / ref.norm()).item()


@pytest.mark.parametrize("new", [16, 32])
@pytest.mark.parametrize("lens", [[1 << 20] * 148, [1 << 20] * 60, [65536, 65408, 65537, 131072, 131073, 200001, 65664, 131200, 300000, 17000] * 30, [3000000]])
@pytest.mark.parametrize("values", ["either sign", "one sign"])
def test_sums_over_very_long_sequences_do_not_drift(ctx, new, lens, values):  # noqa: F811
    """Up to 65536 keys are summed in one piece.  Each of its 4096 steps may be cut off by 2^-23 of what the sum has come to, which grows evenly: 2.4e-4 of the whole,
    for outputs and sums of P together twice that at most, beside the 2^-9 sqrt(1/3) and less that the output's rounding has as its 2-norm: together
    less than 2^-9 (in one piece a million keys came to 0.0029)."""
    from paper_2607_28418_b200 import binding
    dim = 64
    cache, seqs, q, k, v = long_case(ctx, lens, new, dim, len(lens) + new, (lambda x: x) if values == "either sign" else (lambda x: x.abs()))
    bits = binding.tree_ancestors(list(range(-1, new - 1))).cuda().repeat(len(lens), 1)
    o = binding.wide_attn_tree(ctx, q, cache, seqs, 4, 4, bits)
    again = binding.wide_attn_tree(ctx, q, cache, seqs, 4, 4, bits)
    assert torch.isfinite(o).all() and torch.equal(o, again)
    for s in sorted({0, 1, 5, 8, len(lens) // 2, len(lens) - 1} & set(range(len(lens)))):
        rows = slice(new * s, new * s + new)
        assert error(q[rows], k, v, o[rows], lens[s], new, dim) < 2.0 ** -9
