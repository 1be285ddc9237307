"""What the bound of oracle.cache_oracle.attention_with_bound sees: it passes what the kernel's roundings make of the right result,
and nothing that lacks a block of keys, on the sizes that the GPU tests hold against it (no GPU)."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests.cache_util import CacheCase


def case(L, news, share, dim, group, seed=1):
    c = CacheCase([L], [news], 1, dim, group, 16, seed=seed)
    q = co.round_bf16(np.random.default_rng(2).standard_normal((news, share, dim)))
    return c, q, np.ones((news, 1), bool)


@pytest.mark.parametrize("L,news,share,blocks", [(5000, 1, 4, 2), (1777, 1, 4, 4), (3000, 1, 12, 4), (1200, 6, 4, 6)])
@pytest.mark.parametrize("dim,group", [(64, 32), (128, 64), (128, 128)])
def test_a_lost_block_of_keys_is_seen(L, news, share, blocks, dim, group):
    """Without any 16 neighbouring keys some output is off by more than twice the bound: once for the loss, once for what
    the kernel may add to it."""
    c, q, on = case(L, news, share, dim, group)
    ref, bound = co.attention_with_bound(q, c.k[0], c.v[0], group, on, share, blocks=blocks)
    k, v = (x.astype(np.float64) for x in c.held(0))
    n = (L - news) // 16
    for at in sorted({0, 1, n - 1, *range(0, n, max(1, n // 24))}):
        less = co.attention(q, k, v, on, share, True, dim ** -0.5, range(16 * at, 16 * at + 16))
        assert (np.abs(less - ref) > 2 * bound).any(), at


def test_what_the_kernel_does_is_let_through():
    """The kernel's roundings, restated: weighed steps to fp16 under a power of two that follows their largest, then bf16."""
    for dim, group, power in ((64, 32, 0), (128, 128, 0), (64, 32, 30), (128, 64, -40)):
        c, q, on = case(400, 1, 4, dim, group)
        c.v[0][50:60] = co.round_bf16(c.v[0][50:60] * 2.0 ** power)
        ref, bound = co.attention_with_bound(q, c.k[0], c.v[0], group, on, 4)
        kc, ks, km = co.quantise(c.k[0], group)
        vc, vs, vm = (x[:, 0] for x in co.quantise(c.v[0], group))
        kh = (np.repeat(km, group, -1) + np.repeat(ks, group, -1) * kc)[:, 0]
        z = q[0].astype(np.float64) @ kh.T / np.sqrt(dim)
        p = np.exp(z - z.max(-1, keepdims=True))                                      # [heads, keys]
        w = p[:, :, None] * vs                                                        # [heads, keys, sub-groups]
        up = 2.0 ** (2 - np.floor(np.log2(w.max(1, keepdims=True))))
        x = (w * up).astype(np.float16).astype(np.float64) / up
        o = np.einsum("hks,ksc->hsc", x, vc.reshape(400, -1, group) - 8.0) + np.einsum("hk,ks->hs", p, vm + 8 * vs)[..., None]
        o = co.round_bf16(o.reshape(1, 4, dim) / p.sum(-1)[None, :, None])
        assert (np.abs(o - ref) <= bound).all()


def test_it_is_the_oracle():
    c, q, on = case(100, 5, 6, 128, 64)
    on[2] = False
    k, v = (x.astype(np.float64) for x in c.held(0))
    for causal in (True, False):
        got, bound = co.attention_with_bound(q, c.k[0], c.v[0], 64, on, 6, causal, lost=[3, 4])
        want = co.attention(q, k, v, on, 6, causal, 128 ** -0.5, lost=[3, 4])
        np.testing.assert_allclose(got, want, rtol=0, atol=2.0 ** -22)       # `held` rounds m + s n to fp32
        assert (got[2] == 0).all() and (bound[2] == 0).all()
        assert (np.abs(co.round_bf16(got) - got) <= bound).all()
