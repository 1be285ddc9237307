"""Pins of the cache oracle, and the refusals of the calls on a cache and of wide_rope (no GPU)."""
import ctypes
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from tests.cache_util import CacheCase


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("values", [False, True])
def test_every_code_has_a_place_of_its_own_and_tokens_share_no_byte(dim, values):
    places = {(r, d): co.code_place(r, d, values) for r in range(16) for d in range(dim)}
    assert len(set(places.values())) == 16 * dim
    assert max(b for b, _ in places.values()) == 8 * dim - 1
    owner = {}
    for (r, _), (b, _) in places.items():
        assert owner.setdefault(b, r) == r


def test_quantise_hand_worked():
    # min -1, max 2: scale 3 / 15 = 0.2, the next bf16 above is 0.2001953125
    x = np.array([-1.0, 2.0, 0.0, -0.9] + [-1.0] * 28, dtype=np.float32)
    n, s, m = co.quantise(x[None], 32)
    assert m[0, 0] == -1.0 and s[0, 0] == 0.2001953125
    assert list(n[0, :4]) == [0, 15, 5, 0]       # (0 + 1) / s = 4.995, (-0.9 + 1) / s = 0.4995
    # a value on a border belongs to the level above
    x = np.array([0.0, 15.0, 0.5, 1.5, 2.4921875] + [0.0] * 27, dtype=np.float32)
    n, s, m = co.quantise(x[None], 32)
    assert s[0, 0] == 1.0 and list(n[0, :5]) == [0, 15, 1, 2, 2]
    # constant, and not finite
    n, s, m = co.quantise(np.full((1, 32), 3.5, np.float32), 32)
    assert s[0, 0] == 0 and m[0, 0] == 3.5 and not n.any()
    y = co.held(np.array([[np.inf] + [0.0] * 31 + [1.0] * 32], np.float32), 32)
    assert np.isnan(y[0, :32]).all() and (y[0, 32:] == 1).all()


@pytest.mark.parametrize("scale", [1e-38, 1e-20, 1.0, 1e30])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_held_values_are_within_half_a_step(scale, group):
    rng = np.random.default_rng(1)
    x = co.round_bf16(rng.standard_normal((50, 128)) * scale)
    n, s, m = co.quantise(x, group)
    assert n.max() <= 15 and (s >= 0).all()
    err = np.abs(co.held(x, group).astype(np.longdouble) - x).reshape(50, -1, group)
    # half a step, and the fp32 rounding of m + s n (at most 2^-24 of 16 s + |m|; 2^-150 among subnormals)
    assert (err <= s[..., None] / 2 + 2.0 ** -24 * (16 * s + np.abs(m))[..., None] + 2.0 ** -150).all()


def test_store_changes_only_its_tokens():
    c = CacheCase([21], [3], heads=1, dim=64, group=32, page=16)
    pages = c.garbage.copy()
    co.store(pages, 16, 32, c.table[0], 21, c.k[0][18:], c.v[0][18:])
    full = c.full_pages()
    mine = np.zeros_like(pages, dtype=bool)
    for r in (2, 3, 4):   # positions 18..20
        blk = mine[c.table[0, 1], 0, 0]
        for d in range(64):
            blk[co.code_place(r, d, False)[0]] = True
            blk[8 * 64 + co.code_place(r, d, True)[0]] = True
        blk[16 * 64 + r * 8:16 * 64 + r * 8 + 8] = True
        blk[16 * 64 + 128 + r * 8:16 * 64 + 128 + r * 8 + 8] = True
    assert (pages[~mine] == c.garbage[~mine]).all()
    assert (pages[mine] == full[mine]).all()


def test_oracle_attention_is_softmax_attention():
    import torch
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((5, 4, 16)), rng.standard_normal((9, 2, 16)), rng.standard_normal((9, 2, 16))
    got = co.attention(q, k, v, np.ones((5, 2), bool), 2, True, 0.25)
    tq, tk, tv = (torch.from_numpy(a).permute(1, 0, 2) for a in (q, k, v))
    allow = torch.arange(9)[None] <= torch.arange(5)[:, None] + 4
    ref = torch.nn.functional.scaled_dot_product_attention(tq, tk.repeat_interleave(2, 0), tv.repeat_interleave(2, 0), attn_mask=allow)
    np.testing.assert_allclose(got, ref.permute(1, 0, 2).numpy(), atol=1e-12)


def test_oracle_rope_rotates():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((6, 2, 64))
    pos = np.array([[0, 1, 2, 7, 100000, 999999]], dtype=np.int32)
    inv = [10000.0 ** (-2 * i / 32) for i in range(16)]
    y = co.rope(x, pos, inv, [0] * 16, False, False)
    assert (y[0] == x[0]).all() and (y[:, :, 32:] == x[:, :, 32:]).all()
    np.testing.assert_allclose(np.hypot(y[:, :, 3], y[:, :, 19]), np.hypot(x[:, :, 3], x[:, :, 19]), rtol=1e-12)
    a = math.fmod(7 * inv[3], 2 * math.pi)
    np.testing.assert_allclose(y[3, 0, 3], x[3, 0, 3] * math.cos(a) - x[3, 0, 19] * math.sin(a), rtol=1e-12)
    np.testing.assert_allclose(co.rope(y, pos, inv, [0] * 16, False, True), x, atol=1e-12)


# ------------------------------------------------------------------------------ refusals: found on the host, before any launch
@pytest.fixture(scope="module")
def lib():
    from paper_2607_28418_b200 import binding, build
    build.build()
    return binding.load_library()


P = 1 << 20          # an aligned address that is never followed
FAKE = (ctypes.c_ubyte * 4096)()   # stands for a context: a refused call does not look into it


def _cache(**kw):
    from paper_2607_28418_b200 import binding
    a = dict(pages=P, n_pages=4, page_size=16, n_kv_heads=2, head_dim=128, quant_group=64)
    a.update(kw)
    return binding._CacheStruct(*a.values())


def _seqs(**kw):
    from paper_2607_28418_b200 import binding
    a = dict(page_table=P, kv_lens=P, row_start=P, n_seqs=2, max_pages=3)
    a.update(kw)
    return binding._SeqsStruct(*a.values())


BAD_CACHES = [(dict(pages=None), -1), (dict(n_pages=0), -1), (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=512), -2),
              (dict(n_kv_heads=0), -2), (dict(n_kv_heads=257), -2), (dict(head_dim=96), -2), (dict(quant_group=16), -2),
              (dict(head_dim=64, quant_group=128), -2), (dict(pages=P + 8), -3)]
BAD_SEQS = [(dict(page_table=None), -1), (dict(kv_lens=None), -1), (dict(n_seqs=-1), -1), (dict(max_pages=0), -1), (dict(n_seqs=4097), -2),
            (dict(row_start=None, n_seqs=9), -1)]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_bad_cache_is_refused(lib, bad, code):
    args = (ctypes.byref(_cache(**bad)), ctypes.byref(_seqs()))
    for fn in (lib.wide_cache_write, lib.wide_cache_read):
        assert fn(FAKE, None, *args, P, P, 0, 8, 256, 256) == code
    assert lib.wide_attn_cache(FAKE, None, *args, P, 0, 8, 1024, 8 if bad.get("n_kv_heads") != 257 else 257, 1, P, 1, 0.0, P, P, 1 << 30, 0) == code


@pytest.mark.parametrize("bad,code", BAD_SEQS)
def test_bad_sequences_are_refused(lib, bad, code):
    args = (ctypes.byref(_cache()), ctypes.byref(_seqs(**bad)))
    for fn in (lib.wide_cache_write, lib.wide_cache_read):
        assert fn(FAKE, None, *args, P, P, 0, 8, 256, 256) == code
    assert lib.wide_attn_cache(FAKE, None, *args, P, 0, 8, 1024, 8, 4, P, 1, 0.0, P, P, 1 << 30, 0) == code


def test_bad_matrices_are_refused(lib):
    c, s = ctypes.byref(_cache()), ctypes.byref(_seqs())
    for fn in (lib.wide_cache_write, lib.wide_cache_read):
        assert fn(None, None, c, s, P, P, 0, 8, 256, 256) == -1
        assert fn(FAKE, None, None, s, P, P, 0, 8, 256, 256) == -1
        assert fn(FAKE, None, c, None, P, P, 0, 8, 256, 256) == -1
        assert fn(FAKE, None, c, s, None, P, 0, 8, 256, 256) == -1
        assert fn(FAKE, None, c, s, P, P, 7, 8, 256, 256) == -1
        assert fn(FAKE, None, c, s, P, P, 0, -1, 256, 256) == -1
        assert fn(FAKE, None, c, s, P, P, 0, 8, 255, 256) == -1          # rows overlap
        assert fn(FAKE, None, c, s, P, P, 0, 8, 256, 260) == -3          # rows 8 bytes off a boundary
        assert fn(FAKE, None, c, s, P + 4, P, 0, 8, 256, 256) == -3
        assert fn(FAKE, None, c, s, P, P, 0, 1 << 28, 256, 256) == -2

    def attn(q=P, dtype=0, rows=8, stride=1024, heads=8, per=4, o=P, ws=P, size=1 << 30, flags=0):
        return lib.wide_attn_cache(FAKE, None, c, s, q, dtype, rows, stride, heads, per, P, 1, 0.0, o, ws, size, flags)
    assert attn(q=None) == -1 and attn(o=None) == -1 and attn(dtype=5) == -1 and attn(heads=0) == -1 and attn(per=3) == -1
    assert attn(heads=9, per=3, stride=1152) == -1           # not a multiple of the KV heads
    assert attn(flags=1) == -1 and attn(stride=1023) == -1
    assert attn(dtype=1) == -2 and attn(heads=514, per=1, stride=514 * 128) == -2
    assert attn(stride=1028) == -3 and attn(o=P + 2) == -3 and attn(ws=P + 8) == -3
    assert attn(ws=None) == -4 and attn(size=16) == -4


def test_outputs_on_top_of_inputs_are_refused(lib):
    c, s = ctypes.byref(_cache()), ctypes.byref(_seqs())
    assert lib.wide_cache_read(FAKE, None, c, s, P, P, 0, 8, 256, 256) == -1
    assert lib.wide_attn_cache(FAKE, None, c, s, P, 0, 8, 1024, 8, 4, P, 1, 0.0, P, P, 1 << 30, 0) == -1


def test_bad_rope_is_refused(lib):
    def rope(q=P, k=P, dtype=0, tokens=4, hq=2, hk=1, dim=128, rot=128, qs=256, ks=128, pos=P, axes=1, inv=P, axis=None, qo=P, ko=P,
             oqs=256, oks=128):
        return lib.wide_rope(FAKE, None, q, k, dtype, tokens, hq, hk, dim, rot, qs, ks, pos, axes, inv, axis, qo, ko, oqs, oks, 0)
    assert rope(q=None) == -1 and rope(qo=None) == -1 and rope(pos=None) == -1 and rope(inv=None) == -1 and rope(dtype=2) == -1
    assert rope(k=None) == -1 and rope(ko=None) == -1 and rope(hk=0) == -1 and rope(tokens=-1) == -1 and rope(axes=0) == -1
    assert rope(dim=96) == -2 and rope(rot=24) == -2 and rope(dim=64, rot=128) == -2 and rope(axes=9) == -2
    assert rope(qs=255) == -1 and rope(oks=127) == -1 and rope(qs=512) == -1    # in place with another stride
    assert rope(q=P + 8, qo=P * 2) == -3 and rope(qs=260, qo=P * 2) == -3


def test_sizes(lib):
    from paper_2607_28418_b200 import binding
    assert binding.cache_page_bytes(64, 8, 128, 64) == 8 * 4 * (2048 + 256)
    assert binding.cache_page_bytes(16, 1, 64, 32) == 1024 + 256
    assert binding.cache_page_bytes(24, 1, 64, 32) == 0
    assert binding.attn_cache_workspace_bytes(8, 32, 8, 128) > 0 and binding.attn_cache_workspace_bytes(8, 0, 8, 128) == 0
