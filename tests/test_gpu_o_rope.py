"""wide_rope against the oracle: axes, pairings, partial rotation, far positions, gradient, strides."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from tests.cache_util import to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


def tolerance(ref, x, dtype):
    """The angle in half turns is rounded to fp32 (pi 2^-25 of a radian), sine and cosine are off by 2 units of
    2^-24, each product and the sum by one rounding: together below 8 * 2^-24 of |u| + |w|; then the output's rounding."""
    big = np.abs(x).max()
    return 8 * 2.0 ** -24 * 2 * big + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref)


def inputs(T, heads, dim, seed, dtype):
    x = np.random.default_rng(seed).standard_normal((T, heads, dim)).astype(np.float32)
    return co.round_bf16(x) if dtype == "bf16" else x


@pytest.mark.parametrize("dim,rot", [(64, 16), (64, 64), (128, 32), (128, 96), (128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 37, 1300])
def test_against_the_oracle(ctx, dim, rot, interleaved, axes, dtype, T):
    from paper_2607_28418_b200 import binding
    rng = np.random.default_rng(T + dim)
    hq, hk = (5, 2) if T < 1000 else (2, 1)
    q, k = inputs(T, hq, dim, 1, dtype), inputs(T, hk, dim, 2, dtype)
    inv = [500000.0 ** (-2 * i / rot) for i in range(rot // 2)]
    axis = rng.integers(0, axes, rot // 2).astype(np.int32)
    pos = rng.integers(0, 131072, (axes, T)).astype(np.int32)
    for inverse in (False, True):
        qo, ko = binding.wide_rope(ctx, to_device(q.reshape(T, -1), dtype), to_device(k.reshape(T, -1), dtype), torch.from_numpy(pos).cuda(),
                                   torch.tensor(inv, dtype=torch.float64, device="cuda"), axis=torch.from_numpy(axis).cuda(), head_dim=dim,
                                   interleaved=interleaved, inverse=inverse)
        for got, x in ((qo, q), (ko, k)):
            ref = co.rope(x, pos, inv, axis, interleaved, inverse)
            err = np.abs(got.float().cpu().numpy().reshape(ref.shape) - ref)
            assert (err <= tolerance(ref, x, dtype)).all(), err.max()


@pytest.mark.parametrize("offset,extra", [(0, 0), (4, 0), (0, 4), (4, 4), (8, 8)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_f32_rows_at_every_16_bytes(ctx, offset, extra, interleaved):
    """Rows on 16-byte but not on 32-byte boundaries, rotated in place: the same bits, and nothing beside them is touched."""
    from paper_2607_28418_b200 import binding
    T, heads, dim = 21, 3, 64
    x = to_device(inputs(T, heads, dim, 7, "f32").reshape(T, -1), "f32")
    dev = (torch.arange(T, dtype=torch.int32, device="cuda") * 11,
           torch.tensor([10000.0 ** (-2 * i / 48) for i in range(24)], dtype=torch.float64, device="cuda"))
    ref, _ = binding.wide_rope(ctx, x, None, *dev, head_dim=dim, interleaved=interleaved)
    flat = torch.full((offset + T * (192 + extra) + 8,), 7.0, device="cuda")
    rows = flat[offset:offset + T * (192 + extra)].view(T, 192 + extra)
    q = rows[:, :192]
    q.copy_(x)
    binding.wide_rope(ctx, q, None, *dev, head_dim=dim, interleaved=interleaved, q_out=q)
    assert torch.equal(q, ref)
    assert (rows[:, 192:] == 7).all() and (flat[:offset] == 7).all() and (flat[-8:] == 7).all()


def test_far_and_negative_positions(ctx):
    from paper_2607_28418_b200 import binding
    pos = np.array([[0, 1, -1, 999999, 2 ** 31 - 1, -2 ** 31, 16777217, 12345678]], dtype=np.int32)
    x = inputs(8, 2, 64, 3, "f32")
    inv = [1.0, 0.7, 10.0, 1e-3, 1e-9, 0.0, -0.5, 6.283185307179586] * 4
    q, k = binding.wide_rope(ctx, to_device(x.reshape(8, -1), "f32"), None, torch.from_numpy(pos).cuda(),
                             torch.tensor(inv, dtype=torch.float64, device="cuda"), head_dim=64)
    assert k is None
    ref = co.rope(x, pos, inv, [0] * 32, False, False)
    # 2^31 positions times the frequency's 2^-53 relative rounding, times 10: 2.4e-6 of a radian in the oracle's definition and here
    assert (np.abs(q.cpu().numpy().reshape(ref.shape) - ref) <= tolerance(ref, x, "f32") + 2 ** 31 * 10 * 2.0 ** -52 * np.abs(x).max()).all()


def test_gradient(ctx):
    """The rotation's transpose is its inverse: <rope(x), w> = <x, rope^-1(w)>, and by differences."""
    from paper_2607_28418_b200 import binding
    T, heads, dim = 9, 2, 64
    x, w = inputs(T, heads, dim, 4, "f32"), inputs(T, heads, dim, 5, "f32")
    pos = np.arange(T, dtype=np.int32)[None] * 17
    inv = [10000.0 ** (-2 * i / 64) for i in range(32)]
    dev = (torch.from_numpy(pos).cuda(), torch.tensor(inv, dtype=torch.float64, device="cuda"))
    grad, _ = binding.wide_rope(ctx, to_device(w.reshape(T, -1), "f32"), None, *dev, head_dim=dim, inverse=True)
    grad = grad.cpu().numpy().reshape(w.shape).astype(np.float64)

    def loss(z):
        return float((co.rope(z, pos, inv, [0] * 32, False, False) * w).sum())
    for t, h, d in [(0, 0, 0), (3, 1, 40), (8, 0, 31), (5, 1, 63)]:
        z = np.zeros_like(x, dtype=np.float64)
        z[t, h, d] = 0.5
        diff = loss(x + z) - loss(x - z)             # linear: the difference is the derivative
        assert abs(diff - grad[t, h, d]) <= 16 * 2.0 ** -24 * np.abs(w).max() + 1e-9 * abs(loss(x)) + 1e-12
    back, _ = binding.wide_rope(ctx, to_device(co.rope(x, pos, inv, [0] * 32, False, False).reshape(T, -1), "f32"), None, *dev, head_dim=dim, inverse=True)
    assert np.abs(back.cpu().numpy().reshape(x.shape) - x).max() <= 32 * 2.0 ** -24 * np.abs(x).max()


def test_in_place_strided_and_captured(ctx):
    from paper_2607_28418_b200 import binding
    T, dim = 21, 128
    q, k = inputs(T, 4, dim, 6, "bf16"), inputs(T, 2, dim, 7, "bf16")
    pos = np.random.default_rng(8).integers(0, 5000, (1, T)).astype(np.int32)
    inv = [10000.0 ** (-2 * i / 128) for i in range(64)]
    fused = torch.zeros((T, 8 * dim), dtype=torch.bfloat16, device="cuda")
    qs, ks = fused[:, :4 * dim], fused[:, 5 * dim:7 * dim]
    dev = (torch.from_numpy(pos[0]).cuda(), torch.tensor(inv, dtype=torch.float64, device="cuda"))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.wide_rope(ctx, qs, ks, *dev, head_dim=dim, q_out=qs, k_out=ks)
    for _ in range(2):
        fused.fill_(3.0)
        qs.copy_(to_device(q.reshape(T, -1)))
        ks.copy_(to_device(k.reshape(T, -1)))
        g.replay()
        for got, x in ((qs, q), (ks, k)):
            ref = co.rope(x, pos, inv, [0] * 64, False, False)
            assert (np.abs(got.float().cpu().numpy().reshape(ref.shape) - ref) <= tolerance(ref, x, "bf16")).all()
        assert (fused[:, 4 * dim:5 * dim] == 3).all() and (fused[:, 7 * dim:] == 3).all()


def test_bad_axis_and_refusals(ctx):
    from paper_2607_28418_b200 import binding
    q = to_device(inputs(3, 1, 64, 9, "bf16").reshape(3, -1))
    pos = torch.ones((2, 3), dtype=torch.int32, device="cuda")
    inv = torch.ones(32, dtype=torch.float64, device="cuda")
    axis = torch.zeros(32, dtype=torch.int32, device="cuda")
    axis[5], axis[6] = 2, -1
    out, _ = binding.wide_rope(ctx, q, None, pos, inv, axis=axis, head_dim=64)
    assert ctx.status() == binding.ERR_BAD_INDEX
    assert torch.equal(out[:, [5, 6, 37, 38]], q[:, [5, 6, 37, 38]]) and not torch.equal(out, q)
    for bad in (dict(inv_freq=inv.float()), dict(positions=pos[:, :2]), dict(positions=pos.long()), dict(axis=axis[:4]), dict(head_dim=48),
                dict(q_out=torch.empty((3, 64), device="cuda")), dict(positions=pos.cpu())):
        a = dict(q=q, k=None, positions=pos, inv_freq=inv, head_dim=64)
        a.update(bad)
        with pytest.raises(ValueError):
            binding.wide_rope(ctx, **a)
    with pytest.raises(binding.WideError):
        binding.wide_rope(ctx, q, None, pos, inv[:5].contiguous(), head_dim=64)
    assert binding.wide_rope(ctx, q[:0], None, pos[:, :0].contiguous(), inv, head_dim=64)[0].shape == (0, 64)
