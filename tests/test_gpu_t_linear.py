"""wide_linear against the product in 64 bits: token counts from one on, odd sizes, strides, epilogues."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


def make(T, k, n, bias=False, residual=None, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * T + k + n)
    x = torch.randn((T, k + pad), generator=g, device="cuda").to(torch.bfloat16)[:, :k]
    w = (torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).to(torch.bfloat16)
    b = torch.randn(n, generator=g, device="cuda").to(torch.bfloat16) if bias else None
    wide = (n + 7) // 8 * 8 + pad
    r = torch.randn((T, wide), generator=g, device="cuda").to(residual)[:, :n] if residual else None
    return x, w, b, r


def exact(x, w, b, act, r):
    """The definition in 64 bits, and the sum of the magnitudes that it adds up."""
    y = x.double() @ w.double().t()
    size = x.double().abs() @ w.double().abs().t()
    if b is not None:
        y, size = y + b.double(), size + b.double().abs()
    if act == "silu":
        y = y * torch.sigmoid(y)
    elif act == "gelu":
        y = y * 0.5 * torch.special.erfc(-y * math.sqrt(0.5))
    elif act == "gelu_tanh":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    if r is not None:
        y, size = y + r.double(), size + r.double().abs()
    return y, size


def check(got, x, w, b=None, act="none", r=None):
    """The tensor cores add 16 products at a time to an fp32 sum and lose at most 2^-23 of the sum's magnitudes each time, k / 16 times; a
    derivative of an activation is at most 1.13; the activation itself (fast exponential, quotient: 2^-21 each) adds 2^-19 of
    its result; then half a step of the type."""
    ref, size = exact(x, w, b, act, r)
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    tol = 1.13 * size * 2.0 ** -23 * (x.shape[1] / 16 + 2) + (2.0 ** -19 * size if act != "none" else 0) + half * ref.abs()
    assert torch.isfinite(got).all()
    assert ((got.double() - ref).abs() <= tol).all(), ((got.double() - ref).abs() - tol).max()


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 32, 33, 64, 65, 128, 129, 300])
@pytest.mark.parametrize("k,n", [(8, 1), (64, 128), (72, 130), (1000, 777), (4096, 4096)])
def test_sizes(ctx, T, k, n):
    from paper_2607_28418_b200 import binding
    x, w, b, _ = make(T, k, n, bias=True)
    check(binding.wide_linear(ctx, x, w, bias=b), x, w, b)


@pytest.mark.parametrize("T", [1, 48, 257])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True), (True, True)])
def test_epilogues(ctx, T, act, out, bias, residual):
    from paper_2607_28418_b200 import binding
    x, w, b, r = make(T, 256, 391, bias, out if residual else None, pad=24)
    check(binding.wide_linear(ctx, x, w, bias=b, activation=act, residual=r, out_dtype=out), x, w, b, act, r)


@pytest.mark.parametrize("T,k,n", [(1, 16384, 264), (5, 14336, 4096), (700, 4096, 1000), (2048, 1032, 2056), (4097, 512, 520)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_long_sums_and_many_tokens(ctx, T, k, n, out):
    from paper_2607_28418_b200 import binding
    x, w, b, r = make(T, k, n, True, out)
    check(binding.wide_linear(ctx, x, w, bias=b, activation="silu", residual=r), x, w, b, "silu", r)


@pytest.mark.parametrize("T", [1, 9, 40, 130])
def test_in_place_and_nothing_beside(ctx, T):
    """The sum replaces the residual; columns behind n and rows behind the last stay as they were."""
    from paper_2607_28418_b200 import binding
    x, w, b, _ = make(T, 520, 203, True)
    store = torch.randn((T + 3, 216), device="cuda").to(torch.bfloat16)
    before = store.clone()
    y = store[:T, 8:211]
    out = binding.wide_linear(ctx, x, w, bias=b, residual=y, y=y)
    assert out is y
    check(y, x, w, b, "none", before[:T, 8:211])
    store[:T, 8:211] = before[:T, 8:211]
    assert torch.equal(store, before)


@pytest.mark.parametrize("T", [1, 20, 129, 515])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
def test_far_and_missing_values(ctx, T, act):
    """An infinity or a NaN in one row of x stays in that row, one in a row of w in that column; activations of far values are their limits."""
    from paper_2607_28418_b200 import binding
    x, w, _, _ = make(T, 192, 140)
    x[0] = 0
    x[0, 0], w[:, 0], w[5, 0], w[6, 0] = 1.0, 1.0, -3e4, 3e4
    clean = binding.wide_linear(ctx, x, w, activation=act)
    assert torch.isfinite(clean).all()
    assert clean[0, 6] == torch.tensor(3e4).to(torch.bfloat16)
    assert clean[0, 5] == (-torch.tensor(3e4).to(torch.bfloat16) if act == "none" else 0)
    x[T - 1, 3], w[7, 9] = float("inf"), float("nan")
    got = binding.wide_linear(ctx, x, w, activation=act)
    assert torch.isnan(got[:, 7]).all()
    keep = [i for i in range(140) if i != 7]
    assert torch.equal(got[:T - 1, keep], clean[:T - 1, keep])
    assert not torch.isfinite(got[T - 1, keep]).any() or act != "none"


def test_same_bits_every_time_and_replayed(ctx):
    from paper_2607_28418_b200 import binding
    for T in (1, 40, 300):
        x, w, b, _ = make(T, 4096, 1536, True)
        y = binding.wide_linear(ctx, x, w, bias=b)
        out = torch.empty_like(y)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                binding.wide_linear(ctx, x, w, bias=b, y=out)
        for _ in range(5):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, y)


def test_two_calls_at_once(ctx):
    """Calls on two streams through two contexts."""
    from paper_2607_28418_b200 import binding
    other = binding.Context(0)
    x, w, b, _ = make(24, 8192, 4096, True)
    ref = binding.wide_linear(ctx, x, w, bias=b)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append(binding.wide_linear((ctx, other)[i % 2], x, w, bias=b))
    torch.cuda.synchronize()
    assert all(torch.equal(y, ref) for y in got)
    assert other.status() == 0
    other.close()


def test_no_tokens(ctx):
    from paper_2607_28418_b200 import binding
    x, w, _, _ = make(0, 64, 24)
    assert binding.wide_linear(ctx, x, w).shape == (0, 24)


@pytest.mark.parametrize("T", [1, 24, 64, 100, 200, 1500])
@pytest.mark.parametrize("k,n", [(1024, 640), (1032, 640), (2056, 1000), (4096, 2056), (16384, 136), (16384, 16500)])
def test_long_fp32_sums_do_not_drift(ctx, T, k, n):
    """fp32 outputs add their sums up in pieces of 768 products: each of the 48 steps of a piece takes less than 2^-23 of what the piece has come to, which
    grows to its end like a random walk (two thirds of it on average): 48 * 2^-24 * 2 / 3 = 1.9e-6 of a piece, and pieces add in squares like
    their losses; joining them adds 2^-24 each."""
    from paper_2607_28418_b200 import binding
    x, w, _, _ = make(T, k, n, seed=11)
    got = binding.wide_linear(ctx, x, w, out_dtype=torch.float32)
    ref, _ = exact(x, w, None, "none", None)
    assert ((got.double() - ref).norm() / ref.norm()).item() < 1.9e-6
    check(got, x, w)


@pytest.mark.parametrize("T", [3, 128, 600])
@pytest.mark.parametrize("act,residual", [("gelu", True), ("none", False)])
def test_pieces_of_a_sum_with_an_epilogue_replayed(ctx, T, act, residual):
    """Several pieces a tile and several tiles a CTA, over and over."""
    from paper_2607_28418_b200 import binding
    x, w, b, r = make(T, 5000, 20001, bias=True, residual=torch.float32 if residual else None)
    y = binding.wide_linear(ctx, x, w, bias=b, activation=act, residual=r, out_dtype=torch.float32)
    check(y, x, w, b, act, r)
    for _ in range(20):
        assert torch.equal(binding.wide_linear(ctx, x, w, bias=b, activation=act, residual=r, out_dtype=torch.float32), y)
