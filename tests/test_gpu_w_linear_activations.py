"""The activations of wide_linear by themselves, over their whole range: a product of one term is exact, so only the activation rounds."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TOKENS = [5, 64, 400]        # one kernel for few tokens, one for many


@pytest.fixture(scope="module")
def ctx():
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


def ladder(T):
    """T x 130 different numbers from -110 to 80, dense around 0, as x [T, 8] (a number for a token) and w [130, 8]: the product of the two is exact in
    fp32, as both are bf16."""
    n = 130
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = torch.zeros((T, 8), device="cuda"), torch.zeros((n, 8), device="cuda")
    x[:, 0] = (torch.rand(T, generator=g, device="cuda") * 1.9 - 1.1) * 2.0 ** torch.randint(-12, 1, (T,), generator=g, device="cuda")
    x[0, 0], x[T - 1, 0] = 1.0, -1.0
    w[:, 0] = torch.linspace(0.5, 100.0, n, device="cuda")
    x, w = x.bfloat16(), w.bfloat16()
    return x, w, x[:, :1].double() * w[:, 0].double()


def exact(v, act):
    """The activation in 64 bits, and z: where its lower tail is v exp(-z) or smaller."""
    if act == "silu":
        return v * torch.sigmoid(v), torch.zeros_like(v)
    if act == "gelu":
        return v * 0.5 * torch.special.erfc(-v * math.sqrt(0.5)), v * v
    z = 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    return v * torch.sigmoid(z), 3 * z.abs()


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_fp32_outputs_keep_their_digits(ctx, T, act):
    """Units of 2^-23 of the result.  SiLU, v s with s = r or e r, e = exp(-|v|) and r = 1 / (1 + e): e one, which is at most half of it in 1 + e, with half a one
    for that sum; two for the quotient, half a one for each product: below 8.  A GELU (tanh) the same with z for v, where z itself has seen six roundings of half
    a one, 3 z of the tail exp(-z).  A GELU (erf): erfc 4, its argument 1, which is v^2 + 1 of the tail, the product half a one.  Behind the smallest normal number
    (2^-126) steps are 2^-149, of erfc, e and s too, times v."""
    from paper_2607_28418_b200 import binding
    x, w, v = ladder(T)
    ref, tail = exact(v, act)
    got = binding.wide_linear(ctx, x, w, activation=act, out_dtype=torch.float32).double()
    tol = (8 + tail) * 2.0 ** -23 * ref.abs() + 2.0 ** -149 * (4 + 4 * v.abs())
    off = (got - ref).abs() - tol
    assert (off <= 0).all(), (v.flatten()[off.argmax()].item(), got.flatten()[off.argmax()].item(), ref.flatten()[off.argmax()].item())


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_bf16_outputs_keep_their_tails(ctx, T, act):
    """Half a step of bf16, beside which 2^-10 is left for the fast exponential (2 + 1.2 z units of 2^-23, z up to 130 where the result is not 0) and for z
    itself; behind the smallest normal number half a step is 2^-134, and the exponential's own steps there are 2^-149, times v."""
    from paper_2607_28418_b200 import binding
    x, w, v = ladder(T)
    ref, _ = exact(v, act)
    got = binding.wide_linear(ctx, x, w, activation=act).double()
    tol = (2.0 ** -8 + 2.0 ** -10) * ref.abs() + 2.0 ** -134 + v.abs() * 2.0 ** -147
    assert ((got - ref).abs() <= tol).all()


@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_infinities(ctx, T, act, out):
    """+inf stays; -inf stays without an activation, and with one is 0 times infinity in all three formulas: NaN.  The largest finite numbers have their limits."""
    from paper_2607_28418_b200 import binding
    x, w = torch.zeros((T, 8), device="cuda").bfloat16(), torch.zeros((6, 8), device="cuda").bfloat16()
    x[:, 0] = 1.0
    w[:, 0] = torch.tensor([math.inf, -math.inf, math.nan, 3e38, -3e38, 0.0], device="cuda")
    got = binding.wide_linear(ctx, x, w, activation=act, out_dtype=out).float()
    assert (got[:, 0] == math.inf).all()
    assert (got[:, 1] == -math.inf).all() if act == "none" else got[:, 1].isnan().all()
    assert got[:, 2].isnan().all()
    far = w[3, 0].float()
    assert (got[:, 3] == far).all() and (got[:, 4] == (-far if act == "none" else 0)).all() and (got[:, 5] == 0).all()
