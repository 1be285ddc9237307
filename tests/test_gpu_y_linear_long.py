"""wide_linear with sums of many more products than a layer has."""
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


@pytest.mark.parametrize("T", [3, 100, 130, 400])
@pytest.mark.parametrize("k", [131072, 1 << 20])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_sums_of_one_sign_do_not_drift(ctx, T, k, out):
    """What the tensor cores cut off at each of k / 16 additions has one direction in sums of one sign: less than 2^-23 of what the sum has come to, which grows evenly, so
    2^-24 k / 16 of the result in one piece, 2^-8 at a million products.  A piece has 768 products, of bf16 outputs up to 65536, and joining k / 768 of them adds
    2^-24 each in squares (six standard deviations are allowed).  So an output is what some number so near to the exact one rounds to."""
    from paper_2607_28418_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.status() == 0
    c.close()


@pytest.mark.parametrize("T", [3, 100, 130, 400])
@pytest.mark.parametrize("k", [131072, 1 << 20])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_sums_of_one_sign_do_not_drift(ctx, T, k, out):
    """What the tensor cores cut off at each of k / 16 additions has one direction in sums of one sign, up to 2^-24 of the sum each on average: 2^-8 at a million products, were they
    added in one piece.  In pieces an output's error is its rounding's, up to 2^-8 (2^-24) either way, and the average over T * 40 outputs is below
    six standard deviations, plus 48 cuts of 2^-24 a piece, and the joining's 2^-24 a piece, either way."""
    from paper_2607_28418_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(T)
    x, w = torch.rand((T, k), generator=g, device="cuda").bfloat16(), torch.rand((40, k), generator=g, device="cuda").bfloat16()
    ref = sum(x[:, i:i + 65536].double() @ w[:, i:i + 65536].double().t() for i in range(0, k, 65536))
    got = binding.wide_linear(ctx, x, w, out_dtype=out)
    near = 2.0 ** -24 * ((4096 if out == torch.bfloat16 else 48) + 6 * (k / 768) ** 0.5)
    assert (got >= (ref * (1 - near)).to(out)).all() and (got <= (ref * (1 + near)).to(out)).all()
