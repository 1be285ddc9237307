"""wide_status with more than one thing to report."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_bad_index_is_not_lost_behind_an_expired_wait():
    """Both reports come, one a call, whichever was first; in between and after, calls run as usual."""
    from paper_2607_28418_b200 import binding
    ctx = binding.Context(0)
    try:
        ctx.set_wait_limit_ns(1_000_000)
        cache = binding.Cache.empty(2, 1, 64, 64, 16)
        lens = torch.tensor([1], dtype=torch.int32, device="cuda")
        good = binding.Sequences(torch.tensor([[1]], dtype=torch.int32, device="cuda"), lens)
        bad = binding.Sequences(torch.tensor([[7]], dtype=torch.int32, device="cuda"), lens)
        row = torch.full((1, 64), 3.0, dtype=torch.bfloat16, device="cuda")
        for first in ("wait", "index"):
            if first == "wait":
                ctx.selftest_wait()
            binding.wide_cache_write(ctx, cache, bad, row, row)
            if first == "index":
                ctx.selftest_wait()
            binding.wide_cache_write(ctx, cache, good, row, row)
            assert ctx.status() == binding.ERR_TIMEOUT
            assert ctx.status() == binding.ERR_BAD_INDEX
            assert ctx.status() == 0
            k, v = binding.wide_cache_read(ctx, cache, good, 1)
            assert torch.equal(k, row) and torch.equal(v, row)
    finally:
        ctx.close()
