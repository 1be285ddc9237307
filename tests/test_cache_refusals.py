"""Refusals of the calls on a cache and of wide_rope beyond those in test_oracle_cache.py: found on the host, before any
launch and before the device is asked for, so they are the same without a GPU."""
import ctypes

import pytest

P = 1 << 20          # an aligned address that is never followed
FAKE = (ctypes.c_ubyte * 4096)()   # stands for a context: a refused call does not look into it


@pytest.fixture(scope="module")
def lib():
    from paper_2607_28418_b200 import binding, build
    build.build()
    return binding.load_library()


def rope(lib, flags):
    """A call of an unsupported shape (heads of 96): flags are looked at before the shape, so its error tells what became of them."""
    return lib.wide_rope(FAKE, None, P, None, 0, 4, 2, 0, 96, 128, 256, 0, P, 1, P, None, 2 * P, None, 256, 0, flags)


@pytest.mark.parametrize("flags", [1, 2, 128, 1024, 1 << 31, 256 | 1024, 512 | 1])
def test_rope_refuses_flags_that_are_not_its_own(lib, flags):
    from paper_2607_28418_b200 import binding
    assert rope(lib, flags) == binding.ERR_INVALID_ARG


@pytest.mark.parametrize("flags", [0, 256, 512, 768])
def test_rope_takes_its_own_flags(lib, flags):
    from paper_2607_28418_b200 import binding
    assert rope(lib, flags) == binding.ERR_UNSUPPORTED_SHAPE


def cache_and_seqs(heads, seqs, row_start=P):
    from paper_2607_28418_b200 import binding
    return (ctypes.byref(binding._CacheStruct(P, 4, 16, heads, 64, 64)), ctypes.byref(binding._SeqsStruct(P, P, row_start, seqs, 3)))


@pytest.mark.parametrize("heads,seqs,rows", [(256, 4096, 1 << 27), (256, 1, 1 << 27), (255, 1, 1 << 27), (250, 4096, 1 << 27)])
def test_moves_whose_blocks_cannot_be_counted_in_32_bits_are_refused(lib, heads, seqs, rows):
    """rows / 16 + 2 sequences places of blocks for every head."""
    from paper_2607_28418_b200 import binding
    many = (rows // 16 + 2 * seqs) * heads > 2 ** 31 - 1
    assert many == (heads == 256)
    for fn in (lib.wide_cache_write, lib.wide_cache_read):
        # (the pointers are off a 16-byte boundary: a size that is let through ends there, before anything is launched)
        got = fn(FAKE, None, *cache_and_seqs(heads, seqs), P + 2, P + 2, 0, rows, heads * 64, heads * 64)
        assert got == (binding.ERR_UNSUPPORTED_SHAPE if many else binding.ERR_ALIGNMENT)


@pytest.mark.parametrize("heads,rows", [(4096, 1 << 19), (4096, (1 << 18) + 1), (16, 1 << 27), (4096, 1 << 18), (8, 1 << 27)])
def test_attention_with_more_query_rows_than_32_bits_count_is_refused(lib, heads, rows):
    from paper_2607_28418_b200 import binding
    got = lib.wide_attn_cache(FAKE, None, *cache_and_seqs(1, 2), P + 2, 0, rows, heads * 64, heads, heads, P, 1, 0.0, 2 * P, P, 1 << 40, 0)
    assert got == (binding.ERR_UNSUPPORTED_SHAPE if heads * rows > 1 << 30 else binding.ERR_ALIGNMENT)
