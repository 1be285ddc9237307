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
