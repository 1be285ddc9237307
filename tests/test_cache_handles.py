"""Cache and Sequences keep the addresses of their tensors, so the tensors stay the ones they were made of (no GPU)."""
import pytest
import torch


def make():
    from paper_2607_28418_b200 import binding, build
    build.build()
    cache = binding.Cache.empty(3, 2, 64, 64, 16, device="cpu")
    seqs = binding.Sequences(torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    return cache, seqs


def test_their_parts_can_be_read():
    cache, seqs = make()
    assert cache.struct.pages == cache.pages.data_ptr() and cache.struct.n_pages == 3
    assert (cache.n_kv_heads, cache.head_dim, cache.quant_group, cache.page_size) == (2, 64, 64, 16)
    assert seqs.struct.page_table == seqs.page_table.data_ptr() and seqs.struct.kv_lens == seqs.kv_lens.data_ptr()
    assert seqs.struct.row_start == seqs.row_start.data_ptr() and seqs.n_seqs == 2
    seqs.kv_lens.fill_(7)            # in place: what a decode step does
    assert seqs.kv_lens.tolist() == [7, 7]


@pytest.mark.parametrize("name", ["page_table", "kv_lens", "row_start", "n_seqs", "struct"])
def test_sequences_refuse_another_tensor(name):
    """A tensor put in its place would be checked, but the call would use the address of the one before, which may be free."""
    _, seqs = make()
    with pytest.raises(AttributeError):
        setattr(seqs, name, getattr(seqs, name))
    with pytest.raises(AttributeError):
        delattr(seqs, name)


@pytest.mark.parametrize("name", ["pages", "n_kv_heads", "head_dim", "quant_group", "page_size", "struct"])
def test_cache_refuses_another_tensor(name):
    cache, _ = make()
    with pytest.raises(AttributeError):
        setattr(cache, name, getattr(cache, name))
    with pytest.raises(AttributeError):
        delattr(cache, name)
