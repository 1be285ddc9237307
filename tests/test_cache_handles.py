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


def test_they_can_be_derived_from_and_copied():
    """A program's own handle may add what it likes, with or without slots of its own."""
    import copy

    from paper_2607_28418_b200 import binding

    class Batch(binding.Sequences):
        pass

    class Layer(binding.Cache):
        __slots__ = ("index",)
    b = Batch(torch.zeros((2, 4), dtype=torch.int32), torch.ones(2, dtype=torch.int32))
    b.names = ["a", "b"]
    b.names = ["c"]
    del b.names
    assert b.kv_lens.tolist() == [1, 1] and b.row_start is None and b.struct.n_seqs == 2
    layer = Layer.empty(3, 2, 64, 64, 16, device="cpu")
    layer.index = 7
    assert layer.index == 7 and layer.page_size == 16 and layer.struct.n_pages == 3
    b.names = ["a"]
    for one, name in ((b, "names"), (layer, "index")):
        two = copy.copy(one)
        setattr(two, name, None)
        assert getattr(one, name) is not None and two.struct is one.struct
    assert copy.copy(layer).pages is layer.pages and copy.copy(b).kv_lens is b.kv_lens
    for one, name in ((b, "kv_lens"), (layer, "pages")):
        with pytest.raises(AttributeError):
            setattr(one, name, getattr(one, name))
