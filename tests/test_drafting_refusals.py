"""Refusals of wide_cache_append, wide_attn_tree and wide_linear: found on the host, before any launch and before the device is asked
for, so they are the same without a GPU; and the bits of a tree."""
import ctypes

import numpy as np
import pytest

P = 1 << 20          # an aligned address that is never followed
FAKE = (ctypes.c_ubyte * 4096)()   # stands for a context: a refused call does not look into it


@pytest.fixture(scope="module")
def lib():
    from paper_2607_28418_b200 import binding, build
    build.build()
    return binding.load_library()


def places(heads=2, dim=64, seqs=3, row_start=P, pages=P, quant=64, page=16, table=P, max_pages=3, n_pages=4):
    from paper_2607_28418_b200 import binding
    return (ctypes.byref(binding._CacheStruct(pages, n_pages, page, heads, dim, quant)),
            ctypes.byref(binding._SeqsStruct(table, P, row_start, seqs, max_pages)))


APPEND = dict(ctx=FAKE, q=P, k=2 * P, v=3 * P, dtype=0, rows=8, heads=4, rot=64, qs=256, ks=128, vs=128, pos=P, axes=1, inv=P, axis=None, out=4 * P,
              os=256, flags=0)


def append(lib, where=None, **kw):
    a = dict(APPEND, **kw)
    return lib.wide_cache_append(a["ctx"], None, *(where or places()), a["q"], a["k"], a["v"], a["dtype"], a["rows"], a["heads"], a["rot"], a["qs"],
                                 a["ks"], a["vs"], a["pos"], a["axes"], a["inv"], a["axis"], a["out"], a["os"], a["flags"])


INVALID, SHAPE, ALIGNMENT, WORKSPACE = -1, -2, -3, -4


@pytest.mark.parametrize("change", [dict(ctx=None), dict(k=None), dict(v=None), dict(pos=None), dict(inv=None), dict(dtype=2), dict(rows=-1), dict(heads=-1), dict(rot=0),
                                    dict(axes=0), dict(q=None), dict(out=None), dict(heads=0), dict(flags=512), dict(flags=1), dict(flags=256 | 512),
                                    dict(qs=255), dict(ks=127), dict(vs=64), dict(os=128), dict(out=APPEND["q"], os=264), dict(out=APPEND["k"]),
                                    dict(out=APPEND["v"])])
def test_append_refuses_arguments(lib, change):
    assert append(lib, **change) == INVALID


@pytest.mark.parametrize("change", [dict(rot=24), dict(rot=80), dict(axes=9), dict(heads=4097, qs=1 << 20, os=1 << 20), dict(rows=(1 << 27) + 1)])
def test_append_refuses_shapes(lib, change):
    assert append(lib, **change) == SHAPE


@pytest.mark.parametrize("change", [dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=4 * P + 8), dict(qs=257), dict(ks=129), dict(vs=132), dict(os=260),
                                    dict(dtype=1, ks=130)])
def test_append_refuses_rows_off_16_bytes(lib, change):
    assert append(lib, **change) == ALIGNMENT


@pytest.mark.parametrize("where,code", [(dict(pages=None), INVALID), (dict(n_pages=0), INVALID), (dict(table=None), INVALID), (dict(max_pages=0), INVALID),
                                        (dict(page=24), SHAPE), (dict(page=512), SHAPE), (dict(quant=48), SHAPE), (dict(quant=128), SHAPE), (dict(dim=96), SHAPE),
                                        (dict(seqs=4097), SHAPE), (dict(heads=257), SHAPE), (dict(pages=P + 8), ALIGNMENT), (dict(seqs=9, row_start=None), INVALID)])
def test_append_and_tree_refuse_places(lib, where, code):
    assert append(lib, places(**where)) == code
    assert tree(lib, places(**where)) == code


def test_append_without_queries(lib):
    """Keys and values alone are a call of their own: refused here for the key's alignment only."""
    assert append(lib, q=None, out=None, heads=0, qs=0, os=0, k=P + 2) == ALIGNMENT


@pytest.mark.parametrize("heads,rows", [(256, 1 << 27), (255, 1 << 27)])
def test_append_counts_its_blocks(lib, heads, rows):
    many = (rows // 16 + 2) * heads > 2 ** 31 - 1
    got = append(lib, places(heads=heads, seqs=1), rows=rows, k=P + 2, ks=heads * 64, vs=heads * 64)
    assert got == (SHAPE if many else ALIGNMENT) and many == (heads == 256)


TREE = dict(ctx=FAKE, q=P, dtype=0, rows=8, qs=256, heads=4, per=2, mask=P, bits=P, words=2, o=2 * P, ws=P, ws_bytes=1 << 40, flags=0)


def tree(lib, where=None, **kw):
    a = dict(TREE, **kw)
    return lib.wide_attn_tree(a["ctx"], None, *(where or places()), a["q"], a["dtype"], a["rows"], a["qs"], a["heads"], a["per"], a["mask"], a["bits"],
                              a["words"], 0.0, a["o"], a["ws"], a["ws_bytes"], a["flags"])


@pytest.mark.parametrize("change,code", [(dict(ctx=None), INVALID), (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(bits=None), INVALID), (dict(words=0), INVALID),
                                         (dict(words=9), SHAPE), (dict(dtype=1), SHAPE), (dict(dtype=3), INVALID), (dict(rows=-1), INVALID), (dict(heads=0), INVALID),
                                         (dict(heads=5), INVALID), (dict(per=0), INVALID), (dict(per=3), INVALID), (dict(flags=1), INVALID), (dict(qs=255), INVALID),
                                         (dict(qs=257), ALIGNMENT), (dict(q=P + 8), ALIGNMENT), (dict(o=2 * P + 8), ALIGNMENT), (dict(ws=P + 8), ALIGNMENT),
                                         (dict(ws=None), WORKSPACE), (dict(ws_bytes=1 << 20), WORKSPACE), (dict(o=TREE["q"]), INVALID),
                                         (dict(heads=4096, per=4096, rows=(1 << 18) + 1, qs=1 << 18), SHAPE)])
def test_tree_refuses(lib, change, code):
    from paper_2607_28418_b200 import binding
    assert binding.attn_tree_workspace_bytes() > 1 << 20
    assert tree(lib, **change) == code


LINEAR = dict(ctx=FAKE, x=P, dtype=0, tokens=4, k=64, xs=64, w=2 * P, n=10, bias=3 * P, act=0, res=4 * P, rs=16, y=5 * P, out=0, ys=16, flags=0)


def linear(lib, **kw):
    a = dict(LINEAR, **kw)
    return lib.wide_linear(a["ctx"], None, a["x"], a["dtype"], a["tokens"], a["k"], a["xs"], a["w"], a["n"], a["bias"], a["act"], a["res"], a["rs"], a["y"],
                           a["out"], a["ys"], a["flags"])


@pytest.mark.parametrize("change,code", [(dict(ctx=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID), (dict(dtype=1), SHAPE),
                                         (dict(dtype=2), INVALID), (dict(out=2), INVALID), (dict(tokens=-1), INVALID), (dict(k=0), INVALID), (dict(n=0), INVALID),
                                         (dict(act=-1), INVALID), (dict(act=4), INVALID), (dict(flags=1), INVALID), (dict(k=60), SHAPE), (dict(xs=56), INVALID),
                                         (dict(ys=8), INVALID), (dict(rs=8), INVALID), (dict(xs=68), ALIGNMENT), (dict(ys=20), ALIGNMENT), (dict(rs=20), ALIGNMENT),
                                         (dict(x=P + 8), ALIGNMENT), (dict(w=2 * P + 8), ALIGNMENT), (dict(bias=3 * P + 4), ALIGNMENT), (dict(y=5 * P + 8), ALIGNMENT),
                                         (dict(res=4 * P + 8), ALIGNMENT), (dict(y=LINEAR["x"]), INVALID), (dict(y=LINEAR["w"]), INVALID), (dict(y=LINEAR["bias"]), INVALID),
                                         (dict(res=LINEAR["y"], rs=24), INVALID), (dict(tokens=(1 << 27) + 1), SHAPE), (dict(n=(1 << 27) + 1, ys=1 << 28, rs=1 << 28), SHAPE),
                                         (dict(k=1 << 28, xs=1 << 28), SHAPE), (dict(xs=1 << 40), SHAPE), (dict(out=1, ys=18), ALIGNMENT)])
def test_linear_refuses(lib, change, code):
    assert linear(lib, **change) == code


def test_the_bits_of_a_tree():
    from paper_2607_28418_b200 import binding
    bits = binding.tree_ancestors([-1, 0, 0, 1, -1, 3, 2])
    assert bits.dtype.is_signed and bits.shape == (7, 1)
    assert bits[:, 0].tolist() == [1, 0b11, 0b101, 0b1011, 0b10000, 0b101011, 0b1000101]
    chain = binding.tree_ancestors(list(range(-1, 69)))
    assert chain.shape == (70, 3)
    seen = chain.numpy().view(np.uint32)
    for i in range(70):
        assert [(int(seen[i, j // 32]) >> (j % 32)) & 1 for j in range(96)] == [int(j <= i) for j in range(96)]
    assert binding.tree_ancestors([], 2).shape == (0, 2)
    for wrong in ([0], [-2], [-1, 1], [-1, 2, 0]):
        with pytest.raises(ValueError):
            binding.tree_ancestors(wrong)
    with pytest.raises(ValueError):
        binding.tree_ancestors(list(range(-1, 32)), 1)
