"""What a serving step with drafted tokens adds to the routed layer, as it is measured: the dense projections with
their epilogue, keys and values appended to the 4-bit cache with the position rotation applied on the way, and the
attention of a tree of drafted tokens over that cache.

``run`` computes a case with elementary torch operations where ``own`` is false and with the framework's entry points
where it is true; both work on the same buffers, the cache in the byte layout that include/wide.h documents: uint8
[n_pages, n_kv_heads, page_size / 16, block]; a block holds 16 tokens of one head: 8 * head_dim bytes of key codes, as
many of value codes, then 16 * n_sub words of key parameters and as many of value parameters (n_sub = head_dim /
quant_group; low half the bf16 scale, high half the bf16 minimum).  A code n stands for minimum + scale * n.  Token r of a
block and channel d have their code at
    keys:    byte ((((d/64 * 8 + r%8) * 4 + d/8%4) * 2 + d/32%2) * 2 + d/4%2) * 4 + d%2 * 2 + r/8,
             low nibble where d/2%2 is 0
    values:  byte ((((d/64 * 8 + d/4%8) * 4 + r/2%4) * 2 + d/32%2) * 2 + d/2%2) * 4 + r%2 * 2 + r/8,
             low nibble where d%2 is 0
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
HEADS = {"heads": 32, "kv_heads": 8, "head_dim": 128, "quant": 64, "page": 64, "seqs": 1, "new": 1, "lo": 1, "hi": 1}
TREE = dict(HEADS, op="tree", per_group=4, active=8, branch=3)
APPEND = dict(HEADS, op="append", rotary=128, axes=1, interleaved=False, dtype="bf16", branch=1)
LINEAR = {"op": "linear", "tokens": 1, "k": 4096, "n": 4096, "bias": False, "act": "none", "residual": False, "out": "bf16"}


def listed():
    return [
        # one user, a small tree right after a short prompt: latency of the smallest call, half of the head groups routed
        dict(TREE, name="tree_one_short", new=8, lo=200, hi=200, page=16, active=4),
        # one user with a long document and a tree of 61 nodes
        dict(TREE, name="tree_one_32k", new=61, lo=32768, hi=32768),
        # a serving batch: uneven sequences, 16 nodes each, most head groups routed
        dict(TREE, name="tree_batch32_ragged", seqs=32, new=16, lo=17, hi=8192, quant=128, page=32, active=6),
        # heads without sharing, small and finely quantised; wide trees
        dict(TREE, name="tree_small_heads_unshared", seqs=4, new=100, lo=500, hi=4096, heads=40, kv_heads=40, head_dim=64, per_group=1,
             active=30, quant=32, page=16, branch=8),
        # one decode step of a batch of 64: queries rotated, keys and values into the cache
        dict(APPEND, name="append_step64", seqs=64, lo=1, hi=4000, page=16),
        # drafted trees of 16 sequences: siblings share a position
        dict(APPEND, name="append_trees", seqs=16, new=61, lo=62, hi=8192, branch=3),
        # a prefill chunk of four sequences of text and pictures: three position axes
        dict(APPEND, name="append_chunk_3axes", seqs=4, new=2047, lo=2050, hi=9000, axes=3),
        # fp32, neighbouring channels paired, a quarter of the head rotated, many small heads
        dict(APPEND, name="append_ragged_f32", seqs=7, new=300, lo=1, hi=1500, heads=40, kv_heads=40, head_dim=64, rotary=16, quant=32, page=16,
             interleaved=True, dtype="f32"),
        # the fused q, k, v projection of one token, with bias
        dict(LINEAR, name="linear_qkv_one", n=6144, bias=True),
        # the output projection of 48 drafted tokens, added to the residual stream
        dict(LINEAR, name="linear_o_48", tokens=48, residual=True),
        # odd sizes and fp32 results, as a small output head has them
        dict(LINEAR, name="linear_odd_f32", tokens=333, k=1000, n=5003, bias=True, act="gelu", out="f32"),
        # a prefill of 4096 tokens through an up projection
        dict(LINEAR, name="linear_prefill", tokens=4096, n=14336, bias=True, act="silu"),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["tree", "append", "linear"])
    if op == "linear":
        k, n = 8 * log(8, 2048), log(1, 16384)
        tokens = max(1, min(8192, log(1, max(2, 4096 * 4096 * 14336 // (k * n)))))
        return dict(LINEAR, tokens=tokens, k=k, n=n, bias=rng.random() < 0.5, act=rng.choice(["none", "none", "silu", "gelu", "gelu_tanh"]),
                    residual=rng.random() < 0.4, out=rng.choice(["bf16", "bf16", "f32"]))
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([2, 5, 8, 16, 40])
    common = dict(seqs=log(1, 64), kv_heads=kv, head_dim=dim, quant=rng.choice([q for q in (32, 64, 128) if q <= dim]),
                  page=rng.choice([16, 32, 64, 128]), branch=rng.choice([1, 2, 3, 8]))
    share = rng.choice([1, 2, 4, 7, 8]) if kv <= 8 else rng.choice([1, 2])
    if op == "tree":
        hi = max(2, min(32768, log(8, 32 * 8192 * 8 // (common["seqs"] * kv))))
        new = min(log(1, max(2, min(160, 61 * 32 * 32768 // (common["seqs"] * kv * share * hi)))), hi)
        return dict(TREE, **common, new=new, hi=hi, lo=max(1, hi // rng.choice([1, 2, 9])), heads=kv * share, per_group=share,
                    active=rng.randint(1, kv))
    hi = max(2, log(2, 8192 * 8 // kv * 4 // common["seqs"]))
    return dict(APPEND, **common, hi=hi, lo=max(1, hi // rng.choice([1, 2, 9])), new=log(1, max(2, min(hi, 8188 * 8 // (common["seqs"] * kv)))),
                heads=kv * share, rotary=rng.choice([r for r in (16, 32, 48, 64, 128) if r <= dim]), axes=rng.choice([1, 1, 3]),
                interleaved=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]))


# ------------------------------------------------------------------------------ what a case fixes
def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _lens(case):
    """Cache length of every sequence, spread evenly and out of order between lo and hi."""
    part = (np.arange(case["seqs"]) * 0.6180339887498949 + 0.37) % 1.0
    n = case["lo"] + np.rint(part * (case["hi"] - case["lo"])).astype(np.int64)
    if case["seqs"] == 1:
        n[:] = case["hi"]
    return np.maximum(n, 1)


def _rows(case):
    """New tokens of every sequence: the last ones of its cache."""
    return np.minimum(_lens(case), case["new"])


def _block(case):
    return 16 * case["head_dim"] + 128 * (case["head_dim"] // case["quant"])


def _parents(case, seed):
    """For every sequence the parent of each new token (-1: the prefix).  branch 1 is a chain."""
    rng = np.random.default_rng([seed, 7])
    trees = []
    for n in _rows(case):
        i = np.arange(n)
        trees.append(i - 1 if case["branch"] == 1 else np.maximum((i - 1) // case["branch"] - rng.integers(0, 2, n), -1))
    return trees


def _tree(parents):
    """(depth of every node, which nodes it sees [n, n]): its ancestors and itself."""
    n = len(parents)
    sees = np.zeros((n, n), dtype=bool)
    depth = np.zeros(n, dtype=np.int64)
    for i, p in enumerate(parents):
        if p >= 0:
            sees[i] = sees[p]
            depth[i] = depth[p] + 1
        sees[i, i] = True
    return depth, sees


def work(case):
    if case["op"] == "linear":
        t, k, n = case["tokens"], case["k"], case["n"]
        size = 4 if case["out"] == "f32" else 2
        return {"bytes": 2 * (t * k + n * k) + t * n * size * (2 if case["residual"] else 1) + (2 * n if case["bias"] else 0),
                "flops": 2 * t * k * n}
    lens, rows, token = _lens(case), _rows(case), _block(case) / 16  # bytes of keys and values of a token and head
    tables = int(4 * (2 * case["seqs"] + 1 + np.sum(-(-lens // case["page"]))))
    if case["op"] == "tree":
        groups = case["heads"] // case["per_group"]
        share = case["active"] / groups
        used = case["kv_heads"] * (1 - (1 - share) ** rows)  # heads that any new token of the sequence uses
        words = (groups + 31) // 32 + (int(rows.max()) + 31) // 32
        io = int(rows.sum()) * (2 * 2 * case["heads"] * case["head_dim"] + 4 * words)
        pairs = float(np.sum(rows * (lens - rows) + rows))  # the prefix, and a few of the tree
        return {"bytes": int(np.sum(lens * used) * token) + io + tables, "flops": int(4 * pairs * case["heads"] * share * case["head_dim"])}
    size = 4 if case["dtype"] == "f32" else 2
    n, dim = int(rows.sum()), case["head_dim"]
    # queries in and out, keys and values in, stored, and read back as bf16
    dense = n * dim * (2 * size * (case["heads"] + case["kv_heads"]) + 4 * case["kv_heads"])
    return {"bytes": int(dense + 2 * n * case["kv_heads"] * token) + 4 * case["axes"] * n + 12 * case["rotary"] // 2 + tables,
            "flops": 3 * n * (case["heads"] + case["kv_heads"]) * case["rotary"] + 8 * n * case["kv_heads"] * dim}


# ------------------------------------------------------------------------------ inputs
def _generator(seed, part):
    return torch.Generator(device=DEV).manual_seed(seed * 1000 + part)


def _keys_values(case, seed, n):
    """Keys and values [n, kv_heads * head_dim]; some key channels are offset and large, as in trained models."""
    width = case["kv_heads"] * case["head_dim"]
    g = _generator(seed, 1)
    big = torch.rand(width, generator=g, device=DEV) < 0.05
    offset = torch.randn(width, generator=g, device=DEV) * torch.where(big, 2.0, 0.5)
    k = torch.randn((n, width), generator=g, device=DEV).add_(offset)
    return k, torch.randn((n, width), generator=g, device=DEV)


def _places(case, seed):
    """Page table, lengths and row starts, as a serving loop holds them: pages in no order, -1 where a table ends."""
    lens, rows = _lens(case), _rows(case)
    need = -(-lens // case["page"])
    n_pages = int(need.sum()) + 3
    order = torch.randperm(n_pages, generator=_generator(seed, 2), device=DEV).to(torch.int32)
    start = np.concatenate([[0], np.cumsum(need)[:-1]])
    cols = np.arange(int(need.max()))
    at = torch.from_numpy(np.minimum(start[:, None] + cols, n_pages - 1)).to(DEV)
    table = torch.where(torch.from_numpy(cols[None] < need[:, None]).to(DEV), order[at], torch.full_like(order[at], -1))
    starts = torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)).to(DEV)
    pages = torch.zeros((n_pages, case["kv_heads"], case["page"] // 16, _block(case)), dtype=torch.uint8, device=DEV)
    return {"page_table": table, "kv_lens": torch.from_numpy(lens.astype(np.int32)).to(DEV), "row_start": starts, "pages": pages,
            "rows": int(rows.sum())}


def _queries(case, seed):
    """Queries, the routed head groups as bits and as truth values, the trees as bits."""
    n, groups = int(_rows(case).sum()), case["heads"] // case["per_group"]
    g = _generator(seed, 3)
    q = torch.randn((n, case["heads"] * case["head_dim"]), generator=g, device=DEV).to(torch.bfloat16)
    pick = torch.rand((n, groups), generator=g, device=DEV).argsort(1) < case["active"]
    longest = int(_rows(case).max())
    sees = np.zeros((n, longest), dtype=bool)
    at = 0
    for p in _parents(case, seed):
        sees[at:at + len(p), :len(p)] = _tree(p)[1]
        at += len(p)
    return q, _bits(pick), pick, _bits(torch.from_numpy(sees).to(DEV))


def _bits(on):
    """Truth values [n, m] as int32 words [n, ceil(m / 32)]."""
    pad = torch.nn.functional.pad(on, (0, -on.shape[1] % 32)).reshape(on.shape[0], -1, 32).to(torch.int64)
    bits = (pad << torch.arange(32, device=DEV)).sum(2)
    return torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32)


def _append_inputs(case, seed):
    """The fused projection [rows, (heads + 2 kv_heads) * head_dim] and its tokens' positions [axes, rows]."""
    lens, rows, dim = _lens(case), _rows(case), case["head_dim"]
    n = int(rows.sum())
    q = torch.randn((n, case["heads"] * dim), generator=_generator(seed, 3), device=DEV)
    qkv = torch.cat([q, *_keys_values(case, seed, n)], 1).to(_type(case["dtype"]))
    pos = np.concatenate([m - r + _tree(p)[0] if case["branch"] > 1 else np.arange(m - r, m) for m, r, p in zip(lens, rows, _parents(case, seed))])
    far = np.stack([pos // (a + 1) for a in range(case["axes"])])  # time, then coarser axes
    return qkv, torch.from_numpy(far.astype(np.int32)).to(DEV)


def _frequencies(case):
    half = case["rotary"] // 2
    inv = torch.tensor([500000.0 ** (-2.0 * i / case["rotary"]) for i in range(half)], dtype=torch.float64, device=DEV)
    axis = torch.tensor([i * case["axes"] // half for i in range(half)], dtype=torch.int32, device=DEV)
    return inv, axis


def _linear_inputs(case, seed):
    g = _generator(seed, 4)
    t, k, n = case["tokens"], case["k"], case["n"]
    wide = (n + 7) // 8 * 8  # rows of the residual stream start on 16-byte borders
    x = torch.randn((t, k), generator=g, device=DEV).to(torch.bfloat16)
    w = torch.randn((n, k), generator=g, device=DEV).mul_(k ** -0.5).to(torch.bfloat16)
    bias = torch.randn(n, generator=g, device=DEV).to(torch.bfloat16) if case["bias"] else None
    res = torch.randn((t, wide), generator=g, device=DEV).to(_type(case["out"]))[:, :n] if case["residual"] else None
    return x, w, bias, res


def prepare(case, seed):
    if case["op"] == "linear":
        x, w, bias, res = _linear_inputs(case, seed)
        return {"case": case, "x": x, "w": w, "bias": bias, "residual": res}
    state = {"case": case, **_places(case, seed)}
    if case["op"] == "append":
        qkv, pos = _append_inputs(case, seed)
        a, b = case["heads"] * case["head_dim"], case["kv_heads"] * case["head_dim"]
        inv, axis = _frequencies(case)
        return dict(state, q=qkv[:, :a], k=qkv[:, a:a + b], v=qkv[:, a + b:], positions=pos, inv_freq=inv, axis=axis)
    whole = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), state["kv_lens"].long().cumsum(0)])
    k, v = _keys_values(case, seed, int(_lens(case).sum()))
    _put(state, whole, k.to(torch.bfloat16), v.to(torch.bfloat16))  # prefix and drafted tokens, as the calls before left them
    state["q"], state["mask_bits"], _, state["tree_bits"] = _queries(case, seed)
    return state


# ------------------------------------------------------------------------------ the plain forms
def _token_places(row_start, lens, rows):
    """Sequence and cache position of every row, and its place among the sequence's rows."""
    i = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(row_start, i, right=True) - 1
    return seq, lens[seq] - (row_start[seq + 1] - i), i - row_start[seq]


def _quantise(x, quant):
    """Codes (0..15), scale and minimum of groups of `quant` channels: x [..., dim] -> [..., n_sub, quant], [..., n_sub] twice."""
    x = x.reshape(*x.shape[:-1], -1, quant).to(torch.float32)
    low = x.amin(-1)
    bits = low.view(torch.int32)
    low = torch.where(low < 0, (bits + 0xFFFF) & -0x10000, bits & -0x10000).view(torch.float32)  # next bf16 at or below
    wide = (x.amax(-1).double() - low.double()) / 15
    step = wide.float()
    step = torch.where(step.double() < wide, torch.nextafter(step, torch.full_like(step, math.inf)), step)
    step = ((step.view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32)  # next bf16 at or above range / 15
    n = torch.floor((x.double() - low.double()[..., None]) / torch.where(step > 0, step, torch.ones_like(step)).double()[..., None] + 0.5)
    return torch.clamp(n, 0, 15).to(torch.uint8), step, low


def _code_places(dim, values):
    """Byte within the code area and nibble of (token r, channel d): two tensors [16, dim]."""
    r, d = torch.arange(16, device=DEV)[:, None], torch.arange(dim, device=DEV)[None]
    if values:
        word, pair = (((d // 64 * 8 + d // 4 % 8) * 4 + r // 2 % 4) * 2 + d // 32 % 2) * 2 + d // 2 % 2, r % 2
        return word * 4 + pair * 2 + r // 8, (d % 2).expand(16, dim)
    word, pair = (((d // 64 * 8 + r % 8) * 4 + d // 8 % 4) * 2 + d // 32 % 2) * 2 + d // 4 % 2, d % 2
    return word * 4 + pair * 2 + r // 8, (d // 2 % 2).expand(16, dim)


def _put(state, row_start, k, v):
    """Quantise rows of keys and values into the pages."""
    case, pages = state["case"], state["pages"]
    dim, quant, page = case["head_dim"], case["quant"], case["page"]
    rows, heads = k.shape[0], case["kv_heads"]
    seq, at, _ = _token_places(row_start.long(), state["kv_lens"].long(), rows)
    where = state["page_table"].long()[seq, at // page]
    base = (((where * heads)[:, None] + torch.arange(heads, device=DEV)) * (page // 16) + (at % page // 16)[:, None]) * _block(case)
    flat, r = pages.view(-1), at % 16
    _put_one(flat, base, r, k.reshape(rows, heads, dim), quant, 0, 16 * dim, False)
    _put_one(flat, base, r, v.reshape(rows, heads, dim), quant, 8 * dim, 16 * dim + 64 * (dim // quant), True)


def _put_one(flat, base, r, x, quant, codes_at, words_at, values):
    dim = x.shape[-1]
    n, step, low = _quantise(x, quant)
    n = n.reshape(*x.shape)
    byte, nibble = _code_places(dim, values)
    first = torch.argsort(nibble * 100000 + byte, dim=1)  # channels in the order of their bytes: low nibbles, then high ones
    sorted_n = torch.gather(n, 2, first[r][:, None].expand(n.shape))
    packed = sorted_n[..., :dim // 2] | (sorted_n[..., dim // 2:] << 4)
    cells = torch.gather(byte, 1, first[:, :dim // 2])
    flat[base[..., None] + codes_at + cells[r][:, None]] = packed
    size = dim // quant * 4
    words = (((step.view(torch.int32) >> 16) & 0xFFFF) | (low.view(torch.int32) & -0x10000)).contiguous().view(torch.uint8)
    flat[base[..., None] + words_at + r[:, None, None] * size + torch.arange(size, device=DEV)] = words


def _values_of(blocks, dim, quant, codes_at, words_at, values):
    """Blocks of bytes [..., block] -> the fp32 values they stand for [..., 16, dim]."""
    byte, nibble = _code_places(dim, values)
    n = (blocks[..., codes_at + byte] >> (4 * nibble).to(torch.uint8)) & 15
    size = 64 * (dim // quant)
    w = blocks[..., words_at:words_at + size].contiguous().view(torch.int32).reshape(*blocks.shape[:-1], 16, dim // quant, 1)
    step, low = (w << 16).view(torch.float32), (w & -0x10000).view(torch.float32)
    return (low + step * n.reshape(*n.shape[:-1], dim // quant, quant)).reshape(n.shape)


def _unpack(blocks, case):
    dim, quant = case["head_dim"], case["quant"]
    return (_values_of(blocks, dim, quant, 0, 16 * dim, False),
            _values_of(blocks, dim, quant, 8 * dim, 16 * dim + 64 * (dim // quant), True))


def _rotate(x, case, cos, sin):
    dim, rot = case["head_dim"], case["rotary"]
    t = x.shape[0]
    y = x.float().reshape(t, -1, dim)
    part, rest = y[..., :rot], y[..., rot:]
    a, b = (part[..., 0::2], part[..., 1::2]) if case["interleaved"] else (part[..., :rot // 2], part[..., rot // 2:])
    u, w = a * cos - b * sin, a * sin + b * cos
    part = torch.stack([u, w], -1).flatten(-2) if case["interleaved"] else torch.cat([u, w], -1)
    return torch.cat([part, rest], -1).reshape(t, -1).to(x.dtype)


def _append(state):
    case, page, rows = state["case"], state["case"]["page"], state["rows"]
    angle = (state["positions"].double()[state["axis"].long()] * state["inv_freq"][:, None]).t()  # [rows, rotary / 2]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    _put(state, state["row_start"], _rotate(state["k"], case, cos, sin), state["v"])
    seq, at, _ = _token_places(state["row_start"].long(), state["kv_lens"].long(), rows)
    # whole blocks are unpacked once, then the rows are picked
    block_at = state["page_table"].long()[seq, at // page] * (page // 16) + at % page // 16
    used, which = torch.unique(block_at, return_inverse=True)
    k, v = _unpack(state["pages"].transpose(1, 2).flatten(0, 1)[used], case)
    pick = lambda x: x[which, :, at % 16].reshape(rows, -1).to(torch.bfloat16)  # noqa: E731
    return {"q": _rotate(state["q"], case, cos, sin), "k": pick(k), "v": pick(v)}


def _attention(state):
    case = state["case"]
    dim, kv, heads, seqs = case["head_dim"], case["kv_heads"], case["heads"], case["seqs"]
    share, rows, new = heads // kv, state["rows"], int(_rows(case).max())
    lens, starts = state["kv_lens"].long(), state["row_start"].long()
    blocks = state["pages"][state["page_table"].long().clamp(min=0)]       # [seqs, pages, kv, page / 16, block]
    k, v = _unpack(blocks.transpose(2, 3).flatten(1, 2), case)             # [seqs, blocks, kv, 16, dim]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))               # [seqs, kv, keys, dim]
    seq, _, place = _token_places(starts, lens, rows)
    q = torch.zeros((seqs, new, heads * dim), dtype=torch.float32, device=DEV)
    q[seq, place] = state["q"].float()
    q = q.view(seqs, new, kv, share, dim).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(dim)                # [seqs, kv, new * share, keys]
    keys = torch.arange(k.shape[2], device=DEV)
    node = keys - (lens - (starts[1:] - starts[:-1]))[:, None]             # [seqs, keys]: negative in the prefix
    words = state["tree_bits"].long()
    at = node[seq].clamp(0, 32 * words.shape[1] - 1)
    bit = (torch.gather(words, 1, at // 32) >> (at % 32)) & 1              # [rows, keys]
    seen = torch.zeros((seqs, new, keys.numel()), dtype=torch.bool, device=DEV)
    seen[seq, place] = ((node < 0)[seq] | (bit > 0)) & (keys < lens[seq][:, None])
    seen = seen[:, None, :, None].expand(seqs, 1, new, share, -1).flatten(2, 3)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    total = p.sum(-1, keepdim=True)
    held = torch.where((keys < lens[:, None])[:, None, :, None], v, torch.zeros_like(v))
    o = torch.matmul(p, held) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(seqs, kv, new, share, dim).permute(0, 2, 1, 3, 4).reshape(seqs, new, heads, dim)[seq, place]
    g = torch.arange(heads, device=DEV) // case["per_group"]
    on = (state["mask_bits"][:, g // 32] >> (g % 32).to(torch.int32)) & 1
    return (o * on[..., None]).reshape(rows, -1).to(torch.bfloat16)


def _linear(state):
    case = state["case"]
    y = state["x"].float() @ state["w"].float().t()
    if case["bias"]:
        y = y + state["bias"].float()
    if case["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    elif case["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    elif case["act"] == "gelu_tanh":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if case["residual"]:
        y = y + state["residual"].float()
    return y.to(_type(case["out"]))


# ------------------------------------------------------------------------------ the framework's calls
_contexts = {}


def _own_run(state):
    from paper_2607_28418_b200 import binding
    case = state["case"]
    if "ctx" not in _contexts:
        _contexts["ctx"] = binding.Context(torch.cuda.current_device())
    ctx = _contexts["ctx"]
    if case["op"] == "linear":
        return {"y": binding.wide_linear(ctx, state["x"], state["w"], bias=state["bias"], activation=case["act"],
                                         residual=state["residual"], out_dtype=_type(case["out"]))}
    cache = binding.Cache(state["pages"], n_kv_heads=case["kv_heads"], head_dim=case["head_dim"], quant_group=case["quant"],
                          page_size=case["page"])
    seqs = binding.Sequences(state["page_table"], state["kv_lens"], state["row_start"])
    if case["op"] == "tree":
        return {"o": binding.wide_attn_tree(ctx, state["q"], cache, seqs, case["heads"], case["per_group"], state["tree_bits"],
                                            mask_bits=state["mask_bits"])}
    q = binding.wide_cache_append(ctx, cache, seqs, state["q"], state["k"], state["v"], state["positions"], state["inv_freq"],
                                  axis=state["axis"], interleaved=case["interleaved"])
    k, v = binding.wide_cache_read(ctx, cache, seqs, state["rows"], dtype=torch.bfloat16)
    return {"q": q, "k": k, "v": v}


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "linear":
        return {"y": _linear(state)}
    return {"o": _attention(state)} if op == "tree" else _append(state)


# ------------------------------------------------------------------------------ the definition in 64 bits
def _bf16_at(x, up):
    """The nearest bf16 number at or above (up) / at or below a 64-bit value, in 64 bits, by its exponent."""
    _, exp = torch.frexp(x)
    exp = torch.clamp(exp, min=-125)  # below: subnormal bf16 numbers, spaced 2^-133
    unit = torch.ldexp(torch.ones_like(x), exp - 8)
    n = x / unit
    return (torch.ceil(n) if up else torch.floor(n)) * unit


def _held(x, quant):
    """The 64-bit values that a cache holds for x [rows, heads, dim]."""
    y = x.double().unflatten(-1, (-1, quant))
    low = _bf16_at(y.min(-1, keepdim=True).values, False)
    step = _bf16_at((y.max(-1, keepdim=True).values - low) / 15.0, True)
    level = torch.zeros_like(y)
    for i in range(15):  # a value belongs to the level above every border that it reaches
        level += (y - low >= (i + 0.5) * step) & (step > 0)
    return (low + level * step).flatten(-2)


def _exact_linear(case, seed):
    x, w, bias, res = _linear_inputs(case, seed)
    y = torch.einsum("tk,nk->tn", x.double(), w.double())
    if bias is not None:
        y += bias.double()
    if case["act"] == "silu":
        y = y * torch.sigmoid(y)
    elif case["act"] != "none":
        y = torch.nn.functional.gelu(y, approximate="tanh" if case["act"] == "gelu_tanh" else "none")
    return {"y": y if res is None else y + res.double()}


def _exact_append(case, seed):
    qkv, pos = _append_inputs(case, seed)
    inv, axis = _frequencies(case)
    dim, a, half = case["head_dim"], case["heads"], case["rotary"] // 2
    z = qkv.double().view(qkv.shape[0], -1, dim).clone()
    turned = z[:, :a + case["kv_heads"]]
    for i in range(half):
        at = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
        turn = pos[int(axis[i])].double()[:, None] * float(inv[i])
        w = torch.complex(turned[..., at[0]], turned[..., at[1]]) * torch.polar(torch.ones_like(turn), turn)
        turned[..., at[0]], turned[..., at[1]] = w.real, w.imag
    # what is held are levels of the rotated keys as the input's type has them
    k = _held(turned[:, a:].to(qkv.dtype), case["quant"])
    v = _held(z[:, a + case["kv_heads"]:], case["quant"])
    return {"q": turned[:, :a].flatten(1), "k": k.flatten(1), "v": v.flatten(1)}


def _exact_tree(case, seed):
    lens, rows = _lens(case), _rows(case)
    kv, dim, quant = case["kv_heads"], case["head_dim"], case["quant"]
    k, v = (x.to(torch.bfloat16) for x in _keys_values(case, seed, int(lens.sum())))
    q, _, pick, _ = _queries(case, seed)
    share, result, a, b = case["heads"] // kv, [], 0, 0
    for n, m, parents in zip(lens, rows, _parents(case, seed)):
        kk, vv = _held(k[a:a + n].view(n, kv, dim), quant), _held(v[a:a + n].view(n, kv, dim), quant)
        z = q[b:b + m].double().view(m, kv, share, dim)
        s = torch.einsum("mhsd,nhd->mhsn", z, kk) * dim ** -0.5
        hidden = torch.from_numpy(~_tree(parents)[1]).to(DEV)
        s[..., n - m:].masked_fill_(hidden[:, None, None], -math.inf)
        o = torch.einsum("mhsn,nhd->mhsd", torch.softmax(s, -1), vv).reshape(m, case["heads"], dim)
        result.append((o * pick[b:b + m].double().repeat_interleave(case["per_group"], 1)[..., None]).flatten(1))
        a, b = a + n, b + m
    return {"o": torch.cat(result)}


def exact(case, seed):
    return {"linear": _exact_linear, "append": _exact_append, "tree": _exact_tree}[case["op"]](case, seed)
