"""The serving-side operators around the routed attention, as they are measured: the 4-bit key/value
cache (write, read back), the head-group-masked attention over it, and rotary positions.

``run`` computes a case with elementary torch operations where ``own`` is false and with the
framework's entry points where it is true; both work on the same buffers, the cache in the byte layout
that include/wide.h documents.

A cache is uint8 [n_pages, n_kv_heads, page_size / 16, block]; a block holds 16 tokens of one head:
8 * head_dim bytes of key codes, as many of value codes, then 16 * n_sub words of key parameters and as
many of value parameters (n_sub = head_dim / quant_group; low half the bf16 scale, high half the bf16
minimum).  A code n stands for minimum + scale * n.  Token r of a block and channel d have their code at
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
ATTN = {"op": "attn", "seqs": 1, "q_len": 1, "lo": 1, "hi": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "per_group": 4,
        "active": 4, "quant": 64, "page": 64}
STORE = {"op": "store", "seqs": 1, "q_len": 1, "lo": 1, "hi": 1, "kv_heads": 8, "head_dim": 128, "quant": 64, "page": 64, "dtype": "bf16"}
ROPE = {"op": "rope", "tokens": 1, "heads": 32, "kv_heads": 8, "head_dim": 128, "rotary": 128, "axes": 1, "interleaved": False,
        "inverse": False, "dtype": "bf16", "far": 8192}


def listed():
    return [
        # one user, the first tokens of an answer: latency of the smallest call, half of the head groups routed
        dict(ATTN, name="attn_one_short", lo=200, hi=200, page=16),
        # one user with a long document, every head group routed
        dict(ATTN, name="attn_one_32k", lo=32768, hi=32768, active=8),
        # a serving batch of uneven sequences on the 8B shape, half of the head groups routed
        dict(ATTN, name="attn_batch64_ragged", seqs=64, lo=1, hi=16384, quant=128, page=32),
        # the 13B layer's heads: no sharing of keys, 5 of 10 groups of 4 heads
        dict(ATTN, name="attn_batch16_unshared", seqs=16, lo=300, hi=2048, heads=40, kv_heads=40, active=5, quant=128),
        # a drafted answer verified: five tokens a sequence, small heads, fine quantisation, nearly all groups
        dict(ATTN, name="attn_verify5_small_heads", seqs=8, q_len=5, lo=500, hi=4096, head_dim=64, active=6, quant=32, page=16),
        # one decode step of a batch of 64 stores its keys and values (and reads them back)
        dict(STORE, name="store_step64", seqs=64, lo=1, hi=4000, page=16),
        # a prefill chunk of four sequences is stored and read back for the attention among its own tokens
        dict(STORE, name="store_chunk", seqs=4, q_len=2047, lo=2050, hi=9000),
        # a cached document read back for a prefill that attends to it
        dict(STORE, op="load", name="load_32k", lo=32768, hi=32768),
        # uneven sequences, many small heads, read into fp32
        dict(STORE, op="load", name="load_ragged_f32", seqs=7, lo=1, hi=1500, kv_heads=40, head_dim=64, quant=32, page=16, dtype="f32"),
        # queries and keys of one decode step, far positions
        dict(ROPE, name="rope_step64", tokens=64, far=1000000),
        # a prompt of text, pictures and video: time, height and width
        dict(ROPE, name="rope_prompt_3axes", tokens=16384, heads=40, kv_heads=40, axes=3),
        # the gradient of the rotation, fp32, neighbouring channels paired, part of the head rotated
        dict(ROPE, name="rope_gradient_f32", tokens=4099, inverse=True, dtype="f32", interleaved=True, rotary=64),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["attn", "attn", "attn", "store", "load", "rope"])
    dim = rng.choice([64, 128, 128])
    quant = rng.choice([q for q in (32, 64, 128) if q <= dim])
    page = rng.choice([16, 32, 64, 128])
    if op == "attn":
        kv = rng.choice([2, 5, 8, 16, 40])
        share = rng.choice([1, 2, 4, 7, 8]) if kv <= 8 else 1
        seqs = log(1, 64)
        hi = max(2, min(32768, log(8, 64 * 8192 * 8 // (seqs * kv))))
        groups = kv
        return dict(ATTN, seqs=seqs, q_len=min(rng.choice([1, 1, 1, 2, 4, 7]), hi), hi=hi, lo=max(1, min(7, hi), hi // rng.choice([1, 2, 9])),
                    heads=kv * share, kv_heads=kv, head_dim=dim, per_group=share, active=rng.randint(1, groups), quant=quant, page=page)
    if op in ("store", "load"):
        kv = rng.choice([2, 5, 8, 16, 40])
        seqs = log(1, 64)
        hi = max(2, log(2, 32768 * 8 // (seqs * kv)))
        return dict(STORE, op=op, seqs=seqs, q_len=log(1, hi), hi=hi, lo=max(1, hi // rng.choice([1, 2, 9])), kv_heads=kv, head_dim=dim,
                    quant=quant, page=page, dtype=rng.choice(["bf16", "bf16", "f32"]))
    kv = rng.choice([2, 5, 8, 16])
    rotary = rng.choice([r for r in (32, 64, 128) if r <= dim])
    return dict(ROPE, tokens=log(1, 8192), heads=kv * rng.choice([1, 4, 5]), kv_heads=kv, head_dim=dim, rotary=rotary, axes=rng.choice([1, 2, 3]),
                interleaved=rng.random() < 0.5, inverse=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "f32"]), far=log(100, 1000000))


# ------------------------------------------------------------------------------ what a case fixes
def _type(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _lens(case):
    """Cache length of every sequence, spread evenly and out of order between lo and hi."""
    i = np.arange(case["seqs"])
    part = (i * 0.6180339887498949 + 0.37) % 1.0
    n = case["lo"] + np.rint(part * (case["hi"] - case["lo"])).astype(np.int64)
    if case["seqs"] == 1:
        n[:] = case["hi"]
    return np.maximum(n, 1)


def _rows(case):
    """New tokens of every sequence: the last ones of its cache (all of them for a load)."""
    n = _lens(case)
    return n if case["op"] == "load" else np.minimum(n, case["q_len"])


def _block(case):
    return 16 * case["head_dim"] + 128 * (case["head_dim"] // case["quant"])


def work(case):
    if case["op"] == "rope":
        n = case["tokens"] * (case["heads"] + case["kv_heads"])
        size = 4 if case["dtype"] == "f32" else 2
        tables = case["tokens"] * case["axes"] * 4 + case["rotary"] // 2 * 12
        return {"bytes": 2 * n * case["head_dim"] * size + tables, "flops": 3 * n * case["rotary"]}
    lens, rows, token = _lens(case), _rows(case), _block(case) / 16  # bytes of keys and values of a token and head
    tables = int(4 * (2 * case["seqs"] + 1 + np.sum(-(-lens // case["page"]))))
    if case["op"] == "attn":
        groups = case["heads"] // case["per_group"]
        share = case["active"] / groups
        used = case["kv_heads"] * (1 - (1 - share) ** rows)  # heads that any new token of the sequence uses
        io = int(rows.sum()) * (2 * 2 * case["heads"] * case["head_dim"] + 4 * ((groups + 31) // 32))
        pairs = float(np.sum(rows * lens - rows * (rows - 1) / 2))
        return {"bytes": int(np.sum(lens * used) * token) + io + tables, "flops": int(4 * pairs * case["heads"] * share * case["head_dim"])}
    size = 4 if case["dtype"] == "f32" else 2
    n = int(rows.sum()) * case["kv_heads"]
    dense, held = 2 * n * case["head_dim"] * size, int(n * token)
    both = 2 if case["op"] == "store" else 1  # stored, then read back
    return {"bytes": both * (dense + held) + tables, "flops": both * 4 * n * case["head_dim"]}


# ------------------------------------------------------------------------------ inputs
def _generator(seed, part):
    return torch.Generator(device=DEV).manual_seed(seed * 1000 + part)


def _keys_values(case, seed):
    """Keys and values [sum of lens, kv_heads * head_dim]; some key channels are offset and large, as in trained models."""
    n, width = int(_lens(case).sum()), case["kv_heads"] * case["head_dim"]
    g = _generator(seed, 1)
    big = torch.rand(width, generator=g, device=DEV) < 0.05
    offset = torch.randn(width, generator=g, device=DEV) * torch.where(big, 4.0, 0.5)
    k = torch.randn((n, width), generator=g, device=DEV).mul_(torch.where(big, 2.0, 1.0)).add_(offset).to(_type(case))
    v = torch.randn((n, width), generator=g, device=DEV).to(_type(case))
    return k, v


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
    return {"page_table": table, "kv_lens": torch.from_numpy(lens.astype(np.int32)).to(DEV), "row_start": starts, "n_pages": n_pages}


def _queries(case, seed):
    n, groups = int(_rows(case).sum()), case["heads"] // case["per_group"]
    g = _generator(seed, 3)
    q = torch.randn((n, case["heads"] * case["head_dim"]), generator=g, device=DEV).to(torch.bfloat16)
    pick = torch.rand((n, groups), generator=g, device=DEV).argsort(1) < case["active"]
    pad = torch.nn.functional.pad(pick, (0, -groups % 32)).reshape(n, -1, 32).to(torch.int64)
    bits = (pad << torch.arange(32, device=DEV)).sum(2)
    return q, torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32), pick


def _frequencies(case):
    half = case["rotary"] // 2
    inv = torch.tensor([500000.0 ** (-2.0 * i / case["rotary"]) for i in range(half)], dtype=torch.float64, device=DEV)
    axis = torch.tensor([i * case["axes"] // half for i in range(half)], dtype=torch.int32, device=DEV)
    return inv, axis


def _rope_inputs(case, seed):
    g = _generator(seed, 4)
    t, d = case["tokens"], case["head_dim"]
    q = torch.randn((t, case["heads"] * d), generator=g, device=DEV).to(_type(case))
    k = torch.randn((t, case["kv_heads"] * d), generator=g, device=DEV).to(_type(case))
    return q, k, torch.randint(0, case["far"], (case["axes"], t), generator=g, device=DEV).to(torch.int32)


def prepare(case, seed):
    if case["op"] == "rope":
        q, k, pos = _rope_inputs(case, seed)
        inv, axis = _frequencies(case)
        return {"case": case, "q": q, "k": k, "positions": pos, "inv_freq": inv, "axis": axis}
    state = {"case": case, "rows": int(_rows(case).sum()), **_places(case, seed)}
    k, v = _keys_values(case, seed)
    block = _block(case)
    state["pages"] = torch.zeros((state["n_pages"], case["kv_heads"], case["page"] // 16, block), dtype=torch.uint8, device=DEV)
    lens = state["kv_lens"].long()
    whole = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lens.cumsum(0)])
    if case["op"] == "store":
        seq, at, _ = _token_places(state["row_start"].long(), lens, state["rows"])
        state["k"], state["v"] = k[whole[seq] + at].contiguous(), v[whole[seq] + at].contiguous()
        return state
    _put(state, whole, k, v)  # the cache as the tokens before left it
    if case["op"] == "attn":
        state["q"], state["mask_bits"], _ = _queries(case, seed)
    return state


# ------------------------------------------------------------------------------ the plain forms
def _token_places(row_start, lens, rows):
    """Sequence and cache position of every row, and the sequence's first row."""
    i = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(row_start, i, right=True) - 1
    return seq, lens[seq] - (row_start[seq + 1] - i), i - row_start[seq]


def _quantise(x, quant):
    """Codes (0..15), scale and minimum of groups of `quant` channels: x [..., dim] -> [..., n_sub, quant], [..., n_sub] twice."""
    x = x.reshape(*x.shape[:-1], -1, quant).to(torch.float32)
    low = x.amin(-1)
    bits = low.view(torch.int32)
    down = torch.where(low < 0, (bits + 0xFFFF) & -0x10000, bits & -0x10000)  # minimum: next bf16 at or below
    low = down.view(torch.float32)
    wide = (x.amax(-1).double() - low.double()) / 15
    step = wide.float()
    step = torch.where(step.double() < wide, torch.nextafter(step, torch.full_like(step, math.inf)), step)
    step = ((step.view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32)  # scale: next bf16 at or above range / 15
    n = torch.floor((x.double() - low.double()[..., None]) / torch.where(step > 0, step, torch.ones_like(step)).double()[..., None] + 0.5)
    return torch.clamp(n, 0, 15).to(torch.uint8), step, low


def _words(step, low):
    """The parameter words as bytes [..., n_sub * 4]."""
    w = ((step.view(torch.int32) >> 16) & 0xFFFF) | (low.view(torch.int32) & -0x10000)
    return w.contiguous().view(torch.uint8)


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
    _put_one(flat, base, r, k.view(rows, heads, dim), quant, 0, 16 * dim, False)
    _put_one(flat, base, r, v.view(rows, heads, dim), quant, 8 * dim, 16 * dim + 64 * (dim // quant), True)


def _put_one(flat, base, r, x, quant, codes_at, words_at, values):
    dim = x.shape[-1]
    n, step, low = _quantise(x, quant)
    n = n.reshape(*x.shape)
    byte, nibble = _code_places(dim, values)
    first = torch.argsort(nibble * 100000 + byte, dim=1)  # channels in the order of their bytes: low nibbles, then high ones
    order = first[r][:, None].expand(n.shape)
    sorted_n = torch.gather(n, 2, order)
    packed = sorted_n[..., :dim // 2] | (sorted_n[..., dim // 2:] << 4)
    cells = torch.gather(byte, 1, first[:, :dim // 2])
    flat[base[..., None] + codes_at + cells[r][:, None]] = packed
    size = dim // quant * 4
    flat[base[..., None] + words_at + r[:, None, None] * size + torch.arange(size, device=DEV)] = _words(step, low)


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


def _get(state):
    """Read the rows' keys and values back, rounded to the case's type."""
    case, page = state["case"], state["case"]["page"]
    rows = state["rows"]
    seq, at, _ = _token_places(state["row_start"].long(), state["kv_lens"].long(), rows)
    # whole blocks are unpacked once, then the rows are picked
    block_at = state["page_table"].long()[seq, at // page] * (page // 16) + at % page // 16
    used, which = torch.unique(block_at, return_inverse=True)
    blocks = state["pages"].transpose(1, 2).flatten(0, 1)[used]
    k, v = _unpack(blocks, case)
    pick = lambda x: x[which, :, at % 16].reshape(rows, -1).to(_type(case))  # noqa: E731
    return pick(k), pick(v)


def _attention(state):
    case = state["case"]
    dim, kv, heads, seqs = case["head_dim"], case["kv_heads"], case["heads"], case["seqs"]
    share, page, rows = heads // kv, case["page"], state["q"].shape[0]
    lens = state["kv_lens"].long()
    blocks = state["pages"][state["page_table"].long().clamp(min=0)]       # [seqs, pages, kv, page / 16, block]
    k, v = _unpack(blocks.transpose(2, 3).flatten(1, 2), case)             # [seqs, blocks, kv, 16, dim]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))               # [seqs, kv, keys, dim]
    seq, at, place = _token_places(state["row_start"].long(), lens, rows)
    q_len = case["q_len"]
    q = torch.zeros((seqs, q_len, heads * dim), dtype=torch.float32, device=DEV)
    q[seq, place] = state["q"].float()
    q = q.view(seqs, q_len, kv, share, dim).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(dim)                # [seqs, kv, q_len * share, keys]
    last = torch.full((seqs, q_len), -1, dtype=torch.int64, device=DEV)
    last[seq, place] = at
    seen = torch.arange(k.shape[2], device=DEV) <= last[..., None]         # [seqs, q_len, keys]
    seen = seen[:, None, :, None].expand(seqs, 1, q_len, share, -1).flatten(2, 3)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    total = p.sum(-1, keepdim=True)
    seen_v = torch.where((torch.arange(k.shape[2], device=DEV) < lens[:, None])[:, None, :, None], v, torch.zeros_like(v))
    o = torch.matmul(p, seen_v) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(seqs, kv, q_len, share, dim).permute(0, 2, 1, 3, 4).reshape(seqs, q_len, heads, dim)[seq, place]
    g = torch.arange(heads, device=DEV) // case["per_group"]
    on = (state["mask_bits"][:, g // 32] >> (g % 32).to(torch.int32)) & 1
    return (o * on[..., None]).reshape(rows, -1).to(torch.bfloat16)


def _rotate(x, case, cos, sin):
    dim, rot = case["head_dim"], case["rotary"]
    t = x.shape[0]
    y = x.float().view(t, -1, dim)
    part, rest = y[..., :rot], y[..., rot:]
    a, b = (part[..., 0::2], part[..., 1::2]) if case["interleaved"] else (part[..., :rot // 2], part[..., rot // 2:])
    u, w = a * cos - b * sin, a * sin + b * cos
    part = torch.stack([u, w], -1).flatten(-2) if case["interleaved"] else torch.cat([u, w], -1)
    return torch.cat([part, rest], -1).view(t, -1).to(x.dtype)


def _rope(state):
    case = state["case"]
    angle = (state["positions"].double()[state["axis"].long()] * state["inv_freq"][:, None]).t()  # [tokens, rotary / 2]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    sin = -sin if case["inverse"] else sin
    return {"q": _rotate(state["q"], case, cos, sin), "k": _rotate(state["k"], case, cos, sin)}


# ------------------------------------------------------------------------------ the framework's calls
_contexts = {}


def _own_run(state):
    from paper_2607_28418_b200 import binding
    case = state["case"]
    if "ctx" not in _contexts:
        _contexts["ctx"] = binding.Context(torch.cuda.current_device())
    ctx = _contexts["ctx"]
    if case["op"] == "rope":
        q, k = binding.wide_rope(ctx, state["q"], state["k"], state["positions"], state["inv_freq"], axis=state["axis"],
                                 head_dim=case["head_dim"], interleaved=case["interleaved"], inverse=case["inverse"])
        return {"q": q, "k": k}
    cache = binding.Cache(state["pages"], n_kv_heads=case["kv_heads"], head_dim=case["head_dim"], quant_group=case["quant"],
                          page_size=case["page"])
    seqs = binding.Sequences(state["page_table"], state["kv_lens"], state["row_start"])
    if case["op"] == "attn":
        return {"o": binding.wide_attn_cache(ctx, state["q"], cache, seqs, case["heads"], case["per_group"], mask_bits=state["mask_bits"])}
    if case["op"] == "store":
        binding.wide_cache_write(ctx, cache, seqs, state["k"], state["v"])
    k, v = binding.wide_cache_read(ctx, cache, seqs, state["rows"], dtype=_type(case))
    return {"k": k, "v": v}


def run(state):
    if own:
        return _own_run(state)
    case = state["case"]
    if case["op"] == "rope":
        return _rope(state)
    if case["op"] == "attn":
        return {"o": _attention(state)}
    if case["op"] == "store":
        _put(state, state["row_start"], state["k"], state["v"])
    k, v = _get(state)
    return {"k": k, "v": v}


# ------------------------------------------------------------------------------ the definition in 64 bits
def _bf16_at(x, up):
    """The nearest bf16 number at or above (up) / at or below a 64-bit value, in 64 bits, by its exponent."""
    mant, exp = torch.frexp(x)
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


def exact(case, seed):
    if case["op"] == "rope":
        q, k, pos = _rope_inputs(case, seed)
        inv, axis = _frequencies(case)
        out = {}
        for name, x in (("q", q), ("k", k)):
            z = x.double().view(case["tokens"], -1, case["head_dim"]).clone()
            half = case["rotary"] // 2
            for i in range(half):
                at = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
                turn = pos[int(axis[i])].double()[:, None] * float(inv[i]) * (-1 if case["inverse"] else 1)
                w = torch.complex(z[..., at[0]], z[..., at[1]]) * torch.polar(torch.ones_like(turn), turn)
                z[..., at[0]], z[..., at[1]] = w.real, w.imag
            out[name] = z.view(case["tokens"], -1)
        return out
    k, v = _keys_values(case, seed)
    lens, rows = _lens(case), _rows(case)
    kv, dim, quant = case["kv_heads"], case["head_dim"], case["quant"]
    if case["op"] != "attn":
        ends = np.cumsum(lens)
        out = {"k": [], "v": []}
        for e, n in zip(ends, rows):
            out["k"].append(_held(k[e - n:e].view(n, kv, dim), quant).flatten(1))
            out["v"].append(_held(v[e - n:e].view(n, kv, dim), quant).flatten(1))
        return {name: torch.cat(parts) for name, parts in out.items()}
    q, _, pick = _queries(case, seed)
    share, result, a, b = case["heads"] // kv, [], 0, 0
    for n, m in zip(lens, rows):
        kk, vv = _held(k[a:a + n].view(n, kv, dim), quant), _held(v[a:a + n].view(n, kv, dim), quant)
        for i in range(m):
            z = q[b + i].double().view(kv, share, dim)
            n_seen = n - m + i + 1
            s = torch.einsum("hsd,nhd->hsn", z, kk[:n_seen]) * dim ** -0.5
            o = torch.einsum("hsn,nhd->hsd", torch.softmax(s, -1), vv[:n_seen]).reshape(case["heads"], dim)
            o = o * pick[b + i].double().repeat_interleave(case["per_group"])[:, None]
            result.append(o.flatten())
        a, b = a + n, b + m
    return {"o": torch.stack(result)}
