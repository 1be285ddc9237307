"""CPU oracle of the 4-bit cache, the attention over it and the rotary positions: numpy, 64 bits and
more, written from the definitions in include/wide.h.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

from paper_2607_28418_b200 import synth

BORDERS = np.arange(15) + 0.5


def bf16_toward(x: np.ndarray, up: bool) -> np.ndarray:
    """The nearest bf16 number at or above (up) or at or below x, as float64."""
    x = np.asarray(x, dtype=np.longdouble)
    _, e = np.frexp(x.astype(np.float64))
    unit = np.ldexp(np.longdouble(1), np.maximum(e, -125) - 8)   # spacing; bf16 subnormals are 2^-133 apart
    n = x / unit
    return ((np.ceil(n) if up else np.floor(n)) * unit).astype(np.float64)


def reaches(y, a, b):
    """y >= a + b, exactly: the sum is rounded to 64 bits of mantissa, and where y equals it the rounding's exact remainder decides."""
    t = a + b
    v = t - a
    rest = (a - (t - v)) + (b - v)
    return (y > t) | ((y == t) & (rest <= 0))


def quantise(x: np.ndarray, group: int):
    """x [..., dim] (bf16- or fp32-representable) -> codes uint8 [..., dim], scale and minimum float64
    [..., dim / group] (NaN where the sub-group is not finite)."""
    y = np.asarray(x, dtype=np.longdouble).reshape(*x.shape[:-1], -1, group)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0, y)
    m = bf16_toward(y.min(-1), up=False) + 0.0     # a zero minimum is +0
    m80 = m.astype(np.longdouble)
    s = bf16_toward((y.max(-1) - m80) / np.longdouble(15), up=True) + 0.0
    # the quotient is rounded, so the scale is checked by its last level
    short = reaches(y.max(-1), m80, 15 * s.astype(np.longdouble)) & ~reaches(-y.max(-1), -m80, -15 * s.astype(np.longdouble))
    s = np.where(short, bf16_toward(s * (1 + 2.0 ** -12), up=True), s)
    n = np.zeros(y.shape, dtype=np.uint8)
    for b in BORDERS:
        n += reaches(y, m80[..., None], (np.longdouble(b) * s.astype(np.longdouble))[..., None]) & (s[..., None] > 0)
    s, m = np.where(bad, np.nan, s), np.where(bad, np.nan, m)
    return n.reshape(x.shape), s, m


def held(x: np.ndarray, group: int) -> np.ndarray:
    """The values the cache holds for x, computed in float32 with one rounding."""
    n, s, m = quantise(x, group)
    y = m[..., None].astype(np.longdouble) + s[..., None].astype(np.longdouble) * n.reshape(*s.shape, group)
    return y.astype(np.float32).reshape(x.shape)


def word(s: np.ndarray, m: np.ndarray) -> np.ndarray:
    sb = np.where(np.isnan(s), 0x7FC0, np.ascontiguousarray(np.nan_to_num(s).astype(np.float32)).view(np.uint32) >> 16)
    mb = np.where(np.isnan(m), 0x7FC0, np.ascontiguousarray(np.nan_to_num(m).astype(np.float32)).view(np.uint32) >> 16)
    return (sb | (mb << 16)).astype(np.uint32)


def code_place(r: int, d: int, values: bool):
    """(byte within the code area, nibble) of token r of a block and channel d."""
    if values:
        return ((((d // 64 * 8 + d // 4 % 8) * 4 + r // 2 % 4) * 2 + d // 32 % 2) * 2 + d // 2 % 2) * 4 + r % 2 * 2 + r // 8, d % 2
    return ((((d // 64 * 8 + r % 8) * 4 + d // 8 % 4) * 2 + d // 32 % 2) * 2 + d // 4 % 2) * 4 + d % 2 * 2 + r // 8, d // 2 % 2


def store(pages: np.ndarray, page_size: int, group: int, table, length: int, k: np.ndarray, v: np.ndarray):
    """Write the last k.shape[0] positions of one sequence: pages uint8 [n_pages, heads, page_size / 16,
    block] (changed in place), k and v [n, heads, dim]; page numbers out of range drop their tokens."""
    n, heads, dim = k.shape
    ns = dim // group
    for which, x in ((False, k), (True, v)):
        codes, s, m = quantise(x, group)
        words = word(s, m)
        at = np.array([[code_place(r, d, which) for d in range(dim)] for r in range(16)])
        base, wbase = (8 * dim, 16 * dim + 64 * ns) if which else (0, 16 * dim)
        for i in range(n):
            p = length - n + i
            page = int(table[p // page_size])
            if not 0 <= page < pages.shape[0]:
                continue
            r = p % 16
            for h in range(heads):
                block = pages[page, h, p % page_size // 16]
                byte, nibble = at[r, :, 0] + base, at[r, :, 1]
                for nib in (0, 1):
                    b = byte[nibble == nib]
                    keep = 0xF0 if nib == 0 else 0x0F
                    block[b] = (block[b] & keep) | (codes[i, h][nibble == nib] << (4 * nib))
                block[wbase + r * 4 * ns: wbase + (r + 1) * 4 * ns] = words[i, h].astype("<u4").view(np.uint8)


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, on: np.ndarray, heads_per_group: int, causal: bool, scale: float,
              lost=()) -> np.ndarray:
    """One sequence in float64: q [n, n_q_heads, dim] at the last n of the L positions of k, v [L, heads, dim]; on [n, n_groups];
    positions in `lost` are seen by nobody.  Inactive pairs and rows without keys are zero."""
    n, hq, dim = q.shape
    L, hkv, _ = k.shape
    out = np.zeros((n, hq, dim))
    live = np.ones(L, dtype=bool)
    live[list(lost)] = False
    for i in range(n):
        see = live & (np.arange(L) <= (L - n + i if causal else L - 1))
        if not see.any():
            continue
        for h in range(hq):
            if not on[i, h // heads_per_group]:
                continue
            kh, vh = k[see, h // (hq // hkv)].astype(np.float64), v[see, h // (hq // hkv)].astype(np.float64)
            z = kh @ q[i, h].astype(np.float64) * scale
            p = np.exp(z - z.max())
            out[i, h] = p @ vh / p.sum()
    return out


def rope(x: np.ndarray, positions: np.ndarray, inv_freq, axis, interleaved: bool, inverse: bool) -> np.ndarray:
    """x [T, heads, dim] float64; the angle is reduced in extended precision before its sine is taken."""
    half = len(inv_freq)
    y = np.array(x, dtype=np.float64)
    two_pi = np.longdouble(2) * np.longdouble("3.14159265358979323846264338327950288")
    for i in range(half):
        a = np.fmod(positions[axis[i]].astype(np.longdouble) * np.longdouble(inv_freq[i]), two_pi).astype(np.float64)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None] * (-1 if inverse else 1)
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        u, w = x[:, :, lo].astype(np.float64), x[:, :, hi].astype(np.float64)
        y[:, :, lo], y[:, :, hi] = u * c - w * s, u * s + w * c
    return y


def attention_tolerance(ref: np.ndarray, q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float) -> np.ndarray:
    """What wide_attn_cache may be off by.  The output is rounded to bf16: 2^-8 |o|.  Probabilities enter the
    product as fp16 times the step of a value, so each p s n is off by 2^-11 of itself, which sums to 2^-11 of
    the largest |s n| <= 2 max |v|; the fp32 sums of p s n and p m, of p, and their joining are covered by another 2^-11.
    A logit is an fp32 sum of dim products, off by (dim + 16) 2^-23 sum |q k| at most, the minimum's
    part m sum q included (|m| and |s n| are both at most 2 max |k|, hence the 4); p moves by that much, o by twice that times max |v|."""
    if v.size == 0:
        return np.zeros_like(ref)
    dim = q.shape[-1]
    vmax = float(np.abs(v).max())
    logits = float(np.abs(q).sum(-1).max()) * float(np.abs(k).max()) * scale
    return 2.0 ** -8 * np.abs(ref) + 4 * 2.0 ** -11 * vmax + 2 * vmax * 4 * (dim + 16) * 2.0 ** -23 * logits


def attention_with_bound(q: np.ndarray, k: np.ndarray, v: np.ndarray, group: int, on: np.ndarray, heads_per_group: int, causal: bool = True,
                         scale: float = 0.0, lost=(), blocks: int = 2):
    """`attention` of one sequence whose cache was written from k and v [L, heads, dim], with a bound for every output element that
    counts only what the row itself weighs: (o, bound) [n, n_q_heads, dim].  `blocks`: 16-key blocks that one warp takes at most.
    With the natural logits z, p = exp(z - max z) and l = sum p, a value m + s c (code c) and an output o, wide_attn_cache may be off by
      - the output's rounding to bf16: 2^-8 |o|
      - weighed steps p s in fp16: half a unit, 2^-11 of each, or 2^-27 of the row's and sub-group's largest where that is more (its
        product is 2^2 at least and the smallest fp16 numbers are 2^-24 apart), never more than p s itself; each times |c - 8|
      - fp32 sums of p s (c - 8): the tensor core adds at most c + 16 c' + 8 * 17 < 400 times p s (c' the code that shares the byte)
        to a sum and is off by 2^-22 of it at most each time; a block is two such additions, and eight fp32 ones join the parts
      - fp32 sums of p (m + 8 s): every lane adds two keys a block, then five lanes and the parts are joined; 2^-24 each
      - logits: sum_d q (s c + m) is added by the tensor core in dim / 16 <= 8 steps (2^-22 each), the sum of the queries beside the
        minimum in 34 (2^-24 each), and six roundings join them: below 48 * 2^-23 of sum_d |q| (s c + |m|) times scale
      - exponentials: 2^-22 of their own and of the joining, 2^-24 of the argument: with the logits' part each p is off by a share eps, and o by
        sum p eps |v - o| / l.
    The sum is rounded up by 2 % for products of these."""
    n, hq, dim = q.shape
    L, hkv, _ = k.shape
    scale = scale if scale > 0 else dim ** -0.5
    out, bound = np.zeros((n, hq, dim)), np.zeros((n, hq, dim))
    if L == 0:
        return out, bound

    def parts(x):
        c, s, m = quantise(x, group)
        return c.astype(np.float64), *(np.repeat(y.astype(np.float64), group, -1) for y in (s, m))
    kc, ks, km = parts(k)
    vc, vs, vm = parts(v)
    kh, vh = km + ks * kc, vm + vs * vc
    ka = np.abs(km) + ks * kc
    live = np.ones(L, dtype=bool)
    live[list(lost)] = False
    for i in range(n):
        see = live & (np.arange(L) <= (L - n + i if causal else L - 1))
        if not see.any():
            continue
        for h in range(hq):
            if not on[i, h // heads_per_group]:
                continue
            a = h // (hq // hkv)
            x = q[i, h].astype(np.float64)
            z = kh[see, a] @ x * scale
            eps = 48 * 2.0 ** -23 * (ka[see, a] @ np.abs(x)) * scale + 2.0 ** -20 + 2.0 ** -23 * (z.max() - z)
            p = np.exp(z - z.max())
            l, s, c, m, y = p.sum(), vs[see, a], vc[see, a], vm[see, a], vh[see, a]
            o = p @ y / l
            w = p[:, None] * s
            step = np.minimum(w, np.maximum(2.0 ** -11 * w, 2.0 ** -27 * w.max(0)))
            off = 2.0 ** -8 * np.abs(o) + (step * np.abs(c - 8)).sum(0) / l
            off += (2 * blocks + 2) * 2.0 ** -22 * 400 * w.sum(0) / l + (2 * blocks + 40) * 2.0 ** -24 * (p @ np.abs(m + 8 * s)) / l
            off += (p * eps) @ np.abs(y - o) / l
            out[i, h], bound[i, h] = o, 1.02 * off
    return out, bound


def round_bf16(x: np.ndarray) -> np.ndarray:
    return synth.round_to_bf16(np.asarray(x, dtype=np.float32))
