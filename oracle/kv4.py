"""fp64 oracle of the operators around a KV cache held in 4 bits.  TEST INFRASTRUCTURE ONLY.

The format, from its definition: a code is a sign and one of eight magnitudes; 32 channels of a key share a power of two, a
value vector has one bf16 scale; rounding is to the nearest magnitude, ties to the even code.  Codes, scales and
their layout are written out token by token; nothing is vectorised over pages on purpose.

Also here: the tables of a step (a page exchange request by request, then lists row by row) and the norm and
rotation of a head.

Pins (tests/test_oracle_kv4.py): the rounding of every midpoint written out by hand, nearest-neighbour search over all
codes, exponents at and around 6 * 2^e, packing against a hand-made block, a page exchange worked through by hand, rotations that keep
lengths and depend on differences of positions only.
"""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16_round(x):
    """float64 -> the nearest bf16, ties to even, as float64 (normal range and zeros; bf16 subnormals kept)."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(x)                                     # |m| in [1/2, 1)
    e = np.maximum(e, -125)                                # below 2^-126 the step stays
    step = np.ldexp(1.0, e - 8)
    return np.round(x / step) * step


def nearest_code(y: float) -> int:
    """Code of a value: nearest magnitude, ties to the even code; above 6: 6.  The sign is kept, also of a zero."""
    a = abs(float(y))
    d = np.abs(MAGNITUDES - a)
    best = np.flatnonzero(d == d.min())
    code = int(best[0]) if len(best) == 1 else int([c for c in best if c % 2 == 0][0])
    return code | (8 if np.signbit(y) else 0)


def code_value(code):
    code = np.asarray(code)
    return np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code & 7]


def key_exponent(group) -> int:
    """e of the smallest 2^e >= 2^-126 with |x| <= 6 * 2^e for the whole group."""
    top = float(np.abs(group).max())
    e = -126
    while top > 6.0 * 2.0 ** e:
        e += 1
    return e


def quantize_key(k):
    """[D] -> codes [D], scale bytes [D/32]."""
    k = np.asarray(k, dtype=np.float64)
    codes, scales = np.zeros(len(k), dtype=np.uint8), np.zeros(len(k) // 32, dtype=np.uint8)
    for g in range(len(k) // 32):
        x = k[32 * g:32 * g + 32]
        if not np.isfinite(x).all():
            scales[g] = 255
            continue
        e = key_exponent(x)
        scales[g] = e + 127
        codes[32 * g:32 * g + 32] = [nearest_code(np.copysign(abs(v) / 2.0 ** e, v)) for v in x]
    return codes, scales


def quantize_value(v):
    """[D] -> codes [D], scale (float64, a bf16 value or NaN)."""
    v = np.asarray(v, dtype=np.float64)
    if not np.isfinite(v).all():
        return np.zeros(len(v), dtype=np.uint8), np.nan
    s = float(bf16_round(np.abs(v).max() / 6.0))
    if s == 0.0:
        return np.array([nearest_code(np.copysign(0.0, x)) for x in v], dtype=np.uint8), 0.0
    return np.array([nearest_code(x / s) for x in v], dtype=np.uint8), s


class Cache:
    """Codes and scales by (page, head, slot, channel), and the packed arrays they stand in."""

    def __init__(self, pages, heads, page_size, dim):
        self.shape = (pages, heads, page_size, dim)
        self.k = np.zeros(self.shape, dtype=np.uint8)
        self.v = np.zeros(self.shape, dtype=np.uint8)
        self.k_scale = np.ones((pages, heads, page_size, dim // 32), dtype=np.uint8)
        self.v_scale = np.zeros((pages, heads, page_size))

    @classmethod
    def random(cls, rng, pages, heads, page_size, dim, spread=2):
        """Any codes; scales of normal values, `spread` binary orders of them."""
        c = cls(pages, heads, page_size, dim)
        c.k = rng.integers(0, 16, size=c.shape).astype(np.uint8)
        c.v = rng.integers(0, 16, size=c.shape).astype(np.uint8)
        c.k_scale = rng.integers(125 - spread // 2, 126 + (spread + 1) // 2, size=c.k_scale.shape).astype(np.uint8)
        c.v_scale = bf16_round(rng.uniform(0.2, 0.7, size=c.v_scale.shape))
        return c

    def copy(self):
        c = Cache(*self.shape)
        c.k, c.v, c.k_scale, c.v_scale = self.k.copy(), self.v.copy(), self.k_scale.copy(), self.v_scale.copy()
        return c

    def put(self, page, head, slot, k, v):
        self.k[page, head, slot], self.k_scale[page, head, slot] = quantize_key(k)
        self.v[page, head, slot], self.v_scale[page, head, slot] = quantize_value(v)

    def key_values(self):
        e = self.k_scale.astype(np.int64)
        s = np.where(e == 255, np.nan, 2.0 ** (np.minimum(e, 254) - 127.0))
        return code_value(self.k) * np.repeat(s, 32, axis=-1)

    def value_values(self):
        return code_value(self.v) * self.v_scale[..., None]

    def packed(self):
        """The arrays as the library lays them out: k_codes, k_scales, v_codes (uint8) and v_scales (bf16 bit patterns)."""
        P, H, ps, D = self.shape
        k = self.k[..., 0::2] | self.k[..., 1::2] << 4
        v = np.zeros((P, H, ps // 16, 8 * D), dtype=np.uint8)
        for slot in range(ps):
            half, e = slot % 16 // 8, slot % 8
            for ch in range(D):
                at = ((half * 32 + ch % 32) * (D // 32) + ch // 32) * 4 + e // 2
                v[:, :, slot // 16, at] |= self.v[:, :, slot, ch] << (4 * (e % 2))
        bits = (self.v_scale.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
        bits = np.where(np.isnan(self.v_scale), np.uint16(0x7fc0), bits)
        return k, self.k_scale.copy(), v, bits


def append(cache: Cache, k_new, v_new, page_indptr, page_indices, kv_len, row_indptr, verify_len, accept_len):
    """A copy of the cache with rows 0 .. accept_len[i] of every sequence committed, and the new lengths."""
    out, lens = cache.copy(), np.array(kv_len, dtype=np.int64)
    ps = cache.shape[2]
    for i in range(len(kv_len)):
        if verify_len[i] == 0:
            continue
        for j in range(int(accept_len[i]) + 1):
            pos = int(kv_len[i]) + j
            page = int(page_indices[page_indptr[i] + pos // ps])
            for h in range(cache.shape[1]):
                out.put(page, h, pos % ps, k_new[row_indptr[i] + j, h], v_new[row_indptr[i] + j, h])
        lens[i] += int(accept_len[i]) + 1
    return out, lens


def read(cache: Cache, page_indptr, page_indices, start, out_indptr):
    ps = cache.shape[2]
    k, v = cache.key_values(), cache.value_values()
    rows = [(int(page_indices[page_indptr[i] + p // ps]), p % ps)
            for i in range(len(out_indptr) - 1) for p in range(start[i], start[i] + out_indptr[i + 1] - out_indptr[i])]
    if not rows:
        return np.zeros((0, cache.shape[1], cache.shape[3])), np.zeros((0, cache.shape[1], cache.shape[3]))
    return np.stack([k[p, :, s] for p, s in rows]), np.stack([v[p, :, s] for p, s in rows])


# ---- tables of a step -------------------------------------------------------------------------
def step_tables(kv_len, verify_len, mask_rows, block_table, table_len, free_pages, free_count, page_size, mask_vis=None, mask_blocks=None):
    """Request by request, page by page.  Returns a dict of what the call writes (lists as Python lists); short: some request stayed short."""
    table, stack = np.array(block_table, dtype=np.int64), np.array(free_pages, dtype=np.int64)
    held, top, short = [int(x) for x in table_len], int(free_count), False
    B, stride = len(kv_len), table.shape[1]
    need = [min(-(-(int(kv_len[i]) + int(verify_len[i])) // page_size), stride) for i in range(B)]
    for i in range(B):
        for j in range(need[i], held[i]):
            stack[top] = table[i, j]
            top += 1
        held[i] = min(held[i], need[i]) if held[i] > need[i] else held[i]
    for i in range(B):
        while held[i] < need[i]:
            if top == 0:
                short = True
                break
            top -= 1
            table[i, held[i]] = stack[top]
            held[i] += 1
    out = dict(row_indptr=[0], page_indptr=[0], page_indices=[], positions=[], slot_map=[])
    for i in range(B):
        L, k, m = int(kv_len[i]), int(verify_len[i]), int(mask_rows[i])
        nb = 1 if mask_blocks is None else int(mask_blocks[i])
        v = max(k - nb + 1, 0) if mask_vis is None else int(mask_vis[i])
        out["page_indices"] += [int(x) for x in table[i, :held[i]]]
        for r in range(k):
            pos = L + r
            out["positions"].append(pos)
            out["slot_map"].append(int(table[i, pos // page_size]) * page_size + pos % page_size if pos // page_size < held[i] else -1)
        for b in range(nb if m else 0):
            for j in range(m // nb):
                out["positions"].append(L + min(v + b, k) + j)
                out["slot_map"].append(-1)
        out["row_indptr"].append(out["row_indptr"][-1] + k + m)
        out["page_indptr"].append(len(out["page_indices"]))
    out.update(block_table=table, table_len=held, free_pages=stack, free_count=top, short=short)
    return out


# ---- norm and rotation ------------------------------------------------------------------------
def norm_rope(x, weight, positions, inv_freq, eps, interleaved):
    """x [R, H, D] float64.  Returns y and, by element, |a| + |b| of the rotated pair (of the element where it is not rotated)."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * weight
    out, size = y.copy(), np.abs(y)
    half = len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = np.asarray(positions, dtype=np.longdouble) * np.longdouble(inv_freq[i])
        c, s = np.cos(t).astype(np.float64)[:, None], np.sin(t).astype(np.float64)[:, None]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size
