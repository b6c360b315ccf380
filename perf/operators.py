"""The operators around a cache held in 4 bits, as a decoding step uses them: what is measured, and their plain forms.

Kinds
  tables  fd_step_tables: row offsets, page lists, positions and slots of a step from the requests' lengths, with the pages that
          they take from the pool and give back to it
  rope    fd_qk_norm_rope: root-mean-square norm of every query and key head and their rotation by position
  commit  fd_append_kv_q4, then fd_read_kv_q4 of what was committed: the values that the cache now stands for
  read    fd_read_kv_q4: a sequence's keys and values leave the 4-bit cache
  attn    fd_verify_draft_attn_q4: hybrid-mask attention over the 4-bit cache and the step's own rows

The cache in 4 bits.  A code is sign and magnitude 0, 1/2, 1, 3/2, 2, 3, 4, 6.
  k_codes   [pages][heads][slot][dim / 2]: two codes a byte, the even channel low
  k_scales  [pages][heads][slot][dim / 32]: exponent e + 127 of the power of two that 32 channels share
  v_codes   [pages][heads][slot / 16][8 dim]: for each sixteen slots [half h][j < 32][c < dim / 32] four bytes that hold channel 32 c + j of
            slots 8 h .. 8 h + 7, two codes a byte, the even slot low
  v_scales  [pages][heads][slot] bfloat16: one scale a token and head

Lengths are part of a case (drawn from its `lengths` number), so that every state of a case has the same work.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


# ---- cases ------------------------------------------------------------------------------------
def _attn(name, batch, kv, verify, mask_len, *, blocks=1, hq=32, hkv=8, dim=128, page=16, shuffled=True, lengths=1):
    return dict(name=name, kind="attn", batch=batch, hq=hq, hkv=hkv, dim=dim, page=page, kv_lo=kv[0], kv_hi=kv[1], k_lo=verify[0],
                k_hi=verify[1], mask_len=mask_len, blocks=blocks, shuffled=shuffled, lengths=lengths)


def _tables(name, batch, kv, verify, mask_len, *, blocks=1, page=16, lengths=1):
    return dict(name=name, kind="tables", batch=batch, page=page, kv_lo=kv[0], kv_hi=kv[1], k_lo=verify[0], k_hi=verify[1],
                mask_len=mask_len, blocks=blocks, lengths=lengths)


def _rope(name, rows, far, *, hq=32, hkv=8, dim=128, rotary=128, interleaved=False, dtype="bf16", normed=True):
    return dict(name=name, kind="rope", rows=rows, far=far, hq=hq, hkv=hkv, dim=dim, rotary=rotary, interleaved=interleaved, dtype=dtype,
                normed=normed)


def _commit(name, batch, kv, rows, *, prompt=False, hkv=8, dim=128, page=16, lengths=1):
    return dict(name=name, kind="commit", batch=batch, kv_lo=kv[0], kv_hi=kv[1], k_lo=rows[0], k_hi=rows[1], prompt=prompt, hkv=hkv, dim=dim,
                page=page, lengths=lengths)


def _read(name, batch, rows, *, hkv=8, dim=128, page=16, dtype="bf16", lengths=1):
    return dict(name=name, kind="read", batch=batch, k_lo=rows[0], k_hi=rows[1], hkv=hkv, dim=dim, page=page, dtype=dtype, lengths=lengths)


def listed():
    return [
        # a served batch between two steps: 8 drafts to verify and 8 mask tokens each, a few pages change hands
        _tables("tables_b16", 16, (512, 4096), (8, 8), 8),
        # the largest batches with long documents among them, as many rows as the confidence left
        _tables("tables_b1024", 1024, (64, 32768), (1, 16), 8, lengths=2),
        # one interactive user: the bonus token and a block of 15 mask tokens
        _rope("rope_b1", 16, 2064),
        # a float32 model whose heads are rotated in part, pairs side by side, an odd number of rows
        _rope("rope_f32_partial", 333, 32768, hq=16, hkv=4, dim=64, rotary=32, interleaved=True, dtype="f32"),
        # a prompt's rows
        _rope("rope_prompt", 8192, 8192),
        # the accepted rows of a served batch
        _commit("commit_b16", 16, (512, 4096), (8, 8)),
        # four prompts go into the cache
        _commit("commit_prompt", 4, (0, 100), (1500, 2100), prompt=True),
        # four long sequences leave the 4-bit pool
        _read("read_b4", 4, (6000, 8192)),
        # one interactive user: the bonus token and a block of 15 mask tokens over a contiguous cache
        _attn("attn_b1", 1, (2048, 2048), (1, 1), 15, shuffled=False),
        # a served batch of mixed lengths, 8 drafts verified and 8 drafted
        _attn("attn_ragged", 16, (512, 4096), (8, 8), 8),
        # full parallel mode, one mask block per hypothetical number of accepted drafts: 272 new rows a sequence
        _attn("attn_parallel_b2", 2, (2048, 8192), (16, 16), 16, blocks=0),
        # the large-batch mode: verification alone, as many rows as the confidence left
        _attn("attn_verify_b128", 128, (1024, 8192), (1, 16), 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_BYTES, _MOST_FLOPS = 6.4e8, 6.5e10          # the largest listed attention (attn_verify_b128)


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn", "rope", "rope", "tables", "tables", "commit", "commit", "read"])
    lengths = rng.randrange(1 << 20)
    while True:
        if kind == "attn":
            hi, k = _log(rng, 1, 32768), rng.randint(0, 16)
            m = rng.choice([0, 8, 15, 16, rng.randint(1, 16)])
            if k + m == 0:
                continue
            c = _attn("", _log(rng, 1, 128), (max(0, hi // rng.choice([1, 2, 4, 8]) - rng.randint(0, 1)), hi), (min(k, rng.choice([k, 1])), k), m,
                      blocks=rng.choice([1, 1, 1, 0]), hq=rng.choice([32, 32, 16, 40, 64, 8]), dim=rng.choice([128, 128, 128, 64]),
                      page=rng.choice([16, 16, 32, 64]), shuffled=rng.random() < 0.8, lengths=lengths)
        elif kind == "tables":
            hi, k = _log(rng, 16, 32768), rng.randint(1, 16)
            c = _tables("", _log(rng, 1, 1024), (hi // rng.choice([1, 2, 4, 64]), hi), (rng.randint(0, k), k), rng.choice([0, 8, rng.randint(1, 16)]),
                        blocks=rng.choice([1, 1, 0]), page=rng.choice([16, 16, 1, 8, 32, 64, 24]), lengths=lengths)
        elif kind == "rope":
            dim = rng.choice([128, 128, 128, 64, 80, 96, 256])
            c = _rope("", _log(rng, 1, 8192), _log(rng, 64, 1 << 20), hq=rng.choice([32, 16, 40, 64, 8, 5]), hkv=rng.choice([8, 8, 4, 1, 5]), dim=dim,
                      rotary=rng.choice([dim, dim, dim // 16 * 8, 16]), interleaved=rng.random() < 0.3, dtype=rng.choice(["bf16", "bf16", "f32"]),
                      normed=rng.random() < 0.8)
        elif kind == "commit":
            prompt = rng.random() < 0.4
            hi = _log(rng, 17, 2100) if prompt else rng.randint(1, 16)
            kv = _log(rng, 1, 4096)
            c = _commit("", rng.randint(1, 4) if prompt else _log(rng, 1, 128), (kv // rng.choice([1, 2, 8]), kv), (rng.choice([1, hi]), hi), prompt=prompt,
                        hkv=rng.choice([8, 8, 4, 1, 5]), dim=rng.choice([128, 128, 64]), page=rng.choice([16, 16, 32, 48]), lengths=lengths)
        else:
            hi = _log(rng, 1, 8192)
            c = _read("", _log(rng, 1, 16), (rng.choice([0, hi // 2, hi]), hi), hkv=rng.choice([8, 8, 4, 1]), dim=rng.choice([128, 128, 64]),
                      page=rng.choice([16, 16, 32, 48]), dtype=rng.choice(["bf16", "f32"]), lengths=lengths)
        del c["name"]
        w = work(c)
        rows = int(_lengths(c)[2].sum()) if kind in ("attn", "tables") else 1
        if rows and w["bytes"] > 0 and w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS and (kind != "read" or int(_counts(c)[1].sum())):
            return c


# ---- sizes of a case --------------------------------------------------------------------------
def _lengths(c):
    """(prefix lengths, verify rows, new rows, mask blocks) of every sequence."""
    r = np.random.default_rng(c["lengths"])
    kv = r.integers(c["kv_lo"], c["kv_hi"] + 1, size=c["batch"])
    k = r.integers(c["k_lo"], c["k_hi"] + 1, size=c["batch"])
    if c["kind"] == "tables":
        gone = r.random(c["batch"]) < 0.03                    # requests that have ended give back what they hold
        kv[gone], k[gone] = 0, 0
    nb = np.maximum(k, 1) if c["blocks"] == 0 else np.full(c["batch"], c["blocks"])
    m = nb * c["mask_len"]
    if c["kind"] == "tables":
        m[gone] = 0
    return kv, k, k + m, nb


def _held(c):
    """(pages that each request holds, pages that it needs, entries a row of the block table)"""
    kv, k, _, _ = _lengths(c)
    r = np.random.default_rng(c["lengths"] + 1)
    need = -(-(kv + k) // c["page"])
    stride = -(-(c["kv_hi"] + c["k_hi"]) // c["page"]) + 2
    held = need + r.choice([-1, -1, 0, 0, 0, 0, 1], size=c["batch"])
    held = np.where(need == 0, r.integers(0, stride + 1, size=c["batch"]), held)
    return np.clip(held, 0, stride), need, stride


def _counts(c):
    """commit: (prefix lengths, committed rows, verify rows); read: (first token, tokens, tokens that the sequence has)."""
    r = np.random.default_rng(c["lengths"])
    k = r.integers(c["k_lo"], c["k_hi"] + 1, size=c["batch"])
    if c["kind"] == "read":
        start = r.integers(0, 40, size=c["batch"])
        return start, k, start + k + r.integers(0, 40, size=c["batch"])
    kv = r.integers(c["kv_lo"], c["kv_hi"] + 1, size=c["batch"])
    return kv, k if c["prompt"] else r.integers(1, k + 1), k


def _size(dtype):
    return 2 if dtype == "bf16" else 4


def _token_bytes(c):
    return c["hkv"] * (c["dim"] + c["dim"] // 32 + 2)         # both codes of a channel make a byte


def work(case):
    c = case
    if c["kind"] == "attn":
        kv, k, n, nb = _lengths(c)
        rows = int(n.sum())
        new_keys = n * n if c["blocks"] == 1 else n * (k + c["mask_len"])            # what the masks leave, at most
        b = int(kv.sum()) * _token_bytes(c) + rows * ((2 * c["hq"] + 2 * c["hkv"]) * c["dim"] * 2 + c["hq"] * 4)
        return {"bytes": b, "flops": int((n * kv + new_keys).sum()) * c["hq"] * c["dim"] * 4}
    if c["kind"] == "tables":
        kv, k, n, _ = _lengths(c)
        held, need, _ = _held(c)
        moved = int(np.abs(held - need).sum())
        return {"bytes": 4 * (2 * int(need.sum()) + 2 * moved + 7 * c["batch"]) + 12 * int(n.sum()), "flops": 8 * c["batch"]}
    if c["kind"] == "rope":
        x = c["rows"] * (c["hq"] + c["hkv"]) * c["dim"]
        return {"bytes": 2 * x * _size(c["dtype"]) + 4 * c["rows"], "flops": 7 * x}
    _, rows, _ = _counts(c)
    x = int(rows.sum())
    row = c["hkv"] * c["dim"] * 2
    if c["kind"] == "commit":
        return {"bytes": x * (row * 2 + 2 * _token_bytes(c) + row * 4), "flops": x * row * 6}
    return {"bytes": x * (_token_bytes(c) + row * _size(c["dtype"])), "flops": x * row}


# ---- states -----------------------------------------------------------------------------------
def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _indptr(n):
    return np.concatenate([[0], np.cumsum(n)])


def _empty(*shape, dtype=torch.int32):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _random_cache(c, pages, gen):
    """A cache that holds something already.  Scales as those of unit normal values: 2^-2 to 2 for keys, 0.3 to 0.7 for values."""
    H, ps, D = c["hkv"], c["page"], c["dim"]
    byte = lambda *s: torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8)  # noqa: E731
    exps = torch.randint(0, 5, (pages, H, ps, D // 32), generator=gen, device="cuda")
    k_scales = torch.tensor([125, 125, 126, 126, 127], dtype=torch.uint8, device="cuda")[exps]
    return dict(k_codes=byte(pages, H, ps, D // 2), k_scales=k_scales, v_codes=byte(pages, H, ps // 16, 8 * D),
                v_scales=(0.3 + 0.4 * torch.rand(pages, H, ps, generator=gen, device="cuda")).bfloat16())


def _normal_cache(c, pages, gen):
    """A cache of unit normal keys and values."""
    H, ps, D = c["hkv"], c["page"], c["dim"]
    x = torch.randn(pages, H, ps, D, generator=gen, device="cuda")
    codes, k_scales = _k_to_codes(x)
    k_codes = codes[..., 0::2] | codes[..., 1::2] << 4
    x.normal_(generator=gen)
    codes, v_scales = _v_to_codes(x)
    v = codes.view(pages, H, ps // 16, 2, 4, 2, D // 32, 32)             # group, half, byte, nibble, c, j
    v = (v[:, :, :, :, :, 0] | v[:, :, :, :, :, 1] << 4).permute(0, 1, 2, 3, 6, 5, 4)
    return dict(k_codes=k_codes, k_scales=k_scales, v_codes=v.reshape(pages, H, ps // 16, 8 * D), v_scales=v_scales)


def _page_lists(c, tokens, host):
    pages = -(-np.asarray(tokens, dtype=np.int64) // c["page"])
    used = int(pages.sum())
    pool = max(1, used + used // 32)
    ids = host.permutation(pool)[:used] if c.get("shuffled", True) else np.arange(used)
    return pool, _i32(_indptr(pages)), _i32(ids if used else np.zeros(1))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = np.random.default_rng(seed)
    s = dict(case=c, status=_empty(1).zero_())
    if c["kind"] == "attn":
        kv, k, n, nb = _lengths(c)
        R, D = int(n.sum()), c["dim"]
        pool, s["page_indptr"], s["page_indices"] = _page_lists(c, kv, host)
        randn = lambda *x: torch.randn(*x, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        s.update(q=randn(R, c["hq"], D), k_new=randn(R, c["hkv"], D), v_new=randn(R, c["hkv"], D), cache=_normal_cache(c, pool, gen),
                 kv_len=_i32(kv), row_indptr=_i32(_indptr(n)), verify_len=_i32(k), mask_blocks=_i32(nb) if c["blocks"] != 1 else None,
                 kv_max=int(kv.max()), n_max=int(n.max()), out=_empty(R, c["hq"], D, dtype=torch.bfloat16), lse=_empty(R, c["hq"], dtype=torch.float32))
    elif c["kind"] == "tables":
        kv, k, n, nb = _lengths(c)
        held, need, stride = _held(c)
        used, back, taken = int(held.sum()), int(np.maximum(held - need, 0).sum()), int(np.maximum(need - held, 0).sum())
        pool = used + taken + 16 + used // 32
        ids = host.permutation(pool)
        table = host.integers(0, pool, size=(c["batch"], stride))        # what lies behind a request's pages is old
        table[np.arange(stride)[None, :] < held[:, None]] = ids[:used]
        stack = np.concatenate([ids[used:], host.integers(0, pool, size=back)])
        s.update(kv_len=_i32(kv), verify_len=_i32(k), mask_rows=_i32(n - k), mask_blocks=_i32(nb) if c["blocks"] != 1 else None,
                 block_table=_i32(table), table_len=_i32(held), free_pages=_i32(stack), free_count=_i32([pool - used]),
                 row_indptr=_empty(c["batch"] + 1), page_indptr=_empty(c["batch"] + 1), page_indices=_empty(max(1, int(need.sum()))),
                 positions=_empty(int(n.sum())), slot_map=_empty(int(n.sum()), dtype=torch.int64), table_len_out=_empty(c["batch"]), free_count_out=_empty(1))
    elif c["kind"] == "rope":
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        R, Hq, Hkv, D = c["rows"], c["hq"], c["hkv"], c["dim"]
        # queries, keys and values as one projection leaves them
        qkv = torch.randn(R, Hq + 2 * Hkv, D, generator=gen, device="cuda", dtype=dt)
        weight = lambda: (1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(dt)  # noqa: E731
        half = c["rotary"] // 2
        s.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], q_out=_empty(R, Hq, D, dtype=dt), k_out=_empty(R, Hkv, D, dtype=dt),
                 q_weight=weight() if c["normed"] else None, k_weight=weight() if c["normed"] else None,
                 inv_freq=torch.from_numpy((1e6 ** (-np.arange(half) / max(1, half))).astype(np.float32)).cuda(),
                 positions=_i32((host.integers(0, c["far"]) + np.arange(R)) % c["far"]))
    else:
        first, rows, more = _counts(c)
        R = int(rows.sum())
        pool, s["page_indptr"], s["page_indices"] = _page_lists(c, more if c["kind"] == "read" else first + more, host)
        dt = torch.float32 if c["kind"] == "commit" or c["dtype"] == "f32" else torch.bfloat16
        s.update(cache=_random_cache(c, pool, gen), start=_i32(first), out_indptr=_i32(_indptr(rows)), read_k=_empty(R, c["hkv"], c["dim"], dtype=dt),
                 read_v=_empty(R, c["hkv"], c["dim"], dtype=dt))
        if c["kind"] == "commit":
            n = int(more.sum())
            randn = lambda *x: torch.randn(*x, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
            s.update(k_new=randn(n, c["hkv"], c["dim"]), v_new=randn(n, c["hkv"], c["dim"]), row_indptr=_i32(_indptr(more)), verify_len=_i32(more),
                     kv_len=s["start"], accept_len=_i32(rows - 1), kv_len_out=_empty(c["batch"]), kv_max=int(first.max()), n_max=int(more.max()),
                     q=_empty(n, c["hkv"], c["dim"], dtype=torch.bfloat16))
    return s


# ---- plain forms ------------------------------------------------------------------------------
def _magnitude_codes(y):
    """The nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6, ties to the even code."""
    return ((y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)).byte()


def _k_to_codes(x):
    """x [..., dim] float32 -> codes [..., dim], exponents + 127 [..., dim / 32]."""
    g = x.unflatten(-1, (x.shape[-1] // 32, 32))
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = (e - 2 - (m <= 0.75).int()).clamp(-126, 126)                     # the smallest with top <= 6 2^e
    e = torch.where(top == 0, torch.full_like(e, -126), e)
    codes = _magnitude_codes(torch.ldexp(g.abs(), -e)) | torch.signbit(g).byte() << 3
    return codes.flatten(-2), (e + 127).byte().squeeze(-1)


def _v_to_codes(x):
    """x [..., dim] float32 -> codes [..., dim], scales [...] bfloat16."""
    scale = (x.abs().amax(-1) / 6).bfloat16()
    s = scale.float().unsqueeze(-1)
    a = x.abs()
    codes = (a > 0.25 * s).byte() + (a >= 0.75 * s) + (a > 1.25 * s) + (a >= 1.75 * s) + (a > 2.5 * s) + (a >= 3.5 * s) + (a > 5 * s)
    codes = torch.where(s == 0, torch.zeros_like(codes), codes).byte()
    return codes | torch.signbit(x).byte() << 3, scale


def _values(device):
    v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=device)
    return torch.cat([v, -v])


def _pool_values(s):
    """Keys and values that the whole pool stands for: two [pages, slots, heads, dim] float32."""
    t = s["cache"]
    lut = _values(t["k_codes"].device)
    P, H, ps, half = t["k_codes"].shape
    D = 2 * half
    k = torch.stack([t["k_codes"] & 15, t["k_codes"] >> 4], -1).flatten(-2)
    k = lut[k.int()].view(P, H, ps, D // 32, 32) * torch.exp2(t["k_scales"].float() - 127).unsqueeze(-1)
    v = t["v_codes"].view(P, H, ps // 16, 2, 32, D // 32, 4)
    v = torch.stack([v & 15, v >> 4], -1)                               # group, half, j, c, byte, nibble
    v = lut[v.permute(0, 1, 2, 3, 6, 7, 5, 4).reshape(P, H, ps, D).int()] * t["v_scales"].float().unsqueeze(-1)
    return k.view(P, H, ps, D).transpose(1, 2), v.transpose(1, 2)


def _plain_attn(s):
    c = s["case"]
    Hq, Hkv, D, ps = c["hq"], c["hkv"], c["dim"], c["page"]
    G, dev, N, L = Hq // Hkv, s["q"].device, s["n_max"], s["kv_max"]
    B = s["kv_len"].shape[0]
    i64 = {n: s[n].long() for n in ("page_indptr", "page_indices", "kv_len", "row_indptr", "verify_len")}
    k_pool, v_pool = _pool_values(s)
    t = torch.arange(L, device=dev)
    at = (i64["page_indptr"][:-1, None] + t // ps).clamp(max=i64["page_indices"].numel() - 1)
    page = i64["page_indices"][at]
    k, v = k_pool[page, t % ps], v_pool[page, t % ps]                   # [B, L, Hkv, D]
    r = torch.arange(N, device=dev)
    row0, n = i64["row_indptr"][:-1, None], i64["row_indptr"].diff()[:, None]
    rows = (row0 + r).clamp(max=s["q"].shape[0] - 1)
    q = s["q"].float()[rows].view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    keys = torch.cat([k, s["k_new"].float()[rows]], 1).permute(0, 2, 3, 1).contiguous()
    vals = torch.cat([v, s["v_new"].float()[rows]], 1).permute(0, 2, 1, 3).contiguous()
    # who sees whom among the new rows
    kk = i64["verify_len"][:, None]
    nb = s["mask_blocks"].long()[:, None] if s["mask_blocks"] is not None else torch.ones_like(kk)
    ml = ((n - kk) // nb).clamp(min=1)
    first = (kk - nb + 1).clamp(min=0)
    block = ((r - kk) // ml).clamp(min=0)
    is_mask = r >= kk
    sees = torch.where(is_mask, torch.minimum(first + block, kk), r + 1)[:, :, None]
    same = is_mask[:, :, None] & is_mask[:, None, :] & (block[:, :, None] == block[:, None, :])
    new = ((r < sees) | same) & (r < n)[:, None, :]
    seen = torch.cat([(t < i64["kv_len"][:, None])[:, None, :].expand(B, N, L), new], 2)
    x = torch.matmul(q, keys) * (1 / math.sqrt(D))
    x = x.view(B, Hkv, N, G, L + N).masked_fill(~seen[:, None, :, None, :], -math.inf).view(B, Hkv, N * G, L + N)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = (torch.matmul(p, vals) / total).view(B, Hkv, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)
    lse = (top + torch.log(total)).view(B, Hkv, N, G).permute(0, 2, 1, 3).reshape(B, N, Hq)
    at = torch.arange(s["q"].shape[0], device=dev)
    seq = torch.searchsorted(i64["row_indptr"][1:].contiguous(), at, right=True)
    at = at - i64["row_indptr"][seq]
    return {"out": out[seq, at].bfloat16(), "lse": lse[seq, at]}


def _plain_tables(s):
    c = s["case"]
    ps, dev = c["page"], s["kv_len"].device
    kv, k, held = s["kv_len"].long(), s["verify_len"].long(), s["table_len"].long()
    table, stack = s["block_table"], s["free_pages"]
    stride, count = table.shape[1], s["free_count"].long()
    need = (kv + k + ps - 1) // ps
    give, take = (held - need).clamp(min=0), (need - held).clamp(min=0)
    before = lambda x: x.cumsum(0) - x  # noqa: E731
    j = torch.arange(stride, device=dev)
    given = (j >= need[:, None]) & (j < held[:, None])
    to = torch.where(given, count + before(give)[:, None] + j - need[:, None], stack.numel())
    longer = torch.cat([stack, stack.new_zeros(1)])
    longer.scatter_(0, to.flatten(), table.flatten())
    stack.copy_(longer[:-1])
    top = count + give.sum()
    taken = (j >= held[:, None]) & (j < need[:, None])
    at = (top - 1 - before(take)[:, None] - (j - held[:, None])).clamp(0, stack.numel() - 1)
    table.copy_(torch.where(taken, stack[at], table))
    indptr = lambda n: torch.cat([n.new_zeros(1), n.cumsum(0)])  # noqa: E731
    m = s["mask_rows"].long()
    row_indptr, page_indptr = indptr(k + m), indptr(need)
    p = torch.arange(s["page_indices"].numel(), device=dev)
    seq = torch.searchsorted(page_indptr[1:].contiguous(), p, right=True).clamp(max=kv.numel() - 1)
    pages = table[seq, (p - page_indptr[seq]).clamp(max=stride - 1)]
    r = torch.arange(s["positions"].numel(), device=dev)
    seq = torch.searchsorted(row_indptr[1:].contiguous(), r, right=True)
    r = r - row_indptr[seq]
    nb = s["mask_blocks"].long()[seq] if s["mask_blocks"] is not None else torch.ones_like(seq)
    ml = (m[seq] // nb).clamp(min=1)
    rk = r - k[seq]
    block = rk // ml
    ahead = torch.minimum((k[seq] - nb + 1).clamp(min=0) + block, k[seq])
    positions = kv[seq] + torch.where(rk < 0, r, ahead + rk - block * ml)
    pos = (kv[seq] + r)
    slots = torch.where(rk < 0, table[seq, (pos // ps).clamp(max=stride - 1)].long() * ps + pos % ps, -1)
    return {"row_indptr": row_indptr.int(), "page_indptr": page_indptr.int(), "page_indices": pages, "positions": positions.int(), "slot_map": slots,
            "block_table": table, "table_len": need.int(), "free_pages": stack, "free_count": (top - take.sum()).int()}


def _plain_rope(s):
    c = s["case"]
    half, D = c["rotary"] // 2, c["dim"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def one(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        if c["interleaved"]:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([y, x[..., 2 * half:]], -1)

    return {"q": one(s["q"], s["q_weight"]).to(s["q"].dtype), "k": one(s["k"], s["k_weight"]).to(s["k"].dtype)}


def _plain_read(s):
    """The values of tokens start .. of every sequence."""
    ps = s["case"]["page"]
    ip = s["out_indptr"].long()
    at = torch.arange(s["read_k"].shape[0], device=ip.device)
    seq = torch.searchsorted(ip[1:].contiguous(), at, right=True)
    pos = s["start"].long()[seq] + at - ip[seq]
    page = s["page_indices"].long()[s["page_indptr"].long()[seq] + pos // ps]
    t = s["cache"]
    H, D = t["k_codes"].shape[1], 2 * t["k_codes"].shape[3]
    lut = _values(ip.device)
    k = t["k_codes"][page, :, pos % ps]                                  # [R, H, D / 2]
    k = lut[torch.stack([k & 15, k >> 4], -1).int()].view(-1, H, D // 32, 32)
    k = (k * torch.exp2(t["k_scales"][page, :, pos % ps].float() - 127).unsqueeze(-1)).view(-1, H, D)
    e = pos % 16
    v = t["v_codes"].view(-1, H, ps // 16, 2, 32, D // 32, 4)[page, :, pos % ps // 16, e // 8, :, :, e % 8 // 2]   # [R, H, j, c]
    v = v >> (4 * (e % 2)).byte()[:, None, None, None] & 15
    v = lut[v.transpose(2, 3).reshape(-1, H, D).int()] * t["v_scales"][page, :, pos % ps].float().unsqueeze(-1)
    return k.to(s["read_k"].dtype), v.to(s["read_v"].dtype)


def _plain_commit(s):
    c = s["case"]
    ps, H, D = c["page"], c["hkv"], c["dim"]
    t, ip = s["cache"], s["out_indptr"].long()
    at = torch.arange(s["read_k"].shape[0], device=ip.device)
    seq = torch.searchsorted(ip[1:].contiguous(), at, right=True)
    j = at - ip[seq]
    row, pos = s["row_indptr"].long()[seq] + j, s["kv_len"].long()[seq] + j
    page, slot = s["page_indices"].long()[s["page_indptr"].long()[seq] + pos // ps], pos % ps
    codes, scales = _k_to_codes(s["k_new"][row].float())
    t["k_codes"][page, :, slot] = codes[..., 0::2] | codes[..., 1::2] << 4
    t["k_scales"][page, :, slot] = scales
    codes, scales = _v_to_codes(s["v_new"][row].float())
    t["v_scales"][page, :, slot] = scales
    codes = codes.view(-1, H, D // 32, 32).transpose(2, 3)               # [R, H, j, c]
    view = t["v_codes"].view(-1, H, ps // 16, 2, 32, D // 32, 4)
    group, half, byte, odd = slot // 16, slot % 16 // 8, slot % 8 // 2, (slot % 2).bool()

    def put(which, shift):          # the tokens of one parity: no two of them share a byte
        w = torch.nonzero(which).flatten()
        old = view[page[w], :, group[w], half[w], :, :, byte[w]]
        view[page[w], :, group[w], half[w], :, :, byte[w]] = old & (240 >> shift) | codes[w] << shift

    put(~odd, 0)
    put(odd, 4)
    k, v = _plain_read(s)
    return {"k": k, "v": v, "kv_len": (s["kv_len"] + s["accept_len"] + 1)}


# ---- one pass ---------------------------------------------------------------------------------
def _handle(s):
    """What a program keeps beside its tensors: the framework's argument structs over them."""
    from paper_2605_20022_amd import flexdraft as fd
    kind = s["case"]["kind"]
    if kind == "tables":
        s["args"] = fd.make_table_args(s["kv_len"], s["verify_len"], s["block_table"], s["table_len"], s["free_pages"], s["free_count"], s["mask_rows"],
                                       None, s["mask_blocks"], page_size=s["case"]["page"], row_indptr=s["row_indptr"], page_indptr=s["page_indptr"],
                                       page_indices=s["page_indices"], positions=s["positions"], slot_map=s["slot_map"], table_len_out=s["table_len_out"],
                                       free_count_out=s["free_count_out"], status=s["status"])
    elif kind != "rope":
        s["q4"] = fd.Q4Cache(**s["cache"])
        if kind == "attn":
            s["args"] = fd.make_attn_args_q4(s["q"], s["k_new"], s["v_new"], s["q4"], s["page_indptr"], s["page_indices"], s["kv_len"], s["row_indptr"],
                                             s["verify_len"], None, s["mask_blocks"], out=s["out"], lse=s["lse"], max_kv_len=s["kv_max"],
                                             max_new_rows=s["n_max"], status=s["status"])
            s["workspace"] = fd.alloc_workspace(fd.fd_verify_draft_attn_q4_workspace(s["args"]))
            s["args"].workspace, s["args"].workspace_bytes = s["workspace"].data_ptr(), s["workspace"].numel()
        elif kind == "commit":
            s["args"] = fd.make_attn_args_q4(s["q"], s["k_new"], s["v_new"], s["q4"], s["page_indptr"], s["page_indices"], s["kv_len"], s["row_indptr"],
                                             s["verify_len"], out=s["q"], max_kv_len=s["kv_max"], max_new_rows=s["n_max"], status=s["status"])
    s["fd"] = fd


def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        if kind == "commit":
            return _plain_commit(s)
        if kind == "read":
            k, v = _plain_read(s)
            return {"k": k, "v": v}
        return {"attn": _plain_attn, "tables": _plain_tables, "rope": _plain_rope}[kind](s)
    if "fd" not in s:
        _handle(s)
    fd = s["fd"]
    if kind == "attn":
        fd.fd_verify_draft_attn_q4(s["args"], s["q4"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "tables":
        fd.fd_step_tables(s["args"])
        return {"row_indptr": s["row_indptr"], "page_indptr": s["page_indptr"], "page_indices": s["page_indices"], "positions": s["positions"],
                "slot_map": s["slot_map"], "block_table": s["block_table"], "table_len": s["table_len_out"], "free_pages": s["free_pages"],
                "free_count": s["free_count_out"]}
    if kind == "rope":
        fd.fd_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                           eps=1e-6, interleaved=s["case"]["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if kind == "commit":
        fd.fd_append_kv_q4(s["args"], s["q4"], s["accept_len"], s["kv_len_out"])
    fd.fd_read_kv_q4(s["q4"], s["page_indptr"], s["page_indices"], s["start"], s["out_indptr"], s["read_k"], s["read_v"], status=s["status"])
    out = {"k": s["read_k"], "v": s["read_v"]}
    if kind == "commit":
        out["kv_len"] = s["kv_len_out"]
    return out


# ---- the definition in 64 bits ----------------------------------------------------------------
def _exact_tokens(s, i, lo, hi):
    """Keys and values of tokens lo .. hi of sequence i: two [heads, tokens, dim] in 64 bits."""
    t, ps = s["cache"], s["case"]["page"]
    H, D = s["case"]["hkv"], s["case"]["dim"]
    p0 = int(s["page_indptr"][i])
    pages = s["page_indices"][p0 + lo // ps:p0 + -(-hi // ps)].long()
    cut = slice(lo - lo // ps * ps, hi - lo // ps * ps)

    def value(code):                  # sign, two bits of exponent, one of mantissa
        code = code.double()
        neg = (code >= 8).double()
        code = code - 8 * neg
        e, m = torch.div(code, 2, rounding_mode="floor"), torch.remainder(code, 2)
        return torch.where(e == 0, m / 2, 2 ** (e - 1) * (1 + m / 2)) * (1 - 2 * neg)

    kc, ks, vs = t["k_codes"][pages], t["k_scales"][pages], t["v_scales"][pages]
    k = torch.empty(len(pages), H, ps, D, dtype=torch.float64, device=kc.device)
    k[..., 0::2], k[..., 1::2] = value(kc % 16), value(kc // 16)
    k = k * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=kc.device), ks.double() - 127).repeat_interleave(32, dim=-1)
    vc = t["v_codes"][pages].reshape(len(pages), H, ps // 16, 2, 32, D // 32, 4)
    v = torch.empty(len(pages), H, ps // 16, 2, 8, D // 32, 32, dtype=torch.float64, device=kc.device)
    for b in range(4):
        v[:, :, :, :, 2 * b], v[:, :, :, :, 2 * b + 1] = value(vc[..., b] % 16).transpose(-1, -2), value(vc[..., b] // 16).transpose(-1, -2)
    v = v.reshape(len(pages), H, ps, D) * vs.double()[..., None]
    flat = lambda x: x.transpose(0, 1).reshape(H, -1, D)[:, cut]  # noqa: E731
    return flat(k), flat(v)


def _exact_attn(s):
    c = s["case"]
    kv, k, n, nb = _lengths(c)
    G, D, H = c["hq"] // c["hkv"], c["dim"], c["hkv"]
    outs, lses, r0 = [], [], 0
    for i in range(c["batch"]):
        ni, ki = int(n[i]), int(k[i])
        if ni == 0:
            continue
        rows = slice(r0, r0 + ni)
        r0 += ni
        if kv[i]:
            pk, pv = _exact_tokens(s, i, 0, int(kv[i]))
        else:
            pk = pv = torch.empty(H, 0, D, dtype=torch.float64, device="cuda")
        keys = torch.cat([pk, s["k_new"][rows].double().transpose(0, 1)], 1)
        vals = torch.cat([pv, s["v_new"][rows].double().transpose(0, 1)], 1)
        seen = np.zeros((ni, ni), dtype=bool)
        for r in range(ni):
            if r < ki:
                seen[r, :r + 1] = True
            else:
                ml = (ni - ki) // int(nb[i])
                b = (r - ki) // ml
                seen[r, :min(max(ki - int(nb[i]) + 1, 0) + b, ki)] = True
                seen[r, ki + b * ml:ki + (b + 1) * ml] = True
        mask = torch.zeros(ni, int(kv[i]) + ni, dtype=torch.float64, device="cuda")
        mask[:, int(kv[i]):] = torch.where(torch.from_numpy(seen).cuda(), 0.0, -math.inf)
        q = s["q"][rows].double().view(ni, H, G, D).permute(1, 2, 0, 3)                       # [H, G, n, D]
        x = torch.matmul(q, keys.transpose(1, 2).contiguous()[:, None]) / math.sqrt(D) + mask
        lse = torch.logsumexp(x, -1)
        o = torch.matmul(torch.exp(x - lse[..., None]), vals[:, None])
        outs.append(o.permute(2, 0, 1, 3).reshape(ni, c["hq"], D))
        lses.append(lse.permute(2, 0, 1).reshape(ni, c["hq"]))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_rope(s):
    c = s["case"]
    D, half = c["dim"], c["rotary"] // 2
    turn = torch.polar(torch.ones(c["rows"], half, dtype=torch.float64, device="cuda"), torch.outer(s["positions"].double(), s["inv_freq"].double()))

    def one(x, w):
        y = x.double()
        if w is not None:
            y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / D + 1e-6) * w.double()
        at = (torch.arange(half) * 2, torch.arange(half) * 2 + 1) if c["interleaved"] else (torch.arange(half), torch.arange(half) + half)
        z = torch.complex(y[..., at[0].cuda()], y[..., at[1].cuda()]) * turn[:, None]
        y = y.clone()
        y[..., at[0].cuda()], y[..., at[1].cuda()] = z.real, z.imag
        return y

    return {"q": one(s["q"], s["q_weight"]), "k": one(s["k"], s["k_weight"])}


def _exact_commit(s):
    c = s["case"]
    first, rows, more = _counts(c)
    at = np.concatenate([np.arange(r) + o for r, o in zip(rows, _indptr(more)[:-1])])
    at = torch.from_numpy(at).cuda()

    def nearest(y):
        step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
        return (torch.round(y / step) * step).clamp(-6, 6)

    k = s["k_new"][at].double().reshape(-1, c["hkv"], c["dim"] // 32, 32)
    unit = 2.0 ** torch.ceil(torch.log2(k.abs().amax(-1, keepdim=True) / 6))
    v = s["v_new"][at].double()
    scale = (v.abs().amax(-1, keepdim=True) / 6).bfloat16().double()
    return {"k": (nearest(k / unit) * unit).flatten(-2), "v": nearest(v / scale) * scale, "kv_len": None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(s)
    if case["kind"] == "rope":
        return _exact_rope(s)
    if case["kind"] == "commit":
        return _exact_commit(s)
    if case["kind"] == "read":
        first, rows, _ = _counts(case)
        kv = [_exact_tokens(s, i, int(first[i]), int(first[i] + rows[i])) for i in range(case["batch"])]
        return {"k": torch.cat([k.transpose(0, 1) for k, _ in kv]), "v": torch.cat([v.transpose(0, 1) for _, v in kv])}
    return None                       # whole numbers
