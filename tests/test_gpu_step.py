"""GPU parity of the step tables and of the norm and rotation, and a decoding loop of all calls around a 4-bit cache."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import kv4
from tests.q4_harness import bf16, bits_of, device_cache, i32

pytestmark = pytest.mark.gpu


# ---- tables -----------------------------------------------------------------------------------
class Tables:
    def __init__(self, fd, kv, k, m, held, table, stack, count, ps, blocks=None, vis=None, rows=None, entries=None, in_place=False):
        B = len(kv)
        self.kv, self.k, self.m, self.held, self.table, self.stack, self.count, self.ps = kv, k, m, held, table, stack, count, ps
        self.blocks, self.vis = blocks, vis
        need = int(sum(-(-(a + b) // ps) for a, b in zip(kv, k)))
        R = int(np.sum(k) + np.sum(m)) if rows is None else rows
        full = lambda n, dt=torch.int32: torch.full((n,), -9, dtype=dt, device="cuda")  # noqa: E731
        self.t = dict(block_table=i32(table), table_len=i32(held), free_pages=i32(stack), free_count=i32([count]), row_indptr=full(B + 1), page_indptr=full(B + 1),
                      page_indices=full((need if entries is None else entries) + 3), positions=full(R + 3), slot_map=full(R + 3, torch.int64))
        self.t["table_len_out"] = self.t["table_len"] if in_place else full(B)
        self.t["free_count_out"] = self.t["free_count"] if in_place else full(1)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        opt = lambda x: None if x is None else i32(x)  # noqa: E731
        t = self.t
        self.keep = [i32(kv), i32(k), i32(m), opt(vis), opt(blocks)]
        self.args = fd.make_table_args(self.keep[0], self.keep[1], t["block_table"], t["table_len"], t["free_pages"], t["free_count"], self.keep[2], self.keep[3],
                                       self.keep[4], page_size=ps, row_indptr=t["row_indptr"], page_indptr=t["page_indptr"], page_indices=t["page_indices"],
                                       positions=t["positions"], slot_map=t["slot_map"], table_len_out=t["table_len_out"], free_count_out=t["free_count_out"],
                                       status=self.status)

    def check(self, fd):
        fd.fd_step_tables(self.args)
        torch.cuda.synchronize()
        self.compare()

    def compare(self):
        r = kv4.step_tables(self.kv, self.k, self.m, self.table, self.held, self.stack, self.count, self.ps, self.vis, self.blocks)
        got = {n: t.cpu().numpy() for n, t in self.t.items()}
        assert got["row_indptr"].tolist() == r["row_indptr"] and got["page_indptr"].tolist() == r["page_indptr"]
        n, e = r["row_indptr"][-1], r["page_indptr"][-1]
        assert got["page_indices"][:e].tolist() == r["page_indices"] and (got["page_indices"][e:] == -9).all()
        assert got["positions"][:n].tolist() == r["positions"] and (got["positions"][n:] == -9).all()
        assert got["slot_map"][:n].tolist() == r["slot_map"] and (got["slot_map"][n:] == -9).all()
        assert np.array_equal(got["block_table"], r["block_table"]) and got["table_len_out"].tolist() == r["table_len"]
        assert np.array_equal(got["free_pages"], r["free_pages"]) and got["free_count_out"].tolist() == [r["free_count"]]
        assert int(self.status.item()) == (4 if r["short"] else 0)


def _random_tables(fd, rng, B, ps, most, k_hi, m=0, blocks=None, gone=0.1, pool=None, **kw):
    kv, k = rng.integers(0, most + 1, size=B), rng.integers(0, k_hi + 1, size=B)
    end = rng.random(B) < gone
    kv[end], k[end] = 0, 0
    mm = np.where(end, 0, m) if blocks is None else np.where(end, 0, m * blocks)
    need = -(-(kv + k) // ps)
    stride = int(-(-(most + k_hi) // ps)) + 3
    held = np.clip(need + rng.integers(-3, 3, size=B), 0, stride)
    held[end] = rng.integers(0, stride + 1, size=int(end.sum()))
    used = int(held.sum())
    spare = int(np.maximum(need - held, 0).sum()) + 5 if pool is None else pool
    ids = rng.permutation(used + spare)
    table = rng.integers(0, 100, size=(B, stride))
    table[np.arange(stride) < held[:, None]] = ids[:used]
    stack = np.r_[ids[used:], rng.integers(0, 100, size=int(np.maximum(held - need, 0).sum()))]
    return Tables(fd, kv, k, mm, held, table, stack, spare, ps, blocks=blocks, **kw)


@pytest.mark.parametrize("B,ps,most,k_hi", [(1, 16, 2000, 8), (7, 1, 30, 4), (16, 16, 4096, 16), (64, 24, 700, 1), (1023, 16, 300, 5), (1500, 8, 90, 3), (2500, 32, 40, 2)])
@pytest.mark.parametrize("in_place", [False, True])
def test_step_tables(fd, B, ps, most, k_hi, in_place):
    """Requests that end, grow and shrink; one round of the exchange and several (more than 1024 requests)."""
    rng = np.random.default_rng(B + ps)
    _random_tables(fd, rng, B, ps, most, k_hi, m=3, in_place=in_place).check(fd)


def test_step_tables_with_mask_blocks(fd):
    rng = np.random.default_rng(0)
    _random_tables(fd, rng, 20, 16, 500, 6, m=4, blocks=rng.integers(1, 5, size=20)).check(fd)
    Tables(fd, [5, 40], [3, 2], [6, 4], [1, 3], [[7, 0, 0], [1, 2, 3]], [9, 9], 1, 16, blocks=[3, 1], vis=[1, 0]).check(fd)


def test_step_tables_of_a_pool_that_runs_out(fd):
    rng = np.random.default_rng(4)
    _random_tables(fd, rng, 40, 16, 900, 9, gone=0.0, pool=2).check(fd)
    Tables(fd, [0, 0], [0, 0], [0, 0], [0, 0], [[0], [0]], [0], 0, 16).check(fd)              # nothing at all


def test_step_tables_of_bad_device_data(fd):
    """Negative and huge lengths, more pages than a row holds, a count that is no count, too little room in the outputs: clamped and reported."""
    def run(bit, change=None, **kw):
        base = dict(kv=[20, 30], k=[2, 2], m=[1, 1], held=[2, 2], table=[[3, 4, 5], [6, 7, 8]], stack=[9, 10, 11], count=1, ps=16)
        t = Tables(fd, **dict(base, **kw))
        if change:
            change(t)
        fd.fd_step_tables(t.args)
        torch.cuda.synchronize()
        assert int(t.status.item()) & bit, int(t.status.item())
        got = {n: x.cpu().numpy() for n, x in t.t.items()}
        assert 0 <= got["row_indptr"].min() and got["row_indptr"].max() <= len(got["positions"]) and (np.diff(got["row_indptr"]) >= 0).all()
        assert 0 <= got["page_indptr"].min() and got["page_indptr"].max() <= len(got["page_indices"]) and (np.diff(got["page_indptr"]) >= 0).all()
        assert 0 <= got["table_len_out"].min() and got["table_len_out"].max() <= 3 and 0 <= got["free_count_out"][0] <= 3
        return got
    run(1, kv=[-5, 30], rows=4)
    run(1, lambda t: t.keep[0].fill_(2 ** 31 - 1))
    run(2, lambda t: t.keep[1].fill_(-3))
    run(2, lambda t: t.keep[2].fill_(2 ** 31 - 1))
    run(2, blocks=[2, 1])                                           # one mask row in two blocks
    run(2, vis=[3, 0])
    run(4, kv=[20, 300])                                            # more pages than a row of the table
    run(4, held=[7, 2])
    run(4, count=17)
    run(4, entries=-1)                                              # four entries wanted, two there
    got = run(2, rows=-1)                                           # six rows, two places
    assert got["row_indptr"].tolist() == [0, 2, 2]
    # pages given back that the stack has no place for are lost, and reported
    got = run(4, kv=[0, 0], k=[0, 0], m=[0, 0], held=[3, 3], count=1)
    assert got["free_count_out"][0] == 3 and got["free_pages"].tolist() == [9, 3, 4]


# ---- norm and rotation ------------------------------------------------------------------------
def _dev(x, dtype):
    return bf16(bits_of(x)) if dtype == "bf16" else torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()


def _val(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rotary", [(128, 128), (64, 64), (8, 8), (80, 40), (96, 24), (128, 0), (256, 256), (200, 64)])
def test_norm_rope(fd, dtype, interleaved, D, rotary):
    """fp32: a sum of D squares in a tree of 13 additions at most, a root, a quotient, two products, the rotation's two products and
    sum, and an angle within 2^-24 of a turn's half (2 pi 2^-25): below 2^-19 of |a| + |b| in all.  bf16: half a step, 2^-8 of the result, on top."""
    rng = np.random.default_rng(D + rotary)
    R, Hq, Hkv = 37, 5, 3
    x = rng.standard_normal((R, Hq + 2 * Hkv, D)) * rng.choice([0.01, 1.0, 30.0], size=(R, 1, 1))
    qkv = _dev(x, dtype)
    wq, wk = _dev(1 + 0.3 * rng.standard_normal(D), dtype), _dev(1 + 0.3 * rng.standard_normal(D), dtype)
    freq = (1e6 ** (-np.arange(rotary // 2) / max(1, rotary // 2))).astype(np.float32)
    pos = np.r_[0, 1, 2 ** 31 - 1, 2 ** 20 + 1, rng.integers(0, 1 << 20, size=R - 4)]
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    new = lambda h: torch.full((R, h, D), float("nan"), dtype=qkv.dtype, device="cuda")  # noqa: E731
    qo, ko, vo = new(Hq), new(Hkv), new(Hkv)
    fd.fd_qk_norm_rope(q, k, qo, ko, i32(pos), torch.from_numpy(freq).cuda() if rotary else None, q_weight=wq, k_weight=wk, v=v, v_out=vo, eps=1e-5,
                       interleaved=interleaved)
    torch.cuda.synchronize()
    step = 2.0 ** -8 if dtype == "bf16" else 0.0
    for got, src, w in ((qo, q, wq), (ko, k, wk)):
        want, size = kv4.norm_rope(_val(src), _val(w), pos, freq.astype(np.float64), float(np.float32(1e-5)), interleaved)
        assert (np.abs(_val(got) - want) <= 2.0 ** -19 * size + step * np.abs(want) + 1e-37).all()
    assert torch.equal(vo, v)
    # without weights: rotation alone; a row's result does not depend on the others
    qo2, ko2 = new(Hq), new(Hkv)
    fd.fd_qk_norm_rope(q, k, qo2, ko2, i32(pos), torch.from_numpy(freq).cuda() if rotary else None, interleaved=interleaved)
    want, size = kv4.norm_rope(_val(q), None, pos, freq.astype(np.float64), 0.0, interleaved)
    assert (np.abs(_val(qo2) - want) <= 2.0 ** -19 * size + step * np.abs(want) + 1e-37).all()
    one = new(Hq)[:1]
    fd.fd_qk_norm_rope(q[5:6], k[5:6], one, new(Hkv)[:1], i32(pos[5:6]), torch.from_numpy(freq).cuda() if rotary else None, q_weight=wq, k_weight=wk,
                       eps=1e-5, interleaved=interleaved)
    assert torch.equal(one[0], qo[5])


def test_norm_rope_in_place_and_many_rows(fd):
    rng = np.random.default_rng(0)
    for R in (1, 3, 700, 5001):
        q, k = (torch.randn(R, h, 128, device="cuda", dtype=torch.bfloat16) for h in (8, 2))
        f = torch.from_numpy((1e4 ** (-np.arange(64) / 64)).astype(np.float32)).cuda()
        pos = i32(rng.integers(0, 50000, size=R))
        w = torch.rand(128, device="cuda").bfloat16()
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        fd.fd_qk_norm_rope(q, k, qo, ko, pos, f, q_weight=w, k_weight=w)
        sample = rng.integers(0, R, size=5)
        want, size = kv4.norm_rope(_val(q[sample]), _val(w), pos.cpu().numpy()[sample], f.double().cpu().numpy(), float(np.float32(1e-6)), False)
        assert (np.abs(_val(qo[sample]) - want) <= 2.0 ** -19 * size + 2.0 ** -8 * np.abs(want)).all()
        fd.fd_qk_norm_rope(q, k, q, k, pos, f, q_weight=w, k_weight=w)
        assert torch.equal(q, qo) and torch.equal(k, ko)


def test_norm_rope_of_zeros_and_odd_values(fd):
    """A head of zeros stays zero; an infinity or NaN stays in its head; only queries, only keys."""
    q, k = torch.randn(2, 3, 64, device="cuda"), torch.randn(2, 1, 64, device="cuda")
    q[0, 0] = 0
    q[1, 1, 7] = float("inf")
    k[1, 0, 3] = float("nan")
    w, f = torch.ones(64, device="cuda"), torch.ones(32, device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    fd.fd_qk_norm_rope(q, k, qo, ko, i32([3, 4]), f, q_weight=w, k_weight=w)
    assert (qo[0, 0] == 0).all() and torch.isnan(ko[1]).all() and not torch.isfinite(qo[1, 1]).all()
    assert torch.isfinite(qo[0]).all() and torch.isfinite(qo[1, [0, 2]]).all() and torch.isfinite(ko[0]).all()
    only = torch.empty_like(q)
    fd.fd_qk_norm_rope(q, k[:, :0], only, ko[:, :0].contiguous(), i32([3, 4]), f, q_weight=w)
    assert torch.equal(only.nan_to_num(), qo.nan_to_num())


# ---- a decoding loop --------------------------------------------------------------------------
class Loop:
    """A served batch whose cache is held in 4 bits: tables, norm and rotation, attention, commit, step after step, all lengths on the device."""

    def __init__(self, fd, seed, B=4, hq=8, hkv=2, D=128, ps=16, mask=4, rows=9):
        rng = np.random.default_rng(seed)
        self.fd, self.B, self.hq, self.hkv, self.D, self.ps, self.mask, self.rows = fd, B, hq, hkv, D, ps, mask, rows
        self.kv = rng.integers(0, 70, size=B)
        self.stride = 16
        pool = B * self.stride
        held = -(-self.kv // ps)
        ids = rng.permutation(pool)
        table = np.zeros((B, self.stride), dtype=np.int64)
        table[np.arange(self.stride) < held[:, None]] = ids[:held.sum()]
        self.table, self.held, self.stack, self.count = table, held, np.r_[ids[held.sum():], np.zeros(int(held.sum()), dtype=np.int64)], pool - int(held.sum())
        self.cache = kv4.Cache.random(rng, pool, hkv, ps, D)
        self.dev = device_cache(fd, self.cache)
        cap = B * (rows + mask)
        z = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt, device="cuda")  # noqa: E731
        self.t = dict(kv_len=i32(self.kv), verify_len=z(B), mask_rows=i32([mask] * B), accept=z(B), table=i32(table), held=i32(held), stack=i32(self.stack),
                      count=i32([self.count]), row_indptr=z(B + 1), page_indptr=z(B + 1), page_indices=z(B * self.stride), positions=z(cap),
                      slot_map=z(cap, torch.int64), status=z(1))
        self.qkv = torch.zeros(cap, hq + 2 * hkv, D, dtype=torch.bfloat16, device="cuda")
        self.q, self.k, self.v = (torch.zeros(cap, h, D, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
        self.out = torch.zeros_like(self.q)
        self.w = bf16(bits_of(1 + 0.1 * rng.standard_normal(D)))
        self.freq = (1e6 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32)
        self.freq_d = torch.from_numpy(self.freq).cuda()
        t = self.t
        self.tables = fd.make_table_args(t["kv_len"], t["verify_len"], t["table"], t["held"], t["stack"], t["count"], t["mask_rows"], page_size=ps,
                                         row_indptr=t["row_indptr"], page_indptr=t["page_indptr"], page_indices=t["page_indices"], positions=t["positions"],
                                         slot_map=t["slot_map"], status=t["status"])
        self.args = fd.make_attn_args_q4(self.q, self.k, self.v, self.dev, t["page_indptr"], t["page_indices"], t["kv_len"], t["row_indptr"], t["verify_len"],
                                         out=self.out, max_kv_len=self.stride * ps, max_new_rows=rows + mask, status=t["status"])
        self.ws = fd.alloc_workspace(fd.fd_verify_draft_attn_q4_workspace(self.args))
        self.args.workspace, self.args.workspace_bytes = self.ws.data_ptr(), self.ws.numel()

    def enqueue(self):
        fd, hq, hkv = self.fd, self.hq, self.hkv
        fd.fd_step_tables(self.tables)
        x = self.qkv
        fd.fd_qk_norm_rope(x[:, :hq], x[:, hq:hq + hkv], self.q, self.k, self.t["positions"], self.freq_d, q_weight=self.w, k_weight=self.w, v=x[:, hq + hkv:],
                           v_out=self.v)
        fd.fd_verify_draft_attn_q4(self.args, self.dev)
        fd.fd_append_kv_q4(self.args, self.dev, self.t["accept"], self.t["kv_len"])

    def inputs(self, seed):
        rng = np.random.default_rng(seed)
        k = rng.integers(1, self.rows + 1, size=self.B)
        self.k_i, self.acc = k, np.array([rng.integers(0, x) for x in k])
        self.x = bits_of(rng.standard_normal(self.qkv.shape))
        self.t["verify_len"].copy_(i32(k))
        self.t["accept"].copy_(i32(self.acc))
        self.qkv.copy_(bf16(self.x))

    def check(self):
        """The step against the oracle, from the state before it; the oracle's own state moves on."""
        B, hq, hkv = self.B, self.hq, self.hkv
        r = kv4.step_tables(self.kv, self.k_i, [self.mask] * B, self.table, self.held, self.stack, self.count, self.ps)
        n = r["row_indptr"][-1]
        got = {name: t.cpu().numpy() for name, t in self.t.items()}
        assert got["status"][0] == 0 and not r["short"]
        assert got["row_indptr"].tolist() == r["row_indptr"] and got["page_indptr"].tolist() == r["page_indptr"]
        assert got["positions"][:n].tolist() == r["positions"] and got["slot_map"][:n].tolist() == r["slot_map"]
        assert got["held"].tolist() == r["table_len"] and got["count"][0] == r["free_count"]
        x = oa.widen_bf16(self.x)[:n]
        q, qs = kv4.norm_rope(x[:, :hq], _val(self.w), r["positions"], self.freq.astype(np.float64), float(np.float32(1e-6)), False)
        k, ks = kv4.norm_rope(x[:, hq:hq + hkv], _val(self.w), r["positions"], self.freq.astype(np.float64), float(np.float32(1e-6)), False)
        for name, want, size in (("q", q, qs), ("k", k, ks)):
            assert (np.abs(_val(getattr(self, name))[:n] - want) <= 2.0 ** -19 * size + 2.0 ** -8 * np.abs(want)).all()
        # from here on with the rows as they were rounded
        qd, kd, vd = (_val(t)[:n] for t in (self.q, self.k, self.v))
        assert np.array_equal(vd, x[:, hq + hkv:])
        call = lambda v_new, v_cache: oa.verify_draft_attention(qd, kd, v_new, self.cache.key_values(), v_cache, r["page_indptr"], r["page_indices"], self.kv,  # noqa: E731
                                                                r["row_indptr"], self.k_i, None, None, page_size=self.ps)[0]
        ref, size = call(vd, self.cache.value_values()), call(np.abs(vd), np.abs(self.cache.value_values()))
        # (the bounds of the attention tests: two bf16 roundings, and 2^-12 for scores of unit size in fp32)
        assert (np.abs(_val(self.out)[:n] - ref) <= 2.0 ** -8 * (np.abs(ref) + size) + 2.0 ** -12 * size).all()
        self.cache, lens = kv4.append(self.cache, kd, vd, r["page_indptr"], r["page_indices"], self.kv, r["row_indptr"], self.k_i, self.acc)
        assert got["kv_len"].tolist() == lens.tolist()
        want = self.cache.packed()
        assert np.array_equal(self.dev.k_codes.cpu().numpy(), want[0]) and np.array_equal(self.dev.v_codes.cpu().numpy(), want[2])
        self.kv, self.table, self.held, self.stack, self.count = lens, r["block_table"], r["table_len"], r["free_pages"], r["free_count"]


def test_decoding_loop(fd):
    loop = Loop(fd, 1)
    for step in range(6):
        loop.inputs(100 + step)
        loop.enqueue()
        torch.cuda.synchronize()
        loop.check()


def test_decoding_loop_captured(fd):
    """The same loop as one graph, replayed step after step with eager work and synchronisation between the replays."""
    loop = Loop(fd, 2, B=3, mask=8)
    loop.inputs(0)
    fresh = {n: t.clone() for n, t in loop.t.items()}
    codes = [getattr(loop.dev, n).clone() for n in ("k_codes", "k_scales", "v_codes", "v_scales")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loop.enqueue()                                       # modules are loaded before capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loop.enqueue()
    for n, t in loop.t.items():
        t.copy_(fresh[n])
    for n, c in zip(("k_codes", "k_scales", "v_codes", "v_scales"), codes):
        getattr(loop.dev, n).copy_(c)
    for step in range(5):
        loop.inputs(step)
        graph.replay()
        torch.cuda.synchronize()
        loop.check()
