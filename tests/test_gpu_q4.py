"""GPU parity of the calls over a 4-bit cache against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import kv4
from tests.q4_harness import Q4Call, assert_cache_is, bf16, bits_of, device_cache, i32

pytestmark = pytest.mark.gpu


# ---- commit and read-back ---------------------------------------------------------------------
def _commit(fd, call, accept, in_place=False, garbage=None):
    call.upload()
    acc = i32(accept)
    out = call.d["kv_len"] if in_place else torch.full((len(call.kv),), -5, dtype=torch.int32, device="cuda")
    fd.fd_append_kv_q4(call.args, call.dev, acc, out)
    torch.cuda.synchronize()
    return out.cpu().numpy()


@pytest.mark.parametrize("dim,hkv,ps", [(128, 2, 16), (64, 3, 32), (128, 1, 48)])
@pytest.mark.parametrize("in_place", [False, True])
def test_commit_is_exact(fd, dim, hkv, ps, in_place):
    """Codes, scales and every untouched nibble: 1 .. 17 rows from positions 0 .. 33, mask rows never."""
    kv, k = [0, 1, 7, 8, 15, 16, 17, 31, 33, 5], [1, 2, 9, 17, 1, 16, 8, 3, 0, 4]
    call = Q4Call(fd, kv=kv, k=k, m=[2] * 10, hq=hkv, hkv=hkv, dim=dim, ps=ps, room=18, seed=dim + ps)
    accept = [0, 1, 8, 16, 0, 15, 3, 2, 0, 1]
    got = _commit(fd, call, accept, in_place)
    want, lens = kv4.append(call.cache, _wide(call.k_new), _wide(call.v_new), call.page_indptr, call.page_indices, call.kv, call.row_indptr, call.k, accept)
    assert int(call.status.item()) == 0
    assert np.array_equal(got, lens)
    assert_cache_is(call.dev, want)


def _wide(bits):
    return (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def test_commit_of_every_rounding(fd):
    """Values on, above and below each midpoint, at scales from the smallest to the largest; zeros, subnormals, infinities and NaN."""
    rng = np.random.default_rng(3)
    rows = []
    for e in (-126, -125, -60, -3, 0, 4, 120, 125):
        mid = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0])
        near = np.concatenate([mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -8), [6.0, 0.0, -0.0, 0.5, 1.0, 2.0, 3.0, 4.0, -6.0, 1e-3, 0.1]])
        x = np.tile(np.concatenate([near, -near])[:32], 4) * 2.0 ** e
        rows.append(rng.permutation(x))
    rows.append(np.zeros(128))
    rows.append(np.r_[np.full(64, 2.0 ** -133), np.full(64, -(2.0 ** -130))])                 # bf16 subnormals
    rows.append(np.r_[np.full(1, 3.3895e38), np.zeros(127)])                               # the largest bf16
    for odd in (np.inf, -np.inf, np.nan):
        x = rng.standard_normal(128)
        x[70] = odd
        rows.append(x)
    n = len(rows)
    call = Q4Call(fd, kv=[3], k=[n], m=[0], hq=1, hkv=1, room=n)
    call.k_new = bits_of(np.stack(rows))[:, None]
    call.v_new = bits_of(np.stack(rows)[::-1])[:, None]
    got = _commit(fd, call, [n - 1])
    want, lens = kv4.append(call.cache, _wide(call.k_new), _wide(call.v_new), call.page_indptr, call.page_indices, call.kv, call.row_indptr, call.k, [n - 1])
    assert np.array_equal(got, lens)
    assert_cache_is(call.dev, want)


def test_commit_of_a_prompt(fd):
    """Hundreds of rows a sequence, in several work-groups, from a position inside a byte on."""
    call = Q4Call(fd, kv=[5, 0, 40], k=[300, 129, 1], m=[0, 0, 0], hq=2, hkv=2, ps=16, room=300, seed=9)
    accept = [299, 128, 0]
    got = _commit(fd, call, accept, in_place=True)
    want, lens = kv4.append(call.cache, _wide(call.k_new), _wide(call.v_new), call.page_indptr, call.page_indices, call.kv, call.row_indptr, call.k, accept)
    assert np.array_equal(got, lens)
    assert_cache_is(call.dev, want)


def test_commit_reports_bad_device_data(fd):
    call = Q4Call(fd, kv=[10, 20, 16], k=[4, 4, 4], m=[0, 0, 0], room=16)
    call.upload()
    call.d["page_indices"][int(call.page_indptr[1]) + 1] = 10 ** 6           # positions 16 .. 31 of sequence 1
    accept = i32([4, 3, -1])                                                # one more than there are; fewer than none
    out = torch.zeros(3, dtype=torch.int32, device="cuda")
    fd.fd_append_kv_q4(call.args, call.dev, accept, out)
    torch.cuda.synchronize()
    assert int(call.status.item()) == 2 | 4
    assert out.cpu().tolist() == [14, 24, 17]                               # clamped to the verify rows, as fd_append_kv does
    want, _ = kv4.append(call.cache, _wide(call.k_new), _wide(call.v_new), call.page_indptr, call.page_indices, call.kv, call.row_indptr, [4, 0, 4], [3, 0, 0])
    assert_cache_is(call.dev, want)
    # a page list without room: what fits is committed
    call = Q4Call(fd, kv=[14], k=[5], m=[0], room=2)
    got = _commit(fd, call, [4])
    assert int(call.status.item()) == 4 and list(got) == [16]
    want, _ = kv4.append(call.cache, _wide(call.k_new), _wide(call.v_new), call.page_indptr, call.page_indices, call.kv, call.row_indptr, call.k, [1])
    assert_cache_is(call.dev, want)


def test_commit_without_rows_copies_the_lengths(fd):
    call = Q4Call(fd, kv=[10, 20], k=[1, 1], m=[0, 0], room=16).upload()
    call.args.total_rows = 0
    out = torch.zeros(2, dtype=torch.int32, device="cuda")
    fd.fd_append_kv_q4(call.args, call.dev, i32([0, 0]), out)
    assert out.cpu().tolist() == [10, 20]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,hkv,ps", [(128, 2, 16), (64, 3, 32), (128, 1, 48)])
def test_read_is_exact(fd, dtype, dim, hkv, ps):
    rng = np.random.default_rng(dim + ps)
    tokens = [0, 1, 70, 200, 33, 500, 16]
    start = np.array([0, 0, 3, 17, 32, 100, 0])
    rows = np.array([0, 1, 60, 183, 1, 300, 0])
    pages = [-(-t // ps) for t in tokens]
    pool = sum(pages) + 2
    cache = kv4.Cache.random(rng, pool, hkv, ps, dim, spread=20)
    indptr, ids = np.r_[0, np.cumsum(pages)], rng.permutation(pool)[:sum(pages)]
    out_indptr = np.r_[0, np.cumsum(rows)]
    R = int(rows.sum())
    dev = device_cache(fd, cache, heads_first=dim == 64)
    k, v = (torch.full((R + 2, hkv, dim), -3.0, dtype=dtype, device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fd.fd_read_kv_q4(dev, i32(indptr), i32(ids), i32(start), i32(out_indptr), k, v, status=status)
    torch.cuda.synchronize()
    wk, wv = kv4.read(cache, indptr, ids, start, out_indptr)
    if dtype == torch.bfloat16:
        wv = kv4.bf16_round(wv)
    assert int(status.item()) == 0
    assert np.array_equal(k[:R].double().cpu().numpy(), wk) and np.array_equal(v[:R].double().cpu().numpy(), wv)
    assert (k[R:] == -3).all() and (v[R:] == -3).all()                        # rows behind the last sequence stay


def test_read_skips_what_the_page_list_does_not_hold(fd):
    rng = np.random.default_rng(1)
    cache = kv4.Cache.random(rng, 4, 1, 16, 64)
    dev = device_cache(fd, cache)
    k, v = (torch.full((12, 1, 64), -3.0, device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    # sequence 0: tokens 12 .. 19 of one page; sequence 1: tokens -2 .. 1; its page is in the pool
    fd.fd_read_kv_q4(dev, i32([0, 1, 2]), i32([2, 1]), i32([12, -2]), i32([0, 8, 12]), k, v, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 4
    wk, wv = kv4.read(cache, [0, 1, 2], [2, 1], [12, 0], [0, 4, 6])
    at = [0, 1, 2, 3, 10, 11]
    assert np.array_equal(k[at].double().cpu().numpy(), wk) and np.array_equal(v[at].double().cpu().numpy(), wv)
    rest = [4, 5, 6, 7, 8, 9]
    assert (k[rest] == -3).all() and (v[rest] == -3).all()


def test_nan_comes_back_as_nan(fd):
    cache = kv4.Cache(1, 1, 16, 64)
    cache.put(0, 0, 2, np.r_[np.ones(32), np.full(32, np.inf)], np.r_[np.nan, np.ones(63)])
    dev = device_cache(fd, cache)
    k, v = (torch.zeros(16, 1, 64, device="cuda") for _ in range(2))
    fd.fd_read_kv_q4(dev, i32([0, 1]), i32([0]), None, i32([0, 16]), k, v)
    k, v = k.cpu(), v.cpu()
    assert torch.isnan(k[2, 0, 32:]).all() and (k[2, 0, :32] == 1).all() and torch.isnan(v[2]).all()
    k[2], v[2] = 0, 0
    assert (k == 0).all() and (v == 0).all()


# ---- attention --------------------------------------------------------------------------------
LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 127, 128, 129, 300, 700]


@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("k,m", [(1, 0), (0, 1), (3, 5), (8, 8)])
def test_lengths(fd, dim, k, m):
    B = len(LENGTHS)
    call = Q4Call(fd, kv=LENGTHS, k=[k] * B, m=[m] * B, hq=8, hkv=2, dim=dim, seed=k + m).upload()
    call.check(*call.run())
    assert int(call.status.item()) == 0


@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 1), (10, 2), (7, 1), (16, 2), (33, 1)])
@pytest.mark.parametrize("ps", [16, 32, 48])
def test_heads_and_pages(fd, hq, hkv, ps):
    """1, 4, 5, 7, 8 and 33 query heads a KV head; tile rows on both sides of 32, 64, 128 and 256."""
    call = Q4Call(fd, kv=[200, 77, 0, 513, 31], k=[1, 9, 4, 16, 3], m=[0, 8, 1, 16, 30], hq=hq, hkv=hkv, ps=ps, seed=hq + ps).upload()
    call.check(*call.run())
    assert int(call.status.item()) == 0


@pytest.mark.parametrize("kv_chunk", [64, 128, 1024])
@pytest.mark.parametrize("dim", [128, 64])
def test_pieces(fd, kv_chunk, dim):
    """Items in many pieces, the last of which may hold nothing but new rows."""
    call = Q4Call(fd, kv=[1500, 64, 63, 0, 1984, 700], k=[8, 1, 4, 40, 0, 33], m=[8, 0, 3, 0, 70, 15], hq=4, hkv=1, dim=dim, seed=kv_chunk,
                  heads_first=True).upload(kv_chunk=kv_chunk)
    call.check(*call.run())
    assert int(call.status.item()) == 0


@pytest.mark.parametrize("vis", [None, "given"])
def test_mask_blocks(fd, vis):
    """Several isolated blocks a sequence, one per hypothetical number of accepted drafts: more than 128 tile rows and new keys in several blocks of 32."""
    k, nb, per = np.array([16, 4, 1, 3]), np.array([16, 4, 1, 2]), np.array([16, 8, 5, 7])
    call = Q4Call(fd, kv=[500, 90, 33, 0], k=k, m=nb * per, hq=8, hkv=2, blocks=nb, vis=None if vis is None else np.array([0, 2, 1, 1]), seed=5).upload()
    call.check(*call.run())
    assert int(call.status.item()) == 0


def test_larger_batch_without_a_chunk(fd):
    """More items than pieces are aimed at, and sequences whose lengths differ by three orders: whole items beside split ones."""
    rng = np.random.default_rng(0)
    kv = np.r_[rng.integers(0, 60, size=300), 3000]
    call = Q4Call(fd, kv=kv, k=[2] * 301, m=[1] * 301, hq=8, hkv=4, seed=4).upload()
    call.check(*call.run())


@pytest.mark.parametrize("B,hkv", [(64, 8), (65, 2), (100, 1), (130, 4), (257, 1)])
def test_batches(fd, B, hkv):
    """Lengths of up to 64 sequences, of up to 256 and of more; pieces in one round and, the longest first, in several."""
    rng = np.random.default_rng(B)
    kv = np.where(rng.random(B) < 0.1, rng.integers(800, 1500, size=B), rng.integers(0, 200, size=B))
    call = Q4Call(fd, kv=kv, k=rng.integers(0, 3, size=B), m=rng.integers(0, 2, size=B), hq=2 * hkv, hkv=hkv, seed=B).upload()
    call.check(*call.run())
    assert int(call.status.item()) == 0


@pytest.mark.parametrize("dim,hq,ps", [(128, 8, 16), (64, 8, 48), (128, 2, 32)])
def test_long_pieces(fd, dim, hq, ps):
    """More blocks of a wave than lanes that know where they lie, also where the piece ends in the middle of a page."""
    call = Q4Call(fd, kv=[9001, 2049], k=[8, 3], m=[8, 5], hq=hq, hkv=1, dim=dim, ps=ps, seed=31).upload(kv_chunk=8192)
    call.check(*call.run())


def test_scale_and_sharp_scores(fd):
    """Scores that spread over some hundred units of base 2: the running maximum moves often."""
    call = Q4Call(fd, kv=[400, 900], k=[4, 4], m=[4, 4], std=6.0, seed=8).upload(sm_scale=0.3)
    call.check(*call.run(), sm_scale=0.3)


@pytest.mark.parametrize("dim", [128, 64])
def test_one_large_channel(fd, dim):
    """A channel of the query is a thousand times the others, and the scale keeps the softmax from being sharp: the small products count all the same."""
    call = Q4Call(fd, kv=[3, 40, 700, 0], k=[2, 1, 4, 1], m=[0, 3, 4, 0], hq=8, hkv=2, dim=dim, seed=21)
    q = oa.widen_bf16(call.q)
    q[..., 5] *= 1024.0
    call.q = bits_of(q)
    call.upload(sm_scale=2.0 ** -9)
    call.check(*call.run(), sm_scale=2.0 ** -9)


@pytest.mark.parametrize("dim", [128, 64])
def test_lse_of_few_keys(fd, dim):
    """With a handful of keys nothing averages out.  A score is a sum of dim products in fp32, off by at most dim 2^-24 of the sum of their magnitudes, and
    an lse by no more than its worst score; its maximum, exponentials, sum and logarithm add 2^-20 of max(1, |lse|)."""
    call = Q4Call(fd, kv=[1, 2, 3, 5, 4], k=[1, 2, 4, 3, 1], m=[0] * 5, hq=16, hkv=4, dim=dim, seed=22).upload()
    out, lse = call.run()
    call.check(out, lse)
    _, ref = call.oracle()
    kmax = max(np.abs(call.cache.key_values()).max(), np.abs(oa.widen_bf16(call.k_new)).max())
    q = np.abs(oa.widen_bf16(call.q))
    bound = dim * 2.0 ** -24 * q.sum(-1) * kmax / np.sqrt(dim) + 2.0 ** -20 * np.maximum(1, np.abs(ref))
    assert (np.abs(lse - ref) <= bound).all(), float((np.abs(lse - ref) / bound).max())
    # and by far less where errors do not add up: half a step of fp32 a product, independent
    assert np.sqrt(np.mean((lse - ref) ** 2)) <= 2.0 ** -20 * np.sqrt(np.mean(ref ** 2) + 1)


def test_what_lies_behind_the_prefix_does_not_count(fd):
    """Slots behind the last token hold NaN scales and any codes; pages that no list holds, too."""
    call = Q4Call(fd, kv=[1, 20, 47, 100], k=[2, 2, 2, 2], m=[3, 3, 3, 3], seed=6)
    seen = np.zeros(call.cache.shape[::2][:2], dtype=bool)
    for i, L in enumerate(call.kv):
        for pos in range(L):
            seen[call.page_indices[call.page_indptr[i] + pos // 16], pos % 16] = True
    for page, slot in np.argwhere(~seen):
        call.cache.k_scale[page, :, slot] = 255
        call.cache.v_scale[page, :, slot] = np.nan
    call.upload()
    call.check(*call.run())


@pytest.mark.parametrize("odd", [np.inf, -np.inf, np.nan])
def test_odd_values_reach_only_rows_that_see_them(fd, odd):
    """Mask rows with infinities and NaN in K and V: verify rows, and rows of other blocks, do not notice."""
    call = Q4Call(fd, kv=[50, 3, 200], k=[4, 4, 20], m=[8, 8, 40], blocks=np.array([2, 2, 2]), hq=4, hkv=1, seed=2)
    clean_v, clean_k = call.v_new.copy(), call.k_new.copy()
    bad = bits_of(np.array([odd]))[0]
    hit = np.zeros(int(call.n.sum()), dtype=bool)
    for i in range(3):
        r0, k, per = int(call.row_indptr[i]), int(call.k[i]), int(call.n[i] - call.k[i]) // 2
        call.v_new[r0 + k + per, 0, 5] = bad              # the second block's first row
        call.k_new[r0 + k + per + 1, 0, 9] = bad
        hit[r0 + k + per:r0 + k + 2 * per] = True
    call.upload()
    out, lse = call.run()
    call.v_new, call.k_new = clean_v, clean_k
    ref, ref_lse = call.oracle()
    size, _ = call.oracle(magnitudes=True)
    ok = ~hit
    assert np.isfinite(out[ok]).all() and np.isfinite(lse[ok]).all()
    assert (np.abs(out - ref)[ok] <= (2.0 ** -8 * (np.abs(ref) + size) + 2.0 ** -12 * size)[ok]).all()
    if not np.isnan(odd):                                 # an infinite value that is seen shows; the rest of its row's channels do not change for it
        call.v_new[:] = clean_v
        for i in range(3):
            r0, k, per = int(call.row_indptr[i]), int(call.k[i]), int(call.n[i] - call.k[i]) // 2
            call.v_new[r0 + k + per, 0, 5] = bad
        call.upload()
        out, _ = call.run()
        assert (out[hit][:, :, 5] == odd).all()
        rest = np.delete(np.arange(128), 5)
        assert (np.abs(out - ref)[hit][:, :, rest] <= (2.0 ** -8 * (np.abs(ref) + size) + 2.0 ** -12 * size)[hit][:, :, rest]).all()


def test_a_stored_nan_is_seen_by_every_row_of_its_sequence(fd):
    call = Q4Call(fd, kv=[40, 40], k=[2, 2], m=[2, 2], hq=2, hkv=2, seed=3)
    page = call.page_indices[call.page_indptr[1]]
    call.cache.v_scale[page, 0, 4] = np.nan
    call.upload()
    out, lse = call.run()
    n = int(call.row_indptr[1])
    assert np.isfinite(out[:n]).all() and np.isnan(out[n:, 0]).all() and np.isfinite(out[n:, 1]).all()
    assert np.isfinite(lse).all()
    for group in range(4):                                # a NaN among 32 channels of a key
        call.cache.v_scale[page, 0, 4] = 0.5
        call.cache.k_scale[page, 0, 4] = 125
        call.cache.k_scale[page, 0, 4, group] = 255
        out, lse = call.upload().run()
        assert np.isfinite(out[:n]).all() and np.isnan(out[n:, 0]).all() and np.isfinite(out[n:, 1]).all()
        assert np.isnan(lse[n:, 0]).all() and np.isfinite(lse[n:, 1]).all() and np.isfinite(lse[:n]).all()


def test_odd_queries_stay_in_their_row(fd):
    """Queries of zeros, the smallest and the largest bf16s, infinities and NaN, and elements of very different size in one row."""
    call = Q4Call(fd, kv=[300], k=[10], m=[0], hq=4, hkv=2, seed=7)
    q = _wide(call.q)
    q[0] = 0
    q[1] *= 2.0 ** -125
    q[2] *= 2.0 ** -100
    q[3, :, ::2] *= 2.0 ** -20
    q[4, :, 1:] *= 2.0 ** -13
    q[5, :, :64] *= 2.0 ** -9
    call.q = bits_of(q)
    call.upload()
    call.check(*call.run())
    q[6, 1, 3], q[7, 0, 100], q[8, 2, 64] = np.inf, np.nan, -np.inf
    call.q = bits_of(q)
    out, lse = call.upload().run()
    bad = np.zeros((10, 4), dtype=bool)
    bad[6, 1] = bad[7, 0] = bad[8, 2] = True
    assert np.isnan(out[bad]).all() and np.isfinite(out[~bad]).all() and np.isnan(lse[bad]).all() and np.isfinite(lse[~bad]).all()


def test_rows_behind_the_last_sequence_stay(fd):
    call = Q4Call(fd, kv=[100, 20, 0], k=[2, 0, 1], m=[1, 0, 0], spare_rows=3).upload()
    out, lse = call.run()
    call.check(out, lse)
    R = int(call.n.sum())
    assert (out[R:] == -7).all() and (lse[R:] == -7).all()


def test_without_lse_and_empty_calls(fd):
    call = Q4Call(fd, kv=[100, 20], k=[2, 1], m=[1, 0]).upload()
    call.args.lse = None
    out, lse = call.run()
    assert (lse == -7).all()
    call2 = Q4Call(fd, kv=[100, 20], k=[2, 1], m=[1, 0]).upload()
    want, _ = call2.run()
    assert np.array_equal(out, want)
    call2.out.fill_(-7)
    call2.args.total_rows = 0
    out, _ = call2.run()
    assert (out == -7).all()


def test_bad_device_data_is_reported(fd):
    """Lengths above the bound, page ids outside the pool, rows that contradict each other: clamped and reported."""
    for name, at, value, bit in (("kv_len", 1, 10 ** 6, 1), ("kv_len", 0, -4, 1), ("page_indices", 2, -1, 4), ("page_indices", 1, 10 ** 7, 4),
                                 ("page_indptr", 3, 10 ** 6, 4), ("verify_len", 2, 99, 2), ("row_indptr", 1, 1000, 2)):
        call = Q4Call(fd, kv=[64, 100, 30], k=[2, 2, 2], m=[2, 2, 2], seed=1).upload()
        call.d[name][at] = value
        call.run()
        assert int(call.status.item()) & bit, (name, at, value, int(call.status.item()))


def test_offsets_past_32_bits(fd):
    """A pool whose codes take 5 GB an array: pages from its end, and from both sides of 4 GiB."""
    H, D, ps, pool = 8, 128, 16, 620_000
    rng = np.random.default_rng(0)
    call = Q4Call(fd, kv=[90, 33], k=[3, 2], m=[2, 0], hq=8, hkv=H, room=16, seed=12)
    far = np.r_[pool - 1, 4 * 2 ** 30 // (H * 1024) + np.array([-1, 0, 1]), pool - 2 - rng.permutation(20)][:len(call.page_indices)]
    big = fd.Q4Cache(torch.empty(pool, H, ps, D // 2, dtype=torch.uint8, device="cuda"), torch.empty(pool, H, ps, D // 32, dtype=torch.uint8, device="cuda"),
                     torch.empty(pool, H, ps // 16, 8 * D, dtype=torch.uint8, device="cuda"), torch.empty(pool, H, ps, dtype=torch.bfloat16, device="cuda"))
    call.upload()
    src, dst = torch.from_numpy(call.page_indices).cuda(), torch.from_numpy(far).cuda()
    for n in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(big, n)[dst] = getattr(call.dev, n)[src]
    call.d["page_indices"].copy_(i32(far))
    call.args.num_pages = pool
    call.dev = big
    call.check(*call.run())
    # commit there, and read it back
    accept = i32([2, 1])
    out = torch.zeros(2, dtype=torch.int32, device="cuda")
    fd.fd_append_kv_q4(call.args, big, accept, out)
    want, lens = kv4.append(call.cache, _wide(call.k_new), _wide(call.v_new), call.page_indptr, call.page_indices, call.kv, call.row_indptr, call.k, [2, 1])
    rows = np.r_[0, np.cumsum(lens)]
    k, v = (torch.empty(int(rows[-1]), H, D, device="cuda") for _ in range(2))
    fd.fd_read_kv_q4(big, call.d["page_indptr"], call.d["page_indices"], None, i32(rows), k, v)
    wk, wv = kv4.read(want, call.page_indptr, call.page_indices, [0, 0], rows)
    assert np.array_equal(k.double().cpu().numpy(), wk) and np.array_equal(v.double().cpu().numpy(), wv)


def test_two_streams_and_repeats_agree(fd):
    """Two calls at once on two streams, a workspace each; and every repeat gives the same bits."""
    calls = [Q4Call(fd, kv=[900, 40, 333], k=[4, 2, 8], m=[4, 0, 8], hq=8, hkv=2, seed=s).upload() for s in (1, 2)]
    want = [c.run() for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    for c in calls:
        c.out.fill_(-7)
    torch.cuda.synchronize()
    for _ in range(5):
        for c, st in zip(calls, streams):
            fd.fd_verify_draft_attn_q4(c.args, c.dev, stream=st)
    torch.cuda.synchronize()
    for c, (out, lse) in zip(calls, want):
        assert np.array_equal(c.out.float().cpu().numpy(), out) and np.array_equal(c.lse.cpu().numpy(), lse)
