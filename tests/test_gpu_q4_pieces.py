"""How the attention over a 4-bit cache cuts items into pieces, and what its pieces leave of a row: GPU parity against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import kv4
from tests.q4_harness import Q4Call, bits_of

pytestmark = pytest.mark.gpu


def assert_rows_hold(call, out, channels=slice(None)):
    """Every channel by itself, whatever else its row holds.  A probability (times its value's scale) and the result are each rounded to bf16: half a
    step is 2^-8 of the value, so 2^-8 (|o| + sum p |v|).  The rest is fp32, partial rows of items in several pieces included: a score is off by less than
    2^-17 of the sum of its products' magnitudes, which changes a probability by at most twice that, and a sum over n keys by n 2^-23 of its terms' sum."""
    R, D = int(call.n.sum()), call.q.shape[2]
    ref, _ = call.oracle()
    size, _ = call.oracle(magnitudes=True)
    kmax = max(np.abs(call.cache.key_values()).max(), np.abs(oa.widen_bf16(call.k_new[:R])).max())
    score = 2.0 ** -17 * float(np.abs(oa.widen_bf16(call.q[:R])).sum(-1).max() * kmax / np.sqrt(D)) + 2.0 ** -20
    bound = 2.0 ** -8 * (np.abs(ref) + size) + (2 * score + (call.max_kv + call.max_n) * 2.0 ** -23) * size
    worst = float((np.abs(out[:R] - ref) / bound)[..., channels].max())              # (NaN where one is)
    assert worst <= 1.0, f"{worst:.2f} of the bound"


# ---- what a piece leaves of a row -------------------------------------------------------------
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("kv_chunk", [0, 64, 512])
@pytest.mark.parametrize("unit", [1e6, 1.0, 1e-6])
def test_an_infinity_leaves_the_other_channels_of_its_row(fd, dim, kv_chunk, unit):
    """Values of very different size; one channel of one new row is infinite, and every row sees it.  In one piece or in many, the other channels are what they are."""
    call = Q4Call(fd, kv=[1500, 90], k=[4, 3], m=[2, 0], hq=4, hkv=1, dim=dim, seed=41)
    call.cache.v_scale = kv4.bf16_round(call.cache.v_scale * unit)
    call.v_new = bits_of(oa.widen_bf16(call.v_new) * unit)
    odd, clean = call.v_new.copy(), call.v_new
    odd[call.row_indptr[:2], 0, 5] = bits_of([np.inf])[0]                    # each sequence's first row, which all of its rows see
    call.v_new = odd
    out, lse = call.upload(kv_chunk=kv_chunk).run()
    call.v_new = clean
    assert (out[:, :, 5] == np.inf).all() and np.isfinite(lse).all()
    assert_rows_hold(call, out, np.delete(np.arange(dim), 5))


@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("kv_chunk", [0, 64, 512])
def test_small_channels_beside_a_large_one(fd, dim, kv_chunk):
    """One channel of the new rows is a million times the others: those keep their digits in the pieces too."""
    call = Q4Call(fd, kv=[1500, 90, 400], k=[4, 3, 1], m=[2, 0, 8], hq=4, hkv=1, dim=dim, seed=42)
    v = oa.widen_bf16(call.v_new)
    v[..., 9] *= 2.0 ** 20
    call.v_new = bits_of(v)
    out, _ = call.upload(kv_chunk=kv_chunk).run()
    assert_rows_hold(call, out)


# ---- how items are cut ------------------------------------------------------------------------
ROUND = 512                       # work-groups that run at once


def items_of(call, hkv):
    """Items of the call: up to 128 tile rows of a sequence and KV head each."""
    group = call.q.shape[1] // hkv
    return hkv * int((-(-call.n * group // 128)).sum())


@pytest.mark.parametrize("B,hkv,dim", [(64, 8, 128), (64, 9, 64), (65, 8, 128), (130, 4, 128), (200, 3, 64), (256, 2, 128)])
def test_more_items_than_run_at_once(fd, B, hkv, dim):
    """As many items as work-groups run at once, or more, and no more sequences than a wave keeps the lengths of: sequences of very different length, taken the
    longest pieces first, by the variant of up to 64 sequences and the other.  Every sequence has a row."""
    rng = np.random.default_rng(B + hkv)
    kv = np.where(rng.random(B) < 0.1, rng.integers(800, 3000, size=B), rng.integers(0, 300, size=B))
    call = Q4Call(fd, kv=kv, k=rng.integers(1, 4, size=B), m=rng.integers(0, 3, size=B), hq=2 * hkv, hkv=hkv, dim=dim, seed=B)
    assert items_of(call, hkv) >= ROUND and B <= 256
    out, lse = call.upload().run()
    call.check(out, lse)
    assert_rows_hold(call, out)
    assert int(call.status.item()) == 0


@pytest.mark.parametrize("blocks", [None, 4])
def test_more_items_than_run_at_once_of_many_rows(fd, blocks):
    """Eight sequences of up to 272 new rows: whole items beside tails of 32, 64 and 128 tile rows, in several rounds."""
    n = np.array([272, 272, 265, 257, 200, 272, 259, 130])
    k = np.array([16, 16, 9, 1, 200, 12, 3, 130])
    nb = None if blocks is None else np.where((n - k) % blocks == 0, blocks, 1)
    call = Q4Call(fd, kv=[700, 3, 0, 90, 300, 1200, 31, 64], k=k, m=n - k, hq=32, hkv=8, blocks=nb, seed=51)
    assert items_of(call, 8) >= ROUND
    out, lse = call.upload().run()
    call.check(out, lse)
    assert_rows_hold(call, out)
    assert int(call.status.item()) == 0


@pytest.mark.parametrize("B,longest,alone", [(5, 4000, True), (8, 2500, True), (8, 14000, False), (24, 2000, False), (70, 900, False)])
def test_whole_items_and_tails_in_one_round(fd, B, longest, alone):
    """Fewer items than work-groups that run at once, with more of the shortest pieces than those: how far whole items of 128 tile rows and tails are cut is
    found by bisection.  alone: one piece a compute unit; else two."""
    rng = np.random.default_rng(B)
    kv, n = rng.integers(longest // 2, longest + 1, size=B), rng.choice([100, 97, 33, 70, 64], size=B)
    k = np.minimum(n, rng.integers(1, 30, size=B))
    call = Q4Call(fd, kv=kv, k=k, m=n - k, hq=8, hkv=2, seed=B)
    if B == 70:                                                   # (more than a wave's lanes: lengths through LDS)
        n = rng.choice([33, 40], size=B)
        call = Q4Call(fd, kv=kv, k=n, m=0 * n, hq=8, hkv=2, seed=B)
    items, blocks = items_of(call, 2), -(-call.kv // 32) + 4 + 3 * -(-call.n // 32)
    tail = call.n * 4 % 128
    weight = call.n * 4 // 128 * 6 + np.select([tail == 0, tail <= 32, tail <= 64], [0, 2, 3], 6)           # how long a block takes, in halves
    assert (items <= ROUND // 4 and 2 * int((blocks * weight).sum()) <= ROUND // 2 * 192) == alone
    shortest = 2 * int((-(-call.n * 4 // 128) * (blocks // 8 + 1)).sum())
    assert items < ROUND and shortest > (ROUND // 2 if alone else ROUND)
    out, lse = call.upload().run()
    call.check(out, lse)
    assert_rows_hold(call, out)
    assert int(call.status.item()) == 0


# ---- calls beside each other ------------------------------------------------------------------
def _bits(call):
    torch.cuda.synchronize()
    return call.out.view(torch.int16).clone(), call.lse.view(torch.int32).clone()


def test_graphs_that_share_a_workspace(fd):
    """Two captured calls of different shape on one workspace, replayed in turn with eager work in between: nothing in it has to survive, or to be what it was."""
    calls = [Q4Call(fd, kv=[900, 33], k=[4, 2], m=[4, 0], seed=61).upload(), Q4Call(fd, kv=[20, 1500], k=[1, 2], m=[4, 9], seed=62).upload()]
    shared = fd.alloc_workspace(max(c.workspace.numel() for c in calls))
    graphs, want = [], []
    for c in calls:
        c.args.workspace, c.args.workspace_bytes = shared.data_ptr(), shared.numel()
        c.check(*c.run())
        want.append(_bits(c))
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            fd.fd_verify_draft_attn_q4(c.args, c.dev)
    for turn in (0, 1, 0, 0, 1, 1, 0):
        c = calls[turn]
        c.out.fill_(-7)
        shared.random_(0, 255)
        graphs[turn].replay()
        for got, w in zip(_bits(c), want[turn]):
            assert torch.equal(got, w)


def test_pages_that_several_sequences_share(fd):
    """A common prefix: three lists of the same pages."""
    call = Q4Call(fd, kv=[64, 64, 64], k=[2, 3, 1], m=[1, 0, 4], seed=63)
    call.page_indices[4:8] = call.page_indices[8:12] = call.page_indices[:4]
    call.upload()
    out, lse = call.run()
    call.check(out, lse)
    assert_rows_hold(call, out)


@pytest.mark.parametrize("B", [3, 70, 300])
def test_sequences_without_rows(fd, B):
    """A batch none of whose sequences brings a row: nothing is written, and nothing is amiss."""
    call = Q4Call(fd, kv=[50] * B, k=[1] + [0] * (B - 1), m=[0] * B, spare_rows=4, seed=64).upload()
    call.d["row_indptr"].zero_()
    call.d["verify_len"].zero_()
    out, lse = call.run()
    assert (out == -7).all() and (lse == -7).all() and int(call.status.item()) == 0
