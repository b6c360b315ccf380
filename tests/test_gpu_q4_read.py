"""Read-back from a 4-bit cache where its offsets contradict each other, and for very many sequences."""
import numpy as np
import pytest
import torch

from oracle import kv4
from tests.q4_harness import Q4Call, assert_cache_is, device_cache, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offsets,whole", [([0, 8, 4, 12], [0, 2]), ([0, 8, 8, 40], [0, 1]), ([-3, 8, 8, 12], [1, 2]), ([0, 12, 0, 12], []),
                                           ([0, -2 ** 31, 2 ** 31 - 1, 12], [])])
def test_offsets_that_contradict_each_other_are_reported(fd, offsets, whole):
    """Offsets that decrease or leave the output: reported, and no row outside the output is written.  whole: sequences that are checked in the rows
    which no other claims."""
    rng = np.random.default_rng(5)
    cache = kv4.Cache.random(rng, 4, 2, 16, 64)
    dev = device_cache(fd, cache)
    big = [torch.full((40, 2, 64), -3.0, device="cuda") for _ in range(2)]
    k, v = (x[14:26] for x in big)                                                # 12 rows, with others of ours on both sides
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fd.fd_read_kv_q4(dev, i32([0, 1, 2, 3]), i32([2, 0, 3]), None, i32(offsets), k, v, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) & 2, int(status.item())
    for x in big:
        assert (x[:14] == -3).all() and (x[26:] == -3).all()
    for i in whole:
        a, b = offsets[i], offsets[i + 1]
        others = [range(max(offsets[j], 0), min(offsets[j + 1], 12)) for j in range(3) if j != i]
        rows = [r for r in range(a, b) if not any(r in o for o in others)]
        wk, wv = kv4.read(cache, [0, 1, 2, 3], [2, 0, 3], [0, 0, 0], [0] * (i + 1) + [b - a] * (3 - i))
        at = [r - a for r in rows]
        assert np.array_equal(k[rows].double().cpu().numpy(), wk[at]) and np.array_equal(v[rows].double().cpu().numpy(), wv[at])


def test_a_thousand_sequences(fd):
    """Attention, commit and read-back of a batch that takes many rounds of 64 sequences, some without rows or without a prefix."""
    B = 1000
    rng = np.random.default_rng(8)
    kv, k = rng.integers(0, 40, size=B), rng.integers(0, 3, size=B)
    kv[rng.random(B) < 0.2] = 0
    call = Q4Call(fd, kv=kv, k=k, m=rng.integers(0, 2, size=B), hq=4, hkv=2, dim=64, room=2, seed=8).upload()
    call.check(*call.run())
    accept = np.maximum(k - 1, 0)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    fd.fd_append_kv_q4(call.args, call.dev, i32(accept), lens)
    wide = lambda bits: (np.asarray(bits).astype(np.uint32) << 16).view(np.float32).astype(np.float64)  # noqa: E731
    want, after = kv4.append(call.cache, wide(call.k_new), wide(call.v_new), call.page_indptr, call.page_indices, call.kv, call.row_indptr, call.k, accept)
    assert np.array_equal(lens.cpu().numpy(), after)
    assert_cache_is(call.dev, want)
    start = np.minimum(rng.integers(0, 12, size=B), after)
    offsets = np.r_[0, np.cumsum(after - start)]
    out = [torch.full((int(offsets[-1]) + 1, 2, 64), -3.0, device="cuda") for _ in range(2)]
    fd.fd_read_kv_q4(call.dev, call.d["page_indptr"], call.d["page_indices"], i32(start), i32(offsets), *out, status=call.status)
    for x, w in zip(out, kv4.read(want, call.page_indptr, call.page_indices, start, offsets)):
        assert np.array_equal(x[:-1].double().cpu().numpy(), w) and (x[-1] == -3).all()
    assert int(call.status.item()) == 0
