"""Read-back from a 4-bit cache where its offsets contradict each other, and for very many sequences."""
import numpy as np
import pytest
import torch

from oracle import kv4
from tests.q4_harness import device_cache, i32

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
