"""How the attention over a 4-bit cache cuts items into pieces, and what its pieces leave of a row: GPU parity against the fp64 oracle."""
import numpy as np
import pytest

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
