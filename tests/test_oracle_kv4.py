"""Pins of the oracle of the 4-bit cache, the step tables and the rotation."""
import numpy as np
import pytest

from oracle import kv4


def test_midpoints_go_to_the_even_code():
    assert [kv4.nearest_code(x) for x in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)] == [0, 2, 2, 4, 4, 6, 6]
    assert [kv4.nearest_code(x) for x in (0.26, 0.74, 1.26, 1.74, 2.51, 3.49, 5.01, 7.0)] == [1, 1, 3, 3, 5, 5, 7, 7]
    assert kv4.nearest_code(-3.0) == 13 and kv4.nearest_code(-0.0) == 8 and kv4.nearest_code(0.0) == 0
    assert list(kv4.code_value(np.arange(16))) == [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]


def test_key_exponents():
    for e in (-126, -3, 0, 5):
        x = np.zeros(32)
        x[7] = -6.0 * 2.0 ** e
        assert kv4.key_exponent(x) == e
        x[7] = np.nextafter(6.0 * 2.0 ** e, np.inf)
        assert kv4.key_exponent(x) == e + 1
    assert kv4.key_exponent(np.zeros(32)) == -126
    codes, scales = kv4.quantize_key(np.r_[np.full(32, 3.0), np.full(32, -np.inf)])
    assert list(scales) == [126, 255] and (codes[:32] == 7).all() and (codes[32:] == 0).all()       # 3 = 6 * 2^-1


def test_value_scale_is_a_bf16():
    codes, s = kv4.quantize_value(np.linspace(-7, 7, 64))
    assert s == kv4.bf16_round(7 / 6) == 1.1640625 and codes[0] == 15 and codes[-1] == 7
    assert kv4.quantize_value(np.zeros(64))[1] == 0.0
    assert np.isnan(kv4.quantize_value(np.r_[np.nan, np.zeros(63)])[1])


def test_error_is_half_a_step():
    x = np.random.default_rng(1).standard_normal(128)
    codes, scales = kv4.quantize_key(x)
    back = kv4.code_value(codes) * np.repeat(2.0 ** (scales - 127.0), 32)
    unit = np.repeat(2.0 ** (scales - 127.0), 32)
    a = np.abs(x) / unit
    assert (np.abs(back - x) / unit <= np.where(a < 2, .25, np.where(a < 4, .5, 1.0))).all()


def test_packing_of_a_block():
    c = kv4.Cache(1, 1, 16, 64)
    c.k[0, 0, 3, 10], c.k[0, 0, 3, 11] = 5, 9
    c.v[0, 0, 13, 33] = 6                            # half 1, word of j = 1, c = 1, slot 5 of eight: byte 2, high
    k, _, v, _ = c.packed()
    assert k[0, 0, 3, 5] == 5 | 9 << 4 and np.count_nonzero(k) == 1
    assert v[0, 0, 0, ((32 + 1) * 2 + 1) * 4 + 2] == 6 << 4 and np.count_nonzero(v) == 1


def test_page_exchange_by_hand():
    """Page size 4.  Request 0 has ended and holds 2 pages; 1 needs ceil(9 / 4) = 3 of its 1; 2 needs 1 of its 2; 3 needs 2 of its 0."""
    table = [[10, 11, -1], [12, -1, -1], [13, 14, -1], [-1, -1, -1]]
    r = kv4.step_tables([0, 6, 2, 4], [0, 3, 2, 1], [0, 2, 0, 0], table, [2, 1, 2, 0], [20, 21, -1, -1, -1], 2, 4)
    # the stack becomes 20 21 10 11 14; request 1 takes 14 and 11, request 3 takes 10 and 21
    assert r["page_indices"] == [12, 14, 11, 13, 10, 21] and r["page_indptr"] == [0, 0, 3, 4, 6]
    assert r["free_count"] == 1 and r["free_pages"][0] == 20 and not r["short"]
    assert r["row_indptr"] == [0, 0, 5, 7, 8]
    assert r["positions"] == [6, 7, 8, 9, 10, 2, 3, 4]
    assert r["slot_map"] == [14 * 4 + 2, 14 * 4 + 3, 11 * 4, -1, -1, 13 * 4 + 2, 13 * 4 + 3, 21 * 4]
    # with an empty pool behind what is given back the last request stays short
    r = kv4.step_tables([0, 6, 2, 4], [0, 3, 2, 1], [0, 0, 0, 0], table, [2, 1, 2, 0], [0, 0, 0], 0, 4)
    assert r["short"] and r["table_len"] == [0, 3, 1, 1] and r["slot_map"][-1] == -1


def test_positions_of_mask_blocks():
    """Three verify rows and two blocks of two: the blocks follow two and three verify rows."""
    r = kv4.step_tables([100], [3], [4], [[1] * 8], [8], [0] * 8, 0, 16, None, [2])
    assert r["positions"] == [100, 101, 102, 102, 103, 103, 104]
    r = kv4.step_tables([100], [3], [4], [[1] * 8], [8], [0] * 8, 0, 16, [1], [2])
    assert r["positions"] == [100, 101, 102, 101, 102, 102, 103]


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation(interleaved):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((5, 1, 32))
    f = 10.0 ** -np.arange(8)
    one = lambda pos: kv4.norm_rope(x, None, np.full(5, pos), f, 0.0, interleaved)[0]  # noqa: E731
    assert np.allclose(np.linalg.norm(one(7), axis=-1), np.linalg.norm(x, axis=-1))
    assert np.array_equal(one(0), x)
    dots = [(one(a)[0, 0] * one(b)[1, 0]).sum() for a, b in ((3, 5), (103, 105))]
    assert abs(dots[0] - dots[1]) < 1e-12                        # only the difference of positions counts
    assert np.array_equal(one(9)[..., 16:], x[..., 16:])          # what lies behind the rotary dim stays
    y, _ = kv4.norm_rope(x, np.ones(32), np.zeros(5), f, 0.0, interleaved)
    assert np.allclose((y * y).mean(-1), 1.0)
