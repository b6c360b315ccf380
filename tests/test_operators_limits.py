"""Limits of the calls around a 4-bit cache, on both sides, as far as the host decides them."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2605_20022_amd import flexdraft as fd
from tests.test_operators_host import P, ROOT, _attn, _cache, _refused, _rope, _tables


@pytest.mark.parametrize("entries", ["page_indices_len", "free_pages_len"])
def test_step_tables_sum_in_32_bits(entries):
    """A round of 1024 requests moves and lists up to 2^30 pages, which the kernel adds to a number of entries in 32 bits: 2^30 entries would be one too many."""
    for n in (1 << 30, (1 << 31) - 1):
        _refused(_tables(**{entries: n}), 2, "2^30")
    # one fewer is taken: the next check has its turn
    _refused(_tables(**{entries: (1 << 30) - 1, "kv_len": None}), 1, "NULL")


def _weight(rows):
    """How long a block takes a work-group with so many tile rows, in halves (attn_q4.hip)."""
    return 0 if rows == 0 else 2 if rows <= 32 else 3 if rows <= 64 else 6


def test_work_is_counted_in_32_bits_whatever_the_rows_on_the_device(tmp_path):
    """The kernel sums the work of all sequences in units of 2^unit_shift.  Row offsets that overlap can give each of them max_new_rows rows, and the sum must
    hold those too: from it follows how many pieces there are, and where their partial rows go."""
    src = '''#include <stdio.h>
#include "q4_shape.h"
int main() { int a[8]; while (scanf("%d %d %d %d %d %d %d %d", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7) == 8)
  printf("%d\\n", fd::q4_shape(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]).unit_shift); }
'''
    (tmp_path / "t.cpp").write_text(src)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_20022_amd", "csrc"), str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")])
    shapes = [(B, H, G, R, L, n, 0, 128) for B in (1, 16, 64, 65, 256, 1000, 65535) for H in (1, 8) for G in (1, 4, 16) for R in (1, 1000, 65536, 1 << 20)
              for L in (0, 4096, 1 << 21, 1 << 30) for n in (1, 16, 272, 65536, 1 << 20) if n * G <= 1 << 24]
    out = subprocess.run([str(tmp_path / "t")], input="\n".join(" ".join(map(str, s)) for s in shapes), capture_output=True, text=True, check=True).stdout.split()
    assert len(out) == len(shapes)
    for (B, H, G, R, L, n, *_), shift in zip(shapes, map(int, out)):
        n = min(n, R)
        blocks = -(-L // 32) + 4 + 3 * -(-n // 32)
        units = blocks * (n * G // 128 * _weight(128) + _weight(n * G % 128))
        assert B * -(-units // (1 << shift)) < 1 << 31, (B, H, G, R, L, n, shift)
    # where the work is little, as in any ordinary call, it is counted as it is
    assert {int(s) for (B, H, G, R, L, n, *_), s in zip(shapes, out) if B <= 256 and L <= 4096 and n <= 272} == {0}


def _read(total_rows, batch=2, **kw):
    a = dict(page_indptr=P, page_indices=P, out_indptr=P, k_out=P, v_out=P)
    a.update(kw)
    return fd.load().fd_read_kv_q4(C.byref(_cache()), batch, 8, 128, 16, 10, a["page_indptr"], a["page_indices"], 20, None, a["out_indptr"], total_rows, a["k_out"],
                                   a["v_out"], fd.FD_F32, None, None)


def test_read_back_of_too_many_rows_for_a_launch():
    """2^24 work-groups of 256 threads, 64 rows each and up to two more a sequence."""
    for rows, batch in ((1 << 30, 1), ((1 << 31) - 1, 65535), ((1 << 30) - 64 * 4, 2)):
        _refused(_read(rows, batch), 2, "too large")
    _refused(_read((1 << 30) - 64 * 4 - 1, 2, v_out=None), 1, "NULL")


@pytest.mark.parametrize("page_size,pages,heads,stride_page,stride_head", [(16, (1 << 25) + 1, 8, 8, 1), (32, 1 << 24, 8, 8, 1), (16, 1 << 25, 8, 8, 1),
                                                                           (16, (1 << 28) - 7, 1, 1, 1), (16, 64, 4, 1, 1 << 24), (16, 3, 8, 64 * (1 << 20), 1),
                                                                           (16, 1 << 19, 8, 512, 1), (16, (1 << 19) + 1, 8, 512, 1)])
def test_slots_are_numbered_in_32_bits(page_size, pages, heads, stride_page, stride_head):
    """On both sides of 2^32 slots, and with strides that leave blocks out (a pool that 64 layers share)."""
    fits = page_size * ((pages - 1) * stride_page + (heads - 1) * stride_head + 1) <= 1 << 32
    cache = _cache(stride_page=stride_page, stride_head=stride_head)
    args = dict(page_size=page_size, num_pages=pages, num_kv_heads=heads, num_q_heads=heads * 4)
    a, b = _attn(**dict(args, workspace=None)), _attn(**dict(args, k_new=None))
    calls = [fd.load().fd_verify_draft_attn_q4(C.byref(a), C.byref(cache), None), fd.load().fd_append_kv_q4(C.byref(b), C.byref(cache), P, P, None),
             fd.load().fd_read_kv_q4(C.byref(cache), 2, heads, 128, page_size, pages, P, P, 20, None, P, 5, None, P, fd.FD_F32, None, None)]
    assert calls == ([1, 1, 1] if fits else [2, 2, 2])            # (what fits: the missing pointer has its turn)
    if not fits:
        assert b"2^32" in fd.load().fd_last_error()


def test_no_workspace_for_a_call_that_is_refused():
    """Heads and page sizes that the attention refuses need no workspace, 0 says so; the products of the largest sizes do not wrap to a small one."""
    need = lambda **kw: fd.load().fd_verify_draft_attn_q4_workspace(C.byref(_attn(**kw)))  # noqa: E731
    most = (1 << 31) - 1
    for kw in (dict(num_kv_heads=65536, num_q_heads=65536), dict(num_kv_heads=most, num_q_heads=most, batch=65535, max_new_rows=1 << 24, total_rows=most),
               dict(num_kv_heads=65535, num_q_heads=65535, batch=65535, max_new_rows=1 << 24, total_rows=most, max_kv_len=1 << 30, kv_chunk=64),
               dict(page_size=24), dict(page_size=0), dict(page_size=-16)):
        assert need(**kw) == 0, kw
    assert need(num_kv_heads=65535, num_q_heads=65535, batch=1, total_rows=1, max_new_rows=1) > 0


def test_strides_of_dimensions_of_one_do_not_matter():
    """Between rows where there is one row, and between heads where there is one: any number.  (The next check has its turn: the call is not made.)"""
    for kw in (dict(total_rows=1, q_stride_row=1, k_stride_row=-3), dict(num_q_heads=1, q_stride_head=65), dict(num_kv_heads=1, k_stride_head=1),
               dict(num_kv_heads=1, total_rows=1, v=P, v_out=P, v_stride_row=7, v_stride_head=9)):
        _refused(_rope(**dict(kw, q=P + 8)), 1, "aligned")
    for kw in (dict(total_rows=2, q_stride_row=1), dict(num_q_heads=2, q_stride_head=65), dict(num_kv_heads=2, k_stride_head=1)):
        _refused(_rope(**kw), 1, "strides")
