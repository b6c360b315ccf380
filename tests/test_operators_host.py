"""Refusals of the step tables, the norm and rotation and the calls over a 4-bit cache: all before any launch."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2605_20022_amd import flexdraft as fd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096                         # an address that is never dereferenced: the calls fail on the host


def _refused(call, code, words):
    assert call == code, fd.load().fd_last_error()
    assert words.encode() in fd.load().fd_last_error(), fd.load().fd_last_error()


@pytest.mark.parametrize("name,last", [("fd_table_args", "status"), ("fd_rope_args", "positions"), ("fd_q4_cache", "stride_head")])
def test_struct_layouts_match_the_header(name, last):
    mirror = getattr(fd, name)
    src = f'#include <stdio.h>\n#include "flexdraft.h"\nint main(){{printf("%zu %zu\\n", sizeof({name}), __builtin_offsetof({name}, {last}));return 0;}}\n'
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "t.c"), "w").write(src)
        subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), os.path.join(d, "t.c"), "-o", os.path.join(d, "t")])
        size, off = map(int, subprocess.check_output([os.path.join(d, "t")]).split())
    assert size == C.sizeof(mirror) and off == getattr(mirror, last).offset


def _tables(**kw):
    a = fd.fd_table_args()
    a.batch, a.page_size, a.table_stride, a.total_rows, a.page_indices_len, a.free_pages_len = 4, 16, 32, 64, 128, 128
    for n in ("kv_len", "verify_len", "block_table", "table_len", "table_len_out", "free_pages", "free_count", "free_count_out", "row_indptr",
              "page_indptr", "page_indices", "positions", "slot_map"):
        setattr(a, n, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return fd.load().fd_step_tables(C.byref(a), None)


def test_step_tables_refusals():
    assert fd.load().fd_step_tables(None, None) == 1
    for kw, code, words in ((dict(batch=-1), 1, "negative"), (dict(page_size=0), 1, "page_size"), (dict(batch=65536), 2, "batch"),
                            (dict(total_rows=(1 << 20) + 1), 2, "2^20"), (dict(table_stride=(1 << 20) + 1), 2, "2^20"),
                            (dict(free_pages_len=(1 << 30) + 1), 2, "2^30"), (dict(kv_len=None), 1, "NULL"), (dict(free_count=None), 1, "NULL"),
                            (dict(block_table=None), 1, "NULL"), (dict(page_indices=None), 1, "NULL"), (dict(free_pages=None), 1, "NULL"),
                            (dict(page_indptr=None), 1, "NULL")):
        _refused(_tables(**kw), code, words)


def _rope(**kw):
    a = fd.fd_rope_args()
    a.total_rows, a.num_q_heads, a.num_kv_heads, a.head_dim, a.rotary_dim, a.dtype, a.eps = 3, 8, 2, 128, 128, fd.FD_BF16, 1e-6
    a.q_stride_row, a.q_stride_head, a.k_stride_row, a.k_stride_head, a.v_stride_row, a.v_stride_head = 1024, 128, 256, 128, 256, 128
    for n in ("q", "k", "q_out", "k_out", "q_weight", "k_weight", "inv_freq", "positions"):
        setattr(a, n, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return fd.load().fd_qk_norm_rope(C.byref(a), None)


def test_norm_rope_refusals():
    assert fd.load().fd_qk_norm_rope(None, None) == 1
    for kw, code, words in ((dict(total_rows=-1), 1, "negative"), (dict(head_dim=100), 1, "head_dim"), (dict(head_dim=264), 2, "256"),
                            (dict(rotary_dim=136), 1, "rotary_dim"), (dict(rotary_dim=20), 1, "rotary_dim"), (dict(dtype=7), 1, "dtype"),
                            (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"), (dict(q=None), 1, "NULL"), (dict(k_out=None), 1, "NULL"),
                            (dict(v=P), 1, "together"), (dict(v_out=P), 1, "together"), (dict(positions=None), 1, "positions"),
                            (dict(inv_freq=None), 1, "inv_freq"), (dict(k_stride_row=-4), 1, "strides"), (dict(q_stride_head=130), 1, "strides"),
                            (dict(v=P, v_out=P, v_stride_row=2), 1, "strides"), (dict(q=P + 8), 1, "aligned"), (dict(k_weight=P + 2), 1, "aligned"),
                            (dict(num_q_heads=5000), 2, "heads")):
        _refused(_rope(**kw), code, words)
    assert _rope(total_rows=0, q=None, k=None) == 0
    assert _rope(num_q_heads=0, num_kv_heads=0) == 0


def _attn(**kw):
    a = fd.fd_attn_args()
    a.batch, a.num_q_heads, a.num_kv_heads, a.head_dim, a.page_size, a.dtype = 4, 32, 8, 128, 16, fd.FD_BF16
    a.total_rows, a.max_kv_len, a.max_new_rows, a.num_pages, a.page_indices_len = 64, 4096, 16, 2000, 1500
    for n in ("page_indptr", "page_indices", "kv_len", "row_indptr", "verify_len", "q", "k_new", "v_new", "out", "workspace"):
        setattr(a, n, P)
    a.workspace_bytes = 1 << 40
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _cache(**kw):
    c = fd.fd_q4_cache(P, P, P, P, 8, 1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_q4_attention_refusals():
    lib = fd.load()
    call = lambda a, c=_cache(): lib.fd_verify_draft_attn_q4(C.byref(a), None if c is None else C.byref(c), None)  # noqa: E731
    assert lib.fd_verify_draft_attn_q4(None, None, None) == 1 and lib.fd_verify_draft_attn_q4_workspace(None) == 0
    bad = ((dict(dtype=fd.FD_F32), 2, "bf16"), (dict(dtype=5), 1, "dtype"), (dict(head_dim=96), 2, "head_dim"), (dict(num_kv_heads=5), 1, "multiple"),
           (dict(kv_chunk=32), 1, "kv_chunk"), (dict(flags=fd.FD_ATTN_FORCE_GENERIC), 2, "full-precision"), (dict(sm_scale=float("nan")), 1, "sm_scale"),
           (dict(batch=65536), 2, "batch"), (dict(max_kv_len=(1 << 30) + 1), 2, "max_kv_len"), (dict(max_new_rows=(1 << 24)), 2, "2^24"),
           (dict(total_rows=-1), 1, "negative"), (dict(page_indices_len=-1), 1, "page_indices_len"))
    for kw, code, words in bad:
        _refused(call(_attn(**kw)), code, words)
        assert lib.fd_verify_draft_attn_q4_workspace(C.byref(_attn(**kw))) == 0
    for kw, code, words in ((dict(page_size=24), 2, "multiple of 16"), (dict(page_size=0), 1, "page_size"), (dict(q=None), 1, "NULL"),
                            (dict(page_indices=None), 1, "page_indices"), (dict(num_pages=0), 1, "num_pages"), (dict(max_new_rows=0), 1, "max_new_rows"),
                            (dict(workspace=None), 1, "workspace"), (dict(workspace=P + 16), 1, "aligned"), (dict(out=P + 8), 1, "aligned"),
                            (dict(workspace_bytes=lib.fd_verify_draft_attn_q4_workspace(C.byref(_attn())) - 1), 3, "workspace")):
        _refused(call(_attn(**kw)), code, words)
    _refused(call(_attn(), None), 1, "cache is NULL")
    for kw, words in ((dict(k_codes=P + 8), "aligned"), (dict(k_scales=P + 2), "aligned"), (dict(v_scales=P + 8), "aligned"), (dict(stride_page=-1), "strides"),
                      (dict(v_codes=None), "four arrays")):
        _refused(call(_attn(), _cache(**kw)), 1, words)
    assert call(_attn(batch=0)) == 0 and call(_attn(total_rows=0)) == 0


def test_q4_workspace_does_not_grow_with_the_prefix():
    need = lambda **kw: fd.load().fd_verify_draft_attn_q4_workspace(C.byref(_attn(**kw)))  # noqa: E731
    assert need() % 256 == 0 and need(max_kv_len=1 << 20) == need(max_kv_len=1 << 22)
    assert need(max_kv_len=64, batch=1, total_rows=1, max_new_rows=1) < need()
    assert need(kv_chunk=64) > need(kv_chunk=128) > 0


def test_q4_commit_and_read_refusals():
    lib = fd.load()
    call = lambda a, c=_cache(), acc=P, out=P: lib.fd_append_kv_q4(C.byref(a), C.byref(c), acc, out, None)  # noqa: E731
    assert lib.fd_append_kv_q4(None, None, None, None, None) == 1
    for kw, code, words in ((dict(dtype=fd.FD_F32), 2, "bf16"), (dict(head_dim=32), 2, "head_dim"), (dict(page_size=8), 2, "multiple of 16"),
                            (dict(num_kv_heads=0), 1, "num_kv_heads"), (dict(max_new_rows=65536), 2, "max_new_rows"), (dict(k_new=None), 1, "k_new"),
                            (dict(kv_len=None), 1, "NULL"), (dict(num_pages=0), 1, "num_pages"), (dict(v_new=P + 8), 1, "aligned")):
        _refused(call(_attn(**kw)), code, words)
    _refused(call(_attn(), acc=None), 1, "NULL")
    _refused(call(_attn(), out=None), 1, "NULL")
    assert call(_attn(batch=0)) == 0

    def read(c=_cache(), batch=2, heads=8, dim=128, ps=16, pages=10, indptr=P, indices=P, n=20, start=None, out_indptr=P, rows=5, k=P, v=P, dt=fd.FD_F32):
        return lib.fd_read_kv_q4(C.byref(c), batch, heads, dim, ps, pages, indptr, indices, n, start, out_indptr, rows, k, v, dt, None, None)
    for kw, code, words in ((dict(batch=-1), 1, "negative"), (dict(batch=65536), 2, "batch"), (dict(dim=96), 2, "head_dim"), (dict(ps=20), 2, "multiple of 16"),
                            (dict(dt=3), 1, "dtype"), (dict(k=None), 1, "NULL"), (dict(pages=0), 1, "num_pages"), (dict(v=P + 4), 1, "aligned"),
                            (dict(out_indptr=None), 1, "NULL"), (dict(c=_cache(k_scales=None)), 1, "NULL")):
        _refused(read(**kw), code, words)
    assert read(batch=0) == 0 and read(rows=0) == 0


def test_binding_checks_shapes():
    z = lambda *s, dt=torch.uint8: torch.zeros(s, dtype=dt)  # noqa: E731
    good = dict(k_codes=z(6, 2, 32, 64), k_scales=z(6, 2, 32, 4), v_codes=z(6, 2, 2, 1024), v_scales=z(6, 2, 32, dt=torch.bfloat16))
    c = fd.Q4Cache(**good)
    assert (c.num_pages, c.num_kv_heads, c.page_size, c.head_dim, c.c.stride_page, c.c.stride_head) == (6, 2, 32, 128, 2, 1)
    with pytest.raises(TypeError, match="v_codes"):
        fd.Q4Cache(**dict(good, v_codes=z(6, 2, 2, 512)))
    with pytest.raises(TypeError, match="v_scales"):
        fd.Q4Cache(**dict(good, v_scales=z(6, 2, 32)))
    with pytest.raises(TypeError, match="k_scales"):           # heads of another order than the codes'
        fd.Q4Cache(**dict(good, k_scales=z(2, 6, 32, 4).transpose(0, 1)))
    heads_first = {n: t.transpose(0, 1).contiguous().transpose(0, 1) for n, t in good.items()}
    c = fd.Q4Cache(**heads_first)
    assert (c.c.stride_page, c.c.stride_head) == (1, 6)
    q, k = z(3, 8, 128, dt=torch.bfloat16), z(3, 2, 128, dt=torch.bfloat16)
    with pytest.raises(TypeError, match="q_out"):
        fd.fd_qk_norm_rope(q, k, z(3, 8, 64, dt=torch.bfloat16), k, None, None)
    with pytest.raises(TypeError, match="positions"):
        fd.fd_qk_norm_rope(q, k, q, k, z(2, dt=torch.int32), torch.ones(64))
    with pytest.raises(TypeError, match="k_weight"):
        fd.fd_qk_norm_rope(q, k, q, k, None, None, k_weight=torch.ones(128))
    with pytest.raises(TypeError, match="table_len"):
        i = lambda n: z(n, dt=torch.int32)  # noqa: E731
        fd.make_table_args(i(2), i(2), z(2, 4, dt=torch.int32), i(3), i(8), i(1), page_size=16, row_indptr=i(3), page_indptr=i(3), page_indices=i(8))


def test_binding_refuses_tensors_that_no_kernel_may_touch():
    """Tensors in host memory, sizes that contradict each other, a cache of another shape than the call was made for."""
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda n: z(n, dt=torch.int32)  # noqa: E731
    q, k = z(3, 8, 128), z(3, 2, 128)
    with pytest.raises(TypeError, match="CPU"):
        fd.fd_qk_norm_rope(q, k, q, k, i(3), torch.ones(64))
    tables = lambda **kw: fd.make_table_args(i(2), i(2), z(2, 4, dt=torch.int32), i(2), i(8), i(1), page_size=16, row_indptr=i(3), page_indptr=i(3),  # noqa: E731
                                             page_indices=i(8), **kw)
    with pytest.raises(TypeError, match="CPU"):
        fd.fd_step_tables(tables())
    c = fd.alloc_q4_cache(6, 2, 32, 128, device="cpu")
    with pytest.raises(TypeError, match="CPU"):
        fd.fd_read_kv_q4(c, i(3), i(6), None, i(3), z(5, 2, 128), z(5, 2, 128))
    with pytest.raises(TypeError, match="one entry more"):
        fd.fd_read_kv_q4(c, i(2), i(6), None, i(3), z(5, 2, 128), z(5, 2, 128))
    with pytest.raises(TypeError, match="start"):
        fd.fd_read_kv_q4(c, i(3), i(6), i(3), i(3), z(5, 2, 128), z(5, 2, 128))
    good = dict(q=q, k_new=k, v_new=k, cache=c, page_indptr=i(3), page_indices=i(6), kv_len=i(2), row_indptr=i(3), verify_len=i(2), out=q, max_kv_len=9,
                max_new_rows=3)
    args = fd.make_attn_args_q4(**good)
    assert args.device == -1 and args.num_pages == 6
    for kw, words in ((dict(k_new=z(2, 2, 128)), "k_new"), (dict(v_new=z(3, 1, 128)), "v_new"), (dict(out=z(3, 8, 128, dt=torch.float32)), "out"),
                      (dict(lse=z(3, 8)), "lse"), (dict(lse=z(3, 4, dt=torch.float32)), "lse"), (dict(row_indptr=i(2)), "row_indptr"),
                      (dict(page_indptr=i(2)), "page_indptr"), (dict(verify_len=i(3)), "verify_len"), (dict(mask_vis=i(1)), "mask_vis"),
                      (dict(k_new=z(3, 4, 128)), "heads")):
        with pytest.raises(TypeError, match=words):
            fd.make_attn_args_q4(**dict(good, **kw))
    for other in (fd.alloc_q4_cache(5, 2, 32, 128, device="cpu"), fd.alloc_q4_cache(6, 2, 16, 128, device="cpu"), fd.alloc_q4_cache(6, 2, 32, 64, device="cpu"),
                  fd.alloc_q4_cache(6, 4, 32, 128, device="cpu")):
        for call in (lambda: fd.fd_verify_draft_attn_q4(args, other), lambda: fd.fd_append_kv_q4(args, other, i(2), i(2))):
            with pytest.raises(TypeError, match="made for"):
                call()
    with pytest.raises(TypeError, match="CPU"):
        fd.fd_verify_draft_attn_q4(args, c)
    with pytest.raises(TypeError, match="CPU"):
        fd.fd_append_kv_q4(args, c, i(2), i(2))


def test_launches_that_are_too_large_are_refused():
    need = lambda **kw: fd.load().fd_verify_draft_attn_q4_workspace(C.byref(_attn(**kw)))  # noqa: E731
    assert need(batch=65535, num_kv_heads=8, total_rows=1 << 20, max_new_rows=32) > 0
    assert need(batch=65535, num_kv_heads=32, total_rows=1 << 24, max_new_rows=2048) == 0
    _refused(_rope(total_rows=(1 << 25) + 1), 2, "2^25")
