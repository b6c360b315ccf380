"""Inputs and bounds for the GPU tests of the calls over a 4-bit cache."""
from __future__ import annotations

import numpy as np
import torch

from oracle import attention as oa
from oracle import kv4
from paper_2605_20022_amd import workloads as W


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def bf16(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def bits_of(x):
    return W.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


def device_cache(fd, cache: kv4.Cache, heads_first=False):
    k, ks, v, vs = cache.packed()
    t = [torch.from_numpy(k).cuda(), torch.from_numpy(ks).cuda(), torch.from_numpy(v).cuda(), bf16(vs)]
    if heads_first:
        t = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in t]
    return fd.Q4Cache(*t)


def assert_cache_is(dev, cache: kv4.Cache):
    k, ks, v, vs = cache.packed()
    assert np.array_equal(dev.k_codes.cpu().numpy(), k)
    assert np.array_equal(dev.k_scales.cpu().numpy(), ks)
    assert np.array_equal(dev.v_codes.cpu().numpy(), v)
    assert np.array_equal(dev.v_scales.view(torch.int16).cpu().numpy().view(np.uint16), vs)


class Q4Call:
    """One ragged batch: kv, k, m (new mask rows) by sequence; room: tokens beyond prefix that the page lists hold."""

    def __init__(self, fd, *, kv, k, m, hq=8, hkv=2, dim=128, ps=16, blocks=None, vis=None, room=0, seed=0, heads_first=False, std=1.0, spare_rows=0):
        rng = np.random.default_rng(seed)
        kv, k, m = (np.asarray(x, dtype=np.int64) for x in (kv, k, m))
        self.fd, self.kv, self.k, self.n, self.blocks, self.vis, self.ps = fd, kv, k, k + m, blocks, vis, ps
        pages = -(-(kv + room) // ps)
        used = int(pages.sum())
        pool = used + 3
        self.page_indptr = np.concatenate([[0], np.cumsum(pages)])
        self.page_indices = rng.permutation(pool)[:used] if used else np.zeros(1, dtype=np.int64)
        self.row_indptr = np.concatenate([[0], np.cumsum(self.n)])
        self.cache = kv4.Cache.random(rng, pool, hkv, ps, dim)
        R = int(self.n.sum()) + spare_rows
        self.q = bits_of(std * rng.standard_normal((R, hq, dim)))
        self.k_new, self.v_new = bits_of(rng.standard_normal((R, hkv, dim))), bits_of(rng.standard_normal((R, hkv, dim)))
        self.heads_first = heads_first
        self.max_kv, self.max_n = int(kv.max()), int(self.n.max())

    def upload(self, *, kv_chunk=0, sm_scale=0.0, max_kv=None):
        fd = self.fd
        self.dev = device_cache(fd, self.cache, self.heads_first)
        self.d = dict(q=bf16(self.q), k_new=bf16(self.k_new), v_new=bf16(self.v_new), page_indptr=i32(self.page_indptr),
                      page_indices=i32(self.page_indices), kv_len=i32(self.kv), row_indptr=i32(self.row_indptr), verify_len=i32(self.k),
                      mask_vis=None if self.vis is None else i32(self.vis), mask_blocks=None if self.blocks is None else i32(self.blocks))
        d = self.d
        self.out = torch.full(self.q.shape, -7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full(self.q.shape[:2], -7.0, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.args = fd.make_attn_args_q4(d["q"], d["k_new"], d["v_new"], self.dev, d["page_indptr"], d["page_indices"], d["kv_len"], d["row_indptr"],
                                         d["verify_len"], d["mask_vis"], d["mask_blocks"], out=self.out, lse=self.lse,
                                         max_kv_len=self.max_kv if max_kv is None else max_kv, max_new_rows=self.max_n, sm_scale=sm_scale,
                                         kv_chunk=kv_chunk, status=self.status)
        need = fd.fd_verify_draft_attn_q4_workspace(self.args)
        assert need > 0
        self.workspace = torch.full((need,), 0xab, dtype=torch.uint8, device="cuda")         # nothing in it has to start at zero
        self.args.workspace, self.args.workspace_bytes = self.workspace.data_ptr(), need
        return self

    def run(self):
        self.fd.fd_verify_draft_attn_q4(self.args, self.dev)
        torch.cuda.synchronize()
        return self.out.float().cpu().numpy().astype(np.float64), self.lse.cpu().numpy().astype(np.float64)

    def oracle(self, sm_scale=None, magnitudes=False, peaks=False):
        """magnitudes: with |v| for v; peaks: with the largest |v| of its token and head in the place of every channel."""
        k, v = self.cache.key_values(), self.cache.value_values()
        v_new = oa.widen_bf16(self.v_new)
        R = int(self.n.sum())
        f = np.abs if magnitudes else (lambda x: x)
        if peaks:
            f = lambda x: np.broadcast_to(np.abs(x).max(-1, keepdims=True), x.shape)  # noqa: E731
        return oa.verify_draft_attention(self.q[:R], self.k_new[:R], f(v_new[:R]), np.nan_to_num(k, nan=0.0), f(np.nan_to_num(v, nan=0.0)), self.page_indptr,
                                         self.page_indices, self.kv, self.row_indptr, self.k, self.vis, self.blocks, page_size=self.ps, sm_scale=sm_scale)

    def check(self, out, lse, sm_scale=None):
        """The bounds.  A probability (times its value's scale) and the result are each rounded to bf16: half a step is 2^-8 of the value, so
        2^-8 (|o| + sum p |v|) in all.  In fp32: a score sums D = 128 products in order, off by at most 128 * 2^-24 sum |q_d k_d| scale, which
        is below 2^-17 B with B the largest such sum; the base-2 exponential and the scales add 2^-22 of a probability each; the sum of n probabilities n * 2^-24.
        A score that is off by x changes a probability, against the others, by at most 2 x of itself.
        An item in several pieces leaves each piece's row as fp16 numbers over the row's largest entry: off by half a step of [1/2, 1), 2^-12 of that
        entry, which is at most the piece's sum of p max |v|; over all pieces 2^-12 of the whole sum, and fp32 beside it."""
        R = int(self.n.sum())
        ref, ref_lse = self.oracle(sm_scale)
        size, _ = self.oracle(sm_scale, magnitudes=True)
        peak, _ = self.oracle(sm_scale, peaks=True)
        D = self.q.shape[2]
        q, scale = np.abs(oa.widen_bf16(self.q[:R])), sm_scale or 1 / np.sqrt(D)
        kmax = max(np.abs(np.nan_to_num(self.cache.key_values())).max(), np.abs(oa.widen_bf16(self.k_new[:R])).max())
        score = 2.0 ** -17 * float(q.sum(-1).max() * kmax * scale) + 2.0 ** -20
        keys = self.max_kv + self.max_n
        assert np.isfinite(out[:R]).all() and np.isfinite(lse[:R]).all()
        bound = 2.0 ** -8 * (np.abs(ref) + size) + (2 * score + keys * 2.0 ** -23) * size + 2.0 ** -12 * (1 + 2.0 ** -8) * peak + 1e-30
        worst = float((np.abs(out[:R] - ref) / bound).max())
        assert worst <= 1.0, f"{worst:.2f} of the bound"
        off = np.abs(lse[:R] - ref_lse).max()
        assert off <= score + keys * 2.0 ** -24 + 2.0 ** -20 * (1 + np.abs(ref_lse).max()), off
        # what the worst case allows, no run of independent roundings comes near: root mean square of both roundings
        rms = np.sqrt(np.mean((out[:R] - ref) ** 2)) / np.sqrt(np.mean(size ** 2))
        assert rms <= 2.0 ** -8, rms
