"""Values that pass through the norm and rotation: every bit of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.bfloat16, 40), (torch.float32, 64)])
def test_values_are_copied_as_they_are(fd, dtype, D):
    """Every bf16 there is, and floats of every sign, exponent and some mantissas: zeros, subnormals, infinities, NaN of both kinds."""
    if dtype == torch.bfloat16:
        bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    else:
        low = torch.tensor([0, 1, 0x2aaaaa, 0x3fffff, 0x400000, 0x400001, 0x7fffff])
        bits = ((torch.arange(512)[:, None] << 23) + low).flatten().to(torch.int32)
    H = 3
    R = -(-bits.numel() // (H * D))
    bits = torch.cat([bits, bits[:R * H * D - bits.numel()]]).view(R, H, D).cuda()
    v = bits.view(dtype)
    q, k = torch.randn(R, 4, D, device="cuda").to(dtype), torch.randn(R, H, D, device="cuda").to(dtype)
    w = torch.ones(D, device="cuda", dtype=dtype)
    out = [torch.empty_like(x) for x in (q, k, v)]
    fd.fd_qk_norm_rope(q, k, out[0], out[1], torch.arange(R, device="cuda", dtype=torch.int32), torch.ones(D // 2, device="cuda"), q_weight=w, k_weight=w, v=v,
                       v_out=out[2])
    assert torch.equal(out[2].view(bits.dtype), bits)
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[1]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_of_dimensions_of_one(fd, dtype):
    """One row and one key head, whose strides are whatever the view left: the same bits as from dense tensors."""
    D = 128
    q = torch.randn(D, 1, 5, device="cuda").to(dtype).permute(1, 2, 0).contiguous().as_strided((1, 5, D), (3, D, 1))
    k = torch.randn(D, 1, device="cuda").to(dtype)[:, 0].contiguous().as_strided((1, 1, D), (1, 7, 1))
    pos, f = torch.tensor([77], device="cuda", dtype=torch.int32), torch.rand(D // 2, device="cuda")
    w = torch.rand(D, device="cuda").to(dtype)
    outs = []
    for a, b in ((q, k), (torch.empty(1, 5, D, device="cuda", dtype=dtype).copy_(q), torch.empty(1, 1, D, device="cuda", dtype=dtype).copy_(k))):
        outs.append((torch.empty(1, 5, D, device="cuda", dtype=dtype), torch.empty(1, 1, D, device="cuda", dtype=dtype)))
        fd.fd_qk_norm_rope(a, b, *outs[-1], pos, f, q_weight=w, k_weight=w)
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and torch.isfinite(outs[0][0]).all()
