"""The balanced key of an appended token is stored as fp16 of the fp32 product,
like a placed one's."""
import pytest
import torch

from paper_2402_18096_amd import mikv


@pytest.mark.gpu
def test_balanced_append_stores_what_placement_stores():
    B, H, T = 2, 64, 24
    g = torch.Generator(device="cuda").manual_seed(11)
    k, v = (torch.randn(B, H, T, 128, device="cuda", generator=g).half() for _ in range(2))
    balance = torch.rand(B, H, 128, device="cuda", generator=g) * 3 + 0.1
    want = (k.float() * balance[:, :, None]).half().reshape(B * H, T, 128)
    placed, appended = (mikv.MikvCache(B, H, H, 32, 16, 2, T, T, T) for _ in range(2))
    mikv.mikv_quantize_kv(placed, k, v, 0, balance, torch.ones(B, H, T, dtype=torch.uint8, device="cuda"))
    for t in range(T):
        mikv.mikv_quantize_kv(appended, k[:, :, t:t + 1].contiguous(), v[:, :, t:t + 1].contiguous(), t, balance)
    # and through the append that a decode step folds into its attention
    folded = mikv.MikvCache(B, H, H, 32, 16, 2, T, T, T)
    q, out = torch.zeros(B, H, 128, dtype=torch.float16, device="cuda"), torch.empty(B, H, 128, device="cuda")
    for t in range(T):
        mikv.mikv_decode_step(folded, t + 1, q, k[:, :, t].contiguous(), v[:, :, t].contiguous(), out, T, 1,
                              balance=balance, flags=mikv.ATTN_ACCUMULATE)
    for c in (placed, appended, folded):
        assert torch.equal(c.hi_k.view(torch.int16), want.view(torch.int16))
