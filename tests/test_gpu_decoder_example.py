"""The example's decoder step: its parts joined as a user joins them, against the definitions."""
import os
import sys

import pytest
import torch

import decoder_util as du
import paper_2311_05161_amd as w

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_prompt_and_single_tokens(dtype):
    import decoder_attention as ex
    B, width, heads, kv, D, page = 2, 512, 8, 2, 64, 16
    layer = ex.Attention(width, heads, kv, D, dtype=dtype)
    table = torch.randperm(10, device="cuda").reshape(B, 5).to(torch.int32)
    cache = w.KVCacheDint4.empty(10, kv, page, D)
    g = torch.Generator(device="cuda").manual_seed(1)
    start, count = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.tensor([40, 23], dtype=torch.int32, device="cuda")
    for S in (40, 1, 1):
        x, r = (torch.randn((B, S, width), generator=g, device="cuda").to(dtype) for _ in range(2))
        y, h = layer.step(x, r, cache, start, count if S > 1 else None, table, max_len=64)
        assert torch.equal(h.cpu(), (x.cpu().float() + r.cpu().float()).to(dtype))
        q, k, v, _ = layer.project(x, r)                     # (the same bits again: nothing depends on the order of work)
        for n, rows in ((0, k), (2, v)):
            packed, words = du.quantize64(rows.cpu())
            for b in range(B):
                c = int(count[b]) if S > 1 else 1
                pos = int(start[b]) + torch.arange(c)
                at = table[b].cpu().long()[pos // page]
                assert torch.equal(cache[n].cpu()[at, :, pos % page], packed[b, :c])
                assert torch.equal(cache[n + 1].cpu()[at, :, pos % page], words[b, :c])
        o = w.attention_kv_dint4(q, cache, start, count if S > 1 else None, table, max_len=64)
        ref, slack = du.attention64(q.cpu(), [t.cpu() for t in cache], start.tolist(), count.tolist() if S > 1 else None, table.cpu(), D ** -0.5, 64)
        du.assert_attention(o, ref, slack)
        packed, step, zero, s = layer.out
        two = w.w4a8_gemm(*w.quantize_act_int8(o.reshape(-1, heads * D), s), packed, step, zero, width, heads * D, layer.group, out_dtype=dtype)
        assert torch.equal(two.view_as(y), y)
        start = start + (count if S > 1 else 1)


def test_main_runs():
    import decoder_attention as ex
    y = ex.main(width=512, heads=4, kv_heads=2, head_dim=128, prompts=(40, 9, 130), new_tokens=5, page=16)
    assert y.shape == (3, 1, 512) and torch.isfinite(y).all()
