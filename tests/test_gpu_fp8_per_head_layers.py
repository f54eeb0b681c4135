"""Drafting with an index set per attention head over several layers of an 8-bit cache: every layer has its own scales, one
for each head of the CACHE, however many problems the call makes of them."""
import dataclasses

import pytest
import torch

import oracle
from paper_2607_27735_b200 import binding, inputs

pytestmark = pytest.mark.gpu


def test_layers_keep_their_own_scales():
    cfg = inputs.small_config(ctx=(500, 500), n_layers=3, n_q_heads=8, n_kv_heads=2, k_total=64, k_recent=8, draft_steps=1)
    case = inputs.make_case(cfg, device="cuda")
    kv8 = inputs.quantize_kv_fp8(case.kv)
    # room behind the scales, so that a wrong row of them would be read from here
    ks, vs = (torch.full((8, 2), 1000.0, device="cuda") for _ in range(2))
    for wide, scale in ((ks, kv8.k_scale), (vs, kv8.v_scale)):
        wide[:3] = scale * torch.tensor([[1.0], [0.5], [2.0]], device="cuda")
    kv8 = dataclasses.replace(kv8, k_scale=ks[:3], v_scale=vs[:3])
    ctx = case.ctx_len
    idx = torch.arange(0, 480, 8, dtype=torch.int32, device="cuda").expand(3, 1, 8, 60).contiguous()
    n = torch.full((3, 1, 8), 60, dtype=torch.int32, device="cuda")
    q = case.q_draft[0].contiguous()
    out, _, ws = binding.spec_sparse_draft_attn(kv8, q, idx, n, ctx, ctx + 1, 1, per_head=True)
    assert binding.read_status(ws) == 0
    want, _ = oracle.sparse_draft_attn(kv8.cpu(), q.cpu(), idx.cpu(), n.cpu(), ctx.cpu(), (ctx + 1).cpu(), per_head=True)
    assert (out.cpu().double() - want).abs().max().item() <= 2e-3 * 2  # the largest |v| is twice that of the other tests
