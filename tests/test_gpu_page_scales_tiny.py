"""Page scales of V near the least positive fp32 numbers: outputs scale with them, in verification and in drafting.  Tolerances as in
test_gpu_page_scales.py, which are relative to the largest |v|."""
import dataclasses

import pytest
import torch

from paper_2607_27735_b200 import binding
from test_gpu_page_scales import compare, draft_reference, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("n_q", [1, 5, 9])
@pytest.mark.parametrize("power", [-118, -115, -105])
def test_verification(D, n_q, power):
    kv, q, ctx = make(ctx=(700, 260), n_q=n_q, D=D, seed=n_q, poison=False, spread=0.3)
    tiny = dataclasses.replace(kv, v_scale=kv.v_scale * 2.0 ** power)  # scales of about 2^-5.5 before
    assert 2.0 ** -126 <= float(tiny.v_scale.min())
    compare(tiny, q, ctx)


@pytest.mark.parametrize("Hq,H", [(8, 2), (16, 2)])
@pytest.mark.parametrize("power", [-118, -115, -105])
def test_drafting(Hq, H, power):
    kv, q, start = make(ctx=(900,), Hq=Hq, H=H, n_q=1, seed=Hq, poison=False, spread=0.3)
    q = q[:, :, 0].contiguous()
    tiny = dataclasses.replace(kv, v_scale=kv.v_scale * 2.0 ** power)
    assert 2.0 ** -126 <= float(tiny.v_scale.min())
    idx = torch.arange(0, 900, 3, dtype=torch.int32, device="cuda").expand(1, 1, H, 300).contiguous()
    n = torch.full((1, 1, H), 300, dtype=torch.int32, device="cuda")
    out, _, ws = binding.spec_sparse_draft_attn(tiny, q, idx, n, start, start, 0)
    want, _, tol = draft_reference(tiny, q, idx, n, start, start, False)
    assert binding.read_status(ws) == 0
    assert ((out.double() - want).abs() <= tol[..., :1]).all()
