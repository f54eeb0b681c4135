"""Head scales of an 8-bit cache as tensors with a dimension of 1 among theirs give what [layers, heads] gives."""
import dataclasses

import pytest
import torch

from paper_2607_27735_b200 import binding
from test_gpu_page_scales import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(2, 1, 2), (2, 2, 1), (1, 2, 2), (4,)])
def test_the_same_results(shape):
    kv, q, ctx = make(L=2, ctx=(300, 150), n_q=3, seed=1, poison=False)
    ks, vs = (torch.tensor([[0.01, 0.02], [0.03, 0.015]], device="cuda") * f for f in (1.0, 1.5))
    idx = torch.arange(100, dtype=torch.int32, device="cuda").expand(2, 2, 2, 100).contiguous()
    n = torch.full((2, 2, 2), 100, dtype=torch.int32, device="cuda")

    def run(a, b):
        c = dataclasses.replace(kv, k_scale=a, v_scale=b)
        out = binding.spec_verify_attn(c, q, ctx, 300)[:3]
        return [*out, *binding.spec_sparse_draft_attn(c, q[:, :, 0].contiguous(), idx, n, ctx, ctx, 0)[:2]]

    want = run(ks, vs)
    assert all(torch.equal(x, y) for x, y in zip(want, run(ks.view(shape), vs.view(shape))))
