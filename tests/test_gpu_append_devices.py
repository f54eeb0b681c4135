"""spec_qkv_append refuses a cache of which a part that it reads or writes is on another device than the current one.  The part is a tensor
without data that says it is on a second device."""
import dataclasses

import pytest
import torch

from paper_2607_27735_b200 import binding
from test_gpu_page_scales import make
from test_scale_shapes import Said

pytestmark = pytest.mark.gpu


def elsewhere(t):
    return torch.Tensor._make_wrapper_subclass(Said, t.shape, dtype=t.dtype, device=f"cuda:{torch.cuda.device_count()}")


@pytest.mark.parametrize("part", ["k", "v", "k_scale", "v_scale"])
@pytest.mark.parametrize("per_page", [True, False])
def test_a_part_of_the_cache_on_another_device(part, per_page):
    kv, _, _ = make(ctx=(40,), seed=2, poison=False)
    if not per_page:
        kv = dataclasses.replace(kv, k_scale=kv.k_scale[:, 0].contiguous(), v_scale=kv.v_scale[:, 0].contiguous())
    rows = torch.zeros(1, 2, kv.n_kv_heads, 128, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ws = binding.alloc_workspace(4096, "cuda")
    binding.spec_qkv_append(kv, None, rows, rows, None, slots, workspace=ws)
    with pytest.raises(ValueError, match="current CUDA device"):
        binding.spec_qkv_append(dataclasses.replace(kv, **{part: elsewhere(getattr(kv, part))}), None, rows, rows, None, slots, workspace=ws)
