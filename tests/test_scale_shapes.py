"""Which scales an 8-bit cache description has: [layers, pages, heads] is a scale for every page, [layers, heads] one for every head, with or
without a dimension of 1 in it.  No GPU needed: tensors that only say that they are on one."""
import dataclasses

import pytest
import torch

from paper_2607_27735_b200 import binding, inputs


class Said(torch.Tensor):
    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise RuntimeError("no data")


def said(*shape, dtype=torch.float32):
    return torch.Tensor._make_wrapper_subclass(Said, shape, dtype=dtype, device="cuda:0")


def cache(k_scale, v_scale, L=3, pages=7, H=4):
    data = said(L, pages, H, 16, 128, dtype=torch.uint8)
    return inputs.KVCache(k=data, v=data, layer_stride=pages * H * 2048, page_stride=H * 2048, head_stride=2048, slot_stride=128, n_layers=L,
                          page_size=16, page_table=None, max_pages=pages, batch=1, n_q_heads=8, n_kv_heads=H, head_dim=128, n_pages=pages,
                          fp8=True, k_scale=k_scale, v_scale=v_scale)


PER_HEAD = [((3, 4), (3, 4)), ((12,), (12,)), ((3, 1, 4), (3, 1, 4)), ((3, 4, 1), (3, 4, 1)), ((1, 3, 4), (3, 4)), ((3, 4), (3, 1, 4))]
PER_PAGE = [((3, 7, 4), (3, 7, 4))]
NEITHER = [((3, 7, 4), (3, 4)), ((3, 4), (3, 7, 4)), ((3, 6, 4), (3, 6, 4)), ((3, 7, 4), (3, 7, 1)), ((2, 7, 4), (2, 7, 4))]


@pytest.mark.parametrize("shapes,want", [(s, 1) for s in PER_HEAD] + [(s, 2) for s in PER_PAGE])
def test_the_kind_of_the_scales(shapes, want):
    kv = cache(*(said(*s) for s in shapes))
    assert binding._kv_struct(kv).kv_dtype == want
    # a single page's scale is one for every head: either description of it reads the same numbers
    one = dataclasses.replace(cache(said(3, 1, 4), said(3, 1, 4), pages=1))
    assert binding._kv_struct(one).kv_dtype == binding.KV_FP8_E4M3_PAGE


@pytest.mark.parametrize("shapes", NEITHER)
def test_shapes_that_are_neither(shapes):
    kv = cache(*(said(*s) for s in shapes))
    with pytest.raises(ValueError):
        binding._kv_struct(kv)
