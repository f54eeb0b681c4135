"""Verification over a cache with page scales, many units of a few tiles one after the other: the warps that expand tiles take
them in turn, and with an odd number of stages or slots a team comes back to one of them two phases later.  Small shapes, repeated: an order
of events that is rare in one call shows in some of them; every one has to end and to give the same bits."""
import pytest
import torch

from paper_2607_27735_b200 import binding
from test_gpu_page_scales import compare, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_q,Hq,H,longest", [(1, 8, 2, 130), (3, 4, 2, 700), (7, 32, 8, 400), (6, 8, 2, 1200), (9, 8, 2, 300)])
def test_units_of_a_few_tiles(n_q, Hq, H, longest):
    g = torch.Generator().manual_seed(n_q)
    ctx = tuple(int(t) for t in torch.randint(n_q, longest, (40,), generator=g))
    kv, q, ctx = make(ctx=ctx, n_q=n_q, Hq=Hq, H=H, L=3, seed=n_q, ps=16)
    compare(kv, q, ctx, binding.VERIFY_TCGEN05_CACHED)
    T = int(ctx.max())
    out, lse, stats, ws = binding.spec_verify_attn(kv, q, ctx, T)
    first = [x.clone() for x in (out, lse, stats)]
    for _ in range(60):
        binding.spec_verify_attn(kv, q, ctx, T, out=out, lse=lse, stats=stats, workspace=ws)
    assert binding.read_status(ws) == 0
    assert all(torch.equal(a, b) for a, b in zip(first, (out, lse, stats)))
