"""Verification over a cache with page scales, many units of a few tiles one after the other: the warps that expand tiles take
them in turn, and with an odd number of stages or slots a team comes back to one of them two phases later.  Small shapes, repeated: an order
of events that is rare in one call shows in some of them; every one has to end and to give the same bits."""
import dataclasses

import pytest
import torch

from paper_2607_27735_b200 import binding
from test_gpu_page_scales import compare, make, reference

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


@pytest.mark.parametrize("n_q,Hq,H,D", [(1, 8, 2, 128), (7, 8, 2, 128), (9, 8, 2, 128), (5, 8, 2, 64)])
def test_more_units_than_the_work_table_holds(n_q, Hq, H, D):
    """Scales that are all one power of two change no product: the calls give the bits of a scale for each head."""
    g = torch.Generator().manual_seed(D + n_q)
    ctx = tuple(int(t) for t in torch.randint(n_q, 70, (80,), generator=g))
    kv, q, ctx = make(ctx=ctx, n_q=n_q, Hq=Hq, H=H, D=D, L=40, seed=5, ps=16, poison=False)
    L, P, _ = kv.k_scale.shape
    ks, vs = (torch.full((L, H), s, device="cuda") for s in (2.0 ** -6, 2.0 ** -4))
    per_head = dataclasses.replace(kv, k_scale=ks, v_scale=vs)
    per_page = dataclasses.replace(kv, k_scale=ks[:, None].expand(L, P, H).contiguous(), v_scale=vs[:, None].expand(L, P, H).contiguous())
    T = int(ctx.max())
    a, b = binding.spec_verify_attn(per_head, q, ctx, T), binding.spec_verify_attn(per_page, q, ctx, T)
    assert binding.read_status(a[3]) == 0 and binding.read_status(b[3]) == 0
    assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


def test_the_scores_are_counted_as_they_are_written():
    kv, q, ctx = make(ctx=(900, 333), n_q=5, seed=30)
    hist = torch.zeros(1, 2, 2, 2048, dtype=torch.int32, device="cuda")
    _, _, stats, _ = binding.spec_verify_attn(kv, q, ctx, 900, score_hist=hist)
    for b, t in enumerate(ctx.tolist()):
        for h in range(2):
            bins = stats[0, b, h, :t].contiguous().view(torch.int32) >> 21
            assert torch.equal(torch.bincount(bins.long(), minlength=2048).int(), hist[0, b, h])


def test_a_replayed_call_reads_the_scales_as_they_are():
    kv, q, ctx = make(ctx=(700, 400), n_q=3, seed=31, poison=False)
    out, stats = torch.empty(1, 2, 3, 8, 128, device="cuda"), torch.zeros(1, 2, 2, 704, device="cuda")
    ws = binding.alloc_workspace(binding.workspace_bytes(binding.WS_VERIFY, kv, 3, 700), "cuda")
    binding.spec_verify_attn(kv, q, ctx, 700, out=out, stats=stats, workspace=ws, want_lse=False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.v_scale.mul_(0.5)
        kv.k_scale.mul_(1.25)
        binding.spec_verify_attn(kv, q, ctx, 700, out=out, stats=stats, workspace=ws, want_lse=False)
    for _ in range(4):
        graph.replay()
        ref, _, st, tol = reference(kv, q, ctx)
        assert ((out.double() - ref).abs() <= tol[:, :, None, :, :1]).all()
