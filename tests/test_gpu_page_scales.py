"""Attention over an 8-bit cache with a scale for every page and head: verification (the score-cache kernel on the bytes, on
the bf16 copy at head_dim 64, the generic kernels) and sparse drafting, against the formulas in 64 bits.

Tolerances.  A score is an fp32 sum of exact products, off by at most 2^-20 of the sum of their magnitudes `far`
(in units of a factor 2 of the probability) in whatever order it is added, and its exponential by 2^-21, so a probability is within
e = far 2^-20 + 2^-19 of its value; the reference sum that normalises it doubles that.  Probabilities travel in two 16-bit parts:
2^-14 on the bf16 copy (parts cut off), 2^-21 on fp16.  An output is a mean of values: within (2 e + 2^-14) of the
largest |v| of the head; rounding to bf16 adds 2^-8 of the output."""
import dataclasses

import pytest
import torch

import round_ops
from paper_2607_27735_b200 import binding, inputs

pytestmark = pytest.mark.gpu


def make(L=1, ctx=(600,), Hq=8, H=2, D=128, ps=16, n_q=5, extra=0, seed=0, spread=1.0, poison=True):
    """A shuffled pool whose unused pages, scales and rows behind the contexts hold NaN."""
    g = torch.Generator().manual_seed(seed)
    B = len(ctx)
    max_pages = -(-(max(ctx) + extra) // ps) + 1
    n_pages = B * max_pages + 3
    table = torch.randperm(n_pages, generator=g)[:B * max_pages].int().view(B, max_pages)
    k, v = (torch.randint(0, 256, (L, n_pages, H, ps, D), generator=g).to(torch.uint8) for _ in range(2))
    for x in (k, v):  # no NaN among the live bytes, magnitudes around one
        vals = torch.randn(L, n_pages, H, ps, D, generator=g) * 40
        x.copy_(vals.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    ks, vs = (torch.exp(torch.randn(L, n_pages, H, generator=g) * spread) / 45 for _ in range(2))
    if poison:
        live = torch.zeros(n_pages, ps, dtype=torch.bool)
        for b, T in enumerate(ctx):
            for t in range(T + extra):
                live[table[b, t // ps].long(), t % ps] = True
        for x in (k, v):
            x.masked_fill_(~live[None, :, None, :, None], 0x7f)
        for s in (ks, vs):
            s.masked_fill_(~live.any(1)[None, :, None], float("nan"))
    for b, T in enumerate(ctx):  # page numbers behind a context are never looked at either
        table[b, -(-(T + extra) // ps):] = 10 ** 6
    kv = inputs.KVCache(k=k.cuda(), v=v.cuda(), layer_stride=n_pages * H * ps * D, page_stride=H * ps * D, head_stride=ps * D, slot_stride=D,
                        n_layers=L, page_size=ps, page_table=table.cuda(), max_pages=max_pages, batch=B, n_q_heads=Hq, n_kv_heads=H,
                        head_dim=D, n_pages=n_pages, fp8=True, k_scale=ks.cuda(), v_scale=vs.cuda())
    q = (torch.randn(L, B, n_q, Hq, D, generator=g) * 0.6).to(torch.bfloat16).cuda()
    return kv, q, torch.tensor(ctx, dtype=torch.int32, device="cuda")


def reference(kv, q, ctx, per_head=False, group_max=False, window=16):
    L, B, n_q, Hq, D = q.shape
    H, G, T = kv.n_kv_heads, Hq // kv.n_kv_heads, int(ctx.max())
    out = torch.zeros(L, B, n_q, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(L, B, n_q, Hq, dtype=torch.float64, device="cuda")
    stats = torch.zeros(L, B, Hq, T, dtype=torch.float64, device="cuda")
    tol = torch.zeros(L, B, Hq, 2, dtype=torch.float64, device="cuda")  # of an output (without its rounding), of a probability
    for l in range(L):
        for b in range(B):
            t = int(ctx[b])
            last = t - n_q + torch.arange(n_q, device="cuda")
            for h in range(H):
                keys, values = round_ops.cache_rows(kv, l, b, h, range(t), "cuda")
                for hq in range(h * G, h * G + G):
                    o, s, p, far = round_ops.attend(q[l, b, :, hq], keys, values, last)
                    out[l, b, :, hq], lse[l, b, :, hq] = o, s
                    stats[l, b, hq, :t] = p[-min(window, n_q):].sum(0)
                    e = far * 2.0 ** -20 + 2.0 ** -19
                    tol[l, b, hq, 0] = (2 * e + 2.0 ** -14) * float(values.abs().max())
                    tol[l, b, hq, 1] = 2 * e
    if not per_head:
        st = stats.view(L, B, H, G, T)
        stats = st.amax(3) if group_max else st.sum(3)
    return out, lse, stats, tol


def compare(kv, q, ctx, want_impl=None, ref=None, **kw):
    T = int(ctx.max())
    out, lse, stats, ws = binding.spec_verify_attn(kv, q, ctx, T, **kw)
    assert binding.read_status(ws) == 0
    if want_impl is not None:  # (128 rows of a head leave an 8-bit cache too little shared memory: two halves of the rows)
        two = binding.VERIFY_TCGEN05_CACHED_2PASS
        assert binding.last_verify_impl() == (two if want_impl == binding.VERIFY_TCGEN05_CACHED and q.shape[2] * kv.n_q_heads ==
                                              128 * kv.n_kv_heads else want_impl)
    ref = ref or reference(kv, q, ctx, kw.get("per_head", False), kw.get("group_max", False))
    o, s, st, tol = ref
    half = 2.0 ** -8 * o.abs() if kw.get("out_bf16") else 0.0
    assert ((out.double() - o).abs() <= tol[:, :, None, :, :1] + half).all()
    assert ((lse.double() - s).abs() <= tol[:, :, None, :, 1] + 2.0 ** -22 * s.abs()).all()
    H = kv.n_kv_heads
    rel = tol[..., 1] if st.shape[2] != H else tol[..., 1].view(*tol.shape[:2], H, -1).amax(-1)
    for b in range(len(ctx)):
        t = int(ctx[b])
        assert ((stats[:, b, :, :t].double() - st[:, b, :, :t]).abs() <= rel[:, b, :, None] * st[:, b, :, :t] + 2.0 ** -30).all()
        assert (stats[:, b, :, t:] == 0).all()
    return ref


SHAPES = [
    dict(ctx=(600,), n_q=5),
    dict(ctx=(4001,), n_q=1, Hq=32, H=8, ps=64),
    dict(ctx=(1, 2, 129, 128, 127), n_q=1, Hq=4, H=1, ps=8),
    dict(ctx=(5, 900, 256, 2047), n_q=5, ps=128, Hq=10, H=2),
    dict(ctx=(3000, 40, 777), n_q=9, Hq=8, H=2, ps=16, L=2),
    dict(ctx=(1500,), n_q=16, Hq=16, H=2, ps=32),
    dict(ctx=(700, 650), n_q=3, Hq=8, H=8, ps=256),
    dict(ctx=(2500,), n_q=12, Hq=16, H=2, ps=16, spread=3.0),
]


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("shape", SHAPES)
def test_verification_matches_the_formula(shape, D):
    kv, q, ctx = make(D=D, seed=7 * D + shape["ctx"][0], **shape)
    impl = binding.VERIFY_TCGEN05_CACHED if D == 128 else binding.VERIFY_TCGEN05_CACHED_EXPANDED
    ref = compare(kv, q, ctx, impl)
    compare(kv, q, ctx, impl, ref, out_bf16=True)
    binding.set_verify_impl(binding.VERIFY_GENERIC)
    try:
        compare(kv, q, ctx, binding.VERIFY_GENERIC, ref)
    finally:
        binding.set_verify_impl(binding.VERIFY_AUTO)


@pytest.mark.parametrize("ps", [1, 24, 100])
def test_pages_that_end_inside_a_tile(ps):
    kv, q, ctx = make(ctx=(333, 90), ps=ps, seed=ps)
    compare(kv, q, ctx, binding.VERIFY_GENERIC)


@pytest.mark.parametrize("flags", [dict(per_head=True), dict(group_max=True), dict(accumulate=False)])
def test_other_forms_of_the_statistic(flags):
    kv, q, ctx = make(ctx=(500, 1100), seed=3, n_q=6)
    compare(kv, q, ctx, **flags)


def test_many_sequences_and_more_units_than_the_work_table_holds():
    g = torch.Generator().manual_seed(2)
    ctx = tuple(int(t) for t in torch.randint(3, 400, (90,), generator=g))
    kv, q, ctx = make(ctx=ctx, n_q=3, Hq=4, H=2, L=2, seed=5, ps=16)
    compare(kv, q, ctx, binding.VERIFY_TCGEN05_CACHED)


def test_rows_in_two_passes_and_a_long_context():
    kv, q, ctx = make(ctx=(33000,), n_q=32, Hq=16, H=4, seed=8, ps=64)  # 128 rows of a head do not fit the score cache
    T = int(ctx.max())
    out, lse, stats, ws = binding.spec_verify_attn(kv, q, ctx, T)
    assert binding.read_status(ws) == 0
    impl = binding.last_verify_impl()
    compare(kv, q, ctx, impl)


def test_scales_of_every_size_and_one_page_much_larger():
    kv, q, ctx = make(ctx=(1300, 700), n_q=4, seed=11, poison=False, spread=0.3)
    pages = kv.page_table[0].long()
    ks, vs = kv.k_scale.clone(), kv.v_scale.clone()
    vs[:, pages[3]] *= 2.0 ** 20
    vs[:, pages[5]] *= 2.0 ** -30
    ks[:, pages[6]] *= 2.0 ** -40
    compare(dataclasses.replace(kv, k_scale=ks, v_scale=vs), q, ctx, binding.VERIFY_TCGEN05_CACHED)
    tiny = dataclasses.replace(kv, v_scale=kv.v_scale * 2.0 ** -60)
    compare(tiny, q, ctx, binding.VERIFY_TCGEN05_CACHED)
    compare(dataclasses.replace(kv, v_scale=kv.v_scale * 2.0 ** 90), q, ctx, binding.VERIFY_TCGEN05_CACHED)


def test_scales_all_alike_are_a_scale_for_each_head():
    kv, q, ctx = make(ctx=(900, 350), n_q=5, seed=12, poison=False)
    L, P, H = kv.k_scale.shape
    ks, vs = (torch.tensor([0.0107, 0.0231], device="cuda").expand(L, H).contiguous() for _ in range(2))
    per_head = dataclasses.replace(kv, k_scale=ks, v_scale=vs)
    per_page = dataclasses.replace(kv, k_scale=ks[:, None].expand(L, P, H).contiguous(), v_scale=vs[:, None].expand(L, P, H).contiguous())
    T = int(ctx.max())
    a = binding.spec_verify_attn(per_head, q, ctx, T)
    b = binding.spec_verify_attn(per_page, q, ctx, T)
    ref = reference(per_page, q, ctx)
    assert ((a[0] - b[0]).abs().double() <= 2 * ref[3][:, :, None, :, :1]).all()
    assert ((a[1] - b[1]).abs().double() <= 2 * ref[3][:, :, None, :, 1] + 1e-6).all()


def test_a_call_without_a_workspace_and_a_bad_table_entry():
    kv, q, ctx = make(ctx=(600, 300), n_q=4, seed=13, poison=False)
    T = int(ctx.max())
    out, lse, stats, _ = binding.spec_verify_attn(kv, q, ctx, T)
    o2, l2, s2 = binding.spec_verify_attn_noalloc(kv, q, ctx, T)
    ref = reference(kv, q, ctx)
    assert ((o2.double() - ref[0]).abs() <= ref[3][:, :, None, :, :1]).all() and binding.noalloc_read_status() == 0
    table = kv.page_table.clone()
    table[0, 2] = kv.n_pages
    bad = dataclasses.replace(kv, page_table=table)
    for impl in (binding.VERIFY_AUTO, binding.VERIFY_GENERIC):
        binding.set_verify_impl(impl)
        try:
            out, _, _, ws = binding.spec_verify_attn(bad, q, ctx, T)
        finally:
            binding.set_verify_impl(binding.VERIFY_AUTO)
        assert binding.read_status(ws) == -6 and out.isfinite().all()


def draft_reference(kv, q, idx, n, start, cur, per_head):
    L, B, Hq, D = q.shape
    G = Hq // kv.n_kv_heads
    out = torch.zeros(L, B, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((L, B, Hq), -float("inf"), dtype=torch.float64, device="cuda")
    tol = torch.zeros(L, B, Hq, 2, dtype=torch.float64, device="cuda")
    for l in range(L):
        for b in range(B):
            for hq in range(Hq):
                s = hq if per_head else hq // G
                pos = idx[l, b, s, :int(n[l, b, s])].tolist() + list(range(int(start[b]), int(cur[b])))
                if not pos:
                    continue
                keys, values = round_ops.cache_rows(kv, l, b, hq // G, pos, "cuda")
                o, z, _, far = round_ops.attend(q[l, b, hq][None], keys, values, torch.tensor([len(pos)], device="cuda"))
                out[l, b, hq], lse[l, b, hq] = o[0], z[0]
                e = far * 2.0 ** -20 + 2.0 ** -19
                tol[l, b, hq, 0], tol[l, b, hq, 1] = (2 * e + 2.0 ** -14) * float(values.abs().max()), 2 * e
    return out, lse, tol


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("Hq,H,ps,ctx,budget,tail,per_head,L", [
    (8, 2, 16, (600, 90, 1), 128, 3, False, 1),
    (16, 2, 64, (3000, 2000), 1024, 1, False, 2),
    (4, 4, 8, (500,), 64, 0, False, 1),
    (5, 1, 24, (700, 300), 200, 4, False, 1),
    (8, 2, 16, (900, 400), 100, 2, True, 2),
    (32, 8, 16, (9000, 5000, 7000, 100), 2048, 8, False, 1),
])
def test_drafting_matches_the_formula(D, Hq, H, ps, ctx, budget, tail, per_head, L):
    kv, q, start = make(L=L, ctx=ctx, Hq=Hq, H=H, D=D, ps=ps, n_q=1, extra=tail, seed=budget + D)
    q = q[:, :, 0].contiguous()
    sets = Hq if per_head else H
    g = torch.Generator().manual_seed(4)
    idx = torch.full((L, len(ctx), sets, budget), -1, dtype=torch.int32)
    for b, T in enumerate(ctx):
        keep = min(T, budget)
        idx[:, b, :, :keep] = torch.rand(L, sets, T, generator=g).topk(keep).indices.sort(-1).values.int()
    n = (idx >= 0).sum(-1).int()
    n[0, 0, 0] = min(int(n[0, 0, 0]), 7)  # a short set beside long ones
    idx, n, cur = idx.cuda(), n.cuda(), start + tail
    want, lse_w, tol = draft_reference(kv, q, idx, n, start, cur, per_head)
    for early in (False, True):
        out, lse, ws = binding.spec_sparse_draft_attn(kv, q, idx, n, start, cur, tail, per_head=per_head, early_gather=early)
        assert binding.read_status(ws) == 0
        assert ((out.double() - want).abs() <= tol[..., :1]).all()
        some = lse_w > -float("inf")
        assert ((lse.double() - lse_w).abs() <= tol[..., 1] + 2.0 ** -22 * lse_w.abs())[some].all() and (lse[~some] == -float("inf")).all()
    o16, _, _ = binding.spec_sparse_draft_attn(kv, q, idx, n, start, cur, tail, per_head=per_head, out_bf16=True)
    assert torch.equal(o16, out.to(torch.bfloat16))


def test_drafting_over_pages_of_very_different_scale_and_an_empty_set():
    kv, q, start = make(ctx=(800, 300), n_q=1, seed=21, poison=False, spread=0.2)
    q = q[:, :, 0].contiguous()
    vs, ks = kv.v_scale.clone(), kv.k_scale.clone()
    vs[:, kv.page_table[0, 2].long()] *= 2.0 ** 25
    vs[:, kv.page_table[1].long().clamp(max=kv.n_pages - 1)] *= 2.0 ** -50
    kv = dataclasses.replace(kv, k_scale=ks, v_scale=vs)
    idx = torch.arange(0, 300, 3, dtype=torch.int32, device="cuda").expand(1, 2, 2, 100).contiguous()
    n = torch.tensor([[[100, 0], [100, 33]]], dtype=torch.int32, device="cuda")
    out, lse, ws = binding.spec_sparse_draft_attn(kv, q, idx, n, start, start, 0)
    want, lse_w, tol = draft_reference(kv, q, idx, n, start, start, False)
    assert binding.read_status(ws) == 0
    assert ((out.double() - want).abs() <= tol[..., :1]).all()
    assert (out[0, 0, 4:] == 0).all() and (lse[0, 0, 4:] == -float("inf")).all()


def test_the_shapes_of_the_scales_are_checked():
    kv, q, ctx = make(ctx=(100,), n_q=2)
    for bad in (dict(k_scale=kv.k_scale[:, :-1].contiguous()), dict(v_scale=kv.v_scale[..., :1].contiguous()), dict(v_scale=None)):
        with pytest.raises((ValueError, TypeError)):
            binding.spec_verify_attn(dataclasses.replace(kv, **bad), q, ctx, 100)
