"""Rows of Q, K and V normed, rotated and written into the cache, against the formulas in 64 bits.

Tolerances.  A result passes some twenty fp32 roundings (the sum of squares 13, the reciprocal root 2 ulp, two products, the
rotation's three), each at most 2^-24 of the larger element of its pair, hence 2^-19 of the head's largest value; and one
rounding to its type: 2^-8 of the value for bf16, 2^-4 for e4m3, or half a subnormal step, 2^-10 times the scale."""
import dataclasses

import pytest
import torch

import round_ops
from paper_2607_27735_b200 import binding, inputs

pytestmark = pytest.mark.gpu


def make_cache(L, n_pages, H, ps, D, Hq, fmt, seed=0, slot_pad=0, page_pad=0):
    """A cache whose every byte holds something, with gaps between slots and pages, on the CPU (one flat storage)."""
    g = torch.Generator().manual_seed(seed)
    slot = D + slot_pad
    head, page = ps * slot, H * ps * slot + page_pad
    n = L * n_pages * page
    if fmt == "bf16":
        k, v = (torch.randn(n, generator=g).to(torch.bfloat16) for _ in range(2))
        ks = vs = None
    else:
        k, v = ((torch.randn(n, generator=g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2))
        shape = (L, H) if fmt == "head8" else (L, n_pages, H)
        ks, vs = (torch.exp(torch.randn(shape, generator=g) * 0.7 - 4) for _ in range(2))
        if fmt == "page8":  # some pages have never had a scale
            ks.view(-1)[::5] = 0.0
            vs.view(-1)[::7] = float("nan")
    return inputs.KVCache(k=k, v=v, layer_stride=n_pages * page, page_stride=page, head_stride=head, slot_stride=slot, n_layers=L,
                          page_size=ps, page_table=None, max_pages=n_pages, batch=1, n_q_heads=Hq, n_kv_heads=H, head_dim=D,
                          n_pages=n_pages, fp8=fmt != "bf16", k_scale=ks, v_scale=vs)


def row_index(kv, l, page, slot, h):
    base = l * kv.layer_stride + page * kv.page_stride + h * kv.head_stride + slot * kv.slot_stride
    return slice(base, base + kv.head_dim)


def make_rows(L, N, Hq, H, D, seed, packed=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(L, N, Hq + 2 * H, D, generator=g) * torch.exp(torch.randn(L, N, Hq + 2 * H, 1, generator=g))
    x = x.to(torch.bfloat16)
    return x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]


def check(kv0, q, k, v, positions, slots, qw, kw, eps, cos_sin, interleaved, written=None):
    """One call on copies on the GPU; every byte of the cache, the scales and q_out are compared."""
    L, N, H, D = k.shape
    ps, fmt = kv0.page_size, "bf16" if not kv0.fp8 else ("page8" if kv0.k_scale.dim() == 3 else "head8")
    kv = kv0.to("cuda")
    kv = dataclasses.replace(kv, k=kv.k.clone(), v=kv.v.clone(), k_scale=None if kv.k_scale is None else kv.k_scale.clone(),
                             v_scale=None if kv.v_scale is None else kv.v_scale.clone())
    dq = torch.full((L, N, q.shape[2], D), 5.0, dtype=torch.bfloat16, device="cuda") if q is not None else None
    storage = torch.cat([t for t in (q, k, v) if t is not None], 2).cuda()  # the packed projection; its views are the arguments
    at = 0 if q is None else q.shape[2]
    dev = [None if q is None else storage[:, :, :at], storage[:, :, at:at + H], storage[:, :, at + H:]]
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    _, ws = binding.spec_qkv_append(kv, *dev, cuda(positions), slots.cuda(), q_weight=cuda(qw), k_weight=cuda(kw), eps=eps,
                                    cos_sin=cuda(cos_sin), interleaved=interleaved, q_out=dq)
    status = binding.read_status(ws)
    cap = kv0.n_pages * ps
    good = [s >= 0 and s < cap and (cos_sin is None or 0 <= int(positions[i]) < cos_sin.shape[0]) for i, s in enumerate(slots.tolist())]
    assert status == (-6 if any(s >= 0 and not ok for s, ok in zip(slots.tolist(), good)) else 0)

    pos = positions if positions is not None else torch.zeros(N, dtype=torch.int32)
    for l in range(L):
        if q is not None:
            want = round_ops.norm_rope(q[l], None if qw is None else qw[l], eps, cos_sin, pos, interleaved)
            got = dq[l].cpu().double()
            tol = 2.0 ** -8 * want.abs() + 2.0 ** -19 * want.abs().amax(-1, keepdim=True)
            keep = torch.tensor(good)
            assert ((got - want).abs() <= tol)[keep].all()
            assert (got[~keep] == 5.0).all()  # padding rows are left as they were
    rows = {"k": [round_ops.norm_rope(k[l], None if kw is None else kw[l], eps, cos_sin, pos, interleaved) for l in range(L)],
            "v": [v[l].double() for l in range(L)]}
    for name in ("k", "v"):
        before, after = getattr(kv0, name), getattr(kv, name).cpu()
        sc0, sc1 = getattr(kv0, name + "_scale"), getattr(kv, name + "_scale")
        sc1 = None if sc1 is None else sc1.cpu()
        touched = torch.zeros(before.numel(), dtype=torch.bool)
        runs = {}
        for i, s in enumerate(slots.tolist()):
            if good[i] or (fmt == "page8" and 0 <= s < cap):
                runs.setdefault(s // ps, []).append((i, s % ps))
        if fmt == "page8":
            seen = torch.zeros_like(sc0, dtype=torch.bool)
        for l in range(L):
            for h in range(H):
                for page, members in runs.items():
                    vals = {slot: rows[name][l][i, h] for i, slot in members if good[i]}
                    if fmt == "page8":
                        first = members[0][1]
                        seen[l, page, h] = True
                        was = float(sc0[l, page, h])
                        old = was if first > 0 and was > 0 and was < float("inf") else 0.0
                        amax = max((float(x.abs().max()) for x in vals.values()), default=0.0)
                        scale = float(sc1[l, page, h])
                        lo, hi = (max(old, round_ops.pow2_scale(amax * (1 + d))) for d in (-(2.0 ** -19), 2.0 ** -19))
                        assert lo <= scale <= hi, (name, l, page, h, old, amax, scale)
                        for slot in range(first):
                            where = row_index(kv0, l, page, slot, h)
                            touched[where] = True
                            want = before[where] if scale == old else round_ops.requantised(before[where], torch.tensor(old) / torch.tensor(scale))
                            assert torch.equal(after[where], want), (name, l, page, h, slot)
                    elif fmt == "head8":
                        scale = float(sc0[l, h])
                    for slot, want in vals.items():
                        where = row_index(kv0, l, page, slot, h)
                        touched[where] = True
                        err = 2.0 ** -19 * want.abs().max()
                        if fmt == "bf16":
                            got, tol = after[where].double(), 2.0 ** -8 * want.abs() + err
                        else:
                            got = round_ops.e4m3_values(after[where]).double() * scale
                            want = want.clamp(-448 * scale, 448 * scale)
                            tol = 2.0 ** -4 * want.abs() + 2.0 ** -10 * scale + err
                        assert ((got - want).abs() <= tol).all(), (name, l, page, h, slot)
        bits = (lambda t: t.view(torch.int16)) if fmt == "bf16" else (lambda t: t)
        assert torch.equal(bits(after)[~touched], bits(before)[~touched])  # nothing else is written
        if fmt == "page8":
            same = (sc1 == sc0) | (sc1.isnan() & sc0.isnan())
            assert same[~seen].all()
        elif fmt == "head8":
            assert torch.equal(sc0, sc1)
    return kv, dq


def runs_of(spec, ps):
    """(positions, slots) of (first position, rows, pages) triples."""
    pos, slots = [], []
    for first, n, pages in spec:
        for t in range(first, first + n):
            pos.append(t)
            slots.append(pages[t // ps - first // ps] * ps + t % ps)
    return torch.tensor(pos, dtype=torch.int32), torch.tensor(slots, dtype=torch.int32)


@pytest.mark.parametrize("fmt", ["bf16", "head8", "page8"])
@pytest.mark.parametrize("D,Hq,H,rot,interleaved,norm", [(128, 8, 2, 128, False, True), (64, 6, 3, 64, True, True), (128, 5, 1, 32, False, False),
                                                         (64, 2, 2, 16, True, True), (128, 4, 4, 96, False, True), (64, 8, 2, 48, False, False)])
def test_rows_of_several_sequences(fmt, D, Hq, H, rot, interleaved, norm):
    ps, L = 8, 2
    # a run that begins inside a page and crosses two, one that fills a page, single rows, padding behind
    pos, slots = runs_of([(5, 14, [3, 9, 0]), (16, 8, [4]), (31, 1, [7]), (0, 1, [1]), (2, 3, [11])], ps)
    pos, slots = torch.cat([pos, torch.tensor([3, 99999], dtype=torch.int32)]), torch.cat([slots, torch.tensor([-1, -5], dtype=torch.int32)])
    kv = make_cache(L, 12, H, ps, D, Hq, fmt, seed=D + Hq, slot_pad=16, page_pad=32)
    q, k, v = make_rows(L, len(slots), Hq, H, D, seed=rot)
    w = (torch.rand(2, L, D, generator=torch.Generator().manual_seed(1)) + 0.5).to(torch.bfloat16)
    check(kv, q, k, v, pos, slots, w[0] if norm else None, w[1] if norm else None, 1e-6, round_ops.cos_sin_table(40, rot), interleaved)


@pytest.mark.parametrize("fmt", ["bf16", "head8", "page8"])
@pytest.mark.parametrize("ps,n", [(1, 7), (16, 1), (64, 200), (256, 300), (24, 61)])
def test_page_sizes_and_run_lengths(fmt, ps, n):
    Hq, H, D = 4, 2, 128
    pages = -(-(n + 3) // ps) + 1
    first = 3 if ps > 3 else 0
    pos, slots = runs_of([(first, n, list(range(pages))[::-1])], ps)
    kv = make_cache(1, pages, H, ps, D, Hq, fmt, seed=n)
    q, k, v = make_rows(1, n, Hq, H, D, seed=ps)
    check(kv, q, k, v, pos, slots, None, None, 1e-5, round_ops.cos_sin_table(first + n, 128), False)
    check(kv, None, k, v, None, slots, None, None, 1e-5, None, False)  # K and V only, as they are


def test_many_rows_take_whole_rows_per_warp():
    Hq, H, D, ps, n = 12, 2, 64, 16, 10000
    pos, slots = runs_of([(0, n, list(range(n // ps + 1)))], ps)
    kv = make_cache(1, n // ps + 1, H, ps, D, Hq, "bf16")
    q, k, v = make_rows(1, n, Hq, H, D, seed=2)
    w = torch.ones(1, D, dtype=torch.bfloat16)
    table = round_ops.cos_sin_table(n, 64)
    kv_d, dq = kv.to("cuda"), None
    dq, ws = binding.spec_qkv_append(kv_d, q.cuda(), k.cuda(), v.cuda(), pos.cuda(), slots.cuda(), q_weight=w.cuda(), k_weight=w.cuda(),
                                     cos_sin=table.cuda())
    for name, x, got in (("q", q, dq[0].cpu()), ("k", k, kv_d.k.cpu().view(-1, H, ps, D).transpose(1, 2).reshape(-1, H, D)[:n])):
        want = round_ops.norm_rope(x[0], w[0], 1e-6, table, pos, False)
        assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * want.abs().amax(-1, keepdim=True)).all(), name
    assert torch.equal(kv_d.v.cpu().view(-1, H, ps, D).transpose(1, 2).reshape(-1, H, D)[:n], v[0])


def test_a_growing_page_keeps_its_rows():
    """Token after token into one page, each larger than the one before: the earlier rows stay within a step of their values."""
    H, D, ps = 2, 128, 16
    kv = make_cache(1, 2, H, ps, D, 4, "page8", seed=1).to("cuda")
    g = torch.Generator().manual_seed(5)
    truth = torch.zeros(ps, H, D)
    for t in range(ps):
        row = (torch.randn(1, 1, H, D, generator=g) * 2.0 ** (t // 2 - 3)).to(torch.bfloat16)
        truth[t] = row[0, 0].float()
        slot = torch.tensor([ps + t], dtype=torch.int32, device="cuda")
        binding.spec_qkv_append(kv, None, row.cuda(), row.cuda(), None, slot)
        for data, scale in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)):
            s = scale[0, 1].cpu()
            assert ((s.log2() % 1) == 0).all()
            got = round_ops.e4m3_values(data.cpu().view(2, H, ps, D)[1, :, :t + 1]) * s[:, None, None]
            want = truth[:t + 1].transpose(0, 1)
            # one rounding to e4m3, then only halvings: exact, but where a value is subnormal by then (half a step of the present
            # scale, and as much again at each of the up to fifteen times it grew, halved from one to the next)
            tol = 2.0 ** -4 * want.abs() + 2.0 ** -9 * s[:, None, None]
            assert ((got - want).abs() <= tol).all()
    # the page starts afresh with its first slot
    small = torch.full((1, 1, H, D), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    binding.spec_qkv_append(kv, None, small, small, None, torch.tensor([ps], dtype=torch.int32, device="cuda"))
    assert (kv.k_scale[0, 1] == 2.0 ** -18).all() and (kv.v_scale[0, 1] == 2.0 ** -18).all()


def test_zeros_and_values_that_are_no_numbers():
    H, D, ps = 1, 64, 4
    kv = make_cache(1, 3, H, ps, D, 1, "page8", seed=1).to("cuda")
    x = torch.zeros(1, 6, H, D)
    x[0, 4] = 1.0
    x[0, 4, 0, 3] = float("inf")
    x[0, 5, 0, 7] = float("nan")
    x[0, 5, 0, 8] = 2.0
    x = x.to(torch.bfloat16).cuda()
    binding.spec_qkv_append(kv, None, x, x, None, torch.arange(4, 10, dtype=torch.int32, device="cuda"))
    assert float(kv.k_scale[0, 1, 0]) == 2.0 ** -64 and (kv.k.view(3, ps, D)[1] == 0).all()
    s = float(kv.v_scale[0, 2, 0])
    got = round_ops.e4m3_values(kv.v.cpu().view(3, ps, D)[2]) * s
    assert s == 2.0 ** 120 and got[0, 3] == 448 * s and got[1, 7].isnan() and (got[0, :3] == 0).all()
    # an infinity in a cache without page scales: saturated in 8 bits, kept in bf16
    for fmt in ("head8", "bf16"):
        kv = make_cache(1, 3, H, ps, D, 1, fmt, seed=1).to("cuda")
        binding.spec_qkv_append(kv, None, x, x, None, torch.arange(4, 10, dtype=torch.int32, device="cuda"))
        row = kv.k.view(3, ps, D)[2].cpu()
        row = round_ops.e4m3_values(row) if fmt == "head8" else row.float()
        assert row[0, 3] == (448 if fmt == "head8" else float("inf")) and row[1, 7].isnan()


def test_rows_out_of_range_are_reported_and_left_out():
    Hq, H, D, ps = 4, 2, 128, 8
    for fmt in ("bf16", "head8", "page8"):
        kv = make_cache(1, 4, H, ps, D, Hq, fmt, seed=3)
        q, k, v = make_rows(1, 6, Hq, H, D, seed=4)
        pos = torch.tensor([3, 4, 77, 6, -2, 9], dtype=torch.int32)
        slots = torch.tensor([3, 4, 5, 6, 17, 32], dtype=torch.int32)
        check(kv, q, k, v, pos, slots, None, None, 1e-6, round_ops.cos_sin_table(40, 128), False)
        check(kv, None, k, v, None, slots, None, None, 1e-6, None, False)


def test_rows_left_out_do_not_start_a_page_anew():
    Hq, H, D, ps = 4, 2, 128, 8
    kv = make_cache(1, 6, H, ps, D, Hq, "page8", seed=3).to("cuda")
    was = [t.clone() for t in (kv.k, kv.v, kv.k_scale, kv.v_scale)]
    q, k, v = (x.cuda() for x in make_rows(1, 4, Hq, H, D, seed=4))
    pos, slots = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([40, -1, 41, 99], [ps, -1, 3 * ps, 4 * ps + 3]))
    _, ws = binding.spec_qkv_append(kv, q, k, v, pos, slots, cos_sin=round_ops.cos_sin_table(40, 128).cuda())
    assert binding.read_status(ws) == -6
    for t, w in zip((kv.k, kv.v, kv.k_scale, kv.v_scale), was):
        assert torch.equal(t.nan_to_num(), w.nan_to_num())


@pytest.mark.parametrize("rows", [3, 1300])
def test_a_head_that_is_no_number_leaves_its_page_to_the_others(rows):
    """Norms of a head with a NaN, an infinity, or (eps = 0) nothing but zeros are no numbers."""
    Hq, H, D, ps = 4, 2, 128, 4
    kv = make_cache(1, 1 + rows // ps + 1, H, ps, D, Hq, "page8", seed=3).to("cuda")
    k = torch.ones(1, rows, H, D, dtype=torch.bfloat16, device="cuda")
    k[0, 1, 0, 5] = float("nan")
    k[0, 1, 1] = 0
    k[0, 2, 0, 9] = float("inf")
    slots = torch.arange(ps, ps + rows, dtype=torch.int32, device="cuda")
    weight = torch.ones(1, D, dtype=torch.bfloat16, device="cuda")
    binding.spec_qkv_append(kv, None, k, k, None, slots, k_weight=weight, eps=0.0)
    assert (kv.k_scale[0, 1] == 2.0 ** -8).all()  # every other value is 1
    got = round_ops.e4m3_values(kv.k.cpu().view(-1, H, ps, D)[1])
    assert (got[:, 0] == 256).all() and got[:, 1].isnan().all() and (got[1, 2] == 256).all()
    assert (got[0, 2, :9] == 0).all() and got[0, 2, 9].isnan()


def test_q_may_be_rotated_in_place():
    Hq, H, D = 4, 2, 128
    kv = make_cache(2, 4, H, 8, D, Hq, "bf16", seed=3).to("cuda")
    q, k, v = make_rows(2, 9, Hq, H, D, seed=4)
    pos, slots = runs_of([(0, 9, [2, 0])], 8)
    table = round_ops.cos_sin_table(40, 128).cuda()
    want, _ = binding.spec_qkv_append(kv, q.cuda(), k.cuda(), v.cuda(), pos.cuda(), slots.cuda(), cos_sin=table)
    mine = q.contiguous().cuda()
    out, _ = binding.spec_qkv_append(kv, mine, k.cuda(), v.cuda(), pos.cuda(), slots.cuda(), cos_sin=table, q_out=mine)
    assert out is mine and torch.equal(mine, want)


def test_a_replayed_graph_writes_where_the_slots_say():
    Hq, H, D, ps = 4, 2, 128, 8
    kv0 = make_cache(1, 4, H, ps, D, Hq, "page8", seed=3)
    q, k, v = make_rows(1, 3, Hq, H, D, seed=4)
    table = round_ops.cos_sin_table(40, 128).cuda()
    kv, ref = kv0.to("cuda"), kv0.to("cuda")
    dq, dk, dv = q.cuda(), k.cuda(), v.cuda()
    pos, slots = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2))
    out = torch.empty(1, 3, Hq, D, dtype=torch.bfloat16, device="cuda")
    ws = binding.alloc_workspace(binding.append_workspace_bytes(), "cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # a stream of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            binding.spec_qkv_append(kv, dq, dk, dv, pos, slots, cos_sin=table, q_out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    for first, pages in ((0, [2]), (3, [2]), (6, [2, 1]), (9, [1])):
        p, s = runs_of([(first, 3, pages)], ps)
        pos.copy_(p), slots.copy_(s)
        g.replay()
        want, _ = binding.spec_qkv_append(ref, dq, dk, dv, p.cuda(), s.cuda(), cos_sin=table)
        assert torch.equal(out, want) and torch.equal(kv.k, ref.k) and torch.equal(kv.v, ref.v)
        assert torch.equal(kv.k_scale.nan_to_num(), ref.k_scale.nan_to_num()) and binding.read_status(ws) == 0


def test_arguments_are_checked():
    Hq, H, D = 4, 2, 128
    kv = make_cache(1, 4, H, 8, D, Hq, "page8", seed=3).to("cuda")
    q, k, v = (x.cuda() for x in make_rows(1, 3, Hq, H, D, seed=4))
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    table = round_ops.cos_sin_table(40, 128).cuda()
    ok = dict(cos_sin=table)
    with pytest.raises(ValueError):
        binding.spec_qkv_append(kv, q.float(), k, v, pos, pos, **ok)
    with pytest.raises(ValueError):
        binding.spec_qkv_append(kv, q, k[:, :2], v, pos, pos, **ok)
    with pytest.raises(ValueError):
        binding.spec_qkv_append(kv, q, k, v.transpose(2, 3).contiguous().transpose(2, 3), pos, pos, **ok)
    with pytest.raises(ValueError):
        binding.spec_qkv_append(kv, q, k, v, pos.long(), pos, **ok)
    with pytest.raises(ValueError):
        binding.spec_qkv_append(kv, q, k, v, pos, pos, q_weight=torch.ones(D, device="cuda", dtype=torch.bfloat16), **ok)
    with pytest.raises(ValueError):
        binding.spec_qkv_append(kv, q, k, v, pos, pos, q_out=torch.empty_like(q)[:, :2].contiguous(), **ok)
    with pytest.raises(ValueError):
        binding.spec_qkv_append(dataclasses.replace(kv, v_scale=kv.v_scale[0].contiguous()), q, k, v, pos, pos, **ok)
    with pytest.raises(binding.SpecError):
        binding.spec_qkv_append(kv, q, k, v, pos, pos, cos_sin=round_ops.cos_sin_table(40, 24).cuda())  # not in sixteens
    with pytest.raises(binding.SpecError):
        binding.spec_qkv_append(kv, q, k, v, None, pos, **ok)  # a rotation without positions
    with pytest.raises(binding.SpecError):
        binding.spec_qkv_append(dataclasses.replace(kv, head_stride=0), q, k, v, pos, pos, **ok)
    out, _ = binding.spec_qkv_append(kv, q[:, :0], k[:, :0], v[:, :0], pos[:0], pos[:0], **ok)
    assert out.shape == (1, 0, Hq, D)
