"""Calls of more rows than the GPU has warps for at once, whose warps take all heads of a row, batch after batch: head counts that
end inside a batch, against the formulas in 64 bits (tolerances as for the smaller calls: 2^-19 of the head's largest value for the fp32
steps, and one rounding to the type, 2^-8 of the value or 2^-4 of it and half a subnormal step, 2^-10 times the scale)."""
import pytest
import torch

import round_ops
from paper_2607_27735_b200 import binding
from test_gpu_qkv_append import make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "head8", "page8"])
@pytest.mark.parametrize("L,N,Hq,H,D,ps,interleaved,with_q", [
    (1, 2403, 20, 10, 128, 16, False, True),   # three batches of Q, two of K and of V, the last ones not full
    (2, 2050, 22, 22, 64, 64, True, True),     # layers; sixteen heads a batch, six in the second
    (1, 5111, 9, 9, 128, 32, False, False),    # K and V only, one head in the second batch
    (1, 7300, 1, 1, 64, 8, False, True),       # one head
])
def test_many_rows(fmt, L, N, Hq, H, D, ps, interleaved, with_q):
    n_pages = 2 + -(-N // ps)
    kv = make_cache(L, n_pages, H, ps, D, Hq, fmt, seed=N).to("cuda")
    if fmt == "head8":
        kv.k_scale.copy_(kv.k_scale * 0.5), kv.v_scale.copy_(kv.v_scale * 0.5)
    before = {name: getattr(kv, name).clone().view(L, n_pages, H, ps, D) for name in ("k", "v")}
    g = torch.Generator(device="cuda").manual_seed(N + 1)
    x = torch.randn(L, N, Hq + 2 * H, D, generator=g, device="cuda") * torch.exp(torch.randn(L, N, Hq + 2 * H, 1, generator=g, device="cuda"))
    x = x.to(torch.bfloat16)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
    table = round_ops.cos_sin_table(4000, D).cuda()
    pos = torch.arange(N, device="cuda", dtype=torch.int32) * 7 % 4000
    left_out = torch.zeros(N, dtype=torch.bool, device="cuda")
    left_out[[0, N - 1]] = True  # (the first page begins at its slot 1)
    slots = torch.arange(ps, ps + N, device="cuda", dtype=torch.int32)
    slots[left_out] = -1
    qw, kw = (torch.randn(L, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    out = torch.full((L, N, Hq, D), 5.0, dtype=torch.bfloat16, device="cuda") if with_q else None
    _, ws = binding.spec_qkv_append(kv, q if with_q else None, k, v, pos, slots, q_weight=qw, k_weight=kw, cos_sin=table,
                                    interleaved=interleaved, q_out=out)
    assert binding.read_status(ws) == 0
    index = torch.arange(ps, ps + N, device="cuda")[~left_out]
    page, slot = index // ps, index % ps

    def turned(rows, weight, l):  # (the plain form works on the CPU's tensors as on the GPU's, but for its index lists)
        return round_ops.norm_rope(rows[l].cpu(), weight[l].cpu(), 1e-6, table.cpu(), pos.cpu(), interleaved).cuda()

    for l in range(L):
        if with_q:
            want = turned(q, qw, l)
            tol = 2.0 ** -8 * want.abs() + 2.0 ** -19 * want.abs().amax(-1, keepdim=True)
            assert ((out[l].double() - want).abs() <= tol)[~left_out].all() and (out[l][left_out] == 5.0).all()
        for name, want in (("k", turned(k, kw, l)), ("v", v[l].double())):
            want = want[~left_out]
            data = getattr(kv, name).view(L, n_pages, H, ps, D)
            got = data[l, page, :, slot]  # [rows, heads, D]
            err = 2.0 ** -19 * want.abs().amax(-1, keepdim=True)
            if fmt == "bf16":
                assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + err).all()
            else:
                scale = getattr(kv, name + "_scale")
                s = (scale[l][None] if fmt == "head8" else scale[l, page])[..., None].double()
                if fmt == "page8":  # the least power of two that holds the page's largest value
                    most = torch.zeros(n_pages, H, dtype=torch.float64, device="cuda").index_reduce_(0, page, want.abs().amax(-1), "amax")
                    most, own = most[1:-1], scale[l, 1:-1].double()
                    runs_from_0 = torch.ones(n_pages - 2, 1, dtype=torch.bool, device="cuda")
                    runs_from_0[0] = False  # (slot 0 is left out: the page's old scale counts)
                    some = most > 0
                    assert ((own.frexp().mantissa == 0.5) | ~runs_from_0)[some].all()
                    assert (most * (1 - 2.0 ** -19) <= 448 * own)[some].all()
                    assert ((most * (1 + 2.0 ** -19) >= 224 * own) | ~runs_from_0)[some].all()
                want = want.clamp(-448 * s, 448 * s)
                got = got.view(torch.float8_e4m3fn).double() * s
                assert ((got - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * s + err).all()
            # nothing else is written (but for the rows before a page's run, where its scale has grown)
            untouched = torch.ones(n_pages, ps, dtype=torch.bool, device="cuda")
            untouched[page, slot] = False
            if fmt == "page8":
                untouched[1] = False
            same = (data[l] == before[name][l]).all(-1) if fmt != "bf16" else (data[l].view(torch.int16) == before[name][l].view(torch.int16)).all(-1)
            assert same.transpose(1, 2)[untouched].all()
