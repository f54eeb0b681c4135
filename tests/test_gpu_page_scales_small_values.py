"""Drafting over a cache with page scales where all that counts lies in pages of small V scales, beside one page of a much larger scale that
the softmax gives nothing.

Tolerance.  As in test_gpu_page_scales.py, (2 e + 2^-14) of the largest |v|, here of the pages that count (the large page's part of the
result is below 2^-60 of them).  The two 16-bit parts of a probability are off by at most 2^-41 of the largest V scale: with N keys, and V
scales down to 2^-18 of that, N 2^-41 2^18 = N 2^-23 of the largest |v|, below 2^-14 for the 500 keys here."""
import dataclasses

import pytest
import torch

import round_ops
from paper_2607_27735_b200 import binding
from test_gpu_page_scales import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("Hq,H", [(2, 2), (8, 2), (5, 1), (16, 2)])  # both forms of the products
@pytest.mark.parametrize("n", [60, 500])
@pytest.mark.parametrize("small", [10, 18])
def test_small_scales_beside_a_large_one_that_gets_nothing(D, Hq, H, n, small):
    ps, T, G = 16, 640, Hq // H
    kv, q, start = make(ctx=(T,), Hq=Hq, H=H, D=D, ps=ps, n_q=1, seed=n + D + Hq, poison=False, spread=0.2)
    q = q[:, :, 0].contiguous()
    q.view(1, 1, H, G, D)[:] = q.view(1, 1, H, G, D)[:, :, :, :1].clone()  # the heads of a group look the same way
    far = int(kv.page_table[0, 1])                                        # positions 16 to 31
    k, ks, vs = kv.k.clone(), kv.k_scale.clone(), kv.v_scale.clone()
    for h in range(H):
        k[0, far, h] = (-q[0, 0, h * G].float() * 40).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    ks[:, far] = 2.0                                                      # scores of about -40 |q|^2 2 / sqrt(D)
    vs *= 2.0 ** -small
    vs[:, far] *= 2.0 ** small
    kv = dataclasses.replace(kv, k=k, k_scale=ks, v_scale=vs)
    idx = torch.arange(n, dtype=torch.int32, device="cuda").expand(1, 1, H, n).contiguous()
    count = torch.full((1, 1, H), n, dtype=torch.int32, device="cuda")
    out, lse, ws = binding.spec_sparse_draft_attn(kv, q, idx, count, start, start, 0)
    assert binding.read_status(ws) == 0
    for hq in range(Hq):
        keys, values = round_ops.cache_rows(kv, 0, 0, hq // G, range(n), "cuda")
        want, z, p, size = round_ops.attend(q[0, 0, hq][None], keys, values, torch.tensor([n], device="cuda"))
        assert float(p[0, 16:32].sum()) < 2.0 ** -90
        near = torch.ones(n, dtype=torch.bool, device="cuda")
        near[16:32] = False
        e = size * 2.0 ** -20 + 2.0 ** -19
        # (`size` is of the far page's scores; of the others it is less, and they are all that counts)
        e = min(e, float((q[0, 0, hq].double().abs() @ keys[near].abs().T).max()) * D ** -0.5 * 1.4427 * 2.0 ** -20 + 2.0 ** -19)
        assert ((out[0, 0, hq].double() - want[0]).abs() <= (2 * e + 2.0 ** -14) * float(values[near].abs().max())).all()
        assert abs(float(lse[0, 0, hq].double() - z[0])) <= 2 * e + 2.0 ** -22 * abs(float(z[0]))
