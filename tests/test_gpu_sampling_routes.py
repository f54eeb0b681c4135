"""Probabilities and acceptance at the sizes where another kernel or another way through it takes over: rows too long for shared memory,
acceptance by CTAs of 8, 16 and 32 warps, and the second look at a row whose target lies nowhere above the draft, by one CTA and by clusters.
Tolerances as in test_gpu_sampling.py (a thread adds at most 62 terms one after the other here)."""
import pytest
import torch

from paper_2607_27735_b200 import binding
from test_gpu_sampling import _both, _case, _check_probs, _rows

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("vocab,dtype,offset", [(1000003, torch.bfloat16, 3), (1000003, torch.bfloat16, 0), (500009, torch.float32, 1),
                                               (819200, torch.bfloat16, 0), (819199 + 64, torch.bfloat16, 0), (410007, torch.float32, 2)])
def test_rows_longer_than_shared_memory(vocab, dtype, offset):
    rows = 6
    logits, dev = _rows(rows, vocab, dtype, vocab, offset, vocab + 5)
    for x in (logits, dev):
        x[1] = -INF
        x[1, vocab - 3:] = 0.5
        x[2] = torch.finfo(dtype).min
        x[3, vocab // 2] = x[3].max()
        x[4, ::2] = -INF
        x[5] = -INF
    t = torch.tensor([0.8, 0.7, 1.0, 0.0, 1.3, 1.0])
    out = torch.full((rows, vocab + 3), 7.0, device="cuda")
    binding.spec_token_probs(dev, t.cuda(), probs=out[:, 1:vocab + 1])
    _check_probs(logits, t, out[:, 1:vocab + 1])
    assert (out[:, 0] == 7).all() and (out[:, vocab + 1:] == 7).all()
    greedy = binding.spec_token_probs(dev, torch.zeros(rows, device="cuda"))
    _check_probs(logits, torch.zeros(rows), greedy)
    dev[0, vocab - 1] = float("nan")
    assert binding.spec_token_probs(dev, t.cuda())[0].isnan().all()


@pytest.mark.parametrize("B,V", [(37, 50257), (20, 50257), (20, 40000), (30, 32768), (40, 17000), (6, 32000), (6, 128256), (3, 777)])
def test_acceptance_by_every_size_of_a_cta(B, V):
    k = 2
    p, q, draft, u = _case(B, k, V, B + V)
    _both(p, q, draft, u)
    _both(p, None, draft, u)
    # sequences whose first row lies nowhere above the draft's, between ordinary ones
    rows = torch.arange(0, B, 3)
    p[rows, 0] = q[rows, 0] * 0.5
    u[rows, 0] = 0.9
    n, _ = _both(p, q, draft, u)
    assert (n[rows.cuda()] == 0).all()
    # and some without any mass
    p[rows[::2], 0] = 0.0
    _, token = _both(p, q, draft, u)
    assert (token[rows[::2].cuda()] == 0).all()
