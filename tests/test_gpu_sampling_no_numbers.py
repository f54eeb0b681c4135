"""Acceptance where probabilities are no numbers or negative: either counts as 0, the target's and the draft's alike.  The plain form is
written from that rule alone, in 64 bits; the results are whole numbers."""
import pytest
import torch

from paper_2607_27735_b200 import binding

pytestmark = pytest.mark.gpu
NAN = float("nan")


def plain(p, draft, u, q):
    p, q = (torch.where(x > 0, x, 0.0).double() for x in (p, q))  # (a comparison with NaN is false)
    counts, tokens = [], []
    for b in range(p.shape[0]):
        m, k = 0, draft.shape[1]
        while m < k and float(u[b, m]) * float(q[b, m, draft[b, m]]) < float(p[b, m, draft[b, m]]):
            m += 1
        w = (p[b, m] - q[b, m]).clamp_min(0) if m < k else p[b, m]
        if not float(w.sum()) > 0:
            w = p[b, m]
        counts.append(m)
        if not float(w.sum()) > 0:
            tokens.append(0)
            continue
        c = w.cumsum(0)
        past = (c > float(u[b, k]) * float(c[-1])) & (w > 0)
        tokens.append(int(past.nonzero()[0]) if bool(past.any()) else int((w > 0).nonzero()[-1]))
    return counts, tokens


def case(B, k, V, seed):
    g = torch.Generator().manual_seed(seed)
    p = torch.softmax(torch.randn(B, k + 1, V, generator=g) * 2, -1)
    q = torch.softmax(torch.randn(B, k, V, generator=g) * 2, -1)
    return p, q, torch.randint(0, V, (B, k), generator=g).int(), torch.rand(B, k + 1, generator=g)


def both(p, draft, u, q):
    n, token = binding.spec_accept_sample(p.cuda(), draft.cuda(), u.cuda(), draft_probs=q.cuda())
    want = plain(p, draft, u, q)
    assert n.tolist() == want[0] and token.tolist() == want[1]
    return want


@pytest.mark.parametrize("V", [300, 1003, 40000])  # a CTA for each sequence, and clusters of them
def test_values_of_the_draft_that_count_as_nothing(V):
    p, q, draft, u = case(12, 2, V, V)
    rows = torch.arange(12)
    u[:, :2] = u[:, :2].clamp_min(0.1)
    x = draft[:, 0].long()
    q[rows[0:3], 0, x[0:3]] = NAN          # the drafted token's own: 0 accepts whatever has any probability
    q[rows[3:6], 0, x[3:6]] = -0.5
    p[rows[4:6], 0, x[4:6]] = 0.0          # and nothing without any
    q[6:8, 0, ::2] = NAN                   # where the row is drawn from
    q[8:10, 0, ::3] = -1.0
    q[10, 0] = NAN                         # nowhere a number: drawn from p itself
    q[11, 0] = -q[11, 0]
    p[rows[6:12], 0, x[6:12]] = 0.0        # (rejected)
    counts, _ = both(p, draft, u, q)
    assert min(counts[0:4]) >= 1 and counts[4:12] == [0] * 8


@pytest.mark.parametrize("V", [300, 40000])
def test_values_of_both_that_count_as_nothing(V):
    p, q, draft, u = case(9, 3, V, V + 1)
    g = torch.Generator().manual_seed(7)
    for x in (p, q):
        kind = torch.randint(0, 6, x.shape, generator=g)
        x[kind == 0] = NAN
        x[kind == 1] *= -1
    both(p, draft, u, q)
