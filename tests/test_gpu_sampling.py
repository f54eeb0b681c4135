"""Probabilities of logits rows and acceptance of sampled drafts on the GPU, against the formulas in 64 bits.

Tolerance of a probability, from its roundings in fp32 (u = 2^-24): the exponent (z - m) / T passes the difference, the
reciprocal and the product, once relative to a thread's and once to the row's largest logit, 3 u each of |z - m| / T; the
exponentials are within 2 ulp (4 u), twice; the sum adds at most 64 terms one after the other and 18 levels of a tree
(each merge a product and a sum); the quotient, the product and the store 4 more.  Together (6 |z - m| / T + 8 + 64 + 72 + 4) u, taken
as (6 |z - m| / T + 160) u.  Products of two factors below 2^-126 round in steps of 2^-149."""
import pytest
import torch

import round_ops
from paper_2607_27735_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _check_probs(logits, temperature, got):
    got = got.cpu()
    for r in range(logits.shape[0]):
        t = 1.0 if temperature is None else float(temperature[r])
        want = round_ops.token_probs(logits[r], t)
        z = logits[r].double()
        if t <= 0 or float(z.max()) == -float("inf"):
            assert torch.equal(got[r].double(), want), r
            continue
        far = ((z.max() - z) / t).clamp(max=200.0)
        assert ((got[r].double() - want).abs() <= want * (6 * far + 160) * U + 2.0 ** -140).all(), r


def _rows(rows, vocab, dtype, seed, offset=0, stride=None):
    g = torch.Generator().manual_seed(seed)
    stride = vocab if stride is None else stride
    base = torch.zeros(rows * stride + offset + 8, dtype=dtype)
    view = base.as_strided((rows, vocab), (stride, 1), offset)
    x = torch.randn(rows, vocab, generator=g) * (torch.rand(rows, 1, generator=g) * 4 + 0.2)
    x[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] += 12
    view.copy_(x)
    dev = base.cuda().as_strided((rows, vocab), (stride, 1), offset)
    return view, dev


@pytest.mark.parametrize("rows,vocab,dtype,offset,stride", [
    (1, 128256, torch.bfloat16, 0, None),
    (9, 128256, torch.bfloat16, 0, None),
    (5, 128256, torch.float32, 0, None),
    (70, 32000, torch.bfloat16, 0, None),
    (3, 50257, torch.bfloat16, 0, None),       # rows that start on every 2-byte place
    (4, 50257, torch.float32, 1, 50260),
    (3, 151936, torch.bfloat16, 0, None),
    (2, 200003, torch.float32, 0, None),
    (2, 262144 + 77, torch.bfloat16, 3, None),  # more than the registers of a cluster hold
    (300, 1003, torch.bfloat16, 5, 1011),
    (3, 1, torch.float32, 0, None),
    (9, 7, torch.bfloat16, 0, None),
    (5, 16, torch.bfloat16, 1, 17),
])
def test_probs_match_the_formula(rows, vocab, dtype, offset, stride):
    logits, dev = _rows(rows, vocab, dtype, rows + vocab, offset, stride)
    g = torch.Generator().manual_seed(rows)
    t = torch.rand(rows, generator=g) * 1.5 + 0.05
    t[::4] = 0.0
    _check_probs(logits, None, binding.spec_token_probs(dev))
    _check_probs(logits, t, binding.spec_token_probs(dev, t.cuda()))
    # into rows that lie apart: what is between them stays
    wide = torch.full((rows, vocab + 5), 7.0, device="cuda")
    binding.spec_token_probs(dev, t.cuda(), probs=wide[:, 2:vocab + 2])
    _check_probs(logits, t, wide[:, 2:vocab + 2])
    assert (wide[:, :2] == 7).all() and (wide[:, vocab + 2:] == 7).all()


@pytest.mark.parametrize("vocab", [1003, 40000, 300000])
def test_masked_rows_and_values_that_are_no_numbers(vocab):
    inf = float("inf")
    x = torch.randn(8, vocab, generator=torch.Generator().manual_seed(vocab))
    x[0] = -inf                                   # nothing is left
    x[1, 5:] = -inf                               # a few tokens are
    x[2] = torch.finfo(torch.float32).min         # masks of the type's lowest value: equal logits
    x[3, ::2] = torch.finfo(torch.float32).min
    x[4, vocab // 2] = float("nan")
    x[5, vocab - 1] = inf
    x[6, :vocab - 1] = -inf                       # one token in the ragged end
    t = torch.tensor([1.0, 0.7, 1.0, 0.5, 1.0, 1.0, 2.0, 1e-38])
    p = binding.spec_token_probs(x.cuda(), t.cuda()).cpu()
    assert (p[0] == 0).all()
    assert p[4].isnan().all() and p[5].isnan().all()
    for r in (1, 2, 3, 6, 7):
        _check_probs(x[r:r + 1], t[r:r + 1], p[r:r + 1])
    greedy = binding.spec_token_probs(x.cuda(), torch.zeros(8, device="cuda")).cpu()
    assert (greedy[0] == 0).all()
    for r, best in ((1, int(x[1, :5].argmax())), (2, 0), (5, vocab - 1), (6, vocab - 1)):
        assert greedy[r, best] == 1 and greedy[r].sum() == 1


def test_greedy_takes_the_first_of_equal_logits_wherever_they_lie():
    for vocab in (9, 4099, 70000, 300001):
        x = torch.zeros(6, vocab)
        for r, at in enumerate([0, 1, vocab // 3, vocab // 2, vocab - 2, vocab - 1]):
            x[r, at:] = 3.0
        for shift in range(4):
            base = torch.zeros(6 * vocab + shift + 8, device="cuda")
            dev = base[shift:shift + 6 * vocab].view(6, vocab)
            dev.copy_(x)
            p = binding.spec_token_probs(dev, torch.full((6,), -1.0, device="cuda"))
            assert p.argmax(-1).tolist() == [0, 1, vocab // 3, vocab // 2, vocab - 2, vocab - 1]
            assert (p.sum(-1) == 1).all()


def _case(B, k, V, seed, sharp=4.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(B, k + 1, V, generator=g) * sharp
    p = torch.softmax(z, -1)
    y = z[:, :k] + 0.4 * torch.randn(B, k, V, generator=g)
    q = torch.softmax(y, -1)
    draft = (y - (-torch.rand(B, k, V, generator=g).clamp_min(1e-9).log()).log()).argmax(-1).int() if k else torch.zeros(B, 0, dtype=torch.int32)
    return p, q, draft, torch.rand(B, k + 1, generator=g)


def _both(p, q, draft, u, n_draft=None, dev_p=None, dev_q=None):
    got = binding.spec_accept_sample(p.cuda() if dev_p is None else dev_p, draft.cuda(), u.cuda(),
                                     draft_probs=dev_q if dev_q is not None else None if q is None else q.cuda(),
                                     n_draft=None if n_draft is None else n_draft.cuda())
    want = round_ops.accept_sample(p, draft, u, q, n_draft)
    assert got[0].tolist() == want[0].tolist()
    assert got[1].tolist() == want[1].tolist()
    return got


@pytest.mark.parametrize("B,k,V", [(1, 4, 32000), (64, 8, 1003), (3, 1, 128256), (9, 3, 50257), (700, 2, 130), (2, 40, 515), (5, 0, 4096),
                                   (4, 5, 1), (6, 3, 2), (1, 2, 1050007)])
def test_accept_matches_the_formula(B, k, V):
    p, q, draft, u = _case(B, k, V, B + k + V)
    n, _ = _both(p, q, draft, u)
    if B >= 64:
        assert n.min() < n.max()
    _both(p, None, draft, u)  # greedy drafts
    if k:
        n_draft = torch.randint(-1, k + 2, (B,), generator=torch.Generator().manual_seed(V), dtype=torch.int32)
        _both(p, q, draft, u, n_draft)


def test_exact_sums_decide_ties():
    # rows whose sums are exact in 32 bits, and numbers that hit them exactly: c_j > u c_last, not >=
    V = 4096
    p = torch.full((9, 1, V), 1.0 / V)
    u = torch.tensor([[0.0], [1 / V], [2 / V], [0.5], [1 - 1 / V], [1 - 2.0 ** -24], [127 / V], [128 / V], [2047.5 / V]])
    n, token = _both(p, None, torch.zeros(9, 0, dtype=torch.int32), u)
    assert token.tolist() == [0, 1, 2, 2048, 4095, 4095, 127, 128, 2047]
    # acceptance is u q < p: equal rows always stand, and a u of 0 does not save a token without probability
    p, q, draft, u = _case(4, 3, 333, 9)
    q = p[:, :3].clone()
    u[:, :3] = 1 - 2.0 ** -24
    assert _both(p, q, draft, u)[0].tolist() == [3] * 4
    x = draft.long()
    p[torch.arange(4), 0, x[:, 0]] = 0.0
    u[:, 0] = 0.0
    assert _both(p, q, draft, u)[0].tolist() == [0] * 4


def test_rows_without_mass_numbers_out_of_range_and_bad_tokens():
    p, q, draft, u = _case(12, 2, 777, 4)
    nan = float("nan")
    p[0] = 0.0                                     # nothing anywhere: token 0
    p[1, 0] = q[1, 0] * 0.5                        # p <= q everywhere: a rejected token is replaced from p
    u[1, 0] = 0.9
    p[2, 0] = nan
    p[3, 0, ::2] = nan
    draft[4, 0], draft[5, 0] = -1, 777             # no tokens: rejected
    u[6], u[7], u[8] = 1.0, 2.0, -1.0
    u[9] = nan
    p[10, :, 700:] = 0.0
    u[10, 2] = 1.0
    p[11, 0] = -p[11, 0]
    n, token = _both(p, q, draft, u)
    assert n[4] == 0 and n[5] == 0 and token[0] == 0 and 0 <= int(token.min()) and int(token.max()) < 777
    _both(p, None, draft, u)
    with_inf = p.clone()
    with_inf[:, :, 3] = float("inf")
    n, token = binding.spec_accept_sample(with_inf.cuda(), draft.cuda(), u.cuda(), draft_probs=q.cuda())
    assert 0 <= int(token.min()) and int(token.max()) < 777


def test_rows_that_lie_apart_and_start_anywhere():
    p, q, draft, u = _case(5, 3, 1001, 77)
    for shift in (0, 1, 2, 3):
        big_p = torch.full((5, 4, 1010), 9.0, device="cuda")
        big_q = torch.full((6, 4, 1007), 9.0, device="cuda")
        dp, dq = big_p[:, :, shift:shift + 1001], big_q[:5, 1:, shift:shift + 1001]
        dp.copy_(p)
        dq.copy_(q)
        _both(p, q, draft, u, dev_p=dp, dev_q=dq)


def test_committed_tokens_follow_the_target():
    # the first committed token of a round is distributed as p_0, whatever the draft proposes
    V, n = 12, 40000
    g = torch.Generator().manual_seed(3)
    p = torch.softmax(torch.randn(V, generator=g) * 1.5, -1)
    q = torch.softmax(torch.randn(V, generator=g) * 1.5, -1)
    draft = torch.multinomial(q, n, replacement=True, generator=g).int().view(n, 1).cuda()
    u = torch.rand(n, 2, generator=g).cuda()
    m, token = binding.spec_accept_sample(p.cuda().expand(n, 2, V), draft, u, draft_probs=q.cuda().expand(n, 1, V))
    first = torch.where(m > 0, draft[:, 0], token)
    freq = torch.bincount(first.long(), minlength=V).double().cpu() / n
    # six standard deviations of a frequency
    assert ((freq - p.double()).abs() <= 6 * (p.double() * (1 - p.double()) / n).sqrt()).all()
    assert 0 < int(m.sum()) < n


def test_arguments_are_checked():
    p, q, draft, u = (x.cuda() for x in _case(2, 3, 64, 1))
    with pytest.raises(ValueError):
        binding.spec_accept_sample(p.double(), draft, u)
    with pytest.raises(ValueError):
        binding.spec_accept_sample(p, draft[:, :2].contiguous(), u)
    with pytest.raises(ValueError):
        binding.spec_accept_sample(p, draft, u[:, :3].contiguous())
    with pytest.raises(ValueError):
        binding.spec_accept_sample(p, draft, u, draft_probs=q[:, :2])
    with pytest.raises(ValueError):
        binding.spec_accept_sample(p.transpose(1, 2).contiguous().transpose(1, 2), draft, u)
    with pytest.raises(ValueError):
        binding.spec_accept_sample(p.cpu(), draft, u, n_accepted=draft[:, 0].contiguous(), next_token=draft[:, 0].contiguous())
    with pytest.raises(ValueError):
        binding.spec_token_probs(p[0], temperature=torch.ones(3, device="cuda"))
    with pytest.raises(ValueError):
        binding.spec_token_probs(p[0], probs=torch.empty(4, 63, device="cuda"))
    with pytest.raises(ValueError):
        binding.spec_token_probs(p[0].half())
    assert binding.spec_token_probs(p[0, :0]).shape == (0, 64)
    n, token = binding.spec_accept_sample(p[:0], draft[:0], u[:0])
    assert n.numel() == 0 and token.numel() == 0


def test_a_captured_chain_takes_new_logits_and_numbers():
    B, k, V = 3, 2, 5000
    logits = torch.zeros(B * (k + 1), V, device="cuda", dtype=torch.bfloat16)
    t = torch.ones(B * (k + 1), device="cuda")
    probs = torch.empty(B, k + 1, V, device="cuda")
    p, q, draft, u = (x.cuda() for x in _case(B, k, V, 1))
    n, token = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))

    def call():
        binding.spec_token_probs(logits, t, probs=probs.view(-1, V))
        binding.spec_accept_sample(probs, draft, u, draft_probs=q, n_accepted=n, next_token=token)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(5):
        p2, q2, d2, u2 = _case(B, k, V, seed + 20)
        logits.copy_(p2.log().view(-1, V))
        q.copy_(q2), draft.copy_(d2), u.copy_(u2)
        graph.replay()
        want = round_ops.accept_sample(probs.cpu(), d2, u2, q2)
        assert n.tolist() == want[0].tolist() and token.tolist() == want[1].tolist()
        _check_probs(logits.cpu(), None, probs.view(-1, V))
