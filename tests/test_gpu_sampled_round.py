"""Speculation rounds as a serving program would run them on the operators together: pages for the round, drafting steps whose
rows enter the cache one by one, verification of all rows at once, the recall index rebuilt from its statistic, probabilities, sampled
acceptance, the next lengths; eagerly and as a captured graph.  Every stage is checked against the formulas on what
the stage before has left."""
import pytest
import torch

import round_ops
from paper_2607_27735_b200 import binding, inputs

pytestmark = pytest.mark.gpu
L, HQ, H, D, PS, K, VOCAB, BUDGET, SINK, RECENT = 2, 8, 2, 128, 16, 4, 1500, 96, 4, 16
PROMPTS = (150, 33, 301)
B, CAP = len(PROMPTS), 384


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Rounds:
    def __init__(self, fmt):
        self.fmt = fmt
        max_pages = CAP // PS
        n_pages = B * max_pages
        shape = (L, n_pages, H, PS, D)
        data = [torch.zeros(shape, dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device="cuda") for _ in range(2)]
        scale = [None, None] if fmt == "bf16" else [torch.zeros(L, n_pages, H, device="cuda") for _ in range(2)]
        self.table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
        self.kv = inputs.KVCache(k=data[0], v=data[1], layer_stride=n_pages * H * PS * D, page_stride=H * PS * D, head_stride=PS * D, slot_stride=D,
                                 n_layers=L, page_size=PS, page_table=self.table, max_pages=max_pages, batch=B, n_q_heads=HQ, n_kv_heads=H,
                                 head_dim=D, n_pages=n_pages, fp8=fmt != "bf16", k_scale=scale[0], v_scale=scale[1])
        self.n_held, self.pool, self.n_free = _i32([0] * B), _i32(list(range(n_pages))[::-1]), _i32([n_pages])
        self.committed = _i32(PROMPTS)
        self.ctx_verify, self.cur_len = _i32([0] * B), torch.zeros(K, B, dtype=torch.int32, device="cuda")
        self.cos_sin = round_ops.cos_sin_table(CAP, D).cuda()
        g = torch.Generator().manual_seed(6)
        self.qw, self.kw = ((torch.rand(L, D, generator=g) + 0.5).to(torch.bfloat16).cuda() for _ in range(2))
        self.ws_p = binding.alloc_workspace(binding.pages_workspace_bytes(), "cuda")
        self.ws_a = binding.alloc_workspace(binding.append_workspace_bytes(self.kv, sum(PROMPTS)), "cuda")
        self.ws_v = binding.alloc_workspace(binding.workspace_bytes(binding.WS_VERIFY, self.kv, K + 1, CAP), "cuda")
        self.ws_d = binding.alloc_workspace(binding.workspace_bytes(binding.WS_DRAFT, self.kv, k_total=BUDGET + K), "cuda")
        rows = B * (K + 1)
        self.cu, self.pos, self.slots = _i32([0] * (B + 1)), _i32([0] * rows), _i32([-1] * rows)
        self.step_pos, self.step_slots = (torch.zeros(K, B, dtype=torch.int32, device="cuda") for _ in range(2))
        bf = dict(dtype=torch.bfloat16, device="cuda")
        # a round's inputs: projections of the drafting steps and of the verification, logits, drafted tokens, numbers
        self.qkv_d, self.qkv_v = torch.zeros(K, L, B, HQ + 2 * H, D, **bf), torch.zeros(L, rows, HQ + 2 * H, D, **bf)
        self.logits, self.temp = torch.zeros(rows, VOCAB, **bf), torch.ones(rows, device="cuda")
        self.q_probs, self.draft = torch.zeros(B, K, VOCAB, device="cuda"), torch.zeros(B, K, dtype=torch.int32, device="cuda")
        self.u = torch.zeros(B, K + 1, device="cuda")
        # and its results
        self.q_d, self.q_v = torch.zeros(K, L, B, HQ, D, **bf), torch.zeros(L, rows, HQ, D, **bf)
        self.out_d, self.lse_d = torch.zeros(K, L, B, HQ, D, device="cuda"), torch.zeros(K, L, B, HQ, device="cuda")
        self.out_v = torch.zeros(L, B, K + 1, HQ, D, device="cuda")
        self.stats = torch.zeros(L, B, H, CAP, device="cuda")
        self.idx, self.n_idx = torch.zeros(L, B, H, BUDGET, dtype=torch.int32, device="cuda"), torch.zeros(L, B, H, dtype=torch.int32, device="cuda")
        self.probs = torch.zeros(rows, VOCAB, device="cuda")
        self.n_acc, self.token = _i32([0] * B), _i32([0] * B)

    def parts(self, qkv):
        return qkv[..., :HQ, :], qkv[..., HQ:HQ + H, :], qkv[..., HQ + H:, :]

    def append(self, qkv, pos, slots, q_out):
        q, k, v = self.parts(qkv)
        binding.spec_qkv_append(self.kv, q, k, v, pos, slots, q_weight=self.qw, k_weight=self.kw, cos_sin=self.cos_sin, q_out=q_out,
                                workspace=self.ws_a)

    def admit(self, qkv):
        """The prompts' rows, and a recall index from a verification of the last of them."""
        _, pos, slots, _ = binding.spec_assign_pages(_i32([0] * B), self.committed, PS, self.table, self.n_held, self.pool, self.n_free,
                                                     max_rows=sum(PROMPTS) + 3, workspace=self.ws_p)
        pos, slots = pos[:sum(PROMPTS)].contiguous(), slots[:sum(PROMPTS)].contiguous()
        q = torch.zeros(L, sum(PROMPTS), HQ, D, dtype=torch.bfloat16, device="cuda")
        self.append(qkv, pos, slots, q)
        last = torch.tensor(PROMPTS).cumsum(0)
        q = torch.stack([q[:, e - K - 1:e] for e in last.tolist()], 1).contiguous()
        binding.spec_verify_attn(self.kv, q, self.committed, CAP, out=self.out_v, stats=self.stats, workspace=self.ws_v, want_lse=False)
        binding.spec_select_recall(self.stats, self.committed, SINK, RECENT, BUDGET, indices=self.idx, n_indices=self.n_idx)
        binding.spec_advance_lengths(self.committed, None, K, self.ctx_verify, self.cur_len, max_len=CAP)

    def round(self):
        binding.spec_assign_pages(self.committed, self.ctx_verify, PS, self.table, self.n_held, self.pool, self.n_free, cu_rows=self.cu,
                                  positions=self.pos, slots=self.slots, workspace=self.ws_p)
        self.step_pos.copy_(self.pos.view(B, K + 1)[:, :K].T)
        self.step_slots.copy_(self.slots.view(B, K + 1)[:, :K].T)
        for j in range(K):
            self.append(self.qkv_d[j], self.step_pos[j], self.step_slots[j], self.q_d[j])
            binding.spec_sparse_draft_attn(self.kv, self.q_d[j], self.idx, self.n_idx, self.committed, self.cur_len[j], K, out=self.out_d[j],
                                           lse=self.lse_d[j], workspace=self.ws_d)
        self.append(self.qkv_v, self.pos, self.slots, self.q_v)
        binding.spec_verify_attn(self.kv, self.q_v.view(L, B, K + 1, HQ, D), self.ctx_verify, CAP, out=self.out_v, stats=self.stats,
                                 workspace=self.ws_v, want_lse=False)
        binding.spec_token_probs(self.logits, self.temp, probs=self.probs)
        binding.spec_accept_sample(self.probs.view(B, K + 1, VOCAB), self.draft, self.u, draft_probs=self.q_probs, n_accepted=self.n_acc,
                                   next_token=self.token)
        binding.spec_advance_lengths(self.committed, self.n_acc, K, self.ctx_verify, self.cur_len, max_len=CAP)
        binding.spec_select_recall(self.stats, self.committed, SINK, RECENT, BUDGET, indices=self.idx, n_indices=self.n_idx)

    def feed(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.qkv_d.copy_(torch.randn(self.qkv_d.shape, generator=g))
        self.qkv_v.copy_(torch.randn(self.qkv_v.shape, generator=g) * 2)  # larger values: pages' scales have to grow
        z = torch.randn(B, K + 1, VOCAB, generator=g) * 3
        self.logits.copy_(z.view(-1, VOCAB))
        y = z[:, :K] + 0.3 * torch.randn(B, K, VOCAB, generator=g)
        self.q_probs.copy_(torch.softmax(y, -1))
        self.draft.copy_((y - (-torch.rand(B, K, VOCAB, generator=g).clamp_min(1e-9).log()).log()).argmax(-1))
        self.u.copy_(torch.rand(B, K + 1, generator=g))
        self.temp.copy_(torch.rand(B * (K + 1), generator=g) * 0.5 + 0.7)

    def values(self):
        """The cache's contents as numbers, [L, pages, H, PS, D] for K and V."""
        if self.fmt == "bf16":
            return self.kv.k.double(), self.kv.v.double()
        return tuple(d.view(torch.float8_e4m3fn).double() * s.double()[..., None, None]
                     for d, s in ((self.kv.k, self.kv.k_scale), (self.kv.v, self.kv.v_scale)))


def attend(r, q, positions, b, last):
    """Reference over positions of sequence b for every layer and head: q [L, n, HQ, D] -> [L, n, HQ, D]."""
    kx, vx = r.values()
    pos = positions.cuda()
    page = r.table[b].long()[pos // PS]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for l in range(L):
        for hq in range(HQ):
            keys, vals = kx[l, page, hq // (HQ // H), pos % PS], vx[l, page, hq // (HQ // H), pos % PS]
            out[l, :, hq] = round_ops.attend(q[l, :, hq], keys, vals, last.cuda())[0]
    return out


def check_rows(r, qkv, pos, slots):
    """The appended rows in the cache."""
    kx, vx = r.values()
    _, k, v = r.parts(qkv)
    for l in range(L):
        want_k = round_ops.norm_rope(k[l].cpu(), r.kw[l].cpu(), 1e-6, r.cos_sin.cpu(), pos.cpu(), False)
        for got, want, scale in ((kx, want_k, r.kv.k_scale), (vx, v[l].double().cpu(), r.kv.v_scale)):
            for i, s in enumerate(slots.tolist()):
                x = got[l, s // PS, :, s % PS].cpu()
                tol = 2.0 ** -8 * want[i].abs() if r.fmt == "bf16" else 2.0 ** -4 * want[i].abs() + 2.0 ** -10 * scale[l, s // PS].cpu()[:, None]
                assert ((x - want[i]).abs() <= tol + 2.0 ** -19 * want[i].abs().amax(-1, keepdim=True)).all()


@pytest.mark.parametrize("fmt", ["page8", "bf16"])
def test_rounds_stage_by_stage(fmt):
    r = Rounds(fmt)
    prompt = (torch.randn(L, sum(PROMPTS), HQ + 2 * H, D, generator=torch.Generator().manual_seed(1))).to(torch.bfloat16).cuda()
    r.admit(prompt)
    # fp32 sums of exact products and probabilities in two 16-bit parts (2^-14 of the largest value), see the kernels' own tests
    near = lambda got, want: bool(((got.double() - want).abs() <= 2.0 ** -12 * float(r.values()[1].abs().max())).all())  # noqa: E731
    for seed in range(4):
        r.feed(seed)
        committed, idx, n_idx = r.committed.clone(), r.idx.clone(), r.n_idx.clone()
        r.round()
        for ws in (r.ws_p, r.ws_a, r.ws_v, r.ws_d):
            assert binding.read_status(ws) == 0
        pos = torch.cat([torch.arange(c, c + K + 1) for c in committed.tolist()])
        assert r.pos.tolist() == pos.tolist() and int(r.slots.min()) >= 0 and len(set(r.slots.tolist())) == B * (K + 1)
        check_rows(r, r.qkv_v, r.pos, r.slots)
        for b in range(B):
            T = int(committed[b]) + K + 1
            q = r.q_v.view(L, B, K + 1, HQ, D)[:, b]
            assert near(r.out_v[:, b], attend(r, q, torch.arange(T), b, T - K - 1 + torch.arange(K + 1)))
        want = round_ops.accept_sample(r.probs.view(B, K + 1, VOCAB).cpu(), r.draft.cpu(), r.u.cpu(), r.q_probs.cpu())
        assert r.n_acc.tolist() == want[0].tolist() and r.token.tolist() == want[1].tolist()
        for row in range(B * (K + 1)):
            p = round_ops.token_probs(r.logits[row].cpu(), float(r.temp[row]))
            assert ((r.probs[row].cpu().double() - p).abs() <= 2e-5 * p + 1e-30).all()
        assert r.committed.tolist() == [c + m + 1 for c, m in zip(committed.tolist(), r.n_acc.tolist())]
        assert (r.n_held * PS >= committed + K + 1).all()


def test_a_drafting_step_reads_what_was_appended_before_it():
    r = Rounds("page8")
    prompt = (torch.randn(L, sum(PROMPTS), HQ + 2 * H, D, generator=torch.Generator().manual_seed(2))).to(torch.bfloat16).cuda()
    r.admit(prompt)
    r.feed(9)
    committed = r.committed.tolist()
    binding.spec_assign_pages(r.committed, r.ctx_verify, PS, r.table, r.n_held, r.pool, r.n_free, cu_rows=r.cu, positions=r.pos, slots=r.slots,
                              workspace=r.ws_p)
    near = lambda got, want: bool(((got.double() - want).abs() <= 2.0 ** -12 * float(r.values()[1].abs().max())).all())  # noqa: E731
    for j in range(K):
        pos, slots = r.pos.view(B, K + 1)[:, j].contiguous(), r.slots.view(B, K + 1)[:, j].contiguous()
        r.append(r.qkv_d[j], pos, slots, r.q_d[j])
        binding.spec_sparse_draft_attn(r.kv, r.q_d[j], r.idx, r.n_idx, r.committed, r.cur_len[j], K, out=r.out_d[j], lse=r.lse_d[j],
                                       workspace=r.ws_d, early_gather=True)  # (with page scales the promise is not made use of)
        for b in range(B):
            for l in range(L):
                for h in range(H):
                    recalled = r.idx[l, b, h, :int(r.n_idx[l, b, h])].long().cpu()
                    keys = torch.cat([recalled, torch.arange(committed[b], committed[b] + j + 1)])
                    want = attend(r, r.q_d[j][:, b][:, None], keys, b, torch.tensor([len(keys)]))
                    g = slice(h * (HQ // H), (h + 1) * (HQ // H))
                    assert near(r.out_d[j, l, b, g], want[l, 0, g])


@pytest.mark.parametrize("fmt", ["page8", "bf16"])
def test_replayed_rounds_are_the_eager_ones(fmt):
    prompt = (torch.randn(L, sum(PROMPTS), HQ + 2 * H, D, generator=torch.Generator().manual_seed(3))).to(torch.bfloat16).cuda()
    eager, replayed = Rounds(fmt), Rounds(fmt)
    for r in (eager, replayed):
        r.admit(prompt)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):  # captured, not run
        replayed.round()
    for seed in range(5):
        for r in (eager, replayed):
            r.feed(100 + seed)
        eager.round()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("pos", "slots", "table", "n_held", "n_free", "n_acc", "token", "committed", "idx", "out_d", "out_v", "stats", "probs", "q_v"):
            assert torch.equal(getattr(eager, name), getattr(replayed, name)), (seed, name)
        assert torch.equal(eager.kv.k, replayed.kv.k) and torch.equal(eager.kv.v, replayed.kv.v)
        if fmt != "bf16":
            assert torch.equal(eager.kv.k_scale, replayed.kv.k_scale)
