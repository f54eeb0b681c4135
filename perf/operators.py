"""Measured workloads of the operators around a speculation round: page bookkeeping, the rows that enter the
cache, attention over a cache with a scale for each page, and acceptance of sampled drafts.

A case is a dict of plain values.  ``listed()`` holds the fixed ones, ``draw(rng)`` gives another of the same ranges,
``prepare`` makes what a serving program has in hand before a call, ``run`` makes one pass (``own``: through the
package's entry points, else in elementary torch operations), ``exact`` gives the results in 64 bits and ``work``
counts the bytes and operations that a pass cannot do without.

Kinds of pass:
  assign   page table, pool and slot map of the next step from the request lengths
  append   norms and rotation of Q and K for every head, K and V written into the cache
  verify   full-context attention of n_q rows per sequence over an 8-bit cache with page scales
  draft    sparse attention of one row per sequence over recalled rows of such a cache
  probs    probabilities of logits rows at a temperature for each row
  accept   drafted tokens accepted or replaced from given random numbers
"""
from __future__ import annotations

import math
import random
import types

import torch

own = False

# Shapes (query heads, KV heads, head_dim) that the repository's configurations and tests use.
_TINY, _G4, _G5 = (8, 2, 64), (32, 8, 128), (40, 8, 128)
_E4M3_MAX = 448.0
_MIN_EXP = -64


def _attn(name, kind, shape, ctx, page, n_q=1, budget=0, tail=0):
    case = dict(kind=kind, q_heads=shape[0], kv_heads=shape[1], dim=shape[2], ctx=",".join(str(t) for t in ctx), page=page,
                n_q=n_q, budget=budget, tail=tail)
    return dict(case, name=name) if name else case


def _append(name, shape, batch, rows, lo, hi, page, cache, layers=1, interleaved=False, norm=True, rot=0):
    case = dict(kind="append", q_heads=shape[0], kv_heads=shape[1], dim=shape[2], batch=batch, rows=rows, lo=lo, hi=hi,
                page=page, cache=cache, layers=layers, interleaved=interleaved, norm=norm, rot=rot or shape[2])
    return dict(case, name=name) if name else case


def listed():
    return [
        # Between two rounds: 64 running conversations, each gets room for eight drafted tokens and one more.
        dict(name="assign_round_batch64", kind="assign", batch=64, page=16, lo=500, hi=30000, mix="round", rows=9),
        # A scheduler's step that admits prompts, goes on with others and has some that ended.
        dict(name="assign_admit_batch256", kind="assign", batch=256, page=16, lo=100, hi=4000, mix="admit", rows=9),
        # One layer of a verification pass at small batch: nine rows each, every launch paid.
        _append("append_round_page8", _G4, 8, 9, 700, 30000, 64, "page8"),
        # Prompts of odd lengths entering a bf16 cache.
        _append("append_prompt_bf16", _G4, 5, 1639, 0, 700, 16, "bf16"),
        # A long prompt entering the cache with page scales, quantised on the way.
        _append("append_prompt_page8", _G5, 2, 8191, 0, 0, 64, "page8"),
        # Single-token decoding: one row per sequence over a long context.
        _attn("verify_token_page8", "verify", _G4, [32771, 30011, 18444, 25000], 64),
        # A ragged verification batch on small pages.
        _attn("verify_ragged_page8", "verify", _G4, [44631, 9107, 60212, 21940, 35555, 65529, 14003, 50876], 16, n_q=7),
        # Drafting steps of the same batch over the recalled rows.
        _attn("draft_ragged_page8", "draft", _G4, [44631, 9107, 60212, 21940, 35555, 65529, 14003, 50876], 16, budget=1024, tail=6),
        # A single sequence's rows after its verification.
        dict(name="probs_round_batch1", kind="probs", rows=9, vocab=128256, dtype="bf16", masked=False),
        # The verification output of 64 sequences.
        dict(name="probs_round_batch64", kind="probs", rows=576, vocab=128256, dtype="bf16", masked=False),
        # Acceptance for one short draft.
        dict(name="accept_batch1", kind="accept", batch=1, k=4, vocab=32000, draft="probs"),
        # Acceptance for 64 sequences with eight drafted tokens each.
        dict(name="accept_batch64", kind="accept", batch=64, k=8, vocab=128256, draft="probs"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["assign", "append", "append", "verify", "verify", "draft", "probs", "accept"])
    if kind == "assign":
        hi = _log_uniform(rng, 300, 20000)
        batch = _log_uniform(rng, 1, min(256, 1200000 // hi))
        return dict(kind=kind, batch=batch, page=rng.choice([8, 16, 32, 64, 128, 24]), lo=rng.randint(1, hi // 2), hi=hi,
                    mix=rng.choice(["round", "admit"]), rows=rng.randint(1, 17))
    if kind in ("probs", "accept"):
        vocab = rng.choice([1003, 32000, 50257, 128256, 151936])
        if kind == "probs":
            return dict(kind=kind, rows=_log_uniform(rng, 1, 480), vocab=vocab, dtype=rng.choice(["bf16", "bf16", "fp32"]),
                        masked=rng.random() < 0.3)
        return dict(kind=kind, batch=_log_uniform(rng, 1, 48), k=rng.randint(1, 8), vocab=vocab,
                    draft=rng.choice(["probs", "probs", "tokens"]))
    shape = rng.choice([_G4, _G4, _G5, (16, 2, 128), (8, 8, 128), _TINY])
    page = rng.choice([16, 32, 64, 128])
    if kind == "append":
        tokens = _log_uniform(rng, 1, 12000)
        batch = _log_uniform(rng, 1, min(64, tokens))
        return _append(None, shape, batch, max(1, tokens // batch), rng.choice([0, 37]), rng.choice([300, 1000, 5000]), page,
                       rng.choice(["bf16", "head8", "page8", "page8"]), layers=rng.choice([1, 1, 2]) if tokens < 2000 else 1,
                       interleaved=rng.random() < 0.3, norm=rng.random() < 0.7, rot=rng.choice([shape[2], shape[2], shape[2] // 2]))
    total = _log_uniform(rng, 1000, 250000)
    batch = _log_uniform(rng, 1, max(1, min(16, total // 700)))
    ctx = [max(200, min(65536, int(total / batch * rng.uniform(0.4, 1.6)))) for _ in range(batch)]
    if kind == "verify":
        n_q = rng.choice([1, 1, 2, 3, 5, 7, 9, 12])
        while n_q * shape[0] // shape[1] > 64:
            n_q -= 1
        return _attn(None, kind, shape, ctx, page, n_q=n_q)
    budget = max(64, min(rng.choice([256, 500, 1024, 2048]), max(ctx) // 2))
    return _attn(None, kind, shape, ctx, page, budget=budget, tail=rng.randint(1, 8))


# ---- inputs ---------------------------------------------------------------------------------


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _ctx(case):
    return [int(t) for t in case["ctx"].split(",")]


def _pages(tokens, page):
    return -(-tokens // page)


def _lengths(case):
    """Lengths of an assign or append case: (first position written, length afterwards, pages held before)."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    first, new, held = [], [], []
    for _ in range(case["batch"]):
        t = rng.randint(case["lo"], case["hi"])
        f, n, h = t, t + case["rows"], _pages(t, case["page"])
        what = rng.random() if case.get("mix") == "admit" else 1.0
        if what < 0.35:
            f, n, h = 0, t, 0  # a prompt comes in
        elif what < 0.5:
            f, n = 0, 0        # a request has ended: its pages go back
        elif case.get("mix"):
            h += rng.choice([0, 0, 1])  # a page that an earlier round took and did not fill
        first.append(f), new.append(n), held.append(h)
    return first, new, held


def _pow2_scale(amax):
    """The smallest power of two s with amax <= 448 s, at least 2^-64."""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, e, _MIN_EXP).clamp(min=_MIN_EXP))


def _cos_sin(max_pos, rot):
    angle = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * \
        500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    return {"assign": _prepare_assign, "append": _prepare_append, "verify": _prepare_attn, "draft": _prepare_attn,
            "probs": _prepare_probs, "accept": _prepare_accept}[case["kind"]](case, seed)


def run(state):
    return state["run"](state)


def _prepare_assign(case, seed):
    first, new, held = _lengths(case)
    ps, B = case["page"], case["batch"]
    need = [_pages(n, ps) for n in new]
    max_pages = max(max(need), max(held)) + 3
    n_pages = max(sum(need), sum(held)) + sum(max(n - h, 0) for n, h in zip(need, held)) + 17
    order = torch.randperm(n_pages, generator=_generator(seed), device="cuda").int()
    # one block of memory: pages in the pool, pages held by each sequence, the table, the pool (a stack)
    start = torch.zeros(1 + B + B * max_pages + n_pages, dtype=torch.int32, device="cuda")
    n_free = n_pages - sum(held)
    start[0] = n_free
    start[1:1 + B] = _i32(held)
    table = start[1 + B:1 + B + B * max_pages].view(B, max_pages)
    h = _i32(held)
    mask = torch.arange(max_pages, device="cuda")[None] < h[:, None]
    table[mask] = order[n_free:]
    start[1 + B + B * max_pages:][:n_free] = order[:n_free]
    rows = sum(max(n - f, 0) for f, n in zip(first, new)) + 5
    arena = start.clone()
    return dict(run=_run_assign, start=start, arena=arena, n_free=arena[:1], n_held=arena[1:1 + B],
                table=arena[1 + B:1 + B + B * max_pages].view(B, max_pages), pool=arena[1 + B + B * max_pages:],
                first=_i32(first), new=_i32(new), page=ps, cu=torch.empty(B + 1, dtype=torch.int32, device="cuda"),
                positions=torch.empty(rows, dtype=torch.int32, device="cuda"),
                slots=torch.empty(rows, dtype=torch.int32, device="cuda"), ws=None)


def _rows_of(case):
    """(positions, slots, pages in the pool, sequence of a row) of an append case, as lists."""
    first, new, _ = _lengths(case)
    ps = case["page"]
    per = [_pages(n, ps) for n in new]
    pages = list(range(sum(per)))
    random.Random(case["batch"] * 31 + ps).shuffle(pages)
    pos, slots, seq, at = [], [], [], 0
    for b, (f, n) in enumerate(zip(first, new)):
        for t in range(f, n):
            pos.append(t)
            slots.append(pages[at + t // ps] * ps + t % ps)
            seq.append(b)
        at += per[b]
    return pos, slots, len(pages)


def _prepare_append(case, seed):
    gen = _generator(seed)
    L, Hq, Hkv, D, ps = case["layers"], case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    pos, slots, n_pages = _rows_of(case)
    N = len(pos)
    # the packed output of a projection, heads of Q, K and V side by side, a spread of its own for every head
    heads = Hq + 2 * Hkv
    qkv = torch.randn(L, N, heads, D, generator=gen, device="cuda")
    qkv *= torch.rand(L, 1, heads, 1, generator=gen, device="cuda") * 2 + 0.25
    qkv = qkv.to(torch.bfloat16)
    weight = (torch.rand(2, L, D, generator=gen, device="cuda") + 0.5).to(torch.bfloat16)
    rot = case["rot"]
    fmt = case["cache"]
    shape = (L, n_pages, Hkv, ps, D)
    if fmt == "bf16":
        k, v = (torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        ks = vs = None
    else:
        k, v = (torch.randn(shape, generator=gen, device="cuda").mul_(40).clamp_(-448, 448).to(torch.float8_e4m3fn)
                .view(torch.uint8) for _ in range(2))
        sc = (L, Hkv) if fmt == "head8" else (L, n_pages, Hkv)
        ks, vs = (torch.ldexp(torch.ones(sc, device="cuda"), torch.randint(-9, -4, sc, generator=gen, device="cuda"))
                  for _ in range(2))
    kv = types.SimpleNamespace(
        k=k, v=v, layer_stride=n_pages * Hkv * ps * D, page_stride=Hkv * ps * D, head_stride=ps * D, slot_stride=D, n_layers=L,
        page_size=ps, page_table=None, max_pages=n_pages, batch=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, sm_scale=0.0,
        n_pages=n_pages, fp8=fmt != "bf16", k_scale=ks, v_scale=vs)
    return dict(run=_run_append, kv=kv, fmt=fmt, q=qkv[:, :, :Hq], k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:],
                positions=_i32(pos), slots=_i32(slots), q_weight=weight[0] if case["norm"] else None,
                k_weight=weight[1] if case["norm"] else None, eps=1e-6, cos_sin=_cos_sin(max(pos) + 1, rot),
                interleaved=case["interleaved"], q_out=torch.empty(L, N, Hq, D, dtype=torch.bfloat16, device="cuda"), ws=None)


def _prepare_attn(case, seed):
    gen = _generator(seed)
    Hq, Hkv, D, ps = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    ctx, n_q, B = _ctx(case), case["n_q"], len(_ctx(case))
    cap = max(ctx) + case["tail"]
    max_pages = _pages(cap, ps)
    n_pages = B * max_pages
    table = torch.randperm(n_pages, generator=gen, device="cuda").int().view(B, max_pages)
    # every page and head has its own spread, its scale the power of two that holds its largest value
    k, v = (torch.empty(1, n_pages, Hkv, ps, D, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty(1, n_pages, Hkv, device="cuda") for _ in range(2))
    step = max(1, (1 << 26) // (Hkv * ps * D))
    for at in range(0, n_pages, step):
        for data, scale in ((k, ks), (v, vs)):
            x = torch.randn(min(step, n_pages - at), Hkv, ps, D, generator=gen, device="cuda")
            x *= (torch.randn(x.shape[0], Hkv, 1, 1, generator=gen, device="cuda") * 0.4).exp_()
            s = _pow2_scale(x.abs().amax((2, 3)))
            data[0, at:at + step] = (x / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            scale[0, at:at + step] = s
    kv = types.SimpleNamespace(
        k=k, v=v, layer_stride=n_pages * Hkv * ps * D, page_stride=Hkv * ps * D, head_stride=ps * D, slot_stride=D, n_layers=1,
        page_size=ps, page_table=table, max_pages=max_pages, batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, sm_scale=0.0,
        n_pages=n_pages, fp8=True, k_scale=ks, v_scale=vs)
    s = dict(kv=kv, max_ctx=max(ctx), ctx_len=_i32(ctx), ws=None)
    if case["kind"] == "verify":
        s.update(run=_run_verify, q=torch.randn(1, B, n_q, Hq, D, generator=gen, device="cuda").to(torch.bfloat16),
                 out=torch.empty(1, B, n_q, Hq, D, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty(1, B, n_q, Hq, device="cuda"),
                 stats=torch.zeros(1, B, Hkv, _pages(max(ctx), 128) * 128, device="cuda"))
        return s
    K = case["budget"]
    idx = torch.full((1, B, Hkv, K), -1, dtype=torch.int32, device="cuda")
    for b, T in enumerate(ctx):
        keep = min(T, K)
        idx[0, b, :, :keep] = torch.rand(Hkv, T, generator=gen, device="cuda").topk(keep).indices.sort(-1).values.int()
    s.update(run=_run_draft, q=torch.randn(1, B, Hq, D, generator=gen, device="cuda").to(torch.bfloat16), idx=idx,
             n_idx=(idx >= 0).sum(-1).int(), cur_len=_i32([T + case["tail"] for T in ctx]), tail=case["tail"],
             out=torch.empty(1, B, Hq, D, dtype=torch.bfloat16, device="cuda"), lse=torch.empty(1, B, Hq, device="cuda"))
    return s


def _logits(gen, rows, vocab):
    """Next-token logits: a background whose spread differs from row to row and a few boosted tokens."""
    x = torch.randn(rows, vocab, generator=gen, device="cuda") * (torch.rand(rows, 1, generator=gen, device="cuda") * 2.8 + 0.7)
    cols = torch.randint(0, vocab, (rows, 4), generator=gen, device="cuda")
    return x.scatter_add_(1, cols, torch.rand(rows, 4, generator=gen, device="cuda") * 14.0)


def _prepare_probs(case, seed):
    gen = _generator(seed)
    R, V = case["rows"], case["vocab"]
    x = _logits(gen, R, V)
    if case["masked"]:  # a sampler's filter has left a few hundred tokens of every row
        keep = x.topk(min(V, 300), dim=-1).values[:, -1:]
        x = torch.where(x >= keep, x, float("-inf"))
    t = torch.rand(R, generator=gen, device="cuda") * 0.9 + 0.4
    t = torch.where(torch.rand(R, generator=gen, device="cuda") < 0.1, 0.0, t)  # some requests decode greedily
    return dict(run=_run_probs, logits=x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32), temperature=t,
                probs=torch.empty(R, V, device="cuda"))


def _prepare_accept(case, seed):
    gen = _generator(seed)
    B, k, V = case["batch"], case["k"], case["vocab"]
    x = _logits(gen, B * (k + 1), V).view(B, k + 1, V)
    p = torch.softmax(x, -1)
    # the drafting pass sees part of the context: its logits are the target's with some noise
    x = x[:, :k] + 0.3 * torch.randn(B, k, V, generator=gen, device="cuda")
    q = torch.softmax(x, -1)
    noise = -torch.log(-torch.log(torch.rand(B, k, V, generator=gen, device="cuda").clamp_(1e-20, 1 - 1e-7)))
    tokens = (x + noise if case["draft"] == "probs" else x).argmax(-1).int()
    return dict(run=_run_accept, p=p, q=q.contiguous() if case["draft"] == "probs" else None, draft=tokens.contiguous(),
                u=torch.rand(B, k + 1, generator=gen, device="cuda"), n=torch.empty(B, dtype=torch.int32, device="cuda"),
                token=torch.empty(B, dtype=torch.int32, device="cuda"))


# ---- one pass -------------------------------------------------------------------------------


def _run_assign(s):
    s["arena"].copy_(s["start"])  # table and pool as the previous step left them
    if own:
        from paper_2607_27735_b200 import binding
        if s["ws"] is None:
            s["ws"] = binding.alloc_workspace(binding.pages_workspace_bytes(), s["arena"].device)
        binding.spec_assign_pages(s["first"], s["new"], s["page"], s["table"], s["n_held"], s["pool"], s["n_free"],
                                  cu_rows=s["cu"], positions=s["positions"], slots=s["slots"], workspace=s["ws"])
        return dict(cu=s["cu"], positions=s["positions"], slots=s["slots"], arena=s["arena"])
    ps, table, pool, first, new = s["page"], s["table"], s["pool"], s["first"], s["new"]
    B, MP = table.shape
    held = s["n_held"].clone()
    need = (new + (ps - 1)) // ps
    take, give = (need - held).clamp(min=0), (held - need).clamp(min=0)
    j = torch.arange(MP, device=table.device, dtype=torch.int32)[None]
    n_free, n_give = s["n_free"].clone(), give.sum()
    goes = (j >= need[:, None]) & (j < held[:, None])
    stack = torch.cat([pool, pool.new_zeros(1)])  # the last place takes what is not kept
    at = n_free + (give.cumsum(0) - give)[:, None] + j - need[:, None]
    stack.scatter_(0, torch.where(goes, at, pool.numel()).view(-1).long(), table.reshape(-1))
    comes = (j >= held[:, None]) & (j < need[:, None])
    at = n_free + n_give - 1 - ((take.cumsum(0) - take)[:, None] + j - held[:, None])
    table.copy_(torch.where(comes, stack[at.clamp(0, pool.numel() - 1).long()], table))
    pool.copy_(stack[:-1])
    s["n_held"].copy_(need)
    s["n_free"].copy_(n_free + n_give - take.sum())
    cu = torch.cat([new.new_zeros(1), (new - first).clamp(min=0).cumsum(0).int()]).int()
    i = torch.arange(s["slots"].numel(), device=table.device, dtype=torch.int32)
    b = torch.searchsorted(cu[1:].contiguous(), i, right=True)
    real = b < B
    b = b.clamp(max=B - 1)
    pos = first[b] + i - cu[b]
    page = table[b, (pos // ps).clamp(0, MP - 1).long()]
    return dict(cu=cu, positions=torch.where(real, pos, 0), slots=torch.where(real, page * ps + pos % ps, -1), arena=s["arena"])


def _norm_rope(x, weight, eps, cos_sin, positions, interleaved):
    """Rows [L, N, H, D] in 32 bits, normed for each head and rotated at their positions."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * weight.float()[:, None, None]
    half = cos_sin.shape[1] // 2
    cs = cos_sin[positions.long()][None, :, None]
    c, n = cs[..., :half], cs[..., half:]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * c - b * n, b * c + a * n
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * c - b * n, b * c + a * n
    return y


def _e4m3(x):
    return x.clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn)


def _put(cache, scale, x, slots, fmt):
    """Rows [L, N, Hkv, D] into a cache [L, pages, Hkv, slots, D] (and the scales of its pages)."""
    L, P, H, ps, D = cache.shape
    page, at = (slots // ps).long(), (slots % ps).long()
    if fmt == "bf16":
        cache[:, page, :, at] = x.to(torch.bfloat16).transpose(0, 1)
        return
    if fmt == "head8":
        cache[:, page, :, at] = _e4m3(x / scale[:, None, :, None]).view(torch.uint8).transpose(0, 1)
        return
    row = page[None, :, None].expand(L, -1, H)
    most = torch.zeros(L, P, H, device=x.device).scatter_reduce(1, row, x.abs().amax(-1), "amax")
    lowest = torch.full((P,), ps, device=x.device, dtype=torch.int64).scatter_reduce(0, page, at, "amin")
    used = page.unique()
    old = torch.where((lowest > 0)[None, :, None] & (scale > 0) & scale.isfinite(), scale, 0.0)[:, used]
    now = torch.maximum(old, _pow2_scale(most[:, used]))
    there = cache[:, used]
    again = _e4m3(there.view(torch.float8_e4m3fn).float() * (old / now)[..., None, None]).view(torch.uint8)
    keep = (torch.arange(ps, device=x.device)[None] < lowest[used][:, None])[None, :, None, :, None] & (now > old)[..., None, None]
    cache[:, used] = torch.where(keep, again, there)
    scale[:, used] = now
    cache[:, page, :, at] = _e4m3(x / scale[:, page][..., None]).view(torch.uint8).transpose(0, 1)


def _run_append(s):
    kv = s["kv"]
    if own:
        from paper_2607_27735_b200 import binding
        if s["ws"] is None:
            s["ws"] = binding.alloc_workspace(binding.append_workspace_bytes(), s["q"].device)
        binding.spec_qkv_append(kv, s["q"], s["k"], s["v"], s["positions"], s["slots"], q_weight=s["q_weight"],
                                k_weight=s["k_weight"], eps=s["eps"], cos_sin=s["cos_sin"], interleaved=s["interleaved"],
                                q_out=s["q_out"], workspace=s["ws"])
        q = s["q_out"]
    else:
        q = _norm_rope(s["q"], s["q_weight"], s["eps"], s["cos_sin"], s["positions"], s["interleaved"]).to(torch.bfloat16)
        k = _norm_rope(s["k"], s["k_weight"], s["eps"], s["cos_sin"], s["positions"], s["interleaved"])
        _put(kv.k, kv.k_scale, k, s["slots"], s["fmt"])
        _put(kv.v, kv.v_scale, s["v"].float(), s["slots"], s["fmt"])
    if s["fmt"] == "bf16":
        return dict(q=q, k=kv.k, v=kv.v)
    held = dict(q=q, k=kv.k.view(torch.float8_e4m3fn), v=kv.v.view(torch.float8_e4m3fn))
    return held if s["fmt"] == "head8" else dict(held, k_scale=kv.k_scale, v_scale=kv.v_scale)


def _values(data, scale, table, pos):
    """Cache rows at positions [B, n] as values [B, Hkv, n, D] in 32 bits."""
    ps = data.shape[3]
    phys = table.gather(1, (pos // ps).clamp(max=table.shape[1] - 1)).long()
    x = data[0][phys, :, pos % ps].view(torch.float8_e4m3fn).float() * scale[0][phys][..., None]
    return x.transpose(1, 2)


def _run_verify(s):
    kv, q, T = s["kv"], s["q"], s["ctx_len"]
    if own:
        from paper_2607_27735_b200 import binding
        if s["ws"] is None:
            s["ws"] = binding.alloc_workspace(binding.workspace_bytes(binding.WS_VERIFY, kv, q.shape[2], s["max_ctx"]), q.device)
        binding.spec_verify_attn(kv, q, T, s["max_ctx"], out=s["out"], lse=s["lse"], stats=s["stats"], workspace=s["ws"],
                                 out_bf16=True)
        return dict(out=s["out"], lse=s["lse"], stats=s["stats"])
    B, n_q, Hq, D = q.shape[1:]
    H, G = kv.n_kv_heads, kv.n_q_heads // kv.n_kv_heads
    pos = torch.arange(s["max_ctx"], device=q.device)[None].expand(B, -1)
    keys = _values(kv.k, kv.k_scale, kv.page_table, pos)
    x = q[0].float().view(B, n_q, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n_q * G, D)
    score = (x @ keys.transpose(2, 3)).mul_(D ** -0.5)
    del keys
    last = (T[:, None] - n_q + torch.arange(n_q, device=q.device)[None]).repeat_interleave(G, 1)  # [B, n_q G]
    score.masked_fill_(pos[:, None, None] > last[:, None, :, None], float("-inf"))
    m = score.amax(-1, keepdim=True)
    score.sub_(m).exp_()
    total = score.sum(-1, keepdim=True)
    score.div_(total)
    out = score @ _values(kv.v, kv.v_scale, kv.page_table, pos)
    out = out.view(B, H, n_q, G, D).permute(0, 2, 1, 3, 4).reshape(1, B, n_q, Hq, D).to(torch.bfloat16)
    lse = (m + total.log()).view(B, H, n_q, G).permute(0, 2, 1, 3).reshape(1, B, n_q, Hq)
    stats = torch.zeros_like(s["stats"])
    stats[0, :, :, :s["max_ctx"]] = score.sum(2)
    return dict(out=out, lse=lse, stats=stats)


def _run_draft(s):
    kv, q = s["kv"], s["q"]
    if own:
        from paper_2607_27735_b200 import binding
        if s["ws"] is None:
            s["ws"] = binding.alloc_workspace(
                binding.workspace_bytes(binding.WS_DRAFT, kv, k_total=s["idx"].shape[-1] + s["tail"]), q.device)
        binding.spec_sparse_draft_attn(kv, q, s["idx"], s["n_idx"], s["ctx_len"], s["cur_len"], s["tail"], out=s["out"],
                                       lse=s["lse"], workspace=s["ws"], out_bf16=True)
        return dict(out=s["out"], lse=s["lse"])
    B, Hq, D = q.shape[1:]
    H, G = kv.n_kv_heads, kv.n_q_heads // kv.n_kv_heads
    tail = s["ctx_len"][:, None, None] + torch.arange(s["tail"], device=q.device)
    pos = torch.cat([s["idx"][0], tail.expand(B, H, -1)], -1).long()  # [B, H, n]
    some, at = pos >= 0, pos.clamp(min=0)
    ps = kv.page_size
    phys = kv.page_table[torch.arange(B, device=q.device)[:, None, None], at // ps].long()
    h = torch.arange(H, device=q.device)[None, :, None]
    keys, values = (d[0][phys, h, at % ps].view(torch.float8_e4m3fn).float() * c[0][phys, h][..., None]
                    for d, c in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)))
    score = (q[0].float().view(B, H, G, D) @ keys.transpose(2, 3)) * D ** -0.5
    score = score.masked_fill(~some[:, :, None], float("-inf"))
    m = score.amax(-1, keepdim=True)
    p = (score - m).exp()
    total = p.sum(-1, keepdim=True)
    out = (p / total) @ values
    return dict(out=out.reshape(1, B, Hq, D).to(torch.bfloat16), lse=(m + total.log()).reshape(1, B, Hq))


def _run_probs(s):
    if own:
        from paper_2607_27735_b200 import binding
        binding.spec_token_probs(s["logits"], s["temperature"], probs=s["probs"])
        return s["probs"]
    z, t = s["logits"].float(), s["temperature"][:, None]
    m = z.amax(-1, keepdim=True)
    e = ((z - m) / torch.where(t > 0, t, 1.0)).exp()
    p = e / e.sum(-1, keepdim=True)
    v = torch.arange(z.shape[1], device=z.device, dtype=torch.int32)[None]
    best = torch.where(z == m, v, z.shape[1]).amin(-1, keepdim=True)
    return torch.where(t > 0, p, (v == best).float())


def _run_accept(s):
    p, q, x, u = s["p"], s["q"], s["draft"], s["u"]
    if own:
        from paper_2607_27735_b200 import binding
        binding.spec_accept_sample(p, x, u, draft_probs=q, n_accepted=s["n"], next_token=s["token"])
        return dict(n_accepted=s["n"], next_token=s["token"])
    B, k1, V = p.shape
    k = k1 - 1
    px = p[:, :k].gather(2, x.long()[..., None])[..., 0].double()
    qx = q.gather(2, x.long()[..., None])[..., 0].double() if q is not None else torch.ones_like(px)
    m = (u[:, :k].double() * qx < px).int().cumprod(1).sum(1)
    b = torch.arange(B, device=p.device)
    w = p[b, m].double()
    if q is not None:
        less = q[b, m.clamp(max=k - 1)].double()
    else:
        less = torch.zeros_like(w).scatter_(1, x[b, m.clamp(max=k - 1)].long()[:, None], 1.0)
    w = torch.where((m < k)[:, None], (w - less).clamp(min=0), w)
    c = w.cumsum(1)
    token = (c <= u[:, k:].double() * c[:, -1:]).sum(1).clamp(max=V - 1)
    return dict(n_accepted=m.int(), next_token=token.int())


# ---- the definition in 64 bits --------------------------------------------------------------


def exact(case, seed):
    return {"assign": lambda *_: None, "append": _exact_append, "verify": _exact_verify, "draft": _exact_draft,
            "probs": _exact_probs, "accept": _exact_accept}[case["kind"]](case, seed)


def _exact_rows(x, weight, s):
    """One layer's rows [N, H, D] in 64 bits, as complex numbers turned by the angle of their position."""
    x = x.double()
    if weight is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt() * weight.double()
    r = s["cos_sin"].shape[1]
    cs = s["cos_sin"].double()[s["positions"].long()]
    turn = torch.complex(cs[:, :r // 2], cs[:, r // 2:])[:, None]
    part = x[..., :r]
    pair = part.unflatten(-1, (r // 2, 2)) if s["interleaved"] else part.unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
    z = z if s["interleaved"] else z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), x[..., r:]], -1)


def _exact_append(case, seed):
    s = _prepare_append(case, seed)
    L, kv, ps = case["layers"], s["kv"], case["page"]
    wq, wk = s["q_weight"], s["k_weight"]
    q = torch.stack([_exact_rows(s["q"][l], None if wq is None else wq[l], s) for l in range(L)])
    k = torch.stack([_exact_rows(s["k"][l], None if wk is None else wk[l], s) for l in range(L)])
    rows = {"k": k, "v": s["v"].double()}
    page, at = (s["slots"] // ps).long(), (s["slots"] % ps).long()
    if s["fmt"] == "bf16":
        got = {}
        for n, x in rows.items():
            c = getattr(kv, n).double()
            for l in range(L):
                c[l][page, :, at] = x[l]
            got[n] = c
        return dict(q=q, **got)
    if s["fmt"] == "head8":
        return dict(q=q, k=None, v=None)
    scales = {}
    for n, x in rows.items():
        c = getattr(kv, n + "_scale").double().clone()
        began = torch.zeros(c.shape[1], dtype=torch.bool, device=c.device)
        began[page[at == 0]] = True
        c[:, began] = 0.0
        need = torch.zeros_like(c)
        for l in range(L):
            need[l].index_reduce_(0, page, x[l].abs().amax(-1), "amax")
        e = torch.ceil(torch.log2(need / _E4M3_MAX)).clamp(min=_MIN_EXP)
        e = torch.where(need > _E4M3_MAX * torch.exp2(e), e + 1, e)  # a logarithm that came out a hair low
        e = torch.where(need <= _E4M3_MAX * torch.exp2(e - 1), e - 1, e)
        touched = torch.zeros_like(began)
        touched[page] = True
        scales[n + "_scale"] = torch.where(touched[None, :, None], torch.maximum(c, torch.exp2(e.clamp(min=_MIN_EXP))), c)
    return dict(q=q, k=None, v=None, **scales)


def _exact_cache(kv, data, scale, b, pos):
    phys = kv.page_table[b].long()[pos // kv.page_size]
    return data[0][phys, :, pos % kv.page_size].view(torch.float8_e4m3fn).double() * scale[0].double()[phys][..., None]


def _exact_verify(case, seed):
    s = _prepare_attn(case, seed)
    kv, n_q = s["kv"], case["n_q"]
    G = kv.n_q_heads // kv.n_kv_heads
    out, lse = s["out"].double(), s["lse"].double()
    stats = torch.zeros_like(s["stats"], dtype=torch.float64)
    for b, T in enumerate(_ctx(case)):
        pos = torch.arange(T, device="cuda")
        keys, values = (_exact_cache(kv, d, c, b, pos) for d, c in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)))
        for hq in range(kv.n_q_heads):
            z = s["q"][0, b, :, hq].double() @ keys[:, hq // G].T / math.sqrt(case["dim"])
            z = torch.where(pos[None] <= T - n_q + torch.arange(n_q, device="cuda")[:, None], z, -math.inf)
            lse[0, b, :, hq] = torch.logsumexp(z, -1)
            p = torch.softmax(z, -1)
            out[0, b, :, hq] = p @ values[:, hq // G]
            stats[0, b, hq // G, :T] += p.sum(0)
    return dict(out=out, lse=lse, stats=stats)


def _exact_draft(case, seed):
    s = _prepare_attn(case, seed)
    kv = s["kv"]
    G = kv.n_q_heads // kv.n_kv_heads
    out, lse = s["out"].double(), s["lse"].double()
    for b, T in enumerate(_ctx(case)):
        for h in range(kv.n_kv_heads):
            n = int(s["n_idx"][0, b, h])
            pos = torch.cat([s["idx"][0, b, h, :n].long(), torch.arange(T, T + case["tail"], device="cuda")])
            keys, values = (_exact_cache(kv, d, c, b, pos)[:, h] for d, c in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)))
            z = s["q"][0, b, h * G:(h + 1) * G].double() @ keys.T / math.sqrt(case["dim"])
            lse[0, b, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
            out[0, b, h * G:(h + 1) * G] = torch.softmax(z, -1) @ values
    return dict(out=out, lse=lse)


def _exact_probs(case, seed):
    s = _prepare_probs(case, seed)
    out = torch.empty(case["rows"], case["vocab"], dtype=torch.float64, device="cuda")
    for r, t in enumerate(s["temperature"].tolist()):
        z = s["logits"][r].double()
        if t > 0:
            out[r] = torch.softmax(z / t, -1)
        else:
            out[r] = 0
            out[r, int((z == z.max()).nonzero()[0, 0])] = 1
    return out


def _exact_accept(case, seed):
    s = _prepare_accept(case, seed)
    n, token = [], []
    for b in range(case["batch"]):
        m, u = 0, s["u"][b].double().tolist()
        while m < case["k"]:
            x = int(s["draft"][b, m])
            q = float(s["q"][b, m, x]) if s["q"] is not None else 1.0
            if not u[m] * q < float(s["p"][b, m, x]):
                break
            m += 1
        w = s["p"][b, m].double()
        if m < case["k"]:
            if s["q"] is not None:
                w = (w - s["q"][b, m].double()).relu()
            else:
                w[int(s["draft"][b, m])] = 0.0  # its probability is at most one
        c = torch.cumsum(w, 0)
        n.append(m)
        token.append(int(torch.searchsorted(c, (u[-1] * c[-1]).view(1), right=True)[0]))
    return dict(n_accepted=_i32(n), next_token=_i32(token))


# ---- what a pass cannot do without ----------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "assign":
        first, new, held = _lengths(case)
        need = [_pages(n, case["page"]) for n in new]
        moved = sum(abs(n - h) for n, h in zip(need, held))
        rows = sum(max(n - f, 0) for f, n in zip(first, new))
        # lengths and held pages in, held pages out, moved pages read and written, position and slot of every row
        return {"bytes": 4.0 * (5 * case["batch"] + 2 * moved + 2 * rows), "flops": 4.0 * rows}
    if kind == "probs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4.0 + (2 if case["dtype"] == "bf16" else 4)), "flops": 4.0 * n}
    if kind == "accept":
        # the row pair of the first rejection for nearly every sequence; the drafted tokens' probabilities
        n = case["batch"] * case["vocab"] * (2 if case["draft"] == "probs" else 1)
        return {"bytes": 4.0 * n + 20.0 * case["batch"] * case["k"], "flops": 3.0 * n}
    Hq, Hkv, D = case["q_heads"], case["kv_heads"], case["dim"]
    if kind == "append":
        first, new, _ = _lengths(case)
        rows, L = sum(b - a for a, b in zip(first, new)), case["layers"]
        places = len({t for a, b in zip(first, new) for t in range(a, b)})  # rows of the table of angles
        n, es = L * rows, 2 if case["cache"] == "bf16" else 1
        return {"bytes": n * D * (2.0 * (Hq + 2 * Hkv) + 2 * Hq + es * 2 * Hkv) + 8.0 * rows + 4.0 * case["rot"] * places,
                "flops": n * 8.0 * (Hq + Hkv) * D}
    ctx = _ctx(case)
    if kind == "verify":
        tokens, R = sum(ctx), case["n_q"]
        pages = sum(_pages(t, case["page"]) for t in ctx)
        return {"bytes": tokens * Hkv * (2.0 * D + 4) + pages * (8.0 * Hkv + 4) + len(ctx) * R * Hq * (4.0 * D + 4),
                "flops": 4.0 * tokens * Hq * R * D}
    rows = sum(min(t, case["budget"]) + case["tail"] for t in ctx)
    return {"bytes": rows * Hkv * (2.0 * D + 12) + len(ctx) * Hq * (4.0 * D + 4), "flops": 4.0 * rows * Hq * D}
