"""Plain forms, in 64 bits or whole numbers on the CPU, of the operators around a speculation round: page bookkeeping,
the rows that enter the cache, probabilities and acceptance of sampled drafts.  Written from the formulas; used by the tests."""
import math

import torch

E4M3_MAX = 448.0


def assign_pages(first, new, ps, table, held, pool, n_free, max_rows, n_pages):
    """Lists in, (cu_rows, positions, slots, table, held, pool, n_free) out; ``None`` where the call changes nothing."""
    table, held, pool = [list(r) for r in table], list(held), list(pool)
    cap = len(table[0]) * ps if table else 0
    if any(f < 0 or n < 0 or n > cap or h < 0 or h * ps > cap for f, n, h in zip(first, new, held)) or n_free < 0:
        return None
    need = [-(-n // ps) for n in new]
    rows = sum(max(n - f, 0) for f, n in zip(first, new))
    given = [table[b][j] for b in range(len(new)) for j in range(need[b], held[b])]
    wanted = sum(max(n - h, 0) for n, h in zip(need, held))
    if rows > max_rows or n_free + len(given) > n_pages or wanted > n_free + len(given):
        return None
    for page in given:
        pool[n_free] = page
        n_free += 1
    for b in range(len(new)):
        for j in range(held[b], need[b]):
            n_free -= 1
            table[b][j] = pool[n_free]
    cu, positions, slots = [0], [], []
    for b, (f, n) in enumerate(zip(first, new)):
        for t in range(f, n):
            positions.append(t)
            page = table[b][t // ps]
            slots.append(page * ps + t % ps if 0 <= page < n_pages else -1)
        cu.append(len(slots))
    positions += [0] * (max_rows - len(positions))
    slots += [-1] * (max_rows - len(slots))
    return cu, positions, slots, table, need, pool, n_free


def cos_sin_table(max_pos, rot, base=10000.0):
    """fp32 [max_pos, rot]: cosines, then sines, of the angles of every position (computed in 64 bits)."""
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def norm_rope(x, weight, eps, cos_sin, positions, interleaved):
    """One layer's rows [N, H, D] in 64 bits."""
    x = x.double()
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    if cos_sin is None:
        return x
    rot = cos_sin.shape[1]
    half = rot // 2
    cs = cos_sin.double()[positions.long().clamp(0, cos_sin.shape[0] - 1)][:, None]
    c, s = cs[..., :half], cs[..., half:]
    i = torch.arange(half)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y = x.clone()
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def pow2_scale(amax):
    """The smallest power of two s, at least 2^-64, with amax <= 448 s."""
    e = -64
    while amax > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def e4m3_values(data):
    return data.view(torch.float8_e4m3fn).float()


def requantised(data, ratio):
    """Bytes of e4m3 values times ``ratio`` (fp32 arithmetic, rounded to nearest)."""
    return (e4m3_values(data) * ratio).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def accept_sample(probs, draft, uniform, draft_probs=None, n_draft=None):
    """Whole-number results of CPU tensors, probabilities taken to 64 bits."""
    B, k1, V = probs.shape
    counts, tokens = [], []
    for b in range(B):
        nd = k1 - 1 if n_draft is None else min(max(int(n_draft[b]), 0), k1 - 1)
        m = 0
        while m < nd:
            x = int(draft[b, m])
            if not 0 <= x < V:
                break
            q = 1.0 if draft_probs is None else float(draft_probs[b, m, x])
            if not float(uniform[b, m]) * q < float(probs[b, m, x]):
                break
            m += 1
        p = probs[b, m].double()
        w = p.clone()
        if m < nd and draft_probs is not None:
            w = p - draft_probs[b, m].double()
        elif m < nd and 0 <= int(draft[b, m]) < V:
            w[int(draft[b, m])] -= 1.0
        w = torch.where(w > 0, w, 0.0)
        if not float(w.sum()) > 0:
            w = torch.where(p > 0, p, 0.0)
        counts.append(m)
        if not float(w.sum()) > 0:
            tokens.append(0)
            continue
        c = w.cumsum(0)
        past = (c > float(uniform[b, k1 - 1]) * float(c[-1])) & (w > 0)
        tokens.append(int(past.nonzero()[0]) if bool(past.any()) else int((w > 0).nonzero()[-1]))
    return torch.tensor(counts, dtype=torch.int32), torch.tensor(tokens, dtype=torch.int32)


def token_probs(row, t):
    """One row's probabilities in 64 bits."""
    z = row.double()
    m = float(z.max())
    if m == -math.inf:
        return torch.zeros_like(z)
    if t <= 0:
        p = torch.zeros_like(z)
        p[int((z == m).nonzero()[0])] = 1
        return p
    e = ((z - m) / float(t)).exp()
    return e / e.sum()


def cache_rows(kv, layer, b, h, positions, device):
    """Keys and values (64 bits) of one head at `positions` of a cache with a scale for every page."""
    pos = torch.as_tensor(positions, device=device).long()
    page, slot = pos // kv.page_size, pos % kv.page_size
    phys = kv.page_table[b].to(device).long()[page] if kv.page_table is not None else b * kv.max_pages + page
    at = (layer * kv.layer_stride + phys * kv.page_stride + h * kv.head_stride + slot * kv.slot_stride)[:, None] + \
        torch.arange(kv.head_dim, device=device)
    return tuple(e4m3_values(d.to(device).reshape(-1)[at]).double() * s.to(device)[layer, phys, h].double()[:, None]
                 for d, s in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)))


def attend(q, keys, values, last):
    """Rows q [n, D] over keys [T, D], row i over keys 0..last[i]; (out, lse, probabilities, largest sum of |q k| in bits)."""
    scale = q.shape[-1] ** -0.5
    z = q.double() @ keys.T * scale
    far = float((q.double().abs() @ keys.abs().T).max()) * scale / math.log(2)
    z = torch.where(torch.arange(keys.shape[0], device=q.device)[None] <= last[:, None], z, -math.inf)
    lse = torch.logsumexp(z, -1)
    p = (z - lse[:, None]).exp()
    return p @ values, lse, p, far
