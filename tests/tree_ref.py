"""Plain 64-bit statements of the trees of drafts (ancestors, attention, verification, the accepted path), of the weights that attention gives and of
the eviction by them."""
import math

import torch


def ancestors(parents):
    """parents of one sequence (list) -> bool [n, n]: node j is i's own or above it, and how many are above."""
    n = len(parents)
    up = torch.zeros((n, n), dtype=torch.bool)
    for i in range(n):
        a = i
        while True:
            up[i, a] = True
            if not 0 <= parents[a] < a:
                break
            a = parents[a]
    return up, up.sum(-1) - 1


def words_of(rows, words):
    """bool [n, m] -> int32 [n, words]."""
    n, m = rows.shape
    bits = torch.zeros((n, words * 32), dtype=torch.int64)
    bits[:, :min(m, words * 32)] = rows[:, :words * 32].long().cpu()
    w = (bits.view(n, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def seen_of(rows, total, window):
    """rows bool [n, n]: the new tokens that each new token sees -> bool [n, total] over all tokens."""
    n = rows.shape[0]
    before = total - n
    seen = torch.ones((n, total), dtype=torch.bool)
    for i in range(n):
        if window:
            p = before + max(int(rows[i].sum()) - 1, 0)
            seen[i, :max(0, min(max(before, 0), p - window + 1))] = False
        for j in range(max(before, 0), total):
            seen[i, j] = rows[i, j - before]
    return seen


def attention(q, k, v, seen, scale=None):
    """q [n, heads, dim], k, v [total, kv heads, dim] in 64 bits, seen [n, total]: as paged_ref.attention."""
    n, heads, dim = q.shape
    total, kv_heads, _ = k.shape
    group = heads // kv_heads
    scale = dim ** -0.5 if scale is None else scale
    q, seen = q.double(), seen.to(q.device)
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    x = torch.einsum("qhd,khd->hqk", q, k) * scale
    ab = torch.einsum("qhd,khd->hqk", q.abs(), k.abs()) * abs(scale)
    x = x.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(x, -1) if total else torch.full((heads, n), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(x - lse.masked_fill(lse == -math.inf, 0).unsqueeze(-1))
    return torch.einsum("hqk,khd->qhd", p, v), lse.T, torch.einsum("hqk,khd->qhd", p, v.abs()), float(ab.max()) if ab.numel() else 0.0


def f32(x):
    return torch.tensor(x, dtype=torch.float64).float().item()


def draw(r, p, u):
    """The next token from the residual r, or from p where that is empty; -1 where both are."""
    for row in (r, p):
        w = (torch.nan_to_num(row.double(), nan=0.0).clamp(0, 1) * 2.0 ** 38).floor().long().cpu()
        if int(w.sum()) > 0:
            z = min(max(int(float(u) * 2 ** 24), 0), 2 ** 24 - 1)
            return int((w.cumsum(0) > z * int(w.sum()) // 2 ** 24).int().argmax())
    return -1


def verify_tree(target, draft, tokens, parents, cu, max_path, u_accept, u_sample):
    seqs, vocab = len(cu) - 1, target.shape[-1]
    out = torch.full((seqs, max_path + 1), -1, dtype=torch.int32)
    path = torch.full((seqs, max_path), -1, dtype=torch.int32)
    taken = torch.zeros(seqs, dtype=torch.int32)
    target = target.cpu().double()
    draft = None if draft is None else draft.cpu().double()
    tokens, parents, u_accept = tokens.tolist(), parents.tolist(), u_accept.tolist()
    for b in range(seqs):
        lo, hi = cu[b], cu[b + 1]
        if hi <= lo:
            continue
        at, n = 0, 0
        r, s = target[lo].clone(), 1.0
        for c in range(1, hi - lo):
            if parents[lo + c] != at or n == max_path:
                continue
            x = tokens[lo + c]
            real = 0 <= x < vocab
            if real:
                q_x = 1.0 if draft is None else float(draft[lo + at, x])
                if f32(u_accept[lo + c] * f32(s * q_x)) < float(r[x]):
                    out[b, n], path[b, n] = x, c
                    at, n = c, n + 1
                    r, s = target[lo + at].clone(), 1.0
                    continue
            if draft is None:
                if real:
                    r[x] = 0.0
            else:
                r = (r - (s * draft[lo + at]).float().double()).float().double()
                r = torch.nan_to_num(r, nan=0.0).clamp(min=0)
            w = (torch.nan_to_num(r, nan=0.0).clamp(0, 1) * 2.0 ** 38).floor().long()
            s = f32(float(w.sum())) * 2.0 ** -38
        out[b, n] = draw(r, target[lo + at], u_sample[b])
        taken[b] = n
    return out, taken, path


def weights(q, k, lse, causal=True, scale=None):
    """Sums over the rows of exp(scale q k - lse) [total, kv heads] in 64 bits, and the largest |score| and sum |q||k| scale."""
    n, heads, dim = q.shape
    total, kv_heads, _ = k.shape
    scale = dim ** -0.5 if scale is None else scale
    k = k.repeat_interleave(heads // kv_heads, 1)
    x = torch.einsum("qhd,khd->hqk", q.double(), k) * scale
    ab = torch.einsum("qhd,khd->hqk", q.double().abs(), k.abs()) * abs(scale)
    top = float(x.abs().max()) if x.numel() else 0.0
    x = x - lse.double().T.unsqueeze(-1)
    if causal:
        pos = total - n + torch.arange(n, device=q.device)[:, None]
        x = x.masked_fill(torch.arange(total, device=q.device) > pos, -math.inf)
    p = torch.where(lse.T.unsqueeze(-1) == -math.inf, 0.0, torch.exp(x))
    return p.sum(1).view(kv_heads, -1, total).sum(1).T, top, float(ab.max()) if ab.numel() else 0.0


def kept(w, budget, recent):
    """w [n] of one layer, sequence and head -> the places that stay, ascending."""
    n = w.numel()
    if n <= budget:
        return list(range(n))
    order = sorted(range(n - recent), key=lambda j: (-(w[j].item() if w[j] == w[j] else -math.inf), bool(w[j] != w[j]), j))
    return sorted(order[:budget - recent]) + list(range(n - recent, n))
