"""Plain 64-bit statements of the paged key/value cache, the attention over it and the draft verification, and the pages that the
tests run on."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
TOP = {"e4m3": 448.0, "i8": 127.0}


def quantised(x, kind):
    """Rows x [.., dim] -> (codes, exponent byte) by the definition, in 64 bits."""
    x = x.double()
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    y = x.masked_fill(bad, 0)
    a = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(a, -127.0)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):          # the smallest e that lets the row's largest value fit
        up = e + step
        e = torch.where(a > TOP[kind] * torch.exp2(up - 1), up, e)
    c = y / torch.exp2(e)
    # one rounding: fp32 holds c exactly (a shifted fp32 or bf16 value) unless it is far below the smallest code
    codes = c.float().to(torch.float8_e4m3fn) if kind == "e4m3" else c.round().to(torch.int8)
    codes = codes.view(torch.int8).masked_fill(bad, 0).view(codes.dtype)
    return codes, torch.where(bad, torch.full_like(e, 128), e).squeeze(-1).add(127).to(torch.uint8)


def values(codes, exps):
    """What codes stand for, in 64 bits."""
    if exps is None:
        return codes.double()
    scale = torch.exp2(exps.double() - 127).masked_fill(exps == 255, math.nan).unsqueeze(-1)
    return codes.float().double() * scale


def make_pages(kind, layers, pages, page, heads, dim, head_major=False, fill=None, seed=0):
    """(k, v, k_exp, v_exp): pages [layers, pages, tokens, heads, dim] of random rows, or all NaN rows with fill = "nan"."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for _ in range(2):
        x = torch.randn((layers, pages, page, heads, dim), device="cuda", generator=g)
        if fill == "nan":
            x.fill_(math.nan)
        codes, exps = (x.to(torch.bfloat16), None) if kind == "bf16" else quantised(x, kind)
        if kind == "e4m3" and fill == "nan":
            codes = torch.full_like(codes.view(torch.int8), 0x7F).view(codes.dtype)          # NaN codes too
        if head_major:
            codes = codes.view(torch.int8 if kind != "bf16" else codes.dtype).transpose(2, 3).contiguous().transpose(2, 3).view(codes.dtype)
        out.append((codes, None if exps is None else exps.transpose(2, 3).contiguous()))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def attention(q, k, v, q_len, causal=True, window=0, scale=None):
    """One sequence: q [n, heads, dim], k, v [len, kv heads, dim] in 64 bits -> out, lse, and what the error bound needs:
    sum p |v| and the largest sum |q| |k| scale."""
    n, heads, dim = q.shape
    total, kv_heads, _ = k.shape
    group = heads // kv_heads
    scale = dim ** -0.5 if scale is None else scale
    q = q.double()
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    x = torch.einsum("qhd,khd->hqk", q, k) * scale
    ab = torch.einsum("qhd,khd->hqk", q.abs(), k.abs()) * abs(scale)
    pos = total - q_len + torch.arange(n, device=q.device)[:, None]
    j = torch.arange(total, device=q.device)
    seen = torch.ones((n, total), dtype=torch.bool, device=q.device)
    if causal:
        seen &= j <= pos
    if window:
        seen &= j > pos - window
    x = x.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(x, -1) if total else torch.full((heads, n), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(x - lse.masked_fill(lse == -math.inf, 0).unsqueeze(-1))
    out = torch.einsum("hqk,khd->qhd", p, v)
    mass = torch.einsum("hqk,khd->qhd", p, v.abs())
    return out, lse.T, mass, float(ab.max()) if ab.numel() else 0.0


def verify(target, draft, tokens, n_drafts, u_accept, u_sample):
    """Row by row, in whole numbers."""
    seqs, n_max = tokens.shape
    out = torch.full((seqs, n_max + 1), -1, dtype=torch.int32)
    taken = torch.zeros(seqs, dtype=torch.int32)
    vocab = target.shape[-1]
    for b in range(seqs):
        limit = n_max if n_drafts is None else min(max(int(n_drafts[b]), 0), n_max)
        n = 0
        while n < limit:
            x = int(tokens[b, n])
            if not 0 <= x < vocab:
                break
            q_x = 1.0 if draft is None else float(draft[b, n, x])
            if not float(torch.tensor(float(u_accept[b, n]) * q_x, dtype=torch.float32)) < float(target[b, n, x]):
                break
            out[b, n] = x
            n += 1
        p = target[b, n].float()
        r = p.clone()
        if n < limit:
            if draft is not None:
                r = p - draft[b, n].float()
            elif 0 <= int(tokens[b, n]) < vocab:
                r[int(tokens[b, n])] -= 1.0
        for row in (r, p):
            w = (torch.nan_to_num(row.double(), nan=0.0).clamp(0, 1) * 2.0 ** 38).floor().long().cpu()
            if int(w.sum()) > 0:
                break
        total = int(w.sum())
        z = min(max(int(float(u_sample[b]) * 2 ** 24), 0), 2 ** 24 - 1)
        if total:
            out[b, n] = int((w.cumsum(0) > z * total // 2 ** 24).int().argmax())
        taken[b] = n
    return out, taken
