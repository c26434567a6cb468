"""Cases of the operators that carry a cache miss, or a near hit whose stored answer serves as drafted tokens, through the
language model's side: the paged key/value cache quantised as it is written and read back, the attention of a chunk of new
tokens over it, and the verification of drafted tokens.

Every case can be run two ways on the same inputs: in elementary torch operations (`own` false) and through this package's
entry points (`own` true).  `exact` states the same results in 64 bits."""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
_TOP = {"e4m3": 448.0, "i8": 127.0}
_LARGEST = 4.0 * 2048 * 32 * 128 * 33000        # multiplications and additions of the largest listed attention


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one user, one token, a short answer so far: nothing but latency
        _attn("token of one short sequence", 1, 1, 1, 1025, 1025, 32, 8, 128, "bf16", 16),
        # a full decoding batch of unequal lengths over an 8-bit cache
        _attn("token of each of 64 sequences", 64, 1, 1, 201, 8190, 32, 8, 128, "e4m3", 32, layers=2),
        # two very long documents under decoding: few rows, the work is split over the long axis
        _attn("token over a very long cache", 2, 1, 1, 131071, 131071, 16, 2, 128, "i8", 64, layout="head"),
        # stored answers of near hits as drafts: a few tokens for each of a batch, odd head group, odd pages
        _attn("drafts of 24 sequences", 24, 3, 9, 517, 6211, 28, 4, 64, "bf16", 48),
        # prompts of ordinary length that missed, several in one batch
        _attn("prompts of 6 sequences", 6, 129, 903, 903, 2050, 32, 8, 128, "bf16", 64, layout="head"),
        # a prompt's chunk over an 8-bit cache, attention limited to a window
        _attn("chunk in a window, 8 bits", 2, 1000, 1024, 9001, 16385, 32, 8, 128, "e4m3", 64, window=4096),
        # the chunk of a long prompt: the largest
        _attn("chunk over a long cache", 1, 2048, 2048, 33333, 33333, 32, 8, 128, "bf16", 128),
        # the new tokens of one decoding step enter the cache
        _store("store the tokens of a step", 48, 8, 128, "bf16", "e4m3", 16),
        # a long prompt enters the cache, rows that are slices of a fused projection
        _store("store a prompt", 16385, 8, 128, "bf16", "i8", 64),
        # one request, the stored answer's next tokens as drafts (no draft probabilities)
        _verify("drafts from one stored answer", 1, 5, 32000, "f32", False),
        # a serving batch with a drafting model's probabilities
        _verify("drafts of a batch, f32", 64, 4, 128256, "f32", True),
        # a larger batch, probabilities in 16 bits, odd vocabulary
        _verify("drafts of a batch, bf16", 192, 3, 50257, "bf16", True),
    ]


def _attn(name, seqs, q_lo, q_hi, len_lo, len_hi, heads, kv_heads, dim, kind, page, layout="token", window=0, layers=1):
    return {"name": name, "op": "attention", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "len_lo": len_lo, "len_hi": len_hi, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "kind": kind, "page": page, "layout": layout, "window": window, "layers": layers}


def _store(name, tokens, kv_heads, dim, source, kind, page, layout="token"):
    return {"name": name, "op": "store", "tokens": tokens, "kv_heads": kv_heads, "dim": dim, "source": source, "kind": kind, "page": page,
            "layout": layout}


def _verify(name, seqs, drafts, vocab, source, probs):
    return {"name": name, "op": "verify", "seqs": seqs, "drafts": drafts, "vocab": vocab, "source": source, "probs": probs}


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "store", "verify"])
    if kind == "store":
        c = _store("", _log(rng, 1, 16384), rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 96, 128, 256]), rng.choice(["bf16", "f32"]),
                   rng.choice(["e4m3", "i8", "bf16"]), rng.choice([8, 16, 24, 32, 48, 64, 128]), rng.choice(["token", "head"]))
    elif kind == "verify":
        vocab = _log(rng, 1000, 160000)
        c = _verify("", min(_log(rng, 1, 256), 24_000_000 // vocab), _log(rng, 1, 8), vocab, rng.choice(["f32", "bf16"]), rng.random() < 0.6)
    else:
        kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
        dim = rng.choice([64, 128, 128])
        q_hi = _log(rng, 1, 2048)
        q_lo = max(1, int(q_hi * rng.uniform(0.3, 1.0)))
        len_hi = max(q_hi, _log(rng, 32, 65536))
        seqs = max(1, min(_log(rng, 1, 96), 1_500_000 // (len_hi * kv_heads), int(_LARGEST / (4.0 * q_hi * kv_heads * group * dim * len_hi))))
        c = _attn("", seqs, q_lo, q_hi, max(q_hi, int(len_hi * rng.uniform(0.1, 1.0))), len_hi, kv_heads * group, kv_heads, dim,
                  rng.choice(["bf16", "e4m3", "i8"]), rng.choice([8, 16, 32, 48, 64, 128]), rng.choice(["token", "head"]),
                  rng.choice([0, 0, 0, _log(rng, 64, 8192)]), rng.choice([1, 2]))
        if 4.0 * seqs * q_hi * kv_heads * group * dim * len_hi > _LARGEST:
            return draw(rng)
    c.pop("name")
    return c


def _lengths(case):
    """(new tokens, tokens in all) of each sequence: spread evenly over their ranges, in a mixed order."""
    n = case["seqs"]
    at = [(7919 * (i + 1)) % n / max(1, n - 1) for i in range(n)]
    q = [case["q_lo"] + int(a * (case["q_hi"] - case["q_lo"])) for a in at]
    lens = [case["len_lo"] + int(((a * 3.7) % 1.0 if n > 1 else 1.0) * (case["len_hi"] - case["len_lo"])) for a in at]
    lens[0], q[-1] = case["len_hi"], case["q_hi"]
    return q, [max(x, y) for x, y in zip(lens, q)]


def work(case):
    if case["op"] == "store":
        rows = 2 * case["tokens"] * case["kv_heads"]
        size = {"bf16": 2, "f32": 4}
        kept = 2 * case["dim"] if case["kind"] == "bf16" else case["dim"] + 1
        return {"bytes": rows * (case["dim"] * (size[case["source"]] + 2) + kept) + 8 * case["tokens"], "flops": 0}
    if case["op"] == "verify":
        size = {"f32": 4, "bf16": 2}[case["source"]]
        return {"bytes": case["seqs"] * case["vocab"] * size * (2 if case["probs"] else 1), "flops": 0}
    seen = pairs = 0
    q, lens = _lengths(case)
    for n, total in zip(q, lens):
        w = case["window"] or total
        seen += total - max(0, total - n - w + 1)
        pairs += sum(min(p + 1, w) for p in range(total - n, total))
    kept = 2 * case["dim"] if case["kind"] == "bf16" else case["dim"] + 1
    return {"bytes": 2 * seen * case["kv_heads"] * kept + 2 * 2 * sum(q) * case["heads"] * case["dim"], "flops": 4 * pairs * case["heads"] * case["dim"]}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _pow2(n):
    """2^n in 32 bits for whole n in [-127, 127]."""
    return torch.where(n > -127, (n + 127) << 23, torch.full_like(n, 1 << 22)).to(torch.int32).view(torch.float32)


def _quantise(x, kind):
    """Rows of x (32 bits) as 8-bit codes and the smallest power of two that lets the row's largest value fit: (codes, exponent + 127)."""
    mantissa, exponent = torch.frexp(x.abs().amax(-1, keepdim=True))
    top_m, top_e = math.frexp(_TOP[kind])
    e = exponent.to(torch.int32) - top_e + (mantissa > top_m).to(torch.int32)
    e = torch.where(mantissa > 0, e, torch.full_like(e, -127)).clamp(min=-127)
    y = x * _pow2(-e)
    return (y.to(torch.float8_e4m3fn) if kind == "e4m3" else y.round().to(torch.int8)), (e.squeeze(-1) + 127).to(torch.uint8)


def _pool(case, pages, gen, layers=1):
    """Cache pages [layers, pages, tokens, heads, dim] of either memory order with something in every place, and the exponents
    [layers, pages, heads, tokens] of 8-bit ones."""
    page, heads, dim, kind = case["page"], case["kv_heads"], case["dim"], case["kind"]
    token = case["layout"] == "token"
    codes = torch.empty((layers, pages, page, heads, dim) if token else (layers, pages, heads, page, dim), dtype=_TYPES[kind], device="cuda")
    view = codes if token else codes.transpose(2, 3)
    exps = None if kind == "bf16" else torch.empty((layers, pages, heads, page), dtype=torch.uint8, device="cuda")
    for layer in range(layers):
        for at in range(0, pages, 4096):
            n = min(4096, pages - at)
            x = torch.randn((n, page, heads, dim), device="cuda", generator=gen)
            x *= 0.5 + torch.rand((1, 1, heads, dim), device="cuda", generator=gen)
            if exps is None:
                view[layer, at:at + n] = x.to(torch.bfloat16)
            else:
                c, e = _quantise(x, kind)
                view[layer, at:at + n] = c
                exps[layer, at:at + n] = e.transpose(1, 2)
    return view, exps


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"] == "verify":
        b, t, v = case["seqs"], case["drafts"], case["vocab"]
        logits = torch.randn((b, t + 1, v), device="cuda", generator=gen).mul_(2.2)
        target = torch.softmax(logits, -1)
        if case["probs"]:
            draft = torch.softmax(logits[:, :t] + 0.7 * torch.randn((b, t, v), device="cuda", generator=gen), -1)
            tokens = torch.multinomial(draft.reshape(b * t, v), 1, generator=gen).view(b, t)
            s["draft"] = draft.to(_TYPES[case["source"]])
        else:       # a stored answer: mostly tokens that the target might give too
            tokens = torch.multinomial(target[:, :t].reshape(b * t, v).square(), 1, generator=gen).view(b, t)
            s["draft"] = None
        s["target"], s["tokens"] = target.to(_TYPES[case["source"]]), tokens.to(torch.int32)
        s["n_drafts"] = torch.randint(min(1, t), t + 1, (b,), device="cuda", generator=gen, dtype=torch.int32)
        s["u_accept"] = torch.rand((b, t), device="cuda", generator=gen)
        s["u_sample"] = torch.rand((b,), device="cuda", generator=gen)
        return s
    if case["op"] == "store":
        n, heads, dim = case["tokens"], case["kv_heads"], case["dim"]
        pages = -(-n // case["page"]) + 5
        s["k_pages"], s["k_exp"] = _pool(case, pages, gen)
        s["v_pages"], s["v_exp"] = _pool(case, pages, gen)
        fused = torch.randn((n, 6 * heads * dim), device="cuda", generator=gen).to(_TYPES[case["source"]])      # queries, keys, values
        s["k"], s["v"] = (fused[:, i * heads * dim:(i + 1) * heads * dim].view(n, heads, dim) for i in (4, 5))
        order = torch.randperm(pages, device="cuda", generator=gen)
        at = torch.arange(n, device="cuda") + 3
        s["slots"] = order[at // case["page"]] * case["page"] + at % case["page"]
    else:
        q, lens = _lengths(case)
        held = [-(-x // case["page"]) for x in lens]
        pages = sum(held) + 3
        layers = case["layers"]
        s["layer"] = layers - 1
        s["k_pages"], s["k_exp"] = _pool(case, pages, gen, layers)
        s["v_pages"], s["v_exp"] = _pool(case, pages, gen, layers)
        order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
        table = torch.full((len(q), max(held)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(held):
            table[i, :n] = order[at:at + n]
            at += n
        s["table"], s["kv_len"] = table, torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["cu_q"] = torch.tensor([sum(q[:i]) for i in range(len(q) + 1)], dtype=torch.int32, device="cuda")
        s["max_q"] = max(q)
        fused = 1.5 * torch.randn((sum(q), (case["heads"] + 2 * case["kv_heads"]) * case["dim"]), device="cuda", generator=gen)
        s["q"] = fused.to(torch.bfloat16)[:, :case["heads"] * case["dim"]].unflatten(1, (case["heads"], case["dim"]))
    if own:
        import paper_2508_18736_b200 as siso
        s["kv"] = siso.PagedKV(s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2508_18736_b200 as siso
        if op == "store":
            state["kv"].write(state["k"], state["v"], state["slots"])
            return state["kv"].read(state["slots"])
        if op == "verify":
            return siso.verify_drafts(state["target"], state["draft"], state["tokens"], state["n_drafts"], state["u_accept"], state["u_sample"])
        return state["kv"].attention(state["q"], state["cu_q"], state["kv_len"], state["table"], state["max_q"], layer=state["layer"],
                                     window=state["case"]["window"])
    return _plain_store(state) if op == "store" else _plain_verify(state) if op == "verify" else _plain_attention(state)


def _plain_store(s):
    page, kind = s["case"]["page"], s["case"]["kind"]
    p, t = s["slots"] // page, s["slots"] % page
    if kind == "bf16":
        s["k_pages"][0, p, t] = s["k"].to(torch.bfloat16)
        s["v_pages"][0, p, t] = s["v"].to(torch.bfloat16)
        return s["k_pages"][0, p, t], s["v_pages"][0, p, t]
    k, ke = _quantise(s["k"].float(), kind)
    v, ve = _quantise(s["v"].float(), kind)
    s["k_pages"][0].view(torch.int8)[p, t], s["v_pages"][0].view(torch.int8)[p, t] = k.view(torch.int8), v.view(torch.int8)
    s["k_exp"][0].transpose(1, 2)[p, t], s["v_exp"][0].transpose(1, 2)[p, t] = ke, ve
    return _plain_read(s["k_pages"][0], s["k_exp"][0], p, t).to(torch.bfloat16), _plain_read(s["v_pages"][0], s["v_exp"][0], p, t).to(torch.bfloat16)


def _plain_read(pages, exps, p, t):
    """The values in places (page p, token t), in 32 bits."""
    if exps is None:
        return pages[p, t].float()
    codes = pages.view(torch.int8)[p, t].view(pages.dtype).float()
    return codes * _pow2(exps.transpose(1, 2)[p, t].to(torch.int32) - 127).unsqueeze(-1)


def _plain_attention(s):
    c = s["case"]
    b, hk, d, group = c["seqs"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    q_len = s["cu_q"][1:] - s["cu_q"][:-1]
    i = torch.arange(s["max_q"], device="cuda")
    q = s["q"].float()[(s["cu_q"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1)].view(b, -1, hk, group, d)     # padded to max_q tokens
    j = torch.arange(s["table"].shape[1] * c["page"], device="cuda")
    p, t = s["table"].clamp(min=0)[:, j // c["page"]], (j % c["page"]).expand(b, -1)
    in_use = j < s["kv_len"][:, None]
    pick = [None if e is None else e[s["layer"]] for e in (s["k_exp"], s["v_exp"])]
    k = _plain_read(s["k_pages"][s["layer"]], pick[0], p, t).masked_fill_(~in_use[:, :, None, None], 0)
    v = _plain_read(s["v_pages"][s["layer"]], pick[1], p, t).masked_fill_(~in_use[:, :, None, None], 0)
    pos = (s["kv_len"] - q_len)[:, None] + i
    seen = in_use[:, None] & (j <= pos[:, :, None])
    if c["window"]:
        seen &= j > pos[:, :, None] - c["window"]
    seen = seen.unsqueeze(2).expand(-1, -1, group, -1).reshape(b, 1, s["max_q"] * group, -1)
    x = q.permute(0, 2, 1, 3, 4).reshape(b, hk, -1, d) @ k.permute(0, 2, 3, 1)
    x = x.mul_(d ** -0.5).masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(m.masked_fill(m == -math.inf, 0)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ v.transpose(1, 2)) / total.masked_fill(total == 0, 1)
    o = o.view(b, hk, -1, group, d).permute(0, 2, 1, 3, 4).reshape(b * s["max_q"], c["heads"], d)
    row = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(s["cu_q"], row, right=True) - 1
    return o[seq * s["max_q"] + row - s["cu_q"][seq]].to(torch.bfloat16)


def _plain_verify(s):
    target, tokens = s["target"], s["tokens"].long()
    b, t = tokens.shape
    at = tokens.unsqueeze(-1)
    p_x = target[:, :t].gather(-1, at).squeeze(-1).float()
    q_x = torch.ones_like(p_x) if s["draft"] is None else s["draft"].gather(-1, at).squeeze(-1).float()
    i = torch.arange(t + 1, device="cuda")
    accept = (s["u_accept"] * q_x < p_x) & (i[:t] < s["n_drafts"][:, None])
    n = accept.int().cumprod(1).sum(1)
    row = torch.arange(b, device="cuda")
    p_n = target[row, n].float()
    last = n.clamp(max=t - 1)
    q_n = torch.nn.functional.one_hot(tokens[row, last], target.shape[-1]).float() if s["draft"] is None else s["draft"][row, last].float()
    q_n = q_n * (n < s["n_drafts"])[:, None]                      # nothing is taken off where every draft stands
    w = ((p_n - q_n).clamp(0, 1) * 2.0 ** 38).long()
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, (p_n.clamp(0, 1) * 2.0 ** 38).long())
    c = w.cumsum(-1)
    z = (s["u_sample"] * 2.0 ** 24).long()[:, None]
    drawn = ((c << 24) <= z * c[:, -1:]).sum(-1)
    out = torch.cat([tokens, tokens[:, :1]], 1).masked_fill(i > n[:, None], -1)
    out = torch.where(i == n[:, None], drawn[:, None], out)
    return out.to(torch.int32), n.to(torch.int32)


# ---- the same results in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "store":
        return _exact_rows(s["k"], case["kind"]), _exact_rows(s["v"], case["kind"])
    if case["op"] == "verify":
        return _exact_verify(s)
    page, group = case["page"], case["heads"] // case["kv_heads"]
    cu, lens = s["cu_q"].tolist(), s["kv_len"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, total in enumerate(lens):
        table = s["table"][b, :-(-total // page)].long()
        q = s["q"][cu[b]:cu[b + 1]].double()
        at = torch.arange(total, device="cuda")
        pos = total - q.shape[0] + torch.arange(q.shape[0], device="cuda")[:, None]
        hidden = (at > pos) | (at <= pos - (case["window"] or total + 1))
        for h in range(case["kv_heads"]):
            k, v = (_exact_values(p[s["layer"], table, :, h], e if e is None else e[s["layer"], table, h]).reshape(-1, case["dim"])[:total]
                    for p, e in ((s["k_pages"], s["k_exp"]), (s["v_pages"], s["v_exp"])))
            for g in range(h * group, (h + 1) * group):
                x = (q[:, g] @ k.T) / math.sqrt(case["dim"])
                x[hidden] = -math.inf
                out[cu[b]:cu[b + 1], g] = torch.softmax(x, -1) @ v
    return out


def _exact_values(codes, exps):
    return codes.double() if exps is None else codes.double() * torch.exp2(exps.double() - 127).unsqueeze(-1)


def _exact_rows(x, kind):
    """What a row reads back as: the nearest values that its type holds, in units of the row's power of two."""
    x = x.double()
    if kind == "bf16":
        return x.to(torch.bfloat16).double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / _TOP[kind])).clamp(min=-127)
    e = torch.where(top <= _TOP[kind] * torch.exp2(e - 1), e - 1, e)
    e = torch.where(top > _TOP[kind] * torch.exp2(e), e + 1, e)
    y = x / torch.exp2(e)
    if kind == "e4m3":      # steps of 2^-9 up to 2^-6, then an eighth of the value's power of two
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        y = torch.round(y / step) * step
    else:
        y = torch.round(y)
    return y * torch.exp2(e)


def _exact_verify(s):
    out = torch.full((s["tokens"].shape[0], s["tokens"].shape[1] + 1), -1, dtype=torch.int32)
    taken = torch.zeros(s["tokens"].shape[0], dtype=torch.int32)
    tokens, limits, u = s["tokens"].tolist(), s["n_drafts"].tolist(), s["u_accept"].tolist()
    for b, drafts in enumerate(tokens):
        n = 0
        while n < limits[b]:
            x = drafts[n]
            q_x = 1.0 if s["draft"] is None else s["draft"][b, n, x].item()
            if not torch.tensor(u[b][n] * q_x, dtype=torch.float32).item() < s["target"][b, n, x].item():
                break
            out[b, n] = x
            n += 1
        p = s["target"][b, n].double()
        r = p.clone()
        if n < limits[b]:
            if s["draft"] is None:
                r[drafts[n]] -= 1
            else:
                r -= s["draft"][b, n].double()
        r = r.float().double().clamp(0, 1)          # the difference is taken in 32 bits
        w = torch.floor((r if r.max() >= 2.0 ** -38 else p.clamp(0, 1)) * 2.0 ** 38).long()
        c = w.cumsum(0)
        z = int(s["u_sample"][b].item() * 2 ** 24)
        out[b, n] = int((c > (z * int(c[-1])) // 2 ** 24).int().argmax())
        taken[b] = n
    return out.cuda(), taken.cuda()
