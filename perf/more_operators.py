"""Cases of the operators that serve several near hits at once and keep the paged key/value cache small: the attention of a tree of
drafted tokens over the cache, the verification of the tree, the path that stands moved to its place, the weight that attention gives to
each cached token, and the eviction by it.

Every case can be run two ways on the same inputs: in elementary torch operations (`own` false) and through this package's
entry points (`own` true).  `exact` states the same results in 64 bits."""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
_TOP = {"e4m3": 448.0, "i8": 127.0}
_PAIRS = 32.0 * 4096 * 6145            # (query, key) pairs of all heads in the largest listed case


# ---- cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # two stored answers of one user's near hits, a few tokens of each: nothing but latency
        _tree("tree of one short sequence", 1, 9, 9, 1025, 1025, 32, 8, 128, "bf16", 16),
        # stored answers of several near hits each in a serving batch, odd head group, odd pages, two layers
        _tree("trees of 24 sequences", 24, 17, 63, 517, 6211, 28, 4, 128, "bf16", 48, layers=2),
        # wide trees over long documents in 8 bits, head-major pages
        _tree("wide trees, long documents", 4, 129, 255, 16385, 33333, 32, 8, 128, "i8", 64, layout="head"),
        # one request, a tree of stored answers (no draft probabilities)
        _verify("tree of stored answers", 1, 16, 16, 32000, "f32", False),
        # a serving batch, a drafting model's trees with its probabilities
        _verify("drafted trees of a batch", 32, 9, 25, 128256, "bf16", True),
        # the accepted path of one request enters its place in every layer
        _keep("path of one sequence", 1, 9, 9, 6, 8, 8, 128, "bf16", 16),
        # and those of a batch, 8-bit pages
        _keep("paths of 48 sequences", 48, 17, 63, 12, 16, 8, 128, "i8", 32, layout="head"),
        # one decoding step of a batch adds what its tokens attended to
        _weights("weights of a step", 64, 1, 1, 201, 8190, 32, 8, 128, "e4m3", 32, 0.99),
        # the last queries of prompts say what of them to keep, odd head group
        _weights("weights by the last queries", 4, 31, 33, 4097, 16385, 28, 4, 128, "bf16", 64, 0.0),
        # every query of a long prompt's chunk counts: the largest
        _weights("weights by a whole chunk", 1, 4096, 4096, 8193, 8193, 32, 8, 128, "bf16", 64, 1.0),
        # a long prompt is cut down to its heavy and its latest tokens, four layers
        _evict("a long prompt is cut down", 1, 16385, 16385, 2048, 64, 4, 8, 128, "bf16", 64),
        # a batch that has grown past its budget, 8 bits, small pages
        _evict("a batch is cut down", 24, 1100, 4200, 1000, 33, 2, 4, 64, "e4m3", 16),
    ]


def _tree(name, seqs, q_lo, q_hi, len_lo, len_hi, heads, kv_heads, dim, kind, page, layout="token", window=0, layers=1):
    return {"name": name, "op": "tree", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "len_lo": len_lo, "len_hi": len_hi, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "kind": kind, "page": page, "layout": layout, "window": window, "layers": layers}


def _verify(name, seqs, q_lo, q_hi, vocab, source, probs):
    return {"name": name, "op": "verify", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "vocab": vocab, "source": source, "probs": probs, "path": 8}


def _keep(name, seqs, q_lo, q_hi, path, layers, kv_heads, dim, kind, page, layout="token"):
    return {"name": name, "op": "keep", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "len_lo": q_hi + 40, "len_hi": q_hi + 200, "path": path,
            "layers": layers, "kv_heads": kv_heads, "dim": dim, "kind": kind, "page": page, "layout": layout}


def _weights(name, seqs, q_lo, q_hi, len_lo, len_hi, heads, kv_heads, dim, kind, page, decay, layout="token", layers=1):
    return {"name": name, "op": "weights", "seqs": seqs, "q_lo": q_lo, "q_hi": q_hi, "len_lo": len_lo, "len_hi": len_hi, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "kind": kind, "page": page, "decay": decay, "layout": layout, "layers": layers}


def _evict(name, seqs, len_lo, len_hi, budget, recent, layers, kv_heads, dim, kind, page, layout="token"):
    return {"name": name, "op": "evict", "seqs": seqs, "q_lo": 1, "q_hi": 1, "len_lo": len_lo, "len_hi": len_hi, "budget": budget,
            "recent": recent, "layers": layers, "kv_heads": kv_heads, "dim": dim, "kind": kind, "page": page, "layout": layout}


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["tree", "tree", "verify", "keep", "weights", "weights", "evict"])
    kind, layout, page = rng.choice(["bf16", "e4m3", "i8"]), rng.choice(["token", "head"]), rng.choice([8, 16, 32, 48, 64, 128])
    if op == "verify":
        vocab = _log(rng, 1000, 160000)
        q_hi = _log(rng, 2, 60)
        seqs = max(1, min(_log(rng, 1, 96), 90_000_000 // (vocab * q_hi)))
        c = _verify("", seqs, max(2, int(q_hi * rng.uniform(0.3, 1.0))), q_hi, vocab, rng.choice(["f32", "bf16"]), rng.random() < 0.5)
    elif op == "keep":
        q_hi = _log(rng, 2, 200)
        c = _keep("", _log(rng, 1, 48), max(2, int(q_hi * rng.uniform(0.3, 1.0))), q_hi, min(rng.randint(1, 16), q_hi - 1), rng.randint(1, 16),
                  rng.choice([1, 2, 4, 8]), rng.choice([64, 96, 128]), kind, page, layout)
    elif op == "evict":
        len_hi = _log(rng, 100, 32768)
        kv_heads, layers = rng.choice([1, 2, 4, 8]), rng.randint(1, 4)
        budget = _log(rng, max(8, len_hi // 16), max(9, len_hi // 2))
        seqs = max(1, min(_log(rng, 1, 64), 800_000 // (len_hi * kv_heads * layers)))
        c = _evict("", seqs, max(1, int(len_hi * rng.uniform(0.2, 1.0))), len_hi, budget, _log(rng, 1, max(2, budget // 4)), layers, kv_heads,
                   rng.choice([64, 96, 128]), kind, page, layout)
    else:
        kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8])
        dim = rng.choice([64, 128, 128])
        q_hi = _log(rng, 2, 400) if op == "tree" else _log(rng, 1, 4096)
        len_hi = max(q_hi, _log(rng, 64, 40000))
        seqs = max(1, min(_log(rng, 1, 64), 1_000_000 // (len_hi * kv_heads), int(_PAIRS / (q_hi * kv_heads * group * len_hi))))
        if seqs * q_hi * kv_heads * group * len_hi > _PAIRS:
            return draw(rng)
        args = ("", seqs, max(1, int(q_hi * rng.uniform(0.3, 1.0))), q_hi, max(q_hi, int(len_hi * rng.uniform(0.1, 1.0))), len_hi, kv_heads * group,
                kv_heads, dim, kind, page)
        if op == "tree":
            c = _tree(*args, layout, rng.choice([0, 0, 0, _log(rng, 64, 8192)]), rng.choice([1, 2]))
        else:
            c = _weights(*args, rng.choice([0.0, 0.9, 1.0]), layout, rng.choice([1, 2]))
    c.pop("name")
    return c


def _lengths(case):
    """(new tokens, tokens in all) of each sequence: spread evenly over their ranges, in a mixed order."""
    n = case["seqs"]
    at = [(7919 * (i + 1)) % n / max(1, n - 1) for i in range(n)]
    q = [case["q_lo"] + int(a * (case["q_hi"] - case["q_lo"])) for a in at]
    if case["op"] == "verify":
        q[-1] = case["q_hi"]
        return q, q
    lens = [case["len_lo"] + int(((a * 3.7) % 1.0 if n > 1 else 1.0) * (case["len_hi"] - case["len_lo"])) for a in at]
    lens[0], q[-1] = case["len_hi"], case["q_hi"]
    return q, [max(x, y) for x, y in zip(lens, q)]


def _pairs(case):
    """(query, key) pairs of one head in which the query can see the key, and the keys that some query sees, over all sequences."""
    pairs = seen = 0
    for n, total in zip(*_lengths(case)):
        w = case.get("window") or total
        seen += total - max(0, total - n - w + 1)
        pairs += n * (min(total - n, w) + 5) if case["op"] == "tree" else sum(min(p + 1, w) for p in range(total - n, total))
    return pairs, seen


def work(case):
    size = {"f32": 4, "bf16": 2}
    kept = 2 * case["dim"] if case.get("kind") == "bf16" else case.get("dim", 0) + 1             # bytes of a cache row
    q, lens = _lengths(case)
    if case["op"] == "verify":         # one row for each sequence that the next token is drawn from, at least
        return {"bytes": case["seqs"] * case["vocab"] * size[case["source"]] * (2 if case["probs"] else 1) + 12 * sum(q), "flops": 0}
    if case["op"] == "keep":
        return {"bytes": 2 * 2 * case["layers"] * case["kv_heads"] * kept * sum(min(case["path"], n - 1) for n in q), "flops": 0}
    if case["op"] == "evict":
        rows = sum(min(n, case["budget"]) for n in lens)
        return {"bytes": case["layers"] * case["kv_heads"] * (4 * sum(lens) + rows * (2 * 2 * kept + 4 + 4)), "flops": 0}
    pairs, seen = _pairs(case)
    if case["op"] == "weights":
        return {"bytes": case["kv_heads"] * seen * (kept + 8) + sum(q) * case["heads"] * (2 * case["dim"] + 4), "flops": 2 * pairs * case["heads"] * case["dim"]}
    return {"bytes": case["layers"] * (2 * seen * case["kv_heads"] * kept + 2 * 2 * sum(q) * case["heads"] * case["dim"]),
            "flops": case["layers"] * 4 * pairs * case["heads"] * case["dim"]}


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


def _pool(case, pages, gen):
    """Cache pages [layers, pages, tokens, heads, dim] of either memory order with something in every place, and the exponents
    [layers, pages, heads, tokens] of 8-bit ones."""
    page, heads, dim, kind, layers = case["page"], case["kv_heads"], case["dim"], case["kind"], case["layers"]
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


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    q, lens = _lengths(case)
    n = sum(q)
    s = {"case": case, "max_q": max(q), "cu_q": _i32([sum(q[:i]) for i in range(len(q) + 1)])}
    # which sequence each new token belongs to and its place among them; its parent is any earlier one
    seq = torch.repeat_interleave(torch.arange(len(q), device="cuda"), s["cu_q"].diff().long())
    at = torch.arange(n, device="cuda") - s["cu_q"][seq]
    s["seq"], s["at"] = seq, at
    s["parents"] = torch.where(at > 0, (torch.rand(n, device="cuda", generator=gen) * at).long(), -1).to(torch.int32)
    if op == "verify":
        kind, vocab = _TYPES[case["source"]], case["vocab"]
        logits = torch.randn((n, vocab), device="cuda", generator=gen).mul_(2.2)
        target = torch.softmax(logits, -1)
        if case["probs"]:
            guess = torch.softmax(logits.add_(0.7 * torch.randn((n, vocab), device="cuda", generator=gen)), -1)
            s["draft"] = guess.to(kind)
        else:       # stored answers: mostly tokens that the target might give too
            guess, s["draft"] = target.square(), None
        drawn = torch.multinomial(guess, 24, replacement=True, generator=gen)       # a node's children are draws from its row
        s["tokens"] = drawn[s["cu_q"][seq] + s["parents"].clamp(min=0), at % 24].to(torch.int32)
        s["target"] = target.to(kind)
        s["u_accept"] = torch.rand(n, device="cuda", generator=gen)
        s["u_sample"] = torch.rand(len(q), device="cuda", generator=gen)
        return s
    held = [-(-x // case["page"]) for x in lens]
    more = [-(-min(x, case["budget"]) // case["page"]) for x in lens] if op == "evict" else [0] * len(lens)
    pages = sum(held) + sum(more) + 3
    s["k_pages"], s["k_exp"] = _pool(case, pages, gen)
    s["v_pages"], s["v_exp"] = _pool(case, pages, gen)
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    s["kv_len"] = _i32(lens)

    def table(counts, first):
        t = torch.full((len(counts), max(max(counts), 1)), -1, dtype=torch.int32, device="cuda")
        for i, c in enumerate(counts):
            t[i, :c] = order[first:first + c]
            first += c
        return t

    s["table"] = table(held, 0)
    if op in ("weights", "evict"):
        s["weights"] = torch.rand((case["layers"], pages, case["kv_heads"], case["page"]), device="cuda", generator=gen).pow_(6).mul_(8)
    if op == "evict":       # into new pages, so that the old ones can go back to the pool whole
        s["out_table"] = table(more, sum(held))
    if op in ("tree", "weights"):
        fused = 1.5 * torch.randn((n, (case["heads"] + 2 * case["kv_heads"]) * case["dim"]), device="cuda", generator=gen)
        s["q"] = fused.to(torch.bfloat16)[:, :case["heads"] * case["dim"]].unflatten(1, (case["heads"], case["dim"]))
        s["layer"] = case["layers"] - 1
    if op == "weights":
        x = _scores(s, s["layer"], _seen_causal(s))
        s["lse"] = _rows(s, torch.logsumexp(x, -1)).contiguous()
        del x
    if op == "keep":        # any nodes but the first, ascending; as many of them as the longest path, or fewer
        i = torch.arange(s["max_q"], device="cuda")
        there = (i > 0) & (i < s["cu_q"].diff()[:, None])
        longest = min(case["path"], s["max_q"])
        picked = torch.rand((len(q), s["max_q"]), device="cuda", generator=gen).masked_fill(~there, 2).argsort(-1)[:, :longest]
        n_path = [case["path"] if i % 3 == 0 else (5 * i + 3) % (case["path"] + 1) for i in range(len(q))]
        s["accepted"] = torch.minimum(_i32(n_path), there.sum(-1).to(torch.int32))
        stands = torch.arange(longest, device="cuda") < s["accepted"][:, None]
        path = torch.where(stands, picked, s["max_q"]).sort(-1).values
        s["path"] = torch.nn.functional.pad(path.masked_fill(~stands, -1), (0, case["path"] - longest), value=-1).to(torch.int32)
    if own:
        import paper_2508_18736_b200 as siso
        s["kv"] = siso.PagedKV(s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        import paper_2508_18736_b200 as siso
        if op == "tree":
            mask, depth = siso.tree_mask(s["parents"], s["cu_q"], s["max_q"])
            return [depth] + [s["kv"].tree_attention(s["q"], s["cu_q"], s["kv_len"], s["table"], mask, s["max_q"], layer=layer, window=c["window"])
                              for layer in range(c["layers"])]
        if op == "verify":
            return siso.verify_tree(s["target"], s["draft"], s["tokens"], s["parents"], s["cu_q"], c["path"], s["u_accept"], s["u_sample"])
        if op == "keep":
            new_len = s["kv"].keep_path(s["path"], s["accepted"], s["cu_q"], s["kv_len"], s["table"])
            return _buffers(s, [new_len])
        if op == "weights":
            s["kv"].add_weights(s["weights"], s["q"], s["lse"], s["cu_q"], s["kv_len"], s["table"], s["max_q"], layer=s["layer"], decay=c["decay"])
            return s["weights"]
        new_len, kept = s["kv"].evict(s["weights"], s["kv_len"], s["table"], c["budget"], c["recent"], out_pages=s["out_table"])
        return _buffers(s, [new_len, kept, s["weights"]])
    return {"tree": _plain_tree, "verify": _plain_verify, "keep": _plain_keep, "weights": _plain_weights, "evict": _plain_evict}[op](s)


def _buffers(s, more):
    """The pages too: rows are moved as they are, so 8-bit ones are given as the codes and exponents that were moved."""
    codes = [t if t.dtype == torch.bfloat16 else t.view(torch.int8) for t in (s["k_pages"], s["v_pages"])]
    return more + codes + ([] if s["k_exp"] is None else [s["k_exp"], s["v_exp"]])


def _values(pages, exps, p, t):
    """The values in places (page p, token t), in 32 bits."""
    if exps is None:
        return pages[p, t].float()
    codes = pages.view(torch.int8)[p, t].view(pages.dtype).float()
    return codes * _pow2(exps.transpose(1, 2)[p, t].to(torch.int32) - 127).unsqueeze(-1)


def _places(s):
    """(page, token in it) of every token that the sequences could have [seqs, tokens], and which of them they have."""
    page = s["case"]["page"]
    j = torch.arange(s["table"].shape[1] * page, device="cuda")
    return s["table"].clamp(min=0)[:, j // page], (j % page).expand(s["table"].shape[0], -1), j < s["kv_len"][:, None]


def _cached(s, what, layer):
    """Keys ("k") or values ("v") of all sequences [seqs, tokens, kv heads, dim], zeros behind their ends."""
    p, t, there = _places(s)
    exps = s[what + "_exp"]
    return _values(s[what + "_pages"][layer], None if exps is None else exps[layer], p, t).masked_fill_(~there[:, :, None, None], 0)


def _padded(s, x):
    """Rows x [n, ..] of the new tokens as [seqs, max_q, ..]."""
    i = torch.arange(s["max_q"], device="cuda")
    return x[(s["cu_q"][:-1, None] + i).clamp(max=x.shape[0] - 1)]


def _rows(s, x):
    """The reverse for x [seqs, kv heads, max_q * group, ..]: [n, heads, ..]."""
    x = x.unflatten(2, (s["max_q"], -1))[s["seq"], :, s["at"]]
    return x.flatten(1, 2)


def _scores(s, layer, seen):
    """Scores [seqs, kv heads, max_q * group, tokens] in 32 bits, -infinity where a new token does not see the cached one (seen [seqs, max_q, tokens])."""
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    q = _padded(s, s["q"].float()).unflatten(2, (c["kv_heads"], group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    x = (q @ _cached(s, "k", layer).permute(0, 2, 3, 1)).mul_(c["dim"] ** -0.5)
    return x.masked_fill_(~seen.repeat_interleave(group, 1).unsqueeze(1), -math.inf)


def _positions(s):
    """Tokens before the new ones, the places of all, and which of the padded new tokens there are."""
    there = _places(s)[2]
    n_q = s["cu_q"].diff()
    i = torch.arange(s["max_q"], device="cuda")
    return (s["kv_len"] - n_q)[:, None, None], torch.arange(there.shape[1], device="cuda"), (i < n_q[:, None])[:, :, None]


def _seen_causal(s):
    before, j, real = _positions(s)
    i = torch.arange(s["max_q"], device="cuda")[:, None]
    return (j <= before + i) & real


def _plain_tree(s):
    c = s["case"]
    before, j, real = _positions(s)
    # whether node i lies below node a: some power of (identity + parent of) is not zero there
    m = s["max_q"]
    nodes = torch.arange(m, device="cuda")
    up = ((_padded(s, s["parents"]).unsqueeze(-1) == nodes) | (nodes[:, None] == nodes)).float()
    for _ in range(max(1, (m - 1).bit_length())):
        up = (up @ up).clamp_(max=1)
    depth = up.sum(-1) - 1
    new = (j - before).expand(-1, m, -1)
    seen = torch.where(new < 0, torch.ones((), dtype=torch.bool, device="cuda"), up.bool().gather(2, new.clamp(0, m - 1)) & (new < s["cu_q"].diff()[:, None, None]))
    if c["window"]:
        seen &= (new >= 0) | (j > before + depth.unsqueeze(-1).long() - c["window"])
    seen &= real
    outs = [depth[s["seq"], s["at"]].to(torch.int32)]
    for layer in range(c["layers"]):
        x = _scores(s, layer, seen)
        top = x.amax(-1, keepdim=True)
        x = x.sub_(top.masked_fill(top == -math.inf, 0)).exp_()
        total = x.sum(-1, keepdim=True)
        o = (x @ _cached(s, "v", layer).transpose(1, 2)) / total.masked_fill(total == 0, 1)
        outs.append(_rows(s, o).to(torch.bfloat16))
    return outs


def _weigh(r):
    """Weights of 38 bits, which add up to the same sum in any order."""
    return (r.clamp(0, 1) * 2.0 ** 38).long()


def _plain_verify(s):
    target, draft, longest = s["target"], s["draft"], s["case"]["path"]
    first, n_nodes = s["cu_q"][:-1].long(), s["cu_q"].diff()
    b, m = first.shape[0], s["max_q"]
    row, node = torch.arange(b, device="cuda"), torch.arange(m, device="cuda")
    parents = _padded(s, s["parents"]).masked_fill(node >= n_nodes[:, None], -1)
    at, tried, n = (torch.zeros(b, dtype=torch.long, device="cuda") for _ in range(3))
    r, scale = target[first].float(), torch.ones(b, device="cuda")
    path = torch.full((b, longest + 1), -1, dtype=torch.long, device="cuda")
    out = path.clone()
    for _ in range(m - 1):              # every round tries a later node of each sequence
        child = (parents == at[:, None]) & (node > tried[:, None]) & (n < longest)[:, None]
        more = child.any(-1)
        i = torch.where(more, child.int().argmax(-1), at)
        x = s["tokens"].long()[first + i]
        q_x = torch.ones_like(scale) if draft is None else draft[first + at, x].float()
        p_x = r.gather(-1, x[:, None]).squeeze(-1)
        stands = more & (s["u_accept"][first + i] * (scale * q_x) < p_x)
        falls = more & ~stands
        q = torch.zeros_like(r).scatter_(1, x[:, None], 1) if draft is None else draft[first + at].float()
        less = (r - scale[:, None] * q).clamp_(min=0) if draft is not None else r.masked_fill(q > 0, 0)
        r = torch.where(falls[:, None], less, torch.where(stands[:, None], target[first + i].float(), r))
        scale = torch.where(falls, _weigh(r).sum(-1).float() * 2.0 ** -38, torch.where(stands, torch.ones_like(scale), scale))
        path[row, n] = torch.where(stands, i, path[row, n])
        out[row, n] = torch.where(stands, x, out[row, n])
        n, at, tried = n + stands, torch.where(stands, i, at), torch.where(more, i, tried)
    w = _weigh(r)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, _weigh(target[first + at].float()))
    c = w.cumsum(-1)
    z = (s["u_sample"] * 2.0 ** 24).long()[:, None]
    out[row, n] = ((c << 24) <= z * c[:, -1:]).sum(-1)
    return out.to(torch.int32), n.to(torch.int32), path[:, :longest].to(torch.int32)


def _plain_keep(s):
    c = s["case"]
    before = s["kv_len"] - s["cu_q"].diff()
    t = torch.arange(c["path"], device="cuda")
    b, i = (t < s["accepted"][:, None]).nonzero(as_tuple=True)
    source, goal = before[b] + s["path"][b, i], before[b] + 1 + i
    (p0, t0), (p1, t1) = ((s["table"][b, x // c["page"]].long(), x % c["page"]) for x in (source, goal))
    _plain_move(s, p0, t0, p1, t1)
    return _buffers(s, [before + 1 + s["accepted"]])


def _plain_move(s, p0, t0, p1, t1):
    for pages, exps in ((s["k_pages"], s["k_exp"]), (s["v_pages"], s["v_exp"])):
        x = pages if exps is None else pages.view(torch.int8)
        x[:, p1, t1] = x[:, p0, t0]
        if exps is not None:
            y = exps.transpose(2, 3)
            y[:, p1, t1] = y[:, p0, t0]


def _plain_weights(s):
    c = s["case"]
    before = _positions(s)[0]
    x = _scores(s, s["layer"], _seen_causal(s))
    lse = _padded(s, s["lse"]).unflatten(2, (c["kv_heads"], -1)).permute(0, 2, 1, 3).flatten(2, 3)
    w = x.sub_(lse.unsqueeze(-1)).exp_().sum(2).transpose(1, 2)                             # [seqs, tokens, kv heads]
    p, t, there = _places(s)
    held = s["weights"][s["layer"]].transpose(1, 2)
    old = held[p, t]
    w = torch.where(torch.arange(w.shape[1], device="cuda")[:, None] < before, c["decay"] * old, torch.zeros_like(old)) + w
    held[p[there], t[there]] = w[there]
    return s["weights"]


def _plain_evict(s):
    c = s["case"]
    layers, heads, page, budget, recent = c["layers"], c["kv_heads"], c["page"], c["budget"], c["recent"]
    p, t, there = _places(s)
    b = p.shape[0]
    j = torch.arange(p.shape[1], device="cuda")
    lens = s["kv_len"][:, None]
    w = s["weights"].transpose(2, 3)[:, p, t].permute(0, 1, 3, 2)                           # [layers, seqs, kv heads, tokens]
    w = w.masked_fill((j >= lens - recent)[:, None], math.inf).masked_fill(~there[:, None], -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :budget]
    new_len = s["kv_len"].clamp(max=budget)
    gone = torch.arange(order.shape[-1], device="cuda") >= new_len[:, None, None]
    kept = torch.where(gone, p.shape[1], order).sort(-1).values
    kept = torch.nn.functional.pad(kept, (0, budget - kept.shape[-1]), value=p.shape[1])
    kept = kept.masked_fill(kept == p.shape[1], -1)
    la, se, he, to = (kept >= 0).nonzero(as_tuple=True)
    source = kept[la, se, he, to]
    p0, t0 = s["table"][se, source // page].long(), source % page
    p1, t1 = s["out_table"][se, to // page].long(), to % page
    for pages, exps in ((s["k_pages"], s["k_exp"]), (s["v_pages"], s["v_exp"])):
        x = pages if exps is None else pages.view(torch.int8)
        x[la, p1, t1, he] = x[la, p0, t0, he]
        if exps is not None:
            exps[la, p1, he, t1] = exps[la, p0, he, t0]
    s["weights"][la, p1, he, t1] = s["weights"][la, p0, he, t0]
    return _buffers(s, [new_len, kept.to(torch.int32), s["weights"]])


# ---- the same results in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "verify": _exact_verify, "keep": _exact_keep, "weights": _exact_weights, "evict": _exact_evict}[case["op"]](s)


def _exact_rows(s, what, layer, b, head):
    """Rows of sequence b, in 64 bits."""
    n, page = int(s["kv_len"][b]), s["case"]["page"]
    table = s["table"][b, :-(-n // page)].long()
    codes, exps = s[what + "_pages"][layer, table, :, head], s[what + "_exp"]
    x = codes.double() if exps is None else codes.double() * torch.exp2(exps[layer, table, head].double() - 127).unsqueeze(-1)
    return x.reshape(-1, s["case"]["dim"])[:n]


def _exact_tree(s):
    c = s["case"]
    cu, group = s["cu_q"].tolist(), c["heads"] // c["kv_heads"]
    parents = s["parents"].tolist()
    depth = [0] * cu[-1]
    outs = [torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda") for _ in range(c["layers"])]
    for b, total in enumerate(s["kv_len"].tolist()):
        lo, n = cu[b], cu[b + 1] - cu[b]
        before = total - n
        seen = torch.ones((n, total), dtype=torch.bool)
        seen[:, before:] = False
        for i in range(n):
            a = i
            while a >= 0:
                seen[i, before + a] = True
                a = parents[lo + a]
            depth[lo + i] = int(seen[i, before:].sum()) - 1
            if c["window"]:
                seen[i, :max(0, min(before, before + depth[lo + i] - c["window"] + 1))] = False
        hidden = ~seen.cuda()
        for layer in range(c["layers"]):
            for h in range(c["kv_heads"]):
                k, v = (_exact_rows(s, what, layer, b, h) for what in "kv")
                for g in range(h * group, (h + 1) * group):
                    x = (s["q"][lo:lo + n, g].double() @ k.T) / math.sqrt(c["dim"])
                    outs[layer][lo:lo + n, g] = torch.softmax(x.masked_fill_(hidden, -math.inf), -1) @ v
    return [_i32(depth)] + outs


def _exact_verify(s):
    longest, cu = s["case"]["path"], s["cu_q"].tolist()
    tokens, parents, u = s["tokens"].tolist(), s["parents"].tolist(), s["u_accept"].tolist()
    b = len(cu) - 1
    out, path, taken = (torch.full(x, -1, dtype=torch.int32) for x in ((b, longest + 1), (b, longest), (b,)))
    f32 = lambda x: torch.tensor(x, dtype=torch.float64).float().item()                   # one rounding to 32 bits
    for i in range(b):
        lo, at, n = cu[i], 0, 0
        r, scale = s["target"][lo].double(), 1.0
        for node in range(1, cu[i + 1] - lo):
            if parents[lo + node] != at or n == longest:
                continue
            x = tokens[lo + node]
            q_x = 1.0 if s["draft"] is None else s["draft"][lo + at, x].item()
            if f32(u[lo + node] * f32(scale * q_x)) < r[x].item():
                out[i, n], path[i, n] = x, node
                at, n = node, n + 1
                r, scale = s["target"][lo + at].double(), 1.0
                continue
            if s["draft"] is None:
                r[x] = 0.0
            else:                       # products and differences are rounded to 32 bits, as the definition has them
                r = (r - (scale * s["draft"][lo + at].double()).float().double()).float().double().clamp(min=0)
            scale = f32(float(torch.floor(r.clamp(0, 1) * 2.0 ** 38).long().sum())) * 2.0 ** -38
        w = torch.floor(r.clamp(0, 1) * 2.0 ** 38).long()
        if int(w.sum()) == 0:
            w = torch.floor(s["target"][lo + at].double().clamp(0, 1) * 2.0 ** 38).long()
        c = w.cumsum(0)
        out[i, n] = int((c > (int(s["u_sample"][i].item() * 2 ** 24) * int(c[-1])) // 2 ** 24).int().argmax())
        taken[i] = n
    return out.cuda(), taken.cuda(), path.cuda()


def _exact_keep(s):
    c, page = s["case"], s["case"]["page"]
    before = (s["kv_len"] - s["cu_q"].diff()).tolist()
    slot = lambda b, j: (int(s["table"][b, j // page]), j % page)
    for b, n in enumerate(s["accepted"].tolist()):
        for i in range(n):              # ascending, so no row is read after it was written over
            (p0, t0), (p1, t1) = slot(b, before[b] + int(s["path"][b, i])), slot(b, before[b] + 1 + i)
            for t in _buffers(s, [])[:2]:
                t[:, p1, t1] = t[:, p0, t0].clone()
            for e in _buffers(s, [])[2:]:
                e[:, p1, :, t1] = e[:, p0, :, t0].clone()
    return _buffers(s, [_i32([x + 1 + n for x, n in zip(before, s["accepted"].tolist())])])


def _exact_weights(s):
    c, page = s["case"], s["case"]["page"]
    group, cu = c["heads"] // c["kv_heads"], s["cu_q"].tolist()
    w = s["weights"].double()
    for b, total in enumerate(s["kv_len"].tolist()):
        lo, hi = cu[b], cu[b + 1]
        at = torch.arange(total, device="cuda")
        hidden = at > total - (hi - lo) + torch.arange(hi - lo, device="cuda")[:, None]
        p, t = s["table"][b].long()[at // page], at % page
        for h in range(c["kv_heads"]):
            k = _exact_rows(s, "k", s["layer"], b, h)
            got = torch.where(at < total - (hi - lo), c["decay"] * w[s["layer"], p, h, t], torch.zeros((), dtype=torch.float64, device="cuda"))
            for g in range(h * group, (h + 1) * group):
                x = (s["q"][lo:hi, g].double() @ k.T) / math.sqrt(c["dim"]) - s["lse"][lo:hi, g, None].double()
                got = got + torch.exp(x.masked_fill_(hidden, -math.inf)).sum(0)
            w[s["layer"], p, h, t] = got
    return w


def _exact_evict(s):
    c, page = s["case"], s["case"]["page"]
    budget, recent = c["budget"], c["recent"]
    lens = s["kv_len"].tolist()
    kept = torch.full((c["layers"], len(lens), c["kv_heads"], budget), -1, dtype=torch.int32, device="cuda")
    old = [t.clone() for t in _buffers(s, [s["weights"]])]
    new = _buffers(s, [s["weights"]])
    for b, n in enumerate(lens):
        at = torch.arange(n, device="cuda")
        p, t = s["table"][b].long()[at // page], at % page
        for layer in range(c["layers"]):
            for h in range(c["kv_heads"]):
                w = old[0][layer, p, h, t]
                # a token's rank: how many are heavier, or as heavy and earlier
                rank = torch.argsort(torch.argsort(-w[:max(n - recent, 0)].double(), stable=True), stable=True)
                keep = torch.cat([rank < budget - recent, torch.ones(min(n, recent), dtype=torch.bool, device="cuda")]) if n > budget else at >= 0
                k = keep.nonzero().squeeze(-1)
                kept[layer, b, h, :k.numel()] = k.to(torch.int32)
                to = torch.arange(k.numel(), device="cuda")
                p1, t1 = s["out_table"][b].long()[to // page], to % page
                new[0][layer, p1, h, t1] = old[0][layer, p[k], h, t[k]]
                for x, y in zip(new[1:3], old[1:3]):
                    x[layer, p1, t1, h] = y[layer, p[k], t[k], h]
                for x, y in zip(new[3:], old[3:]):
                    x[layer, p1, h, t1] = y[layer, p[k], h, t[k]]
    return [_i32([min(n, budget) for n in lens]), kept] + new
