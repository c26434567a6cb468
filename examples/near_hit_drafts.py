"""A near hit of the semantic cache as drafts for the language model.

A query is looked up in the semantic cache.  Above the threshold the stored answer is the answer.  Below it, but near, the stored
answer's tokens are drafts: a few at a time they go through the model as one chunk over the paged key/value cache, and the model's
own probabilities say how many of them stand.  The answer is distributed as if the model had written it alone; it takes fewer passes.

    python examples/near_hit_drafts.py [e4m3 | i8 | bf16]

The model is a small decoder with random weights (no checkpoint is needed); its matrix products are torch's."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2508_18736_b200 as siso  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
PAGE = 16


class Decoder:
    """Random weights; keys and values of all layers live in a paged cache."""

    def __init__(self, vocab=512, dim=256, heads=8, kv_heads=2, head_dim=64, layers=2, kind="e4m3", pages=64, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim, self.layers = heads, kv_heads, head_dim, layers
        wide = (heads + 2 * kv_heads) * head_dim
        draw = lambda *s: torch.randn(s, device="cuda", generator=g).mul_(s[0] ** -0.5).to(torch.bfloat16)
        self.embed = torch.randn((vocab, dim), device="cuda", generator=g).to(torch.bfloat16)
        self.place = torch.randn((PAGE * pages, dim), device="cuda", generator=g).mul_(0.3).to(torch.bfloat16)
        self.w = [(draw(dim, wide), draw(heads * head_dim, dim), draw(dim, 4 * dim), draw(4 * dim, dim)) for _ in range(layers)]
        self.kv = siso.PagedKV.allocate(layers, pages, PAGE, kv_heads, head_dim, TYPES[kind])
        self.free = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)

    def probabilities(self, tokens, seen, attend=None):
        """Probabilities [n, vocab] after each of `tokens` [n], which follow `seen` tokens that are in the cache already."""
        n = tokens.numel()
        table = self.free[None]
        pos = torch.arange(seen, seen + n, device="cuda")
        slots = self.free[pos // PAGE].long() * PAGE + pos % PAGE
        cu_q, kv_len = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [seen + n]))
        x = self.embed[tokens.long()] + self.place[pos]
        for layer, (qkv, out, up, down) in enumerate(self.w):
            y = torch.nn.functional.rms_norm(x, x.shape[-1:]) @ qkv
            y = y.view(n, self.heads + 2 * self.kv_heads, self.head_dim)
            q, k, v = y.split((self.heads, self.kv_heads, self.kv_heads), 1)
            if attend is not None:
                a = attend(layer, q, k, v)
            else:
                self.kv.write(k, v, slots, layer=layer)
                a = self.kv.attention(q, cu_q, kv_len, table, n, layer=layer)
            x = x + a.reshape(n, -1) @ out
            y = torch.nn.functional.rms_norm(x, x.shape[-1:]) @ up
            x = x + torch.nn.functional.silu(y) @ down
        return torch.softmax(3.0 * (torch.nn.functional.rms_norm(x, x.shape[-1:]) @ self.embed.T).float() / x.shape[-1] ** 0.5, -1)

    def answer(self, prompt, length, drafts=None, at_once=4, seed=0):
        """(tokens [length], passes through the model): sampled, with `drafts` [..] as guesses for the tokens to come."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        seen, last, got, passes = 0, prompt, [], 0
        while len(got) < length:
            guess = drafts[len(got):len(got) + at_once] if drafts is not None else prompt[:0]
            chunk = torch.cat([last, guess])
            p = self.probabilities(chunk, seen)[-1 - guess.numel():]
            passes += 1
            u = torch.rand(guess.numel() + 1, device="cuda", generator=g)
            out, n = siso.verify_drafts(p[None].contiguous(), None, guess[None].to(torch.int32), None, u[None, :-1].contiguous(), u[-1:])
            n = int(n)
            got += out[0, :n + 1].tolist()
            seen += last.numel() + n            # rejected drafts stay in the pages, beyond what counts; the next chunk overwrites them
            last = out[0, n:n + 1].to(prompt.dtype)
        return torch.tensor(got[:length], device="cuda"), passes


def main(kind="e4m3", length=48, verbose=True):
    g = torch.Generator(device="cuda").manual_seed(1)
    model = Decoder(kind=kind)
    unit = lambda x: torch.nn.functional.normalize(x, dim=-1).to(torch.bfloat16)
    # the semantic cache: queries that have been answered, and their answers
    prompts = torch.randint(0, 512, (32, 20), device="cuda", generator=g)
    queries = torch.randn((32, 64), device="cuda", generator=g)
    cache = siso.SisoCache(64, 64, "bf16")
    slots = cache.insert(unit(queries)).tolist()
    answers = {slots[i]: model.answer(prompts[i], length, seed=i)[0] for i in (3, 17)}
    # a new query, close to number 17 but not close enough to take its answer
    query, prompt = unit(queries[17:18] + 0.06 * torch.randn((1, 64), device="cuda", generator=g) * queries.norm(dim=-1).mean()), prompts[17].clone()
    prompt[2] = (prompt[2] + 1) % 512
    idx, sim, hit = cache.lookup(query, 0.97)
    near = not bool(hit) and float(sim) > 0.8
    alone, passes_alone = model.answer(prompt, length, seed=99)
    drafted, passes = model.answer(prompt, length, answers[int(idx)] if near else None, seed=99)
    if verbose:
        print(f"best entry {int(idx)} at {float(sim):.3f}: {'hit' if bool(hit) else 'near hit' if near else 'miss'}")
        print(f"{length} tokens alone in {passes_alone} passes, with the stored answer as drafts in {passes}")
    model.kv.check_status()
    cache.close()
    return model, near, passes_alone, passes, drafted


if __name__ == "__main__":
    main(*sys.argv[1:2])
