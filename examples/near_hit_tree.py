"""Several near hits of the semantic cache at once, and a long prompt's cache kept small.

A lookup for the best few entries may find several just below the threshold.  Their stored answers' next tokens, shared beginnings once, make a
tree of drafts that goes through the model in one pass over the paged key/value cache: each node sees the tokens before the tree and the nodes
above it.  The model's own probabilities say which path stands; its rows are moved to their place and the next pass follows.  Before that the prompt's
cache is cut down to the tokens that its last queries gave most weight, and the latest ones.

    python examples/near_hit_tree.py [e4m3 | i8 | bf16]

The model is the small decoder with random weights of near_hit_drafts.py."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2508_18736_b200 as siso  # noqa: E402
from near_hit_drafts import PAGE, Decoder  # noqa: E402


def tree_of(answers, longest):
    """Lists of tokens as a tree below node 0: (tokens, parents) of the nodes from 1 on, shared beginnings once, parents first."""
    tokens, parents, child = [], [], {}
    for answer in answers:
        at = 0
        for token in answer[:longest]:
            if (at, token) not in child:
                tokens.append(token)
                parents.append(at)
                child[at, token] = len(tokens)
            at = child[at, token]
    return tokens, parents


class TreeDecoder(Decoder):
    """Keeps how many tokens are in the cache and the position of the next one, which eviction lets drift apart."""

    def start(self, prompt, budget=None, recent=8, look=8):
        """Takes the prompt but its last token into the cache; cuts it down to `budget` tokens by what its last `look` queries attend to."""
        n = prompt.numel() - 1
        self.weights, self.seen, self.at = self.kv.new_weights(), 0, 0
        self.last_queries = []
        self.nodes(prompt[:-1], list(range(-1, n - 1)), keep_queries=min(look, n))
        self.seen = self.at = n
        if budget is not None and n > budget:
            look = min(look, n)
            cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, look], [n]))
            for layer, (q, lse) in enumerate(self.last_queries):
                self.kv.add_weights(self.weights, q, lse, cu, lens, self.free[None], look, layer=layer, decay=0.0)
            new_len, _ = self.kv.evict(self.weights, lens, self.free[None], budget, recent)
            self.seen = int(new_len)

    def nodes(self, tokens, parents, keep_queries=0):
        """Probabilities [n, vocab] after each node of a tree below what is in the cache; the nodes' keys and values are left behind it."""
        n, table = tokens.numel(), self.free[None]
        cu, lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [self.seen + n]))
        mask, depth = siso.tree_mask(torch.tensor(parents, dtype=torch.int32, device="cuda"), cu, n)
        where = torch.arange(self.seen, self.seen + n, device="cuda")
        slots = self.free[where // PAGE].long() * PAGE + where % PAGE
        x = self.embed[tokens.long()] + self.place[self.at + depth.long()]
        for layer, (qkv, out, up, down) in enumerate(self.w):
            y = torch.nn.functional.rms_norm(x, x.shape[-1:]) @ qkv
            q, k, v = y.view(n, -1, self.head_dim).split((self.heads, self.kv_heads, self.kv_heads), 1)
            self.kv.write(k, v, slots, layer=layer)
            a, lse = self.kv.tree_attention(q, cu, lens, table, mask, n, layer=layer, want_lse=True)
            if keep_queries:
                self.last_queries.append((q[-keep_queries:], lse[-keep_queries:]))
            x = x + a.reshape(n, -1) @ out
            x = x + torch.nn.functional.silu(torch.nn.functional.rms_norm(x, x.shape[-1:]) @ up) @ down
        self.cu, self.lens, self.table = cu, lens, table
        return torch.softmax(3.0 * (torch.nn.functional.rms_norm(x, x.shape[-1:]) @ self.embed.T).float() / x.shape[-1] ** 0.5, -1)

    def write_answer(self, prompt, length, stored=(), at_once=4, seed=0, budget=None):
        """(tokens [length], passes after the prompt's): sampled, with the stored answers as guesses for the tokens to come."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.start(prompt, budget)
        last, got, passes = int(prompt[-1]), [], 0
        while len(got) < length:
            tokens, parents = tree_of([a[len(got):] for a in stored], at_once)
            tokens = torch.tensor([last] + tokens, dtype=torch.int32, device="cuda")
            parents = [-1] + parents
            p = self.nodes(tokens, parents)
            passes += 1
            u = torch.rand(len(parents) + 1, device="cuda", generator=g)
            out, n, path = siso.verify_tree(p, None, tokens, torch.tensor(parents, dtype=torch.int32, device="cuda"), self.cu, at_once, u[:-1], u[-1:])
            self.kv.keep_path(path, n, self.cu, self.lens, self.table)
            n = int(n)
            got += out[0, :n + 1].tolist()
            last = got[-1]
            self.seen += 1 + n
            self.at += 1 + n
        return torch.tensor(got[:length], device="cuda"), passes


def main(kind="e4m3", length=48, budget=None, verbose=True):
    g = torch.Generator(device="cuda").manual_seed(1)
    model = TreeDecoder(kind=kind)
    unit = lambda x: torch.nn.functional.normalize(x, dim=-1).to(torch.bfloat16)
    # the semantic cache: queries that have been answered, two of them much alike
    prompts = torch.randint(0, 512, (32, 20), device="cuda", generator=g)
    queries = torch.randn((32, 64), device="cuda", generator=g)
    queries[18] = queries[17] + 0.2 * torch.randn(64, device="cuda", generator=g)
    prompts[18] = prompts[17]
    cache = siso.SisoCache(64, 64, "bf16")
    slots = cache.insert(unit(queries)).tolist()
    answers = {slots[i]: model.write_answer(prompts[i], length, seed=i)[0].tolist() for i in (17, 18)}
    # a new query, close to both but not close enough to take an answer
    query, prompt = unit(queries[17:19].mean(0, keepdim=True) + 0.1 * torch.randn((1, 64), device="cuda", generator=g)), prompts[17].clone()
    prompt[2] = (prompt[2] + 1) % 512
    idx, sim, hit = cache.lookup(query, 0.999, k=2)
    near = [i for i, s in zip(idx[0].tolist(), sim[0].tolist()) if s > 0.8 and i in answers]
    alone, passes_alone = model.write_answer(prompt, length, seed=99, budget=budget)
    drafted, passes = model.write_answer(prompt, length, [answers[i] for i in near], seed=99, budget=budget)
    if verbose:
        print(f"near hits {near} at {[round(s, 3) for s in sim[0].tolist()]}, cache of the prompt cut to {budget}")
        print(f"{length} tokens alone in {passes_alone} passes, with the tree of stored answers in {passes}")
    model.kv.check_status()
    cache.close()
    return model, near, passes_alone, passes, drafted


if __name__ == "__main__":
    main(*sys.argv[1:2])
    main(*sys.argv[1:2], budget=12)
