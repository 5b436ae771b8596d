"""A small serving loop: adaptive-depth MoE layers behind attention over a paged cache.

    python examples/paged_serving.py [--share] [--blocks N]

Prompts of different lengths are prefilled in one packed step, one of them is
branched into two continuations that share its pages, and then every sequence is
decoded.  A round drafts a tree of candidate tokens for each sequence, runs the tree
through the model in one step (each draft attends to its ancestors), keeps the
longest path that the model agrees with, and drops the rest of the tree from the
cache.  Per layer:

    q = cache.append(layer, norm(h) Wqkv)     norms, rotation, keys and values into pages
    h = h + cache.attend(layer, q) Wo         live tokens of prompts, drafted trees, decoding
                                              (--share: the branch's common pages read once;
                                              --blocks: over the N most promising pages per token)
    engine.layer_step(layer, tokens)          skip / exit / execute and the experts

A token that exits keeps the state that entered the layer, and goes on supplying keys
and values.  (The exit decision reads the state behind this attention; inside the full
block it reads the one before it.)  The weights are random; the projections are plain
matrix products.  A token's decisions hang on its own state and on its sequence's access
server, so what a round accepts is what decoding one token at a time would have
produced, up to rounding (which can tip a decision that stands at its threshold).
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_00573_gb300 import binding as B          # noqa: E402
from paper_2608_00573_gb300 import workload as W         # noqa: E402


class Model:
    """Attention layers over a PagedCache, each followed by the engine's MoE layer."""

    def __init__(self, cfg, q_heads, kv_heads, head_dim, vocab, cache, engine, seed=0):
        self.cfg, self.cache, self.engine = cfg, cache, engine
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)

        d, N = cfg.d, cfg.N
        self.embed = normal(vocab, d, std=1.0)
        self.w_qkv = normal(N, d, (q_heads + 2 * kv_heads) * head_dim, std=d ** -0.5)
        self.w_o = normal(N, q_heads * head_dim, d, std=(q_heads * head_dim) ** -0.5)
        self.gamma_q, self.gamma_k = (torch.ones(N, head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def __call__(self, ids, pos=None, tree=None, server=0, groups=None, blocks=0):
        """Most likely next token after each of the step's tokens (ids int64 [T]); server: the access server of each
        token's sequence, where the token starts (decisions hang on it, not on the place in the step); groups: how
        many of the step's sequences in a row share a prompt; blocks: pages before the step that a token attends to
        (0: all)."""
        T = ids.shape[0]
        state = W.make_tokens(self.cfg, T=T)
        tok = self.engine.tokens_to_device(state)
        tok["hidden"].copy_(self.embed[ids])
        tok["s"][:] = server
        h, alive = tok["hidden"], tok["alive"]
        if groups is not None:
            self.cache.share(groups)
        for layer in range(self.cfg.N):
            entering, live = h.clone(), (alive != 0)[:, None]
            # Every token supplies keys and values, also one that has exited; attention runs for live ones.
            x = torch.nn.functional.rms_norm(h, (self.cfg.d,), eps=1e-6)
            q = self.cache.append(layer, x @ self.w_qkv[layer], gamma_q=self.gamma_q[layer], gamma_k=self.gamma_k[layer],
                                  theta=1e4, pos=pos)
            if blocks:
                self.cache.summarize(layer)
                seen = self.cache.attend_blocks(layer, q, self.cache.select(layer, q, blocks), tree=tree)
            else:
                seen = self.cache.attend(layer, q, tree=tree)
            h += torch.where(live, seen @ self.w_o[layer], 0)
            self.engine.layer_step(layer, tok)
            # A token that exits at a layer leaves with the state that entered it.
            h.copy_(torch.where(live & (alive == 0)[:, None], entering, h))
        return (torch.nn.functional.rms_norm(h, (self.cfg.d,)) @ self.embed.T).argmax(-1)


def tree_of(width, depth):
    """A root and `width` chains of `depth` drafts: depths, mask words, parents."""
    parent = [-1] + [max(0, i - width) if i > width else 0 for i in range(1, 1 + width * depth)]
    deep, words = [0], [1]
    for i in range(1, len(parent)):
        deep.append(deep[parent[i]] + 1)
        words.append(words[parent[i]] | 1 << i)
    return deep, words, parent


def longest_path(drafts, following, parent):
    """Nodes of the tree that the model agrees with, from the root down."""
    path = [0]
    while True:
        nxt = [i for i, p in enumerate(parent) if p == path[-1] and i > 0 and drafts[i] == following[path[-1]]]
        if not nxt:
            return path
        path.append(nxt[0])


def run(rounds=6, width=3, depth=3, prompts=(200, 37, 130), seed=0, verbose=True, share=False, blocks=0):
    """share: the branch and its origin are listed side by side, as a group; blocks: pages per token (at least two)."""
    cfg = W.WorkloadConfig(name="paged", N=3, d=512, E=8, k=2, F=256, C=1, M=6, H=3, act=W.ACT_SWIGLU, T=512, seed=seed + 3)
    small = W.make_small_weights(cfg, calib=None)
    engine = B.Engine(cfg, W.make_tables(cfg, small["W_r"], calib=None), small, W.make_expert_weights_host(cfg), T_max=1024)
    heads, kv_heads, head_dim, page, vocab = 8, 2, 64, 16, 200
    n = len(prompts) + 1                                   # the last sequence branches off the first
    cache = B.PagedCache.empty(cfg.N, 256, heads, kv_heads, head_dim, page, max_seqs=n, max_pages=64, T_max=1024,
                               bounds=blocks > 0)
    model = Model(cfg, heads, kv_heads, head_dim, vocab, cache, engine, seed)
    rng = np.random.default_rng(seed)
    text = [rng.integers(0, vocab, p).tolist() for p in prompts]
    server = np.random.default_rng([seed, 1]).integers(0, cfg.M, len(prompts)).tolist()
    server.append(server[0])

    def start(per_sequence):
        """Access server of each packed token."""
        return torch.tensor(np.repeat(server[:len(per_sequence)], per_sequence), dtype=torch.uint8, device="cuda")

    # Prefill: all prompts in one step.
    cache.step(range(len(prompts)), prompts)
    following = model(torch.tensor(sum(text, []), device="cuda"), server=start(prompts), blocks=blocks)
    ends = np.cumsum(prompts) - 1
    for s, t in enumerate(following[torch.tensor(ends, device="cuda")].tolist()):
        text[s].append(t)
    # Branch: the continuation starts from another token and shares the prompt's pages.
    cache.fork([0], [n - 1])
    text.append(text[0][:-1] + [(text[0][-1] + 1) % vocab])

    # The order in which a round lists the sequences.
    order = [0, n - 1, *range(1, n - 1)] if share else list(range(n))
    groups = [2] + [1] * (n - 2) if share else None
    deep, words, parent = tree_of(width, depth)
    m = len(deep)
    tree = torch.tensor(words * n, dtype=torch.int64, device="cuda")
    accepted = 0
    for _ in range(rounds):
        base = cache.length.tolist()                       # (for the positions; a server would keep them)
        cache.step(order, [m] * n)
        # Drafts: a crude guesser, the bigrams seen so far and random tokens.
        drafts = {}
        for s in range(n):
            bigram = dict(zip(text[s], text[s][1:]))
            d = [text[s][-1]]
            for i in range(1, m):
                guess = bigram.get(d[parent[i]], None) if i <= width and i == 1 or i > width else None
                d.append(int(rng.integers(0, vocab)) if guess is None else guess)
            drafts[s] = d
        pos = torch.tensor([base[s] + k for s in order for k in deep], dtype=torch.int32, device="cuda")
        after = model(torch.tensor(sum((drafts[s] for s in order), []), device="cuda"), pos=pos, tree=tree,
                      server=torch.tensor(np.repeat([server[s] for s in order], m), dtype=torch.uint8, device="cuda"),
                      groups=groups, blocks=blocks)
        after = dict(zip(order, after.view(n, m).tolist()))
        paths = [longest_path(drafts[s], after[s], parent) for s in range(n)]
        table = torch.tensor([p + [0] * (depth + 1 - len(p)) for p in paths], dtype=torch.int32, device="cuda")
        cache.accept(range(n), torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda"), table)
        for s in range(n):
            text[s] += [drafts[s][i] for i in paths[s][1:]] + [after[s][paths[s][-1]]]
            accepted += len(paths[s]) - 1
    stats = cache.stats()
    if verbose:
        print(f"{n} sequences, {rounds} rounds: {sum(map(len, text)) - sum(prompts) - prompts[0]} tokens, "
              f"{accepted} of them drafted; lengths {cache.length.tolist()}, {stats['free_pages']} pages free")
    return dict(text=text, cache=cache, model=model, stats=stats, accepted=accepted, engine=engine)


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--share", action="store_true")
    parser.add_argument("--blocks", type=int, default=0)
    run(**vars(parser.parse_args()))
