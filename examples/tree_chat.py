"""Chats over long contexts: trees of drafts, and caches held at a budget.

A small decoder with random weights runs what a serving program runs, one sequence
and its own cache per chat:

* the prompt goes through every layer in blocks of 64 rows (kv_append, tree_attention
  with the masks of a chain); the attention weight that the last block's rows give to
  the tokens in front of them is kept per key (attention_mass);
* every step drafts a tree: the likeliest next tokens, some after each of those, ..;
  tree_mask makes the nodes' masks and positions, all nodes go through add_rms_norm,
  the q/k/v projection, kv_append, tree_attention and the output projection, layer by
  layer, sample gives the target's token after every node, and tree_commit follows
  the target through the tree, moves the path's keys and values behind the context and
  prepares lengths and pages for the next tree;
* the weight that the path's rows gave to the context is added up, and where a context
  has outgrown its budget, kv_evict keeps the tokens of most weight.

With --check the rows of every step's path are compared with the same tokens as a chain
through verify_attention.

    python examples/tree_chat.py --chats 4 --budget 256 --check
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.shared_video import BF16, I32, PAGE, Model, layers_forward  # noqa: E402
from paper_2505_12728_gb300 import specflash_verify as sfv  # noqa: E402

BLOCK = 64


class Cache:
    """All layers' pages of `chats` sequences of at most `most` tokens, and each KV
    head's weight per key."""

    def __init__(self, model, layers, chats, most):
        each = -(-most // PAGE)
        shape = (layers, chats * each, model.kv_heads, PAGE, model.d)
        self.k = torch.zeros(shape, dtype=BF16, device="cuda")
        self.v = torch.zeros(shape, dtype=BF16, device="cuda")
        self.mass = torch.zeros(layers, chats, model.kv_heads, each * PAGE, device="cuda")
        self.table = torch.full((chats, each), -1, dtype=I32, device="cuda")
        self.lens = torch.zeros(chats, dtype=I32, device="cuda")
        self.free = torch.arange(chats * each, dtype=I32, device="cuda")
        self.free_count = torch.tensor([chats * each], dtype=I32, device="cuda")

    def map(self, tokens):
        """Pages for the first `tokens` positions of every chat, off the free stack."""
        pages, chats = -(-tokens // PAGE), self.table.shape[0]
        left = int(self.free_count) - pages * chats
        self.table[:, :pages] = self.free[left:left + pages * chats].view(chats, pages)
        self.free_count.fill_(left)
        self.lens.fill_(tokens)


def forward(model, cache, tokens, positions, attention):
    """Rows [chats][n] of tokens behind each chat's context (cache.lens counts them).
    Returns the final hidden states and every layer's (q, lse)."""
    chats, n = tokens.shape
    seen = []

    def attend(layer, q, k, v):
        q = sfv.kv_append(q, k, v, positions.flatten()[None].contiguous(), model.inv_freq, cache.k[layer], cache.v[layer],
                          cache.table, cache.lens).view(chats, n, model.heads, model.d)
        out, lse = attention(q, cache.k[layer], cache.v[layer])
        seen.append((q, lse))
        return out.view(chats * n, model.heads, model.d)

    return layers_forward(model, model.embed[tokens.flatten()], attend).view(chats, n, -1), seen


def prompt(model, cache, tokens):
    """The prompts [chats][tokens], in blocks."""
    chats, length = tokens.shape
    chain = torch.tensor([(2 << i) - 1 if i < 63 else -1 for i in range(BLOCK)], device="cuda")
    for at in range(0, length, BLOCK):
        lens = torch.full((chats,), at + BLOCK, dtype=I32, device="cuda")
        cache.lens.copy_(lens)
        positions = (at + torch.arange(BLOCK, device="cuda")).to(I32).expand(chats, -1)
        _, seen = forward(model, cache, tokens[:, at:at + BLOCK], positions,
                          lambda q, k, v: sfv.tree_attention(q, k, v, cache.table, lens, chain))
    for layer, (q, lse) in enumerate(seen):  # what the last block's rows looked at
        sfv.attention_mass(q, lse, cache.k[layer], cache.table, lens, out=cache.mass[layer])


def draft(model, last, parents):
    """Tokens [chats][n] of the trees' nodes: below each node the likeliest tokens of the
    target without its attention, the first child the likeliest one."""
    tokens = last.new_zeros(last.shape[0], len(parents))
    tokens[:, 0] = last
    rank = [parents[:i].count(p) for i, p in enumerate(parents)]
    for i in range(1, len(parents)):
        scores = model.embed[tokens[:, parents[i]]].float() @ model.head.float().t()
        tokens[:, i] = scores.topk(rank[i] + 1, 1)[1][:, -1]
    return tokens


def as_chain(model, cache, tokens, positions, lens):
    """The same rows as a chain over verify_attention; what they append is taken back."""
    kept = cache.k.clone(), cache.v.clone(), cache.lens.clone()
    cache.lens.copy_(lens)
    hidden, _ = forward(model, cache, tokens, positions,
                        lambda q, k, v: sfv.verify_attention(q, k, v, cache.table, lens))
    first = cache.k[0].clone()  # layer 0's keys depend on tokens and positions alone
    cache.k.copy_(kept[0])
    cache.v.copy_(kept[1])
    cache.lens.copy_(kept[2])
    return hidden, first


def run(chats=4, length=320, steps=6, budget=256, slack=32, layers=2, heads=14, kv_heads=2, d=128, vocab=500, tau=0.0,
        check=False):
    """Returns every chat's tokens, the contexts' lengths after each step, and with check
    the largest difference of a path's final hidden states to the chain's."""
    model = Model(layers, heads, kv_heads, d, vocab)
    gen = torch.Generator(device="cuda").manual_seed(3)
    # three tokens after the root, two after the first two of those, ..
    parents = [-1, 0, 0, 0, 1, 1, 2, 2, 4, 4, 6, 8, 8, 11]
    n = len(parents)
    cache = Cache(model, layers, chats, max(length, budget + slack) + steps * n + n)
    cache.map(length)
    prompt(model, cache, torch.randint(vocab, (chats, length), generator=gen, device="cuda"))
    up = torch.tensor([parents] * chats, dtype=I32, device="cuda")
    at = torch.full((chats,), length, dtype=I32, device="cuda")  # the roots' positions, whatever the cache keeps
    last = torch.randint(vocab, (chats,), generator=gen, device="cuda")
    temperature = torch.full((chats * n,), tau, device="cuda")
    said, lengths, worst = [[] for _ in range(chats)], [], 0.0
    # room for the first tree
    pages = -(-(length + n) // PAGE)
    have = -(-length // PAGE)
    if pages > have:
        left = int(cache.free_count) - (pages - have) * chats
        cache.table[:, have:pages] = cache.free[left:left + (pages - have) * chats].view(chats, -1)
        cache.free_count.fill_(left)
    cache.lens.fill_(length + n)
    for _ in range(steps):
        tokens = draft(model, last, parents)
        mask, positions = sfv.tree_mask(up, at)
        lens = cache.lens.clone()
        hidden, seen = forward(model, cache, tokens, positions,
                               lambda q, k, v: sfv.tree_attention(q, k, v, cache.table, cache.lens, mask))
        logits = (hidden.flatten(0, 1).float() @ model.head.float().t()).contiguous()
        u = torch.rand(chats * n, generator=gen, device="cuda")
        _, target = sfv.sample(logits, u, temperature)
        table = cache.table.clone()
        kept, out, path, weights = sfv.tree_commit(tokens.to(I32), target.view(chats, n), up, cache.k, cache.v, cache.table,
                                                   cache.lens, n_q_next=n, free_pages=cache.free,
                                                   free_count=cache.free_count)
        for layer, (q, lse) in enumerate(seen):
            sfv.attention_mass(q, lse, cache.k[layer], table, lens, cache.mass[layer], row_weights=weights,
                               out=cache.mass[layer])
        if check:
            now = cache.table.clone()
            for b, a in enumerate(kept.tolist()):
                rows = path[b:b + 1, :a + 1].long()
                chain_len = lens.clone()
                chain_len += a + 1 - n
                cache.table.copy_(table)
                all_rows = rows.expand(chats, -1).contiguous()
                got, keys = as_chain(model, cache, tokens.gather(1, all_rows), positions.gather(1, all_rows).to(I32), chain_len)
                cache.table.copy_(now)
                worst = max(worst, float((got[b].float() - hidden[b, rows[0]].float()).abs().max()))
                for r in range(a + 1):
                    t = int(lens[b]) - n + r
                    page = int(table[b, t // PAGE])
                    assert torch.equal(keys[page, :, t % PAGE], cache.k[0, page, :, t % PAGE])
        at += kept + 1
        for b, (a, row) in enumerate(zip(kept.tolist(), out.tolist())):
            said[b] += row[:a + 1]
        last = out.gather(1, kept.long()[:, None])[:, 0].long()
        if int(cache.lens.max()) - n > budget + slack:
            sfv.kv_evict(cache.mass, cache.k, cache.v, cache.table, cache.lens, budget, first=4, recent=32, n_q=n,
                         free_pages=cache.free, free_count=cache.free_count)
        lengths.append((cache.lens - n).tolist())
    return said, lengths, worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--chats", type=int, default=4)
    ap.add_argument("--length", type=int, default=320, help="prompt tokens, a multiple of 64")
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--budget", type=int, default=256)
    ap.add_argument("--tau", type=float, default=0.0)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    said, lengths, worst = run(a.chats, a.length, a.steps, a.budget, tau=a.tau, check=a.check)
    for b, tokens in enumerate(said):
        print(f"chat {b}: {tokens}")
    print("context lengths:", lengths)
    if a.check:
        print(f"largest difference of the hidden states to the chain's: {worst:.3g}")


if __name__ == "__main__":
    main()
