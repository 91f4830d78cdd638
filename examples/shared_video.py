"""Several questions about one video, verified together over one copy of its cache.

A small decoder with random weights runs what a serving program runs:

* the prompt: the video's tokens (frames of 12 x 12 visual tokens, positions with
  three axes: time, height, width) go through every layer once; kv_append writes their
  keys and values into the pages that all questions share;
* the questions' own tokens follow, each question's in pages of its own;
* verification steps: draft rows of all questions go through add_rms_norm, the q/k/v
  projection, kv_append, shared_prefix_attention, the output projection and
  add_rms_norm, layer by layer; the fused LM head and acceptance (verify_lm_head_accept)
  says which drafts stay, and kv_commit prepares the caches for the next step.

With --check every step is compared with the same step over verify_attention, for
which the prefix' pages stand in front of every question's own block table.

    python examples/shared_video.py --questions 8 --frames 16 --check
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_12728_gb300 import specflash_verify as sfv  # noqa: E402

PAGE = sfv.PAGE_SIZE
BF16, I32 = torch.bfloat16, torch.int32


class Model:
    """Random weights of a pre-norm decoder without an MLP."""

    def __init__(self, layers, heads, kv_heads, d, vocab, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.d, self.hidden = heads, kv_heads, d, heads * d
        rand = lambda *s: (torch.randn(*s, generator=gen, device="cuda") * s[-1] ** -0.5).to(BF16)  # noqa: E731
        self.embed = rand(vocab, self.hidden) * self.hidden ** 0.5
        self.head = rand(vocab, self.hidden) * 4
        self.norms = [torch.ones(self.hidden, dtype=BF16, device="cuda") for _ in range(layers + 1)]
        self.qkv = [rand((heads + 2 * kv_heads) * d, self.hidden) for _ in range(layers)]
        self.out = [rand(self.hidden, self.hidden) for _ in range(layers)]
        half = d // 2
        self.inv_freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        # time, height and width share the frequencies 1/4, 3/8, 3/8
        cut = [half // 4, half * 3 // 8, half - half // 4 - half * 3 // 8]
        self.axis = torch.tensor([a for a, n in enumerate(cut) for _ in range(n)], dtype=I32, device="cuda")

    def split(self, x, layer):
        """The fused projection's q, k and v rows, as strided views."""
        y = torch.nn.functional.linear(x, self.qkv[layer])
        sizes = [self.heads * self.d, self.kv_heads * self.d, self.kv_heads * self.d]
        return [t.unflatten(1, (-1, self.d)) for t in y.split(sizes, 1)]


class Cache:
    """One layer's pages, and who holds which: the video's, then `most` tokens a question."""

    def __init__(self, model, layers, prefix, questions, most):
        shared, own = -(-prefix // PAGE), -(-most // PAGE)
        shape = (shared + questions * own + 64, model.kv_heads, PAGE, model.d)
        self.k = [torch.empty(shape, dtype=BF16, device="cuda") for _ in range(layers)]
        self.v = [torch.empty(shape, dtype=BF16, device="cuda") for _ in range(layers)]
        page = torch.arange(shape[0], dtype=I32, device="cuda")
        self.prefix_table = page[None, :shared].contiguous()
        self.prefix_lens = torch.tensor([prefix], dtype=I32, device="cuda")
        self.group_starts = torch.tensor([0, questions], dtype=I32, device="cuda")
        self.table = page[shared:shared + questions * own].view(questions, own).clone()
        self.lens = torch.zeros(questions, dtype=I32, device="cuda")
        self.free = page[shared + questions * own:].clone()
        self.free_count = torch.tensor([64], dtype=I32, device="cuda")


def layers_forward(model, x, attend):
    """x [T][hidden] through every layer; attend(layer, q, k, v) is the layer's attention."""
    residual = torch.zeros_like(x)
    for layer in range(len(model.qkv)):
        y, residual, _ = sfv.add_rms_norm(x, model.norms[layer], residual, residual_out=residual)
        x = torch.nn.functional.linear(attend(layer, *model.split(y, layer)).flatten(1), model.out[layer])
    return sfv.add_rms_norm(x, model.norms[-1], residual)[0]


def prompt(model, cache, frames):
    """The video's tokens: causal over the prompt in blocks of one frame's tokens, each
    block appended and then attended to over what lies before it."""
    n = 144
    gen = torch.Generator(device="cuda").manual_seed(1)
    visual = torch.randn(frames * n, model.hidden, generator=gen, device="cuda").to(BF16)
    at = torch.arange(n, device="cuda")
    for f in range(frames):
        pos = torch.stack([torch.full_like(at, f), at // 12, at % 12]).to(I32)
        upto = torch.tensor([(f + 1) * n], dtype=I32, device="cuda")

        def attend(layer, q, k, v):
            q = sfv.kv_append(q, k, v, pos, model.inv_freq, cache.k[layer], cache.v[layer], cache.prefix_table, upto,
                              axis=model.axis)
            # rows in blocks of 16 queries over the frames so far: nine sequences that
            # share everything before them, and see the frame up to their own block
            rows = q.view(n // 16, 16, model.heads, model.d)
            before = torch.tensor([f * n], dtype=I32, device="cuda")
            ends = 16 * torch.arange(1, n // 16 + 1, dtype=I32, device="cuda")
            own = cache.prefix_table[:, f * n // PAGE:(f + 1) * n // PAGE].expand(n // 16, -1).contiguous()
            starts = torch.tensor([0, n // 16], dtype=I32, device="cuda")
            return sfv.shared_prefix_attention(rows, cache.k[layer], cache.v[layer], cache.prefix_table, before, starts,
                                               own, ends)[0].view(n, model.heads, model.d)

        layers_forward(model, visual[f * n:(f + 1) * n], attend)


def block(model, cache, tokens, frames, unshared=False):
    """Token rows [questions][n] behind what each question has (cache.lens counts them):
    append and attention in every layer.  Returns the final hidden states."""
    questions, n = tokens.shape
    text = frames + cache.lens[:, None] - n + torch.arange(n, device="cuda")  # one time step a text token
    pos = text.to(I32).flatten().expand(3, -1).contiguous()
    prefix = cache.prefix_table.shape[1]
    if unshared:  # (here: verify_attention reads both before it waits for the kernel in front of it)
        table = torch.cat([cache.prefix_table.expand(questions, prefix), cache.table], 1)
        lens = cache.lens + prefix * PAGE

    def attend(layer, q, k, v):
        q = sfv.kv_append(q, k, v, pos, model.inv_freq, cache.k[layer], cache.v[layer], cache.table, cache.lens,
                          axis=model.axis).view(questions, n, model.heads, model.d)
        if unshared:
            out = sfv.verify_attention(q, cache.k[layer], cache.v[layer], table, lens)[0]
        else:
            out = sfv.shared_prefix_attention(q, cache.k[layer], cache.v[layer], cache.prefix_table, cache.prefix_lens,
                                              cache.group_starts, cache.table, cache.lens)[0]
        return out.view(questions * n, model.heads, model.d)

    return layers_forward(model, model.embed[tokens.flatten()], attend).view(questions, n, -1)


def run(questions=8, frames=8, steps=4, drafts=4, layers=2, heads=14, kv_heads=2, d=128, vocab=2000, check=False):
    """Returns the tokens of every question and, with check, the largest difference of
    the final hidden states between the two attentions."""
    model = Model(layers, heads, kv_heads, d, vocab)
    prefix = frames * 144
    cache = Cache(model, layers, prefix, questions, 64 + steps * (drafts + 1) + PAGE)
    prompt(model, cache, frames)

    gen = torch.Generator(device="cuda").manual_seed(2)
    said = [[] for _ in range(questions)]
    n = drafts + 1
    last = torch.randint(vocab, (questions, 1), generator=gen, device="cuda")
    # the questions: sixteen tokens each
    cache.lens += 16
    block(model, cache, torch.randint(vocab, (questions, 16), generator=gen, device="cuda"), frames)
    cache.lens += n
    worst = 0.0
    tau = torch.full((questions,), 0.7, device="cuda")
    for _ in range(steps):
        # a draft model's proposals: here the target's own, one position at a time
        # over a flat distribution
        q = torch.full((questions, drafts, vocab), 1.0 / vocab, device="cuda")
        proposed = torch.randint(vocab, (questions, drafts), generator=gen, device="cuda")
        tokens = torch.cat([last, proposed], 1)
        if check:  # (first: the keys and values that stay are those of the shared attention)
            other = block(model, cache, tokens, frames, unshared=True)
        hidden = block(model, cache, tokens, frames)
        if check:
            worst = max(worst, float((hidden.float() - other.float()).abs().max()))
        u = torch.rand(questions, n, generator=gen, device="cuda")
        _, kept, out, _ = sfv.verify_lm_head_accept(hidden, model.head, q, proposed.to(I32), u, tau)
        sfv.kv_commit(cache.lens, cache.table, cache.free, cache.free_count, kept, n, n)
        for b, (a, row) in enumerate(zip(kept.tolist(), out.tolist())):
            said[b] += row[:a + 1]
        last = out.gather(1, kept.long()[:, None]).long()
    return said, worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--questions", type=int, default=8)
    ap.add_argument("--frames", type=int, default=8)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    said, worst = run(a.questions, a.frames, a.steps, a.drafts, check=a.check)
    for b, tokens in enumerate(said):
        print(f"question {b}: {tokens}")
    if a.check:
        print(f"largest difference of the hidden states to the unshared attention: {worst:.3g}")


if __name__ == "__main__":
    main()
