"""The work that the operators of tree drafts and of a bounded cache are measured on.

A draft may be a tree of tokens instead of a chain: all its nodes are verified
in one pass, each seeing the cached context and its own ancestors, and the
context afterwards keeps one path of it.  A long (mostly visual) context may
be held at a budget by dropping the keys that queries attend to least.

* ``mask``: a tree's ancestor masks and positions from its parents
  (``tree_mask``);
* ``attend``: verification attention of a tree's nodes over the paged cache
  (``tree_attention``);
* ``commit``: the path that the target's tokens take through the tree, and its
  keys and values in all layers' caches moved to follow the context
  (``tree_commit``);
* ``mass``: the attention weight that each cached key got from some query rows,
  per KV head (``attention_mass``);
* ``evict``: the keys of most weight kept, in all layers, the caches compacted
  in place (``kv_evict``).

Shapes follow the library's workloads (paper_2505_12728_gb300/workloads.py):
32/32 heads of 128 with 3008-token image prompts, 28/4 heads with 4864-token
video prompts and contexts of up to 32768 tokens, 8/8 heads of 64 as the small
one; trees have up to 64 nodes.

With ``own`` false, `run` computes plain forms in elementary operations; with
``own`` true it calls the library.
"""
import math
import random

import torch

own = False

PAGE = 16
DEVICE = "cuda"
HEADS = [(8, 8, 64), (16, 4, 64), (12, 3, 128), (20, 4, 128), (28, 4, 128), (32, 32, 128)]


# --------------------------------------------------------------------------- #
# the cases                                                                   #
# --------------------------------------------------------------------------- #
def _mask(**kw):
    c = dict(op="mask", B=1, nodes=26)
    c.update(kw)
    return c


def _attend(**kw):
    c = dict(op="attend", B=1, nodes=26, lo=3008, hi=3008, heads=32, kv_heads=32, d=128, idle=0)
    c.update(kw)
    return c


def _commit(**kw):
    c = dict(op="commit", layers=32, B=1, nodes=26, lo=3008, hi=3008, kv_heads=32, d=128, idle=0)
    c.update(kw)
    return c


def _mass(**kw):
    c = dict(op="mass", B=1, rows=5, lo=3008, hi=3008, heads=32, kv_heads=32, d=128, weighted=False, add=True)
    c.update(kw)
    return c


def _evict(**kw):
    c = dict(op="evict", layers=32, B=1, lo=3008, hi=3008, kv_heads=32, d=128, budget=1024, first=4, recent=128)
    c.update(kw)
    return c


def listed():
    return [
        # one sequence's tree, built anew by the draft model: latency
        _mask(name="mask_step", B=1, nodes=26),
        # the trees of a large batch
        _mask(name="mask_batch", B=256, nodes=61),
        # a small model's tree of five nodes, two sequences: latency
        _attend(name="attend_tiny", B=2, nodes=5, lo=640, hi=640, heads=8, kv_heads=8, d=64),
        # the tree of one image chat, one KV head per query head
        _attend(name="attend_image", B=1, nodes=26, lo=3008, hi=3008),
        # four videos, seven query heads per KV head
        _attend(name="attend_video", B=4, nodes=32, lo=4864, hi=4864, heads=28, kv_heads=4),
        # 16 long videos of different lengths, large trees, one slot of the batch idle
        _attend(name="attend_long", B=16, nodes=61, lo=8192, hi=32768, heads=28, kv_heads=4, idle=1),
        # one image chat's accepted path, in the 32 layers' caches: latency
        _commit(name="commit_image"),
        # a batch of long videos, 28 layers
        _commit(name="commit_batch", layers=28, B=16, nodes=61, lo=8192, hi=32768, kv_heads=4, idle=1),
        # the draft rows of one image chat, the accepted ones counted, added to
        # what the keys have got before: each step of decoding
        _mass(name="mass_step", weighted=True),
        # the last 32 rows of 16 long video prompts, once per prompt
        _mass(name="mass_prompt", B=16, rows=32, lo=8192, hi=32768, heads=28, kv_heads=4, add=False),
        # an image chat of 32 layers back to its budget
        _evict(name="evict_image"),
        # the prompts of four long videos of 28 layers down to 4096 tokens
        _evict(name="evict_prompt", layers=28, B=4, lo=8192, hi=32768, kv_heads=4, budget=4096, recent=256),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["mask", "attend", "attend", "commit", "mass", "evict"])
    nodes = rng.randint(1, 64)
    if op == "mask":
        return _mask(B=_log_int(rng, 1, 256), nodes=nodes)
    h, kv, d = rng.choice(HEADS)
    hi = _log_int(rng, 1, 32768)
    lo = _log_int(rng, max(1, hi // 4), hi)
    if op == "commit":
        layers = rng.randint(1, 32)
        B = _log_int(rng, 1, max(1, min(32, 28 * 16 * 4 * 128 // (layers * kv * d))))
        return _commit(layers=layers, B=B, nodes=nodes, lo=lo, hi=hi, kv_heads=kv, d=d, idle=rng.randint(0, B // 4))
    if op == "evict":
        layers = rng.randint(1, 32)
        hi = max(64, min(hi, 28 * 4 * 32768 * 4 * 128 // (layers * kv * d)))
        lo = min(max(lo, 1), hi)
        B = _log_int(rng, 1, max(1, min(8, 28 * 4 * 32768 * 4 * 128 // (layers * hi * kv * d))))
        # at most the rows that the largest listed case moves
        budget = min(_log_int(rng, max(1, hi // 16), hi), max(1, 28 * 4 * 4096 * 4 * 128 // (layers * B * kv * d)))
        first = rng.randint(0, min(8, budget))
        return _evict(layers=layers, B=B, lo=lo, hi=hi, kv_heads=kv, d=d, budget=budget, first=first,
                      recent=rng.randint(0, min(256, budget - first)))
    B = _log_int(rng, 1, 16)
    rows = min(nodes, 512 * kv // h)
    # at most the rows x keys of the longest listed case, and its cache
    most = 16 * 61 * 28 if op == "attend" else 16 * 32 * 28
    hi = max(1, min(hi, most * 20480 // (B * rows * h), 16 * 20480 * 4 * 128 // (B * kv * d)))
    lo = min(lo, hi)
    if op == "attend":
        return _attend(B=B, nodes=rows, lo=lo, hi=hi, heads=h, kv_heads=kv, d=d, idle=rng.randint(0, B // 4))
    return _mass(B=B, rows=rows, lo=lo, hi=hi, heads=h, kv_heads=kv, d=d, weighted=rng.random() < 0.5,
                 add=rng.random() < 0.5)


# --------------------------------------------------------------------------- #
# sizes of a case (the same for every seed)                                   #
# --------------------------------------------------------------------------- #
def _sizes(case):
    """Context lengths (None: an idle slot) and the depths of the accepted paths."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    B = case["B"]
    idle = set(rng.sample(range(B), case.get("idle", 0)))
    lens = [None if b in idle else rng.randint(case["lo"], case["hi"]) for b in range(B)]
    return lens, [rng.randint(0, 5) for _ in range(B)]


def work(case):
    B = case["B"]
    if case["op"] == "mask":
        return {"bytes": 16 * B * case["nodes"], "flops": 0}
    lens, depths = _sizes(case)
    kv, d = case["kv_heads"], case["d"]
    live = [n for n in lens if n is not None]
    if case["op"] == "commit":
        rows = sum(min(a, case["nodes"] - 1) for n, a in zip(lens, depths) if n is not None)
        return {"bytes": 8 * case["layers"] * kv * d * rows + 12 * B * case["nodes"], "flops": 0}
    if case["op"] == "evict":
        cut = [n for n in live if n > case["budget"]]
        moved = len(cut) * (case["budget"] - case["first"])
        return {"bytes": case["layers"] * kv * (8 * d * moved + 4 * sum(live) + 8 * sum(min(n, case["budget"]) for n in live)),
                "flops": 0}
    h = case["heads"]
    if case["op"] == "mass":
        R = case["rows"] * h
        return {"bytes": 2 * kv * d * sum(live) + 4 * kv * sum(live) * (1 + case["add"]) + B * R * (2 * d + 4),
                "flops": 2 * d * R * sum(live)}
    n = case["nodes"]
    return {"bytes": 4 * kv * d * sum(x + n for x in live) + len(live) * n * (h * (4 * d + 4) + 8),
            "flops": 4 * d * h * n * sum(x + 1 for x in live)}


# --------------------------------------------------------------------------- #
# inputs                                                                      #
# --------------------------------------------------------------------------- #
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _trees(rng, B, n):
    """Parents of B trees of n nodes, node 0 the root; -2 from a tree's last node on."""
    t = []
    for _ in range(B):
        used = n if n < 4 or rng.random() < 0.5 else rng.randint(n - n // 4, n)
        t.append([-1] + [rng.randint(max(0, i - 8), i - 1) if i < used else -2 for i in range(1, n)])
    return t


def _ancestors(parents):
    """One 64-bit word per node: bit j for node j itself or above it."""
    words = []
    for p in parents:
        row = []
        for i, a in enumerate(p):
            row.append(0 if a < -1 else (1 << i) | (row[a] if a >= 0 else 0))
        words.append([w - (1 << 64) if w >> 63 else w for w in row])
    return torch.tensor(words, dtype=torch.int64, device=DEVICE)


def _table(rng, totals, shared=None):
    """A block table over randomly ordered pages, and how many pages there are.  With
    `shared`, the pages in front of page shared[b] of a row are the same few."""
    pages = [-(-t // PAGE) for t in totals]
    first = [0] * len(pages) if shared is None else shared
    pool = sum(p - f for p, f in zip(pages, first)) + 3
    ids = rng.sample(range(pool), pool)
    width = max(1, max(pages))
    t, at = [], 0
    for p, f in zip(pages, first):
        t.append([ids[-1]] * f + ids[at:at + p - f] + [-1] * (width - p))
        at += p - f
    return _ints(t), pool


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    rng = random.Random(seed)
    B = case["B"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE).to(torch.bfloat16)

    s = dict(op=case["op"])
    if case["op"] == "mask":
        n = case["nodes"]
        s["parents"] = _ints(_trees(rng, B, n))
        s["start"] = _ints([rng.randint(0, 32768) for _ in range(B)])
        s["mask"] = torch.empty(B, n, dtype=torch.int64, device=DEVICE)
        s["positions"] = torch.empty(B, n, dtype=torch.int32, device=DEVICE)
        if own:
            from paper_2505_12728_gb300 import specflash_verify as sfv
            s["workspace"] = sfv.new_workspace(sfv.tree_mask_workspace_size())
        return s

    kv, d = case["kv_heads"], case["d"]
    lens, depths = _sizes(case)
    if case["op"] == "evict":
        totals = [n or 0 for n in lens]
        s["table"], pool = _table(rng, totals)
        s["lens"] = _ints(totals)
        s["k"] = torch.stack([normal(pool, kv, PAGE, d) for _ in range(case["layers"])])
        s["v"] = torch.stack([normal(pool, kv, PAGE, d) for _ in range(case["layers"])])
        width = s["table"].shape[1] * PAGE
        # a few keys get most of the weight, and some none at all
        mass = torch.randn(case["layers"], B, kv, width, generator=gen, device=DEVICE).mul(2).exp()
        s["mass"] = mass * (torch.rand(mass.shape, generator=gen, device=DEVICE) > 0.05)
        s["mass_out"] = torch.empty_like(s["mass"])
        s["lens_out"] = torch.empty_like(s["lens"])
        s["kept"] = torch.empty(case["layers"], B, kv, case["budget"], dtype=torch.int32, device=DEVICE)
        s["budget"], s["first"], s["recent"] = case["budget"], case["first"], case["recent"]
        if own:
            from paper_2505_12728_gb300 import specflash_verify as sfv
            s["workspace"] = sfv.new_workspace(sfv.kv_evict_workspace_size(case["layers"], B, kv, case["budget"]))
        return s

    if case["op"] == "mass":
        n, h = case["rows"], case["heads"]
        # the rows' own keys are behind the context, as in the attention in front
        totals = [x + n for x in lens]
        s["table"], pool = _table(rng, totals)
        s["lens"] = _ints(totals)
        s["q"], s["k"] = normal(B, n, h, d), normal(pool, kv, PAGE, d)
        s["lse"] = torch.empty(B, n, h, device=DEVICE)
        for b, x in enumerate(lens):  # what that attention gave
            keys = s["k"][s["table"][b, :-(-totals[b] // PAGE)].long()].transpose(0, 1).reshape(kv, -1, d)
            q = s["q"][b].view(n, kv, h // kv, d).transpose(0, 1).reshape(kv, -1, d)
            score = torch.bmm(q, keys[:, :x].transpose(1, 2)).float() * d ** -0.5
            s["lse"][b] = torch.logsumexp(score, 2).view(kv, n, h // kv).transpose(0, 1).reshape(n, h)
        s["weights"] = None
        if case["weighted"]:
            s["weights"] = (torch.rand(B, n, generator=gen, device=DEVICE) < 0.6).float()
        width = s["table"].shape[1] * PAGE
        s["mass"] = torch.rand(B, kv, width, generator=gen, device=DEVICE) if case["add"] else None
        s["mass_out"] = torch.zeros(B, kv, width, device=DEVICE)
        if own:
            from paper_2505_12728_gb300 import specflash_verify as sfv
            s["workspace"] = sfv.new_workspace(sfv.attention_mass_workspace_size())
        return s

    n = case["nodes"]
    totals = [0 if x is None else x + n for x in lens]
    s["lens"] = _ints(totals)
    trees = _trees(random.Random(repr((B, n, lens))), B, n)  # a program keeps its trees
    if case["op"] == "attend":
        h = case["heads"]
        s["table"], pool = _table(rng, totals)
        s["q"], s["k"], s["v"] = normal(B, n, h, d), normal(pool, kv, PAGE, d), normal(pool, kv, PAGE, d)
        s["mask"] = _ancestors(trees)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(B, n, h, device=DEVICE)
        if own:
            from paper_2505_12728_gb300 import specflash_verify as sfv
            s["workspace"] = sfv.new_workspace(sfv.tree_attention_workspace_size(B, n, h, kv, d, s["table"].shape[1]))
        return s

    # the caches hold the pages of the tree's rows; those of the context in front
    # are the same few, as nothing here reads them
    s["table"], pool = _table(rng, totals, [0 if x is None else x // PAGE for x in lens])
    s["k"] = torch.stack([normal(pool, kv, PAGE, d) for _ in range(case["layers"])])
    s["v"] = torch.stack([normal(pool, kv, PAGE, d) for _ in range(case["layers"])])
    tokens, sampled = [], []
    for p, want in zip(trees, depths):
        # siblings carry different tokens; the target follows the path to a node
        # `want` levels down (or as deep as the tree goes), then leaves the tree
        children = [[c for c in range(n) if p[c] == i] for i in range(n)]
        t, at = [rng.randint(0, 31999) for _ in range(n)], 0
        for c in children:
            for i, x in zip(c, rng.sample(range(32000), len(c))):
                t[i] = x
        o = [rng.randint(32000, 63999) for _ in range(n)]
        for _ in range(want):
            if children[at]:
                child = rng.choice(children[at])
                o[at], at = t[child], child
        tokens.append(t)
        sampled.append(o)
    s["parents"], s["tokens"], s["sampled"] = _ints(trees), _ints(tokens), _ints(sampled)
    s["accepted"] = torch.empty(B, dtype=torch.int32, device=DEVICE)
    s["out_tokens"] = torch.empty(B, n, dtype=torch.int32, device=DEVICE)
    s["path"] = torch.empty(B, n, dtype=torch.int32, device=DEVICE)
    s["weights"] = torch.empty(B, n, device=DEVICE)
    if own:
        from paper_2505_12728_gb300 import specflash_verify as sfv
        s["workspace"] = sfv.new_workspace(sfv.tree_commit_workspace_size())
    return s


# --------------------------------------------------------------------------- #
# one pass                                                                    #
# --------------------------------------------------------------------------- #
def run(s):
    if own:
        return _library(s)
    return {"mask": _plain_mask, "attend": _plain_attend, "commit": _plain_commit, "mass": _plain_mass,
            "evict": _plain_evict}[s["op"]](s)


def _library(s):
    from paper_2505_12728_gb300 import specflash_verify as sfv
    if s["op"] == "mask":
        return sfv.tree_mask(s["parents"], s["start"], mask=s["mask"], positions=s["positions"],
                             workspace=s["workspace"])
    if s["op"] == "attend":
        return sfv.tree_attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["mask"], out=s["out"],
                                  lse=s["lse"], workspace=s["workspace"])
    if s["op"] == "commit":
        # (the layers' caches side by side; a list of them will do as well)
        got = sfv.tree_commit(s["tokens"], s["sampled"], s["parents"], s["k"], s["v"], s["table"], s["lens"],
                              num_accepted=s["accepted"], out_tokens=s["out_tokens"], path=s["path"],
                              row_weights=s["weights"], workspace=s["workspace"])
        return tuple(got) + (s["k"], s["v"])
    if s["op"] == "mass":
        return sfv.attention_mass(s["q"], s["lse"], s["k"], s["table"], s["lens"], s["mass"],
                                  row_weights=s["weights"], out=s["mass_out"], workspace=s["workspace"])
    sfv.kv_evict(s["mass"], s["k"], s["v"], s["table"], s["lens"], s["budget"], first=s["first"], recent=s["recent"],
                 mass_out=s["mass_out"], seq_lens_out=s["lens_out"], kept=s["kept"], workspace=s["workspace"])
    return s["k"], s["v"], s["mass_out"], s["lens_out"], s["kept"]


def _twice(r):
    """Reachability in up to twice as many steps."""
    return (r @ r).clamp(max=1)


def _reach(parents):
    """[B][n][n]: 1 where j is i or above it, 0 for rows that are not part of the tree."""
    n = parents.shape[1]
    node = torch.arange(n, device=DEVICE)
    up = (parents[:, :, None] == node).float() + torch.eye(n, device=DEVICE)
    reach = _twice(_twice(_twice(_twice(_twice(_twice(up))))))
    return reach * (parents >= -1)[:, :, None]


def _plain_mask(s):
    reach = _reach(s["parents"])
    n = reach.shape[1]
    bits = torch.ones(n, dtype=torch.int64, device=DEVICE) << torch.arange(n, device=DEVICE)
    mask = (reach.long() * bits).sum(2)
    depth = (reach.sum(2) - 1).clamp(min=0)
    return mask, (s["start"][:, None] + depth).to(torch.int32)


def _pages(cache, table):
    """The tokens of each row of a block table, [rows][heads][tokens][d] in fp32."""
    x = cache[table.clamp(min=0).long()].float()  # [rows][pages][heads][16][d]
    return x.transpose(1, 2).flatten(2, 3)


def _rows(q, kv):
    """[B][n][h][d] as the rows of each KV head, [B][kv][n * h / kv][d] in fp32."""
    B, n, h, d = q.shape
    return q.float().view(B, n, kv, h // kv, d).transpose(1, 2).reshape(B, kv, n * (h // kv), d)


def _plain_attend(s):
    B, n, h, d = s["q"].shape
    kv = s["k"].shape[1]
    g = h // kv
    q = _rows(s["q"], kv) * d ** -0.5
    k, v = _pages(s["k"], s["table"]), _pages(s["v"], s["table"])
    before = s["lens"].long() - n  # the context's length (negative: an idle slot)
    at = torch.arange(k.shape[2], device=DEVICE) - before[:, None]  # [B][keys]: place within the tree
    sees = (s["mask"][:, :, None] >> at.clamp(0, 63)[:, None, :]) & 1
    sees = ((at < 0)[:, None] | ((at < n)[:, None] & (sees > 0))) & (before >= 0)[:, None, None]
    score = (q @ k.transpose(2, 3)).masked_fill(~sees.repeat_interleave(g, 1)[:, None], -math.inf)
    m = score.amax(3, keepdim=True).clamp(min=-3e38)
    p = (score - m).exp()
    l = p.sum(3, keepdim=True)
    o = (p @ v) / l.clamp(min=1e-38)
    lse = m + l.log()
    out = o.view(B, kv, n, g, d).transpose(1, 2).reshape(B, n, h, d).to(torch.bfloat16)
    return out, lse.view(B, kv, n, g).transpose(1, 2).reshape(B, n, h)


def _plain_commit(s):
    parents, n = s["parents"].long(), s["parents"].shape[1]
    node = torch.arange(n, device=DEVICE)
    up = parents.clamp(min=0)
    # a node continues its parent where it carries the target's token, the first such child
    fits = (s["tokens"] == s["sampled"].gather(1, up)) & (parents >= 0)
    rival = (parents[:, :, None] == parents[:, None, :]) & fits[:, None, :] & (node[None, :] < node[:, None])
    goes = (fits & ~rival.any(2)) | (node == 0)
    on = ((_reach(s["parents"]) > 0) & ~goes[:, None, :]).sum(2) == 0
    on = on & _reach(s["parents"])[:, :, 0].bool() & (s["lens"] > 0)[:, None]
    count = on.sum(1)
    path = torch.sort((~on).long() * n + node, 1)[0]
    taken = node < count[:, None]
    path = torch.where(taken, path, -1)
    out_tokens = torch.where(taken, s["sampled"].gather(1, path.clamp(min=0)), -1)
    b, i = taken.nonzero(as_tuple=True)
    before, table = s["lens"].long() - n, s["table"].long()
    to, source = before[b] + i, before[b] + path[b, i]
    page, source_page = table[b, to // PAGE], table[b, source // PAGE]
    s["k"][:, page, :, to % PAGE] = s["k"][:, source_page, :, source % PAGE]
    s["v"][:, page, :, to % PAGE] = s["v"][:, source_page, :, source % PAGE]
    return ((count - 1).clamp(min=0).to(torch.int32), out_tokens.to(torch.int32), path.to(torch.int32), on.float(),
            s["k"], s["v"])


def _plain_mass(s):
    B, n, h, d = s["q"].shape
    kv = s["k"].shape[1]
    g = h // kv
    k = _pages(s["k"], s["table"])
    lse = s["lse"].view(B, n, kv, g).transpose(1, 2).reshape(B, kv, n * g, 1)
    p = (_rows(s["q"], kv) * d ** -0.5 @ k.transpose(2, 3) - lse).exp()
    if s["weights"] is not None:
        p = p * s["weights"].repeat_interleave(g, 1)[:, None, :, None]
    total = p.sum(2)
    if s["mass"] is not None:
        total = total + s["mass"]
    inside = torch.arange(k.shape[2], device=DEVICE) < (s["lens"] - n)[:, None, None]
    s["mass_out"].copy_(torch.where(inside, total, s["mass_out"]))
    return s["mass_out"]


def _plain_evict(s):
    layers, B, kv, width = s["mass"].shape
    budget, lens = s["budget"], s["lens"].long()
    at = torch.arange(width, device=DEVICE)
    must = (at < s["first"]) | (at >= (lens - s["recent"])[:, None])
    inside = at < lens[:, None]
    key = s["mass"].masked_fill(must[None, :, None], math.inf).masked_fill(~inside[None, :, None], -math.inf)
    best = torch.sort(key, dim=3, descending=True, stable=True)[1][..., :budget]
    kept = torch.sort(best, 3)[0]
    if kept.shape[3] < budget:
        kept = torch.nn.functional.pad(kept, (0, budget - kept.shape[3]))
    i = torch.arange(budget, device=DEVICE)
    new = lens.clamp(max=budget)
    # (a sequence within its budget keeps all its keys, in their places)
    kept = torch.where((lens > budget)[None, :, None, None], kept, i)
    valid = (i < new[:, None])[None, :, None].expand_as(kept)
    mass = s["mass"].gather(3, kept.clamp(max=width - 1)).masked_fill(~valid, 0)
    s["mass_out"].zero_()
    s["mass_out"][..., :min(width, budget)] = mass[..., :min(width, budget)]
    s["lens_out"].copy_(new)
    s["kept"].copy_(torch.where(valid, kept, -1))
    l, b, h, j = (valid & (lens > budget)[None, :, None, None]).nonzero(as_tuple=True)
    source, table = kept[l, b, h, j], s["table"].long()
    page, source_page = table[b, j // PAGE], table[b, source // PAGE]
    s["k"][l, page, h, j % PAGE] = s["k"][l, source_page, h, source % PAGE]
    s["v"][l, page, h, j % PAGE] = s["v"][l, source_page, h, source % PAGE]
    return s["k"], s["v"], s["mass_out"], s["lens_out"], s["kept"]


# --------------------------------------------------------------------------- #
# the definitions in 64 bits                                                  #
# --------------------------------------------------------------------------- #
def exact(case, seed):
    if case["op"] == "evict":
        return None  # values are chosen and moved, none is computed
    s = prepare(case, seed)
    B = case["B"]
    if case["op"] == "mask":
        parents = s["parents"].tolist()
        depth = [[max(0, bin(w & (2 ** 64 - 1)).count("1") - 1) for w in row] for row in _ancestors(parents).tolist()]
        return _ancestors(parents), torch.tensor(depth, dtype=torch.int32, device=DEVICE) + s["start"][:, None]
    lens, _ = _sizes(case)
    if case["op"] == "commit":
        n, accepted, out_tokens, paths = case["nodes"], [], [], []
        parents, tokens, sampled = s["parents"].tolist(), s["tokens"].tolist(), s["sampled"].tolist()
        for b in range(B):
            path = [] if lens[b] is None else [0]
            while path:
                more = [c for c in range(n) if parents[b][c] == path[-1] and tokens[b][c] == sampled[b][path[-1]]]
                if not more:
                    break
                path.append(more[0])
            accepted.append(max(0, len(path) - 1))
            out_tokens.append([sampled[b][i] for i in path] + [-1] * (n - len(path)))
            paths.append(path + [-1] * (n - len(path)))
        weights = torch.tensor([[float(i in p) for i in range(n)] for p in paths], device=DEVICE)
        return _ints(accepted), _ints(out_tokens), _ints(paths), weights, None, None
    kv, d, h = case["kv_heads"], case["d"], case["heads"]

    def tokens_of(cache, b, count):
        pages = s["table"][b, :-(-count // PAGE)].long()
        return cache[pages].transpose(0, 1).reshape(kv, -1, d)[:, :count].double()

    if case["op"] == "mass":
        out = s["mass_out"].double()
        for b, x in enumerate(lens):
            q = s["q"][b].double().view(-1, kv, h // kv, d)
            lse = s["lse"][b].double().view(-1, kv, h // kv, 1)
            p = torch.exp(torch.einsum("nkgd,ktd->nkgt", q, tokens_of(s["k"], b, x)) / math.sqrt(d) - lse)
            if s["weights"] is not None:
                p = p * s["weights"][b].double()[:, None, None, None]
            out[b, :, :x] = p.sum((0, 2)) + (0 if s["mass"] is None else s["mass"][b, :, :x].double())
        return out
    n = case["nodes"]
    out = torch.zeros(B, n, h, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, n, h), -math.inf, dtype=torch.float64, device=DEVICE)
    words = s["mask"].tolist()
    for b, x in enumerate(lens):
        if x is None:
            continue
        k, v = tokens_of(s["k"], b, x + n), tokens_of(s["v"], b, x + n)
        for i in range(n):
            own_keys = [x + j for j in range(n) if words[b][i] >> j & 1]
            place = torch.cat([torch.arange(x), torch.tensor(own_keys, dtype=torch.long)]).to(DEVICE)
            score = torch.einsum("kgd,ktd->kgt", s["q"][b, i].double().view(kv, h // kv, d), k[:, place]) / math.sqrt(d)
            lse[b, i] = torch.logsumexp(score, 2).flatten()
            out[b, i] = torch.einsum("kgt,ktd->kgd", torch.softmax(score, 2), v[:, place]).reshape(h, d)
    return out, lse
