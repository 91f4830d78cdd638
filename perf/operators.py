"""The work that the decoder-layer operators around the verification attention are measured on.

Three operators that a program calls in every layer of a verification step:

* ``norm``: residual addition and root-mean-square norm, with bf16 output or
  8-bit (e4m3) output and scales (``add_rms_norm``);
* ``append``: rotation of the new queries and keys by positions with one or
  three axes, and the keys' and values' way into the paged cache
  (``kv_append``);
* ``shared``: verification attention of a batch whose sequences share long
  prefixes, each read once for its whole group (``shared_prefix_attention``).

Shapes follow the library's workloads (paper_2505_12728_gb300/workloads.py):
32/32 heads of 128 with 3008-token image prompts, 28/4 heads with 4864-token
video prompts and contexts of up to 32768 tokens, 8/8 heads of 64 as the small
one, drafts of 1 to 8 rows, hidden sizes 4096 and 3584.

With ``own`` false, `run` computes plain forms in elementary fp32 operations;
with ``own`` true it calls the library.
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
def _norm(**kw):
    c = dict(op="norm", T=5, d=4096, wide=False, residual=True, out="bf16", group=0)
    c.update(kw)
    return c


def _append(**kw):
    c = dict(op="append", prompt=False, B=1, rows=5, lo=3008, hi=3008, heads=32, kv_heads=32, d=128, rotary=128,
             interleaved=False, axes=1, wide=False, idle=0)
    c.update(kw)
    return c


def _shared(**kw):
    c = dict(op="shared", B=8, groups=1, rows=5, prefix_lo=3008, prefix_hi=3008, own_lo=20, own_hi=200, heads=32,
             kv_heads=32, d=128, idle=0)
    c.update(kw)
    return c


def listed():
    return [
        # the draft rows of one image chat between two layers: launch latency
        _norm(name="norm_step", T=5, d=4096),
        # the rows of 16 long-video sequences, 8-bit rows with a scale per 128
        # columns for an 8-bit projection
        _norm(name="norm_batch_8bit", T=128, d=3584, out="e4m3", group=128),
        # a projection's fp32 rows of an odd hidden size and a ragged number of
        # tokens onto an fp32 residual stream
        _norm(name="norm_odd_wide", T=1037, d=2187, wide=True),
        # the prompt of several long videos, 8-bit rows with one scale each
        _norm(name="norm_prompt_8bit", T=32768, d=3584, out="e4m3", group=0),
        # the draft rows of one image chat: latency
        _append(name="append_step", B=1, rows=5, lo=3008, hi=3008),
        # the draft rows of a batch of long videos, three position axes, two
        # slots of the captured batch idle
        _append(name="append_batch", B=16, rows=8, lo=8192, hi=32768, heads=28, kv_heads=4, axes=3, idle=2),
        # the prompts of eight videos of different lengths, three position axes
        _append(name="append_prompt", prompt=True, B=8, lo=1200, hi=8192, heads=28, kv_heads=4, axes=3),
        # ragged prompts of a small model that rotates half of each head in
        # neighbouring pairs, from a projection's fp32 rows
        _append(name="append_odd_wide", prompt=True, B=5, lo=97, hi=1203, heads=16, kv_heads=4, d=64, rotary=32,
                interleaved=True, wide=True),
        # two questions about one image, one token each: latency
        _shared(name="shared_tiny", B=2, rows=1, prefix_lo=640, prefix_hi=640, own_lo=9, own_hi=64, heads=8, kv_heads=8,
                d=64),
        # eight questions about one set of images, one KV head per query head
        _shared(name="shared_image", B=8, rows=5, prefix_lo=3008, prefix_hi=3008),
        # four videos with eight questions each, and two idle slots
        _shared(name="shared_video", B=32, groups=4, rows=8, prefix_lo=4000, prefix_hi=4864, own_lo=32, own_hi=512,
                heads=28, kv_heads=4, idle=2),
        # 64 questions or samples over one long video
        _shared(name="shared_long", B=64, rows=8, prefix_lo=32768, prefix_hi=32768, own_lo=64, own_hi=1024, heads=28,
                kv_heads=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "append", "shared", "shared"])
    if op == "norm":
        d = _log_int(rng, 64, 8192)
        if rng.random() < 0.7:
            d = max(64, d // 64 * 64)
        d += d == 3072
        T = _log_int(rng, 1, min(32768, 32768 * 3584 // d))
        out = rng.choice(["bf16", "e4m3"])
        return _norm(T=T, d=d, wide=rng.random() < 0.4, residual=rng.random() < 0.8, out=out,
                     group=rng.choice([0, 128]) if out == "e4m3" else 0)
    h, kv, d = rng.choice(HEADS)
    if op == "append":
        c = dict(heads=h, kv_heads=kv, d=d, rotary=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.3,
                 axes=rng.choice([1, 3]), wide=rng.random() < 0.3)
        if rng.random() < 0.5:
            most = 36864 * 36 * 128 // ((h + 2 * kv) * d * 3)
            lo = _log_int(rng, 1, 4096)
            hi = min(_log_int(rng, lo, 8192), most)
            return _append(prompt=True, B=_log_int(rng, 1, max(1, min(16, most // hi))), lo=min(lo, hi), hi=hi, **c)
        lo = _log_int(rng, 1, 16384)
        B = _log_int(rng, 1, 64)
        return _append(B=B, rows=rng.randint(1, 16), lo=lo, hi=_log_int(rng, lo, 32768), idle=rng.randint(0, B // 4), **c)
    B, rows = _log_int(rng, 1, 64), rng.randint(1, 8)
    hi = _log_int(rng, 1, 32768)
    lo = _log_int(rng, max(1, hi // 4), hi)
    own_lo = _log_int(rng, rows, 256)
    # at most the rows x keys of the longest listed case, and its cache
    hi = max(1, min(hi, 64 * 8 * 28 * 32768 // (B * rows * h), 16 * 4 * 32768 * 128 // (kv * d)))
    lo = min(lo, hi)
    groups = _log_int(rng, 1, min(B, 8))
    return _shared(B=B, groups=groups, rows=rows, prefix_lo=lo, prefix_hi=hi, own_lo=own_lo,
                   own_hi=_log_int(rng, own_lo, 1024), heads=h, kv_heads=kv, d=d, idle=rng.randint(0, B // 4))


# --------------------------------------------------------------------------- #
# sizes of a case (the same for every seed)                                   #
# --------------------------------------------------------------------------- #
def _lengths(case):
    """Prompt or context lengths, group sizes and the like, from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    B = case["B"]
    idle = set(rng.sample(range(B), case["idle"]))
    if case["op"] == "append":
        lens = [0 if b in idle else rng.randint(case["lo"], case["hi"]) for b in range(B)]
        if case["prompt"]:
            return dict(n=lens, before=[0] * B)
        return dict(n=[case["rows"]] * B, before=[None if b in idle else lens[b] for b in range(B)])
    cuts = sorted(rng.sample(range(1, B), case["groups"] - 1))
    starts = [0] + cuts + [B]
    prefix = [rng.randint(case["prefix_lo"], case["prefix_hi"]) for _ in range(case["groups"])]
    lo = max(case["own_lo"], case["rows"])
    lens = [0 if b in idle else rng.randint(lo, max(lo, case["own_hi"])) for b in range(B)]
    return dict(starts=starts, prefix=prefix, own=lens)


def work(case):
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        e = 4 if case["wide"] else 2
        move = T * d * (e + 2 * e * case["residual"] + (1 if case["out"] == "e4m3" else 2)) + 2 * d
        if case["out"] == "e4m3":
            move += 4 * T * (-(-d // case["group"]) if case["group"] else 1)
        return {"bytes": move, "flops": 6 * T * d}
    h, kv, d = case["heads"], case["kv_heads"], case["d"]
    s = _lengths(case)
    if case["op"] == "append":
        T = sum(s["n"])
        live = sum(n for n, b in zip(s["n"], s["before"]) if b is not None)
        e = 4 if case["wide"] else 2
        return {"bytes": T * h * d * (e + 2) + live * 2 * kv * d * (e + 2) + 4 * T * case["axes"],
                "flops": 3 * case["rotary"] * (T * h + live * kv)}
    keys = sum(s["prefix"]) + sum(s["own"])
    rows = flops = 0
    for g in range(case["groups"]):
        for b in range(s["starts"][g], s["starts"][g + 1]):
            if s["own"][b]:
                rows += case["rows"]
                flops += 4 * h * d * sum(s["prefix"][g] + s["own"][b] - i for i in range(case["rows"]))
    return {"bytes": keys * kv * d * 4 + rows * h * (4 * d + 4), "flops": flops}


# --------------------------------------------------------------------------- #
# inputs                                                                      #
# --------------------------------------------------------------------------- #
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _tables(counts, ids, width):
    """Block tables: each row's pages from the permutation `ids`, -1 after them."""
    t, at = [], 0
    for n in counts:
        t.append(ids[at:at + n] + [-1] * (width - n))
        at += n
    return t


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device=DEVICE).to(dtype)

    s = dict(op=case["op"])
    if case["op"] == "norm":
        T, d = case["T"], case["d"]
        kind = torch.float32 if case["wide"] else torch.bfloat16
        # a few channels carry values far above the others, as residual streams do
        loud = 1 + 30 * (torch.rand(d, generator=gen, device=DEVICE) < 0.004)
        s["x"] = normal(T, d, dtype=kind)
        s["residual"] = (3 * normal(T, d, dtype=torch.float32) * loud).to(kind) if case["residual"] else None
        s["weight"] = (1 + 0.2 * normal(d, dtype=torch.float32)).to(torch.bfloat16)
        s["eps"], s["group"] = 1e-6, case["group"]
        s["dtype"] = torch.float8_e4m3fn if case["out"] == "e4m3" else torch.bfloat16
        s["out"] = torch.empty(T, d, dtype=s["dtype"], device=DEVICE)
        s["residual_out"] = torch.empty_like(s["x"]) if case["residual"] else None
        s["scales"] = None
        if case["out"] == "e4m3":
            s["scales"] = torch.empty(T, -(-d // case["group"]) if case["group"] else 1, device=DEVICE)
        return s

    rng = random.Random(seed)
    h, kv, d = case["heads"], case["kv_heads"], case["d"]
    sizes = _lengths(case)
    if case["op"] == "append":
        n, before = sizes["n"], sizes["before"]
        total = [0 if b is None else b + m for b, m in zip(before, n)]
        pages = [-(-t // PAGE) for t in total]
        width = max(1, max(pages))
        # the cache holds the pages of the new rows; those of the tokens before
        # them are the same few, as nothing here reads them
        touched = [0 if b is None else p - b // PAGE for b, p in zip(before, pages)]
        pool = max(1, sum(touched) + 3)
        ids = rng.sample(range(pool), pool)
        t, at = [], 0
        for b in range(case["B"]):
            first = pages[b] - touched[b]
            t.append([ids[-1]] * first + ids[at:at + touched[b]] + [-1] * (width - pages[b]))
            at += touched[b]
        T = sum(n)
        kind = torch.float32 if case["wide"] else torch.bfloat16
        # q, k and v of a token lie side by side, as a fused projection leaves them
        qkv = normal(T, (h + 2 * kv) * d, dtype=kind)
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in qkv.split([h * d, kv * d, kv * d], 1))
        s["k_cache"], s["v_cache"] = normal(pool, kv, PAGE, d), normal(pool, kv, PAGE, d)
        s["block_table"], s["seq_lens"] = _ints(t), _ints(total)
        s["rows"] = None if case["prompt"] else case["rows"]
        starts = [0]
        for m in n:
            starts.append(starts[-1] + m)
        s["row_starts"] = _ints(starts)
        half = case["rotary"] // 2
        s["inv_freq"] = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEVICE) / half)
        row = torch.arange(T, device=DEVICE)
        seq = torch.searchsorted(s["row_starts"][1:].long(), row, right=True)
        at = row - s["row_starts"].long()[seq] + _ints([b or 0 for b in before]).long()[seq]
        if case["axes"] == 3:
            # frames of 12 x 12 visual tokens, then nothing else: time, height, width
            s["positions"] = torch.stack([at // 144, at % 144 // 12, at % 12]).to(torch.int32)
            s["axis"] = _ints([0] * (half // 4) + [1] * (half * 3 // 8) + [2] * (half - half // 4 - half * 3 // 8))
        else:
            s["positions"], s["axis"] = at.to(torch.int32)[None], None
        s["interleaved"] = case["interleaved"]
        s["q_out"] = torch.empty(T, h, d, dtype=torch.bfloat16, device=DEVICE)
        if own:
            from paper_2505_12728_gb300 import specflash_verify as sfv
            s["workspace"] = sfv.new_workspace(sfv.kv_append_workspace_size())
        return s

    B, n, G = case["B"], case["rows"], case["groups"]
    p_pages = [-(-x // PAGE) for x in sizes["prefix"]]
    o_pages = [-(-x // PAGE) for x in sizes["own"]]
    pool = sum(p_pages) + sum(o_pages) + 3
    ids = rng.sample(range(pool), pool)
    s["q"] = normal(B, n, h, d)
    s["k_cache"], s["v_cache"] = normal(pool, kv, PAGE, d), normal(pool, kv, PAGE, d)
    s["prefix_table"] = _ints(_tables(p_pages, ids, max(p_pages)))
    s["block_table"] = _ints(_tables(o_pages, ids[sum(p_pages):], max(1, max(o_pages))))
    s["prefix_lens"], s["group_starts"], s["seq_lens"] = _ints(sizes["prefix"]), _ints(sizes["starts"]), _ints(sizes["own"])
    s["most"] = max(b - a for a, b in zip(sizes["starts"], sizes["starts"][1:]))  # the largest group
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(B, n, h, device=DEVICE)
    if own:
        from paper_2505_12728_gb300 import specflash_verify as sfv
        s["workspace"] = sfv.new_workspace(sfv.shared_prefix_attention_workspace_size(
            B, n, h, kv, d, G, s["prefix_table"].shape[1], s["block_table"].shape[1]))
    return s


# --------------------------------------------------------------------------- #
# one pass                                                                    #
# --------------------------------------------------------------------------- #
def run(s):
    if own:
        return _library(s)
    return {"norm": _plain_norm, "append": _plain_append, "shared": _plain_shared}[s["op"]](s)


def _library(s):
    from paper_2505_12728_gb300 import specflash_verify as sfv
    if s["op"] == "norm":
        return sfv.add_rms_norm(s["x"], s["weight"], s["residual"], eps=s["eps"], group=s["group"], out=s["out"],
                                residual_out=s["residual_out"], scales=s["scales"])
    if s["op"] == "append":
        q = sfv.kv_append(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["k_cache"], s["v_cache"],
                          s["block_table"], s["seq_lens"], axis=s["axis"],
                          row_starts=s["row_starts"] if s["rows"] is None else None, interleaved=s["interleaved"],
                          q_out=s["q_out"], workspace=s["workspace"])
        return q, s["k_cache"], s["v_cache"]
    return sfv.shared_prefix_attention(s["q"], s["k_cache"], s["v_cache"], s["prefix_table"], s["prefix_lens"],
                                       s["group_starts"], s["block_table"], s["seq_lens"], out=s["out"], lse=s["lse"],
                                       workspace=s["workspace"])


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + s["eps"]) * s["weight"].float()
    r = None if s["residual"] is None else h.to(s["x"].dtype)
    if s["scales"] is None:
        return y.to(s["dtype"]), r, None
    T, d = y.shape
    width = s["group"] or d
    parts = torch.nn.functional.pad(y, (0, -d % width)).view(T, -1, width)
    scales = (parts.abs().amax(2) / 448).clamp(min=2.0 ** -126)
    out = (parts / scales[..., None]).view(T, -1)[:, :d].clamp(-448, 448)
    return out.to(s["dtype"]), r, scales


def _plain_rotate(x, cos, sin, interleaved):
    half = cos.shape[1]
    turn, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if interleaved else (turn[..., :half], turn[..., half:])
    cos, sin = cos[:, None], sin[:, None]
    a, b = a * cos - b * sin, a * sin + b * cos
    turn = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turn, rest], -1)


def _plain_append(s):
    f = s["inv_freq"].float()
    at = s["positions"].float()
    angle = at[0][:, None] * f if s["axis"] is None else at[s["axis"].long()].t() * f
    cos, sin = angle.cos(), angle.sin()
    q = _plain_rotate(s["q"].float(), cos, sin, s["interleaved"]).to(torch.bfloat16)
    k = _plain_rotate(s["k"].float(), cos, sin, s["interleaved"]).to(torch.bfloat16)
    v = s["v"].to(torch.bfloat16)
    starts, lens = s["row_starts"].long(), s["seq_lens"].long()
    row = torch.arange(q.shape[0], device=DEVICE)
    seq = torch.searchsorted(starts[1:], row, right=True)
    place = lens[seq] - starts[seq + 1] + row
    place = torch.where(lens[seq] > 0, place, -1)
    keep = (place >= 0).nonzero()[:, 0]  # the rows of idle slots are not written
    seq, place = seq[keep], place[keep]
    page = s["block_table"].long()[seq, place // PAGE]
    s["k_cache"][page, :, place % PAGE] = k[keep]
    s["v_cache"][page, :, place % PAGE] = v[keep]
    return q, s["k_cache"], s["v_cache"]


def _pages(cache, table):
    """The tokens of each row of a block table, [rows][heads][tokens][d] in fp32."""
    x = cache[table.clamp(min=0).long()].float()  # [rows][pages][heads][16][d]
    return x.transpose(1, 2).flatten(2, 3)


def _plain_shared(s):
    q = s["q"].float()
    B, n, h, d = q.shape
    kv = s["k_cache"].shape[1]
    R = n * (h // kv)
    starts, lens = s["group_starts"].long(), s["seq_lens"].long()
    G = starts.shape[0] - 1
    b = torch.arange(B, device=DEVICE)
    group = torch.searchsorted(starts[1:], b, right=True)
    slot = b - starts[group]
    # rows of a sequence and KV head: [B][kv][n * heads per KV head][d]
    q = q.view(B, n, kv, h // kv, d).transpose(1, 2).reshape(B, kv, R, d) * d ** -0.5
    # the prefix: the queries of a group against its keys, in one product
    kp, vp = _pages(s["k_cache"], s["prefix_table"]), _pages(s["v_cache"], s["prefix_table"])
    Lp = kp.shape[2]
    grouped = q.new_zeros(G, s["most"], kv, R, d)
    grouped[group, slot] = q
    sp = grouped.transpose(1, 2).reshape(G, kv, -1, d) @ kp.transpose(2, 3)
    sp = sp.masked_fill(torch.arange(Lp, device=DEVICE) >= s["prefix_lens"][:, None, None, None], -math.inf)
    sp = sp.view(G, kv, s["most"], R, Lp).transpose(1, 2)[group, slot]
    # the sequence's own tokens, draft row i up to its own position
    ko, vo = _pages(s["k_cache"], s["block_table"]), _pages(s["v_cache"], s["block_table"])
    Lo = ko.shape[2]
    last = lens[:, None] - n + torch.arange(n, device=DEVICE)
    last = last.repeat_interleave(h // kv, 1)[:, None, :, None]
    so = (q @ ko.transpose(2, 3)).masked_fill(torch.arange(Lo, device=DEVICE) > last, -math.inf)
    idle = (lens == 0)[:, None, None, None]
    m = torch.maximum(sp.amax(3, keepdim=True), so.amax(3, keepdim=True))
    pp, po = (sp - m).exp(), (so - m).exp()
    l = pp.sum(3, keepdim=True) + po.sum(3, keepdim=True)
    back = q.new_zeros(G, s["most"], kv, R, Lp)
    back[group, slot] = pp
    o = (back.transpose(1, 2).reshape(G, kv, -1, Lp) @ vp).view(G, kv, s["most"], R, d).transpose(1, 2)[group, slot]
    o = ((o + po @ vo) / l).masked_fill(idle, 0)
    lse = (m + l.log()).masked_fill(idle, -math.inf)
    out = o.view(B, kv, n, h // kv, d).transpose(1, 2).reshape(B, n, h, d).to(torch.bfloat16)
    return out, lse.view(B, kv, n, h // kv).transpose(1, 2).reshape(B, n, h)


# --------------------------------------------------------------------------- #
# the definitions in 64 bits                                                  #
# --------------------------------------------------------------------------- #
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
        y = h / ((h * h).sum(1, keepdim=True) / case["d"] + s["eps"]).sqrt() * s["weight"].double()
        r = None if s["residual"] is None else h
        if case["out"] == "bf16":
            return y, r, None
        w = case["group"] or case["d"]
        tops = torch.stack([c.abs().amax(1) for c in y.split(w, 1)], 1) / 448
        # the values before their rounding to 8 bits
        return y / tops.repeat_interleave(w, 1)[:, :case["d"]], r, tops
    sizes = _lengths(case)
    if case["op"] == "append":
        half = case["rotary"] // 2
        axis = [0] * half if s["axis"] is None else s["axis"].tolist()
        angle = torch.stack([s["positions"][a].double() * s["inv_freq"][j] for j, a in enumerate(axis)], 1)
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        rotated = []
        for x in (s["q"], s["k"]):
            x = x.double()
            y = x.clone()
            first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else \
                (slice(0, half), slice(half, 2 * half))
            z = torch.complex(x[..., first], x[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            rotated.append(y)
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        table, at = s["block_table"].tolist(), 0
        for b, (m, before) in enumerate(zip(sizes["n"], sizes["before"])):
            if before is not None and m:
                place = range(before, before + m)
                page = torch.tensor([table[b][t // PAGE] for t in place], device=DEVICE)
                slot = torch.tensor([t % PAGE for t in place], device=DEVICE)
                kc[page, :, slot] = rotated[1][at:at + m]
                vc[page, :, slot] = s["v"][at:at + m].double()
            at += m
        return rotated[0], kc, vc
    B, n, h, kv, d = case["B"], case["rows"], case["heads"], case["kv_heads"], case["d"]
    out = torch.zeros(B, n, h, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((B, n, h), -math.inf, dtype=torch.float64, device=DEVICE)
    for g in range(case["groups"]):
        P = sizes["prefix"][g]
        for b in range(sizes["starts"][g], sizes["starts"][g + 1]):
            L = sizes["own"][b]
            if not L:
                continue
            tokens = [c[torch.cat([s["prefix_table"][g, :-(-P // PAGE)], s["block_table"][b, :-(-L // PAGE)]]).long()]
                      for c in (s["k_cache"], s["v_cache"])]
            pad = -P % PAGE
            k, v = (t.transpose(0, 1).reshape(kv, -1, d) for t in tokens)
            k, v = (torch.cat([t[:, :P], t[:, P + pad:P + pad + L]], 1).double() for t in (k, v))
            for i in range(n):
                end = P + L - n + i + 1
                x = s["q"][b, i].double().view(kv, h // kv, d)
                score = torch.einsum("kgd,ktd->kgt", x, k[:, :end]) / math.sqrt(d)
                lse[b, i] = torch.logsumexp(score, 2).flatten()
                out[b, i] = torch.einsum("kgt,ktd->kgd", torch.softmax(score, 2), v[:, :end]).reshape(h, d)
    return out, lse
