"""Timed cases of a rolling paged cache: the operators around long streams of video and text.

Three kinds of work, each one a part of serving a request whose sequences outgrow what a model attends to:

  window  attention of the newest 1 to 9 tokens of each sequence, which see the last ``window`` keys and the
          first ``sinks`` keys of the sequence (a draft or a target with a sliding window)
  rope    rotary positions of a call's queries and keys, and the append of the keys and values to the cache
  pages   the block tables of a paged cache: a tick reserves the pages that the next tokens are written to and
          frees those that fell out of the window; a fork lets sequences go on as several branches that share
          their pages, each with a copy of the page that it writes to next; a compaction moves the used pages
          to the front of the pool

``run`` makes the framework's calls where ``own`` is true, and computes the same from plain tensor operations
otherwise.  Sequences of a batch are ragged: their lengths follow from ``tokens`` and the batch index.  Head
shapes and lengths are those of the workloads and tests of this repository, or generic.
"""
import math

import numpy as np
import torch

own = False

HEADS = ((28, 4, 128), (64, 8, 128), (40, 8, 128), (8, 2, 64), (4, 1, 64))       # (query heads, KV heads, head_dim)
BASE = 1000000.0                                                                # of the rotary frequencies


def _window(name, layers, batch, heads, n_q, tokens, window, sinks, page):
    return dict(name=name, kind="window", layers=layers, batch=batch, q_heads=heads[0], kv_heads=heads[1],
                head_dim=heads[2], n_q=n_q, tokens=tokens, window=window, sinks=sinks, page=page)


def _rope(name, layers, batch, heads, n_new, tokens, page, rot_dim, interleaved, axes, scale, ragged, counted):
    return dict(name=name, kind="rope", layers=layers, batch=batch, q_heads=heads[0], kv_heads=heads[1],
                head_dim=heads[2], n_new=n_new, tokens=tokens, page=page, rot_dim=rot_dim, interleaved=interleaved,
                axes=axes, scale=scale, ragged=ragged, counted=counted)


def _pages(name, step, layers, heads, page, pool, batch, tokens, **more):
    return dict(name=name, kind="pages", step=step, layers=layers, kv_heads=heads[1], head_dim=heads[2], page=page,
                pool=pool, batch=batch, tokens=tokens, **more)


def listed():
    return [
        # a draft layer's decode call behind a 32-frame video: the smallest call of a layer-by-layer program
        _window("window-layer", 1, 1, HEADS[0], 1, 6400, 1024, 4, 0),
        # the draft step of all 28 layers for eight long streams, pages out of the window given back
        _window("window-draft", 28, 8, HEADS[0], 1, 50304, 2048, 64, 64),
        # one target layer's verification of a chain of five drafted tokens for four streams
        _window("window-verify-layer", 1, 4, HEADS[1], 6, 12672, 4096, 128, 64),
        # the same of twenty layers over a contiguous cache
        _window("window-verify", 20, 4, HEADS[1], 6, 8192, 4096, 4, 0),
        # a small model with a short window that no tile boundary fits
        _window("window-short", 6, 16, HEADS[3], 3, 5000, 333, 5, 64),
        # one token of one layer: what every layer of every draft step does first (the step's first layer has counted it)
        _rope("rope-token", 1, 1, HEADS[0], 1, 6400, 0, 128, False, 1, 1.0, False, True),
        # a verification window in all 28 layers of sixteen streams, positions of time, height and width
        _rope("rope-step", 28, 16, HEADS[0], 6, 6400, 64, 128, False, 3, 1.0, False, False),
        # one layer of the prompts of four streams, padded to the longest; half of each head is rotated, in
        # neighbouring pairs, with frequencies stretched for a context eight times as long
        _rope("rope-prompt", 1, 4, HEADS[1], 6528, 0, 64, 64, True, 1, 8.0, True, True),
        # a tick of 64 streams on a pool of 16 384 pages: six more tokens each, the window moves on
        _pages("pages-tick", "tick", 1, HEADS[4], 64, 16384, 64, 12500, n_new=6, window=4096, sinks=64),
        # two streams go on as sixteen branches of a draft with 28 layers
        _pages("pages-fork", "fork", 28, HEADS[0], 64, 256, 2, 6300, n_new=6, batch_out=16),
        # a small pool, half of it free in pieces
        _pages("pages-compact-small", "compact", 2, HEADS[3], 64, 300, 5, 1900),
        # the pool of a 28-layer draft after two thirds of its streams have ended
        _pages("pages-compact", "compact", 28, HEADS[0], 64, 900, 6, 4700),
    ]


_MOST = 1.2e9            # bytes of a drawn case, below the largest listed ones


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("window", "window", "rope", "rope", "tick", "fork", "compact"))
    heads = rng.choice(HEADS)
    layers, batch = _log(rng, 1, 28), _log(rng, 1, 16)
    if kind == "window":
        n_q = rng.choice((1, 1, 1, 2, 3, 6, 8, 9))
        window, sinks = _log(rng, 16, 8192), rng.choice((0, 1, 4, 33, 64, 200))
        c = _window("", layers, batch, heads, n_q, _log(rng, 64, 30000), window, sinks, rng.choice((0, 64, 64, 256)))
        full = c["page"] == 0                                # a contiguous cache keeps every row
        while c["layers"] > 1 and (work(c)["bytes"] > _MOST or full and _cache_bytes(c) > 4e9):
            c["layers"] -= 1
        while c["batch"] > 1 and (work(c)["bytes"] > _MOST or full and _cache_bytes(c) > 4e9):
            c["batch"] -= 1
    elif kind == "rope":
        rot = 16 * rng.randint(1, heads[2] // 16)
        c = _rope("", layers, batch, heads, _log(rng, 1, 6528), rng.choice((0, 1, 63, 700, 6400)), rng.choice((0, 64, 128)),
                  rot, rng.random() < 0.4, rng.choice((1, 3)) if rot >= 32 else 1, rng.choice((1.0, 4.0, 8.0)),
                  rng.random() < 0.5, rng.random() < 0.5)
        while c["layers"] > 1 and (work(c)["bytes"] > 9e8 or _cache_bytes(c) > 4e9):
            c["layers"] -= 1
        while c["batch"] > 1 and (work(c)["bytes"] > 9e8 or _cache_bytes(c) > 4e9):
            c["batch"] -= 1
    else:
        page = rng.choice((64, 128))
        tokens = _log(rng, 100, 12000)
        need = batch * (-(-tokens // page) + 2)
        if kind == "tick":
            c = _pages("", "tick", 1, rng.choice(HEADS[3:]), page, need + _log(rng, 16, 8000), batch, tokens,
                       n_new=_log(rng, 1, 700), window=_log(rng, 64, 8192), sinks=rng.choice((0, 1, 64, 100)))
            c["pool"] += batch * (c["n_new"] // page + 2)
        elif kind == "fork":
            out = _log(rng, 1, 32)
            c = _pages("", "fork", layers, heads, page, need + out * 3 + rng.randint(1, 50), batch, tokens,
                       n_new=_log(rng, 1, 9), batch_out=out)
        else:
            c = _pages("", "compact", layers, heads, page, 3 * need + rng.randint(0, 50), batch, tokens)
        while c["layers"] > 1 and _pool_bytes(c) > 3e9:
            c["layers"] -= 1
        if _pool_bytes(c) > 3e9:
            return draw(rng)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ shapes
def _ragged(tokens, batch):
    """Lengths of a batch: the first sequence is the longest, the others are down to a half shorter."""
    return [max(1, tokens - (b * 37 % 64) * tokens // 127) for b in range(batch)] if tokens else [0] * batch


def _new_lens(c):
    return [max(1, c["n_new"] - (b * 29 % 32) * c["n_new"] // 64) if c["ragged"] else c["n_new"] for b in range(c["batch"])]


def _capacity(c):
    return (c["tokens"] if c["kind"] == "window" else c["tokens"] + c["n_new"])


def _cache_bytes(c):
    return 4 * c["layers"] * c["batch"] * c["kv_heads"] * _capacity(c) * c["head_dim"]


def _pool_bytes(c):
    return 4 * c["layers"] * c["pool"] * c["kv_heads"] * c["page"] * c["head_dim"]


def _visible(c):
    """Keys that some query of each sequence sees."""
    n_vis = []
    for n in _ragged(c["tokens"], c["batch"]):
        lo = max(0, n - c["n_q"] - c["window"] + 1)
        n_vis.append(n - lo + min(c["sinks"], lo))
    return n_vis


def _parents(c):
    """Who goes on: branch i continues sequence i (i + 3) / 2 modulo the sequences, so that some have more branches."""
    return [i * (i + 3) // 2 % c["batch"] for i in range(c["batch_out"])]


def work(case):
    """Every row that the operator cannot do without read or written once; tables and counts with it."""
    c, D = case, case["head_dim"]
    if c["kind"] == "window":
        row, qrow, keys = c["kv_heads"] * D * 2, c["q_heads"] * D, sum(_visible(c))
        return {"bytes": c["layers"] * (2 * keys * row + c["batch"] * c["n_q"] * (4 * qrow + 4 * c["q_heads"])),
                "flops": 4 * c["layers"] * c["n_q"] * qrow * keys}
    if c["kind"] == "rope":
        new = sum(_new_lens(c)) * c["layers"]
        return {"bytes": new * (c["q_heads"] + 2 * c["kv_heads"]) * D * 4 + 4 * c["axes"] * sum(_new_lens(c)),
                "flops": new * 3 * (c["q_heads"] + c["kv_heads"]) * c["rot_dim"]}
    row = 4 * c["layers"] * c["kv_heads"] * D               # K and V of a token in all layers
    lens = _ragged(c["tokens"], c["batch"])
    held = sum(-(-n // c["page"]) for n in lens)
    if c["step"] == "tick":
        return {"bytes": 4 * c["pool"] + 8 * held, "flops": c["pool"]}
    if c["step"] == "fork":
        par = _parents(c)
        rows = sum((par.count(b) - 1) * (n % c["page"]) for b, n in enumerate(lens) if b in par)
        return {"bytes": 4 * c["pool"] + 4 * held + 4 * sum(-(-lens[p] // c["page"]) for p in par) + 2 * rows * row,
                "flops": c["pool"]}
    moved = held * (c["pool"] - held) // c["pool"]            # pages drawn at random: this many lie behind the first `held`
    return {"bytes": 8 * c["pool"] + 8 * held + 2 * moved * c["page"] * row, "flops": c["pool"]}


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 17)
    return g


def _randn(shape, g):
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    return x.normal_(generator=g)


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _frequencies(c):
    """Rotary frequencies (radians a position, 64 bits); with scale > 1 those of long waves are lowered by it and those
    between an eighth and a half of the trained context blended, as models stretched to longer contexts have them."""
    f = BASE ** (-torch.arange(0, c["rot_dim"], 2, dtype=torch.float64, device="cuda") / c["rot_dim"])
    if c["scale"] > 1.0:
        waves = 8192.0 * f / (2 * math.pi)                    # turns within the trained context
        keep = ((waves - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / c["scale"])
    return f


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=c)
    L, H, D = c["layers"], c["kv_heads"], c["head_dim"]
    rng = np.random.RandomState(seed % (1 << 31))
    lens = _ragged(c["tokens"], c["batch"])
    if c["kind"] != "pages":
        page, caps = c["page"], lens
        if c["kind"] == "rope":
            caps = [n + m for n, m in zip(lens, _new_lens(c))]
        s["max_len"] = max(caps)
        live = []
        for n in caps:
            blocks = set(range(-(-n // page))) if page else set()
            if page and c["kind"] == "window":               # pages out of sight have been given back
                lo = max(0, n - c["n_q"] - c["window"] + 1)
                blocks = {j for j in blocks if j * page < c["sinks"] or (j + 1) * page > lo}
            live.append(sorted(blocks))
        if page:
            pool = sum(map(len, live)) + 3
            order, table, at = rng.permutation(pool), np.full((c["batch"], -(-s["max_len"] // page)), -1, np.int32), 0
            for b, blocks in enumerate(live):
                table[b, blocks] = order[at:at + len(blocks)]
                at += len(blocks)
            s["table"], shape = _int(table), (L, pool, H, page, D)
        else:
            s["table"], shape = None, (L, c["batch"], H, s["max_len"], D)
        s["k"], s["v"] = _randn(shape, g), _randn(shape, g)
        s["lens"] = _int(lens)
    if c["kind"] == "window":
        shape = (L, c["batch"], c["n_q"], c["q_heads"])
        s["q"] = _randn(shape + (D,), g)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(shape, dtype=torch.float32, device="cuda")
        s["scale"] = 1.0 / math.sqrt(D)
    elif c["kind"] == "rope":
        # queries, keys and values lie side by side in the rows of one projection
        qkv = _randn((L, c["batch"], c["n_new"], c["q_heads"] + 2 * H, D), g)
        s["q"], s["new_k"], s["new_v"] = qkv.split((c["q_heads"], H, H), dim=3)
        s["q_out"] = torch.zeros((L, c["batch"], c["n_new"], c["q_heads"], D), dtype=torch.bfloat16, device="cuda")
        s["lens0"] = s["lens"].clone()
        if c["counted"]:
            s["lens"] += _int(_new_lens(c))
        s["new_lens"] = _int(_new_lens(c)) if c["ragged"] else None
        s["freq"] = _frequencies(c)
        half = c["rot_dim"] // 2
        s["sections"] = (half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8) if c["axes"] == 3 else None
        s["factor"] = 0.1 * math.log(c["scale"]) + 1.0
        s["positions"] = None
        if c["axes"] == 3:                                     # time, height and width run at paces of their own
            t = torch.arange(c["n_new"], device="cuda")
            x = torch.stack([t // 196, t % 196 // 14, t % 14])[:, None, :] + s["lens0"][None, :, None]
            s["positions"] = (x + int(rng.randint(0, 40000))).to(torch.int32).contiguous()
    elif c["kind"] == "pages":
        page, pool, B = c["page"], c["pool"], c["batch"]
        s["k"], s["v"] = (_randn((L, pool, H, page, D), g) for _ in range(2))
        more = c.get("n_new", 0)
        table = np.full((B, -(-(max(lens) + more) // page)), -1, np.int32)
        order, at = rng.permutation(pool), 0
        for b, n in enumerate(lens):
            need = -(-n // page)
            table[b, :need] = order[at:at + need]
            at += need
        s["table0"] = _int(table)
        ref = np.zeros(pool, np.int32)
        ref[order[:at]] = 1
        s["ref0"], s["lens"], s["max_len"] = _int(ref), _int(lens), max(lens) + more
        s["table"], s["ref"] = s["table0"].clone(), s["ref0"].clone()
        if c["step"] == "fork":
            s["parents"] = _int(_parents(c))
            s["table_out"] = torch.empty((c["batch_out"], table.shape[1]), dtype=torch.int32, device="cuda")
            s["lens_out"] = torch.empty(c["batch_out"], dtype=torch.int32, device="cuda")
        s["n_used"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_window(s):
    c = s["case"]
    L, B, n_q, Hq, D = s["q"].shape
    H, W, S = c["kv_heads"], c["window"], c["sinks"]
    n = s["lens"].long()[:, None]
    lo = (n - n_q - W + 1).clamp_min(0)
    reach = min(W + n_q - 1, s["max_len"])
    j = torch.cat([torch.arange(S, device="cuda").expand(B, S), lo + torch.arange(reach, device="cuda")], 1)
    there = j < n
    there[:, :S] &= j[:, :S] < lo                              # a sink inside the window counts once
    at = torch.where(there, j, n - 1)
    blk = torch.arange(B, device="cuda")[:, None].expand_as(at)
    if s["table"] is not None:
        blk, at = s["table"].long().gather(1, at // c["page"]), at % c["page"]
    p = n - n_q + torch.arange(n_q, device="cuda")             # position of each query
    j, p, there = j[:, None, :], p[:, :, None], there[:, None, :]
    seen = there & (j <= p) & ((j > p - W) | (j < S))          # [B][n_q][keys]
    k, v = (x[:, blk, :, at].permute(2, 0, 3, 1, 4).float() for x in (s["k"], s["v"]))       # [L][B][H][keys][D]
    q = s["q"].float().view(L, B, n_q, H, Hq // H, D).permute(0, 1, 3, 2, 4, 5)
    x = torch.matmul(q.reshape(L, B, H, -1, D), k.transpose(3, 4)) * s["scale"]
    x = x.view(L, B, H, n_q, Hq // H, -1).masked_fill(~seen[None, :, None, :, None, :], float("-inf"))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m.isinf(), torch.zeros_like(m), m)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(L, B, H, -1, e.shape[-1]), v).view(L, B, H, n_q, Hq // H, D) / total.clamp_min(1e-30)
    lse = (m + torch.log(total)).squeeze(-1)
    s["out"].copy_(o.permute(0, 1, 3, 2, 4, 5).reshape(L, B, n_q, Hq, D))
    s["lse"].copy_(lse.permute(0, 1, 3, 2, 4).reshape(L, B, n_q, Hq))
    return dict(out=s["out"], lse=s["lse"])


def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return y.to(torch.bfloat16)


def _plain_rope(s):
    c = s["case"]
    B, n = c["batch"], c["n_new"]
    t = torch.arange(n, device="cuda")
    start = s["lens0"].long()[:, None]
    count = s["new_lens"].long()[:, None] if s["new_lens"] is not None else torch.full((B, 1), n, device="cuda")
    real = t < count                                           # [B][n]
    half = c["rot_dim"] // 2
    if s["positions"] is None:
        pos = (start + t)[:, :, None].expand(B, n, half)
    else:
        axis = (torch.arange(half, device="cuda")[:, None] >= torch.tensor(s["sections"], device="cuda").cumsum(0)[:2]).sum(1)
        pos = s["positions"].permute(1, 2, 0)[:, :, axis]
    angle = pos.double() * s["freq"]
    cos, sin = ((f(angle) * s["factor"]).float()[None, :, :, None, :] for f in (torch.cos, torch.sin))
    q, k = (_rotate(x, cos, sin, c["rot_dim"], c["interleaved"]) for x in (s["q"], s["new_k"]))
    s["q_out"].copy_(torch.where(real[None, :, :, None, None], q, s["q_out"]))
    # rows of padding take the place, and the values, of their sequence's first new row
    first = torch.where(real, t, 0)
    b = torch.arange(B, device="cuda")[:, None].expand(B, n)
    at = start + first
    blk = b
    if s["table"] is not None:
        blk, at = s["table"].long().gather(1, at // c["page"]), at % c["page"]
    for_cache = [x.permute(1, 2, 0, 3, 4)[b, first] for x in (k, s["new_v"])]                # [B][n][L][H][D]
    s["k"][:, blk, :, at] = for_cache[0]
    s["v"][:, blk, :, at] = for_cache[1]
    if not c["counted"]:
        s["lens"] += count[:, 0]
    return dict(q=s["q_out"], k=s["k"], v=s["v"], lens=s["lens"])


def _plain_fork(s, page):
    table, lens, par, ref = s["table"].long(), s["lens"].long(), s["parents"].long(), s["ref"]
    B, M = table.shape
    takers = (par[None, :] == torch.arange(B, device="cuda")[:, None]).sum(1)
    kept = torch.arange(M, device="cuda") < ((lens + page - 1) // page)[:, None]
    change = torch.where(kept, takers[:, None] - 1, -1) * (table >= 0)
    ref.index_add_(0, table.clamp_min(0).view(-1), change.view(-1).to(torch.int32))
    s["table_out"].copy_(torch.where((par[:, None] >= 0) & kept[par.clamp_min(0)], table[par.clamp_min(0)], -1))
    s["lens_out"].copy_(torch.where(par >= 0, lens[par.clamp_min(0)], 0))


def _plain_reserve(s, table, lens, page, n_new):
    ref, (B, M), pool = s["ref"], table.shape, s["ref"].numel()
    old, n = table.long(), lens.long()
    first, j = n // page, torch.arange(M, device="cuda")
    inside = (j >= first[:, None]) & (j <= ((n + n_new - 1) // page)[:, None])
    held = ref.long()[old.clamp_min(0)]
    begun = (j == first[:, None]) & (n % page > 0)[:, None] & (old >= 0)
    # of the sequences that share the page they go on in, the last one keeps it
    mine = old.gather(1, first.clamp_max(M - 1)[:, None])[:, 0]
    writes = (n % page > 0) & (mine >= 0)
    b = torch.arange(B, device="cuda")
    before = ((mine[:, None] == mine[None, :]) & writes[None, :] & (b[None, :] < b[:, None])).sum(1)
    copies = writes & (ref.long()[mine.clamp_min(0)] - before > 1)
    fresh = inside & torch.where(begun, copies[:, None], (old < 0) | (held > 1))
    free = ref == 0
    place = torch.where(free, free.cumsum(0) - 1, pool)
    lowest = torch.zeros(pool + 1, dtype=torch.long, device="cuda").scatter_(0, place, torch.arange(pool, device="cuda"))
    fresh &= fresh.sum() <= free.sum()                         # all or nothing
    order = (fresh.view(-1).cumsum(0) - 1).view(B, M)
    new = torch.where(fresh, lowest[order.clamp(0, pool)], old)
    ref.index_add_(0, old.clamp_min(0).view(-1), -(fresh & (old >= 0)).view(-1).to(torch.int32))
    ref.index_add_(0, new.clamp_min(0).view(-1), fresh.view(-1).to(torch.int32))
    table.copy_(new)
    # the rows that the copied pages hold; a sequence that copies nothing writes its last page over itself
    at = torch.where(copies, first, (n - 1) // page)[:, None]
    src, dst = old.gather(1, at)[:, 0], new.gather(1, at)[:, 0]
    rows = (torch.arange(page, device="cuda") < (n % page)[:, None])[None, :, None, :, None]
    for x in (s["k"], s["v"]):
        x[:, dst] = torch.where(rows, x[:, src], x[:, dst])


def _plain_release(s, table, lens, page, window, sinks):
    ref, M = s["ref"], table.shape[1]
    old, n, j = table.long(), lens.long()[:, None], torch.arange(M, device="cuda")
    gone = (j * page >= n) | ((j * page >= sinks) & ((j + 1) * page <= n - window))
    gone &= old >= 0
    ref.index_add_(0, old.clamp_min(0).view(-1), -gone.view(-1).to(torch.int32))
    table.copy_(torch.where(gone, -1, old))


def _plain_compact(s):
    ref, pool = s["ref"], s["ref"].numel()
    used, i = ref > 0, torch.arange(pool, device="cuda")
    n_used = used.sum()
    hole, mover = ~used & (i < n_used), used & (i >= n_used)
    spare = torch.zeros(pool + 1, dtype=torch.long, device="cuda")
    h, m = hole.cumsum(0) - 1, mover.cumsum(0) - 1             # the i-th page behind the front fills the i-th hole
    holes = spare.scatter(0, torch.where(hole, h, pool), i)
    movers = spare.scatter(0, torch.where(mover, m, pool), i)
    to = torch.where(mover, holes[m.clamp_min(0)], i)
    source = torch.where(hole, movers[h.clamp_min(0)], i)
    old = s["table"].long()
    s["table"].copy_(torch.where(old >= 0, to[old.clamp_min(0)], old))
    ref.copy_(torch.where(i < n_used, ref[source], 0))
    for x in (s["k"], s["v"]):
        x.copy_(x[:, source])
    s["n_used"].copy_(n_used)


def _plain_pages(s):
    c = s["case"]
    if c["step"] == "tick":
        _plain_reserve(s, s["table"], s["lens"], c["page"], c["n_new"])
        _plain_release(s, s["table"], s["lens"], c["page"], c["window"], c["sinks"])
    elif c["step"] == "fork":
        _plain_fork(s, c["page"])
        _plain_reserve(s, s["table_out"], s["lens_out"], c["page"], c["n_new"])
    else:
        _plain_compact(s)


# ------------------------------------------------------------------------------------------ the framework's calls
def _handles(s):
    """What a program makes once beside its cache: the cache's descriptor, the rotation and the scratch memory."""
    from paper_2508_16201_b200 import specvlm
    if "cache" in s:
        return specvlm
    c = s["case"]
    s["cache"] = specvlm.KvCache(s["k"], s["v"], s["lens"], s["max_len"], s["table"])
    if c["kind"] == "window":
        nbytes = specvlm.window_attn_workspace_bytes(s["cache"], c["batch"], c["q_heads"], c["n_q"], c["window"], c["sinks"])
    elif c["kind"] == "rope":
        s["rope"] = specvlm.Rope(s["freq"], interleaved=c["interleaved"], factor=s["factor"], sections=s["sections"])
        return specvlm
    elif c["step"] == "fork":
        s["branches"] = specvlm.KvCache(s["k"], s["v"], s["lens_out"], s["max_len"], s["table_out"])
        nbytes = specvlm.pages_workspace_bytes(s["branches"], c["batch_out"])
    else:
        nbytes = specvlm.pages_workspace_bytes(s["cache"], c["batch"])
    s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda")
    return specvlm


def run(state):
    s, c = state, state["case"]
    # an append and a change of the tables start from the same sequences again
    if c["kind"] == "rope" and not c["counted"]:
        s["lens"].copy_(s["lens0"])
    elif c["kind"] == "pages":
        s["ref"].copy_(s["ref0"])
        s["table"].copy_(s["table0"])
    if not own:
        if c["kind"] == "window":
            return _plain_window(s)
        if c["kind"] == "rope":
            return _plain_rope(s)
        _plain_pages(s)
    else:
        specvlm = _handles(s)
        if c["kind"] == "window":
            specvlm.window_attn(s["cache"], s["q"], c["window"], c["sinks"], s["scale"], out=s["out"], lse=s["lse"], ws=s["ws"])
            return dict(out=s["out"], lse=s["lse"])
        if c["kind"] == "rope":
            specvlm.rope_append_kv(s["cache"], s["rope"], s["q"], s["new_k"], s["new_v"], q_out=s["q_out"],
                                   positions=s["positions"], new_lens=s["new_lens"], counted=c["counted"])
            return dict(q=s["q_out"], k=s["k"], v=s["v"], lens=s["lens"])
        if c["step"] == "tick":
            specvlm.reserve_pages(s["cache"], s["ref"], c["n_new"], ws=s["ws"])
            specvlm.release_pages(s["cache"], s["ref"], window=c["window"], n_sinks=c["sinks"])
        elif c["step"] == "fork":
            specvlm.fork_pages(s["cache"], s["ref"], s["parents"], s["table_out"], s["lens_out"])
            specvlm.reserve_pages(s["branches"], s["ref"], c["n_new"], ws=s["ws"])
        else:
            specvlm.compact_pages(s["cache"], s["ref"], n_used=s["n_used"], ws=s["ws"])
    if c["step"] == "fork":
        return dict(table=s["table_out"], lens=s["lens_out"], ref=s["ref"], k=s["k"], v=s["v"])
    if c["step"] == "tick":
        return dict(table=s["table"], ref=s["ref"])
    return dict(table=s["table"], ref=s["ref"], n_used=s["n_used"], k=s["k"], v=s["v"])


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """The computed outputs in 64 bits, from the definitions: one sequence and one layer after the other."""
    c = case
    if c["kind"] == "pages":
        return None                                            # tables, counts and copies: nothing is computed
    if c["kind"] == "window" and c["layers"] * c["batch"] * c["n_q"] > 6000:
        return None
    s = prepare(c, seed)
    L, B, H, D = c["layers"], c["batch"], c["kv_heads"], c["head_dim"]
    if c["kind"] == "window":
        group = c["q_heads"] // H
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, float("-inf"), dtype=torch.float64, device="cuda")
        for b, n in enumerate(_ragged(c["tokens"], B)):
            for t in range(c["n_q"]):
                p = n - c["n_q"] + t
                keys = [j for j in range(p + 1) if j < c["sinks"] or p - j < c["window"]]
                if not keys:
                    continue
                keys = torch.tensor(keys, device="cuda")
                for layer in range(L):
                    if s["table"] is None:
                        k, v = (x[layer, b, :, keys].double() for x in (s["k"], s["v"]))
                    else:
                        blk = s["table"][b, keys // c["page"]].long()
                        k, v = (x[layer, blk, :, keys % c["page"]].transpose(0, 1).double() for x in (s["k"], s["v"]))
                    q = s["q"][layer, b, t].double().view(H, group, D)
                    x = torch.einsum("hgd,hkd->hgk", q, k) * s["scale"]
                    out[layer, b, t] = torch.einsum("hgk,hkd->hgd", torch.softmax(x, -1), v).reshape(-1, D)
                    lse[layer, b, t] = torch.logsumexp(x, -1).reshape(-1)
        return dict(out=out, lse=lse)
    # one complex number a pair of channels, turned by exp(i angle)
    rot, half = c["rot_dim"], c["rot_dim"] // 2
    q_out, k, v = (s[x].double() for x in ("q_out", "k", "v"))
    parts = s["sections"] or (half,)
    for b, (n, m) in enumerate(zip(_ragged(c["tokens"], B), _new_lens(c))):
        rows = torch.arange(n, n + m, device="cuda")
        pos = s["positions"][:, b, :m].double() if c["axes"] == 3 else rows.double()[None]
        angle = torch.cat([pos[a][:, None] * f for a, f in enumerate(s["freq"].split(list(parts)))], 1)
        turn = torch.polar(torch.full_like(angle, s["factor"]), angle)[None, :, None, :]
        for x, is_q in ((s["q"], True), (s["new_k"], False)):
            y = x[:, b, :m].double()
            pairs = y[..., :rot].unflatten(-1, (half, 2) if c["interleaved"] else (2, half))
            z = torch.complex(*(pairs.unbind(-1) if c["interleaved"] else pairs.unbind(-2))) * turn
            y = torch.cat([torch.stack([z.real, z.imag], -1 if c["interleaved"] else -2).flatten(-2), y[..., rot:]], -1)
            if is_q:
                q_out[:, b, :m] = y
            else:
                blk, at = (s["table"][b, rows // c["page"]].long(), rows % c["page"]) if c["page"] else (b, rows)
                if c["page"]:
                    k[:, blk, :, at] = y.transpose(0, 1)
                    v[:, blk, :, at] = s["new_v"][:, b, :m].double().transpose(0, 1)
                else:
                    k[:, b, :, n:n + m] = y.transpose(1, 2)
                    v[:, b, :, n:n + m] = s["new_v"][:, b, :m].double().transpose(1, 2)
    return dict(q=q_out, k=k, v=v, lens=None)
