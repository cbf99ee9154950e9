"""Timed cases of the operators that keep a sequence's cache bounded: norms and
rotary positions of new queries and keys on their way into the blocks,
attention in a sliding window behind a few first tokens, the weight that each
cached token got, and eviction of the tokens with the least.

A case's lengths follow from the case alone, and its data from the seed.  The
plain forms are elementary torch operations in 32 bits (angles in 64).
"""

import math
import random

import torch

own = False

NONE = -1  # a table entry that names no block (0xFFFFFFFF as a 32-bit pattern)


# ------------------------------------------------------------------ cases


def _rows(name, op, heads, group, dim, seqs, new, cached, **more):
    """``heads`` KV heads of ``dim``, each serving ``group`` query heads;
    ``seqs`` sequences of new[0]..new[1] rows after cached[0]..cached[1]
    tokens."""
    c = dict(name=name, op=op, layers=1, layer=0, block_size=16, heads=heads, group=group, dim=dim,
             e4m3=False, seqs=seqs, new_lo=new[0], new_hi=new[1], cached_lo=cached[0],
             cached_hi=cached[1], salt=1)
    c.update(more)
    return c


def _evict(name, geometry, seqs, tokens, keep, sinks, recent, **more):
    """``seqs`` sequences of tokens[0]..tokens[1] over blocks of (layers, block
    size, heads, dim, element bytes), each cut to ``keep`` tokens; ``children``
    more of them share their parents' full blocks."""
    layers, block_size, heads, dim, elem_bytes = geometry
    c = dict(name=name, op="evict", layers=layers, block_size=block_size, heads=heads, dim=dim,
             elem_bytes=elem_bytes, seqs=seqs, tokens_lo=tokens[0], tokens_hi=tokens[1], keep=keep,
             sinks=sinks, recent=recent, children=0, salt=1)
    c.update(more)
    return c


def listed():
    return [
        # one layer of one decoding step: a token for each of 48 running sequences, whose
        # positions are kept apart from the cache's length
        _rows("rotate-step", "rotate", 8, 4, 128, 48, (1, 1), (0, 4000), rot=128, norm=True, axes=1),
        # one layer of a prefill batch with pictures in it: time, height and width, e4m3 blocks
        _rows("rotate-prompts-axes-e4m3", "rotate", 4, 7, 128, 24, (100, 1500), (0, 0), e4m3=True,
              k_scale=0.031, v_scale=0.017, rot=128, norm=True, axes=3),
        # one long document of a model that rotates half of each head, in neighbouring pairs,
        # without norms
        _rows("rotate-prompt-long", "rotate", 8, 4, 64, 1, (16384, 16384), (0, 0), rot=32, norm=False,
              axes=0, interleaved=True),
        # a demo's decoding step
        _rows("window-few", "window", 2, 2, 64, 4, (1, 1), (0, 400), window=64, sinks=4),
        # 64 long chats in a window of 4096 tokens
        _rows("window-step-64", "window", 8, 4, 128, 64, (1, 1), (2000, 12000), window=4096, sinks=4,
              lse=True),
        # one long document through a layer with a window of 4096
        _rows("window-prompt-long", "window", 8, 4, 128, 1, (16384, 16384), (0, 0), window=4096, sinks=4),
        # ragged prompts after cached tokens, a short window, e4m3 blocks
        _rows("window-prompts-e4m3", "window", 4, 7, 128, 12, (33, 1500), (0, 4000), e4m3=True,
              k_scale=0.031, v_scale=0.017, window=1000, sinks=20, lse=True),
        # a demo's step: what its cached tokens got
        _rows("weigh-few", "weigh", 2, 2, 64, 4, (1, 1), (0, 400), window=0, sinks=0),
        # the same for one layer of 64 running sequences
        _rows("weigh-step-64", "weigh", 8, 4, 128, 64, (1, 1), (100, 8192), window=0, sinks=0),
        # a prompt's weights, all of its rows over all of its tokens
        _rows("weigh-prompt", "weigh", 8, 4, 128, 1, (8192, 8192), (0, 0), window=0, sinks=0),
        # a demo's pool, forked samples among the sequences
        _evict("evict-few", (2, 16, 2, 64, 2), 3, (60, 200), 64, 4, 16, children=2),
        # 8 chats over 16 layers of 8B-shaped blocks are cut to 2048 tokens
        _evict("evict-chats", (16, 16, 8, 128, 2), 8, (1900, 4000), 2048, 4, 256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: 1 to 8 KV heads of 64 or 128, 1 to 16
    query heads to each, blocks of 8 to 64 tokens in bf16 and e4m3, 1 to 64
    sequences, up to 16384 rows and 32768 tokens, windows of 16 to 8192."""
    op = rng.choice(["rotate", "window", "window", "weigh", "weigh", "evict"])
    salt = rng.randrange(1 << 30)
    if op == "evict":
        geometry = (_log_int(rng, 1, 32), rng.choice([8, 16, 16, 24, 64]), rng.choice([1, 2, 4, 8]),
                    rng.choice([64, 128]), rng.choice([1, 2]))
        token = 2 * geometry[0] * geometry[2] * geometry[3] * geometry[4]
        seqs = _log_int(rng, 1, 32)
        children = rng.choice([0, 0, 1, seqs])
        hi = max(40, min(_log_int(rng, 64, 16384), (1 << 30) // (token * (seqs + children))))
        keep = rng.randint(hi // 4, hi * 3 // 4)
        sinks = rng.choice([0, 1, 4, 16])
        sinks = min(sinks, keep // 2)
        return _unnamed(_evict("", geometry, seqs, (hi // 2, hi), keep, sinks,
                               rng.randint(0, keep - sinks), salt=salt,
                               children=children))
    more = dict(block_size=rng.choice([8, 16, 16, 16, 24, 32, 64]), salt=salt)
    if rng.random() < 0.4:
        more.update(e4m3=True, k_scale=rng.uniform(0.02, 0.05), v_scale=rng.uniform(0.01, 0.03))
    heads, group, dim = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16]), rng.choice([64, 128, 128])
    seqs = _log_int(rng, 1, 64)
    if rng.random() < 0.4:  # a decoding step
        new = (1, 1)
        cached_hi = _log_int(rng, 1, min(16384, 400000 // seqs))
    else:
        new_hi = _log_int(rng, 2, 16384 // seqs)
        cached_hi = 0 if rng.random() < 0.5 else _log_int(rng, 1, 32768 // seqs)
        new = (max(1, new_hi // 8), new_hi)
    if op == "rotate":
        more.update(rot=rng.choice([dim, dim, dim // 2, 16]), norm=rng.random() < 0.6,
                    axes=rng.choice([0, 1, 2, 3, 4]), interleaved=rng.random() < 0.3)
    else:
        if op == "window" or rng.random() < 0.3:
            more.update(window=_log_int(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 20, 100]))
        else:
            more.update(window=0, sinks=0)
        if op == "window":
            more.update(lse=rng.random() < 0.5)
        new_hi = new[1]
        most = 1e9 if op == "weigh" else 2e9
        while heads * group * seqs * new_hi * min(new_hi / 2 + cached_hi, more["window"] or 1e9) > most:
            new_hi, cached_hi = new_hi * 2 // 3 + 1, cached_hi * 2 // 3
        new = (min(new[0], new_hi), new_hi)
    return _unnamed(_rows("", op, heads, group, dim, seqs, new, (0, cached_hi), **more))


def _unnamed(c):
    del c["name"]
    return c


def _lengths(c):
    """(rows, tokens cached before them) of each sequence."""
    r = random.Random(c["salt"])
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["seqs"])]
    return new, [r.randint(c["cached_lo"], c["cached_hi"]) for _ in range(c["seqs"])]


def _held(c):
    """Tokens of each sequence, and the parents of those after the first ones."""
    r = random.Random(c["salt"])
    got = [r.randint(c["tokens_lo"], c["tokens_hi"]) for _ in range(c["seqs"])]
    parents = [r.randrange(c["seqs"]) for _ in range(c["children"])]
    return got + [got[p] for p in parents], parents


def _cdiv(a, b):
    return -(-a // b)


# ------------------------------------------------------------------ inputs


def _handle(s, c, blocks):
    """What a serving program keeps: the pool's handle and its sequences."""
    from paper_2606_01387_amd import claimkv, sequences
    from paper_2606_01387_amd.synth import Geometry

    geometry = Geometry(c["layers"], 2, c["block_size"], c["heads"], c["dim"],
                        c.get("elem_bytes", 1 if c.get("e4m3") else 2), blocks)
    pool = claimkv.Pool(geometry, 7, s["kv"].view(torch.uint8), max_claims=256, max_footprint=1 << 14,
                        event_capacity=1 << 10)
    s["pool"] = pool
    s["seqs"] = sequences.Sequences(pool, tables=s["tables"], lengths=s["lengths"], refs=s["refs"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_evict if case["op"] == "evict" else _prepare_rows)(case, g)


def _prepare_rows(c, g):
    dev = "cuda"
    H, G, D, bs = c["heads"], c["group"], c["dim"], c["block_size"]
    new, cached = _lengths(c)
    total = [n + m for n, m in zip(new, cached)]
    need = [_cdiv(t, bs) for t in total]
    used = sum(need)
    blocks = used + used // 8 + 8
    perm = torch.randperm(blocks, generator=g, device=dev)[:used].to(torch.int32)
    tables = torch.full((c["seqs"], max(need)), NONE, device=dev, dtype=torch.int32)
    inside = torch.arange(max(need), device=dev)[None] < torch.tensor(need, device=dev)[:, None]
    tables[inside] = perm
    lengths = torch.tensor(total, device=dev, dtype=torch.int32)
    refs = torch.zeros(blocks, device=dev, dtype=torch.int32)
    refs[perm.long()] = 1
    offsets = torch.zeros(c["seqs"] + 1, device=dev, dtype=torch.int32)
    offsets[1:] = torch.cumsum(torch.tensor(new, device=dev), 0)
    T = sum(new)

    # keys have a few large channels, as rotary keys do
    chan = 1 + 3 * (torch.rand(D, generator=g, device=dev) < 0.06).float()
    kv = torch.empty(2 * c["layers"], blocks, bs, H, D, device=dev, dtype=torch.bfloat16)
    kv.normal_(generator=g)
    kv[0::2] *= chan.to(torch.bfloat16)
    if c["e4m3"]:
        kv[0::2] *= 0.5 / c["k_scale"] / 16
        kv[1::2] *= 0.5 / c["v_scale"] / 16
        kv = kv.to(torch.float8_e4m3fn)
    s = dict(c, kv=kv, tables=tables, lengths=lengths, refs=refs, offsets=offsets, new=new, total=total,
             k_scale=c.get("k_scale", 1.0), v_scale=c.get("v_scale", 1.0))
    if c["op"] == "rotate":
        # a slice of one fused projection, as a layer has them
        qkv = torch.empty(T, (G + 2) * H * D, device=dev, dtype=torch.bfloat16).normal_(generator=g)
        s["q"] = qkv[:, :G * H * D].view(T, G * H, D)
        s["k"] = qkv[:, G * H * D:(G + 1) * H * D].view(T, H, D)
        s["v"] = qkv[:, (G + 1) * H * D:].view(T, H, D)
        half = c["rot"] // 2
        s["freqs"] = 500000.0 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        s["q_norm"] = s["k_norm"] = s["positions"] = s["sections"] = None
        if c["norm"]:
            s["q_norm"], s["k_norm"] = (
                (1 + 0.2 * torch.randn(D, generator=g, device=dev)).to(torch.bfloat16) for _ in range(2))
        if c["axes"]:
            # positions past the cache's length, as after evictions
            far = torch.randint(0, 100000, (T, 1), generator=g, device=dev)
            near = torch.randint(0, 64, (T, c["axes"]), generator=g, device=dev)
            s["positions"] = (far + near).to(torch.int32)
            s["sections"] = _sections(c)
        s["row_seq"], s["row_pos"] = _row_places(s)
    else:
        s["q"] = (1.5 * torch.randn(T, H * G, D, generator=g, device=dev)).to(torch.bfloat16)
        if c["op"] == "weigh":
            s["weights"] = torch.zeros(c["seqs"], max(need) * bs, device=dev)
            s["lse"] = _row_sums(s)
    if own:
        _handle(s, c, blocks)
    return s


def _sections(c):
    """Pairs of each axis: the first axis has what is left."""
    half, n = c["rot"] // 2, c["axes"]
    rest = half * 3 // (4 * (n - 1)) if n > 1 else 0
    return (half - rest * (n - 1),) + (rest,) * (n - 1)


def _row_places(s):
    """Each packed row's sequence and position."""
    offsets, rows = s["offsets"].long(), s["q"].shape[0]
    at = torch.arange(rows, device=offsets.device)
    seq = torch.searchsorted(offsets, at, right=True) - 1
    return seq, s["lengths"].long()[seq] - offsets[seq + 1] + at


def _prepare_evict(c, g):
    dev, bs = "cuda", c["block_size"]
    held, parents = _held(c)
    n, seqs = len(held), c["seqs"]
    need = [_cdiv(t, bs) for t in held]
    # children share full blocks and have a last one of their own
    fresh = [need[i] if i < seqs else need[i] - held[i] // bs for i in range(n)]
    used, spare = sum(fresh), sum(_cdiv(c["keep"], bs) for _ in held) if parents else 0
    nb = used + used // 8 + 8 + spare
    kv = torch.randint(-2**62, 2**62, (2 * c["layers"], nb, bs, c["heads"] * c["dim"] * c["elem_bytes"] // 8),
                       generator=g, device=dev)
    wide = max(need)
    perm = torch.randperm(nb, generator=g, device=dev)[:used].to(torch.int32)
    tables = torch.full((n, wide), NONE, device=dev, dtype=torch.int32)
    col = torch.arange(wide, device=dev)
    first = sum(fresh[:seqs])
    tables[:seqs][col < torch.tensor(need[:seqs], device=dev)[:, None]] = perm[:first]
    at = first
    for i, p in enumerate(parents, seqs):
        full = held[i] // bs
        tables[i, :full] = tables[p, :full]
        tables[i, full:full + fresh[i]] = perm[at:at + fresh[i]]
        at += fresh[i]
    refs = torch.zeros(nb + 1, device=dev, dtype=torch.int32)
    named = tables.flatten().long()
    refs = refs.scatter_add_(0, named.where(named >= 0, nb), torch.ones_like(named, dtype=torch.int32))[:-1].clone()
    # accumulated weights have a heavy tail, and some tokens got nothing yet
    weights = torch.exp(2 * torch.randn(n, wide * bs, generator=g, device=dev))
    weights[torch.rand(n, wide * bs, generator=g, device=dev) < 0.1] = 0
    lengths = torch.tensor(held, device=dev, dtype=torch.int32)
    s = dict(c, kv=kv, tables=tables, lengths=lengths, refs=refs, weights=weights, n=n,
             before=[x.clone() for x in (tables, lengths, refs, weights)])
    if own:
        _handle(s, c, nb)
    return s


# ------------------------------------------------------------------ one pass


def run(state):
    return (_run_own if own else _run_plain)(state)


def _restore(s):
    """An eviction's own state as it was, so that a pass can be made again."""
    for name, x in zip(("tables", "lengths", "refs", "weights"), s["before"]):
        s[name].copy_(x)


def _run_own(s):
    q = s["seqs"]
    if s["op"] == "rotate":
        out = q.write_rotated(s["layer"], s["q"], s["k"], s["v"], s["freqs"], positions=s["positions"],
                              sections=s["sections"], q_norm=s["q_norm"], k_norm=s["k_norm"],
                              neighbours=s.get("interleaved", False), offsets=s["offsets"],
                              k_scale=s["k_scale"], v_scale=s["v_scale"])
        return out, s["kv"]
    if s["op"] == "window":
        lse = torch.empty(s["q"].shape[:2], device="cuda") if s.get("lse") else None
        out = q.attend_window(s["layer"], s["q"], s["window"], sinks=s["sinks"], offsets=s["offsets"],
                              k_scale=s["k_scale"], v_scale=s["v_scale"], lse=lse)
        return (out, lse) if s.get("lse") else out
    if s["op"] == "weigh":
        s["weights"].zero_()
        q.weigh(s["layer"], s["q"], s["lse"], s["weights"], window=s["window"] or None, sinks=s["sinks"],
                offsets=s["offsets"], k_scale=s["k_scale"])
        return s["weights"]
    _restore(s)
    status, kept = q.evict(None, s["weights"], s["keep"], sinks=s["sinks"], recent=s["recent"])
    return s["kv"], s["tables"], s["lengths"], s["refs"], s["weights"], status, kept


def _run_plain(s):
    if s["op"] == "rotate":
        return _plain_rotate(s)
    if s["op"] == "window":
        return _plain_window(s)
    if s["op"] == "weigh":
        s["weights"].zero_()
        return _plain_weigh(s)
    _restore(s)
    return _plain_evict(s)


def _plain_rotate(s):
    T, half = s["q"].shape[0], s["rot"] // 2
    pos = s["row_pos"][:, None].expand(T, half)
    if s["positions"] is not None:
        axis = torch.repeat_interleave(torch.arange(len(s["sections"])), torch.tensor(s["sections"]))
        pos = s["positions"].long()[:, axis.to(pos.device)]
    angle = pos.double() * s["freqs"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turn(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
        y = x.clone()
        if s.get("interleaved"):
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
        return y

    k, v = turn(s["k"], s["k_norm"]), s["v"].float()
    if s["e4m3"]:
        k, v = (k / s["k_scale"]).clamp(-448, 448), (v / s["v_scale"]).clamp(-448, 448)
    block = s["tables"].long()[s["row_seq"], s["row_pos"] // s["block_size"]]
    token = s["row_pos"] % s["block_size"]
    held = s["kv"].view(torch.uint8) if s["e4m3"] else s["kv"]
    held[2 * s["layer"]][block, token] = k.to(s["kv"].dtype).view(held.dtype)
    held[2 * s["layer"] + 1][block, token] = v.to(s["kv"].dtype).view(held.dtype)
    return turn(s["q"], s["q_norm"]).to(torch.bfloat16), s["kv"]


def _tokens(s, plane, seq, pos, scale):
    """Rows of a plane at positions ``pos`` [..., n] of sequences ``seq``, as
    [..., head, n, dim] in 32 bits."""
    bs = s["block_size"]
    raw = s["kv"][plane].view(torch.uint8) if s["e4m3"] else s["kv"][plane]
    x = raw[s["tables"].long()[seq, pos // bs].clamp(min=0), pos % bs]
    x = x.view(s["kv"].dtype).float() * scale
    return x.transpose(-3, -2).contiguous()


def _chunks(s):
    """Pieces of the work as (sequences, rows, query positions [S, N], visible
    positions [S, M], which of them are keys at all): all single tokens
    together, or rows of one sequence whose scores fit 2 GiB."""
    dev, window, sinks = s["kv"].device, s["window"] or 1 << 40, s["sinks"]
    if max(s["new"]) == 1:
        L = s["lengths"].long()[:, None]
        first = (L - window).clamp(min=sinks)
        span = min(max(s["total"]), s["window"] or 1 << 40)
        near = first + torch.arange(span, device=dev)
        pos = torch.cat([torch.arange(sinks, device=dev).expand(len(s["new"]), -1), near], 1)
        rows = torch.arange(len(s["new"]), device=dev)[:, None]
        yield rows, rows, L - 1, pos, pos < L
        return
    row = 0
    for b, (n, L) in enumerate(zip(s["new"], s["total"])):
        most = min(2048, (1 << 29) // (s["heads"] * s["group"] * min(L, window + 2048)))
        for r in range(0, n, most):
            e = min(n, r + most)
            lo, hi = max(0, L - n + r + 1 - window), L - n + e
            few = min(sinks, lo)
            pos = torch.cat([torch.arange(few, device=dev), torch.arange(lo, hi, device=dev)])[None]
            yield (torch.full((1, 1), b, device=dev), torch.arange(row + r, row + e, device=dev)[None],
                   torch.arange(L - n + r, hi, device=dev)[None], pos, pos >= 0)
        row += n


def _scores(s, seq, rows, at, pos, there):
    """(scores [S, H, G, N, M] in 32 bits, -inf where not visible)."""
    H, G, D = s["heads"], s["group"], s["dim"]
    S, N = rows.shape
    q = s["q"][rows].float().view(S, N, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * N, D)
    k = _tokens(s, 2 * s["layer"], seq, pos.clamp(max=s["tables"].shape[1] * s["block_size"] - 1), s["k_scale"])
    a = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(D**-0.5).view(S, H, G, N, -1)
    seen = (pos[:, None] <= at[..., None]) & there[:, None]
    if s["window"]:
        seen &= (pos[:, None] > at[..., None] - s["window"]) | (pos[:, None] < s["sinks"])
    return a.masked_fill_(~seen[:, None, None], float("-inf"))


def _plain_window(s):
    H, G, D = s["heads"], s["group"], s["dim"]
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], device=out.device)
    for seq, rows, at, pos, there in _chunks(s):
        a = _scores(s, seq, rows, at, pos, there)
        S, _, _, N, M = a.shape
        top = a.amax(-1, keepdim=True)
        p = a.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        v = _tokens(s, 2 * s["layer"] + 1, seq, pos.clamp(max=s["tables"].shape[1] * s["block_size"] - 1),
                    s["v_scale"])
        o = torch.matmul(p.view(S, H, G * N, M), v).view(S, H, G, N, D).div_(total)
        out[rows] = o.permute(0, 3, 1, 2, 4).reshape(S, N, H * G, D).to(torch.bfloat16)
        lse[rows] = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(S, N, H * G)
    return (out, lse) if s.get("lse") else out


def _row_sums(s):
    """The logarithms of the rows' sums of exponentials [rows, heads], which
    attention over the same rows has given."""
    lse = torch.empty(s["q"].shape[:2], device="cuda")
    for seq, rows, at, pos, there in _chunks(s):
        a = torch.logsumexp(_scores(s, seq, rows, at, pos, there), -1)
        lse[rows] = a.permute(0, 3, 1, 2).reshape(*rows.shape, -1)
    return lse


def _plain_weigh(s):
    H, G = s["heads"], s["group"]
    for seq, rows, at, pos, there in _chunks(s):
        a = _scores(s, seq, rows, at, pos, there)
        S, N = rows.shape
        p = a.sub_(s["lse"][rows].view(S, N, H, G).permute(0, 2, 3, 1)[..., None]).exp_()
        got = p.sum((1, 2, 3))
        s["weights"].index_put_((seq.expand_as(pos), pos.where(there, 0)), got.where(there, 0.0), accumulate=True)
    return s["weights"]


def _plain_evict(s):
    bs, keep, tables, refs = s["block_size"], s["keep"], s["tables"], s["refs"]
    n, wide = tables.shape
    dev, L = tables.device, s["lengths"].long()[:, None]
    new = L.clamp(max=keep)
    # kept: the first, the last, and of the others those of the most weight
    p = torch.arange(wide * bs, device=dev).expand(n, -1)
    w = s["weights"].masked_fill((p < s["sinks"]) | (p >= L - s["recent"]), float("inf"))
    w = w.masked_fill(p >= L, -1.0)
    kept = torch.sort(w, dim=1, descending=True, stable=True)[1][:, :keep].sort(1)[0]
    j = torch.arange(kept.shape[1], device=dev)
    inside = j < new
    cut = (L > keep).squeeze(1)
    # blocks that get other tokens, or a last one that is not full
    last = _cdiv(new, bs)
    moves = (kept != j) & inside
    first = torch.where(moves.any(1), moves.to(torch.uint8).argmax(1), kept.shape[1])[:, None]
    if keep % bs:
        first = first.clamp(max=keep - 1)
    col = torch.arange(wide, device=dev)
    touched = (col >= first // bs) & (col < last) & cut[:, None]
    held = tables.long().clamp(min=0)
    replaced = touched & (refs[held] > 1)
    order = torch.sort((refs > 0).to(torch.uint8), stable=True)[1].to(torch.int32)
    rank = (torch.cumsum(replaced.flatten(), 0) - 1).view(n, wide)
    old = tables.clone()
    rows = torch.where(replaced, order[rank.clamp(min=0)], tables)
    rows = torch.where((col < last) | ~cut[:, None], rows, NONE)
    dropped = (old != rows) & (old >= 0)
    refs.scatter_add_(0, held.flatten(), -dropped.flatten().to(torch.int32))
    refs.scatter_add_(0, rows.long().clamp(min=0).flatten(), replaced.flatten().to(torch.int32))
    tables.copy_(rows)
    s["lengths"].copy_(new.squeeze(1).to(torch.int32))
    goes = inside & touched.gather(1, (j // bs).expand(n, -1))
    at = kept.clamp(max=wide * bs - 1)
    src_b, src_t = old.long().gather(1, at // bs)[goes], (at % bs)[goes]
    dst_b, dst_t = rows.long().gather(1, (j // bs).expand(n, -1))[goes], (j % bs).expand(n, -1)[goes]
    for plane in s["kv"]:
        plane[dst_b, dst_t] = plane[src_b, src_t]
    took = s["weights"].gather(1, at)
    s["weights"].masked_fill_((p >= new) & (p < L), 0.0)
    s["weights"][:, :kept.shape[1]] = torch.where(inside, took, s["weights"][:, :kept.shape[1]])
    kept = torch.where(inside, kept, NONE).to(torch.int32)
    if kept.shape[1] < keep:
        kept = torch.cat([kept, kept.new_full((n, keep - kept.shape[1]), NONE)], 1)
    return s["kv"], tables, s["lengths"], refs, s["weights"], torch.zeros(n, device=dev, dtype=torch.int32), kept


# ------------------------------------------------------------------ work


def work(case):
    c, bs = case, case["block_size"]
    if c["op"] == "evict":
        # what is kept of a longer sequence, but for its first tokens, is read and written,
        # its weights too; all weights are read
        token = 2 * c["layers"] * c["heads"] * c["dim"] * c["elem_bytes"]
        held, _ = _held(c)
        moved = sum(c["keep"] - c["sinks"] for t in held if t > c["keep"])
        entries = sum(_cdiv(t, bs) + _cdiv(min(t, c["keep"]), bs) for t in held)
        return {"bytes": 2 * moved * (token + 4) + 4 * sum(held) + 4 * sum(min(t, c["keep"]) for t in held)
                + 4 * entries, "flops": 0}
    new, cached = _lengths(c)
    H, G, D, e = c["heads"], c["group"], c["dim"], 1 if c["e4m3"] else 2
    T = sum(new)
    if c["op"] == "rotate":
        return {"bytes": 2 * T * H * D * (2 + e) + 4 * T * H * G * D + 4 * T * (1 + c["axes"]),
                "flops": T * H * (G + 1) * (3 * c["rot"] + (4 * D if c["norm"] else 0))}
    W, sinks = c["window"] or 1 << 40, c["sinks"]
    pairs = keys = 0
    for n, m in zip(new, cached):
        lo = max(0, m + 1 - W)
        keys += m + n - lo + min(sinks, lo)
        # the rows at m .. m + n - 1 see position + 1 tokens, or W and the first ones
        for a, b in ((m, min(m + n, W)), (max(m, W), m + n)):
            if b <= a:
                continue
            if b <= W:
                pairs += (a + 1 + b) * (b - a) // 2
            else:  # position a sees W, and those of the first that are behind the window
                behind = [a + 1 - W, b - W]
                short = max(0, min(behind[1], sinks) - behind[0] + 1) if behind[0] <= sinks else 0
                pairs += (b - a) * W + short * (behind[0] + behind[0] + short - 1) // 2
                pairs += (b - a - short) * sinks
    rows = 2 * T * H * G * D
    if c["op"] == "weigh":
        return {"bytes": keys * (H * D * e + 8) + rows + 4 * T * H * G + 4 * _cdiv(keys, bs),
                "flops": 2 * D * H * G * pairs}
    return {"bytes": 2 * keys * H * D * e + 2 * rows + (4 * T * H * G if c.get("lse") else 0)
            + 4 * _cdiv(keys, bs), "flops": 4 * D * H * G * pairs}


# ------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    if case["op"] == "evict":
        return None  # whole tokens and whole numbers: there is nothing to be off from
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"rotate": _exact_rotate, "window": _exact_attend, "weigh": _exact_attend}[case["op"]](case, s)


def _exact_rotate(case, s):
    new, cached = _lengths(case)
    bs, half, kv = case["block_size"], case["rot"] // 2, s["kv"].double()
    at = torch.cat([torch.arange(m, m + n, device="cuda") for n, m in zip(new, cached)])
    turns = []
    for i in range(half):
        pos = at
        if case["axes"]:
            edges = [sum(s["sections"][:a + 1]) for a in range(case["axes"])]
            pos = s["positions"][:, next(a for a, e in enumerate(edges) if i < e)]
        turns.append(pos.double() * s["freqs"][i])
    turn = torch.polar(torch.ones(len(at), half, device="cuda", dtype=torch.float64), torch.stack(turns, 1))

    def rotated(x, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x**2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * weight.double()
        i = torch.arange(half, device="cuda")
        a, b = (2 * i, 2 * i + 1) if case.get("interleaved") else (i, i + half)
        z = torch.complex(x[..., a], x[..., b]) * turn[:, None]
        x = x.clone()
        x[..., a], x[..., b] = z.real, z.imag
        return x

    row = 0
    k, v = rotated(s["k"], s["k_norm"]), s["v"].double()
    for b, (n, m) in enumerate(zip(new, cached)):
        where = torch.arange(m, m + n, device="cuda")
        block, token = s["tables"][b].long()[where // bs], where % bs
        kv[2 * case["layer"], block, token] = k[row:row + n] / s["k_scale"]
        kv[2 * case["layer"] + 1, block, token] = v[row:row + n] / s["v_scale"]
        row += n
    return rotated(s["q"], s["q_norm"]), kv


def _exact_attend(case, s):
    """Attention's outputs, and the logarithms of its sums, or the weights."""
    new, cached = _lengths(case)
    G, D, bs, W = case["group"], case["dim"], case["block_size"], case["window"] or 1 << 40
    weigh = case["op"] == "weigh"
    out = torch.empty(s["q"].shape, device="cuda", dtype=torch.float64)
    lse = torch.empty(s["q"].shape[:2], device="cuda", dtype=torch.float64)
    got = torch.zeros(len(new), s["tables"].shape[1] * bs, device="cuda", dtype=torch.float64)
    row = 0
    for b, (n, m) in enumerate(zip(new, cached)):
        where = torch.arange(m + n, device="cuda")
        block, token = s["tables"][b].long()[where // bs], where % bs
        for h in range(case["heads"]):
            view = s["kv"].view(torch.uint8) if case["e4m3"] else s["kv"]
            k, v = (view[2 * case["layer"] + i][:, :, h][block, token].view(s["kv"].dtype).double()
                    for i in (0, 1))
            for r in range(0, n, 1024):  # rows whose scores are in hand at once
                e = min(n, r + 1024)
                from_ = max(0, m + r + 1 - W)
                lo = min(from_, case["sinks"])  # keys 0 .. lo - 1, then from_ on
                pick = torch.cat([where[:lo], where[from_:m + e]])
                q = s["q"][row + r:row + e, h * G:(h + 1) * G].double().transpose(0, 1)
                a = (q.reshape(-1, D) @ k[pick].T * (s["k_scale"] / math.sqrt(D))).view(G, e - r, -1)
                P = torch.arange(m + r, m + e, device="cuda")[:, None]
                hidden = (pick > P) | ((pick <= P - W) & (pick >= case["sinks"]))
                a[hidden.expand(G, -1, -1)] = -math.inf
                if weigh:
                    mine = s["lse"][row + r:row + e, h * G:(h + 1) * G].double().T
                    got[b, pick] += torch.exp(a - mine[..., None]).sum((0, 1))
                    continue
                lse[row + r:row + e, h * G:(h + 1) * G] = torch.logsumexp(a, -1).T
                o = (torch.softmax(a, -1).view(-1, len(pick)) @ v[pick] * s["v_scale"]).view(G, e - r, D)
                out[row + r:row + e, h * G:(h + 1) * G] = o.transpose(0, 1)
        row += n
    if weigh:
        return got
    return (out, lse) if case.get("lse") else out
