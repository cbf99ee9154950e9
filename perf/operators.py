"""Timed cases of the operators on a pool's sequences: writing keys and values
into blocks, attention over a prompt, attention of a decoding batch with a
shared prefix, and the block operations (free, fork, grow, compact).

A case's lengths follow from the case alone, and its data from the seed.  The
plain forms are elementary torch operations in 32 bits: keys and values are
gathered from the blocks into padded tensors, scores are masked, exponentiated,
summed and multiplied.
"""

import math
import random

import torch

own = False

NONE = -1  # a table entry that names no block (0xFFFFFFFF as a 32-bit pattern)


# ------------------------------------------------------------------ cases


def _attend(name, op, heads, group, dim, seqs, new, cached, **more):
    """``heads`` KV heads of ``dim``, each serving ``group`` query heads;
    ``seqs`` sequences of new[0]..new[1] rows after cached[0]..cached[1]
    tokens (and after ``prefix`` tokens that all of them share)."""
    c = dict(name=name, op=op, layers=2, layer=1, block_size=16, heads=heads, group=group, dim=dim,
             e4m3=False, seqs=seqs, new_lo=new[0], new_hi=new[1], cached_lo=cached[0],
             cached_hi=cached[1], prefix=0, salt=1)
    c.update(more)
    return c


def _blocks(name, op, geometry, parents, children, tokens, **more):
    """Sequences of tokens[0]..tokens[1] over a pool (layers, planes, block
    size, heads, dim, element bytes, blocks)."""
    layers, planes, block_size, heads, dim, elem_bytes, blocks = geometry
    c = dict(name=name, op=op, layers=layers, planes=planes, block_size=block_size, heads=heads,
             dim=dim, elem_bytes=elem_bytes, blocks=blocks, parents=parents, children=children,
             tokens_lo=tokens[0], tokens_hi=tokens[1], grow_lo=1, grow_hi=1, salt=1)
    c.update(more)
    return c


def listed():
    return [
        # one layer of one decoding step: a token's K and V for each of 48 running sequences
        _attend("write-step", "write", 8, 4, 128, 48, (1, 1), (0, 4000)),
        # one layer of a prefill batch, rounded to e4m3 on the way in
        _attend("write-prompts-e4m3", "write", 4, 7, 128, 24, (100, 1500), (0, 0), e4m3=True,
                k_scale=0.031, v_scale=0.017),
        # a unit test's or a demo's prompts: a few tokens each
        _attend("prompt-short", "prompt", 2, 2, 64, 5, (1, 60), (0, 0)),
        # one long document, nothing cached: 16384 causal tokens, 32 query heads over 8
        _attend("prompt-long", "prompt", 8, 4, 128, 1, (16384, 16384), (0, 0)),
        # requests whose prefixes were restored: ragged prompts after cached tokens, 7 query
        # heads to a KV head, e4m3 blocks
        _attend("prompt-resumed-e4m3", "prompt", 4, 7, 128, 12, (33, 1500), (0, 4000), e4m3=True,
                k_scale=0.031, v_scale=0.017),
        # a small decoding step: 4 sequences behind a short common instruction
        _attend("shared-few", "shared", 2, 2, 64, 4, (1, 1), (0, 100), prefix=256),
        # 64 sequences behind one 8192-token system prompt
        _attend("shared-64", "shared", 8, 4, 128, 64, (1, 1), (0, 1024), prefix=8192),
        # one GPU's KV head of a tensor-parallel model, 200 samples of a 20000-token
        # document, e4m3 blocks
        _attend("shared-200-e4m3", "shared", 1, 8, 128, 200, (1, 1), (0, 2000), prefix=20000,
                e4m3=True, k_scale=0.031, v_scale=0.017),
        # a demo's pool: 3 finished samples are freed, forked anew and grown by a token
        _blocks("branch-tiny", "branch", (2, 2, 16, 2, 64, 2, 64), 2, 3, (8, 128)),
        # 8B-shaped blocks (2 MiB): 64 samples are freed, forked from 16 prompts and grown
        _blocks("branch-8b", "branch", (32, 2, 16, 8, 128, 2, 1200), 16, 64, (64, 700)),
        # half of a small pool's sequences end; the rest moves to the front
        _blocks("compact-tiny", "compact", (2, 2, 16, 2, 64, 2, 64), 4, 4, (8, 100)),
        # latent blocks (61 layers, 36 KiB chunks) of a long-running server are compacted
        _blocks("compact-latent", "compact", (61, 1, 64, 1, 576, 1, 2000), 40, 40, (200, 2300)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: 1 to 8 KV heads of 64 or 128, 1 to 16
    query heads to each, blocks of 8 to 64 tokens in bf16 and e4m3, 1 to 256
    sequences, up to 16384 rows and 32768 tokens; pools of 64 to 4000 blocks."""
    op = rng.choice(["write", "prompt", "prompt", "shared", "shared", "branch", "compact"])
    salt = rng.randrange(1 << 30)
    if op in ("branch", "compact"):
        while True:
            planes = rng.choice([1, 2, 2])
            geometry = (_log_int(rng, 1, 80), planes, rng.choice([8, 16, 16, 24, 64]),
                        1 if planes == 1 else rng.randint(1, 8),
                        576 if planes == 1 else rng.choice([64, 80, 128]), rng.choice([1, 2]),
                        _log_int(rng, 64, 4000))
            chunk = geometry[2] * geometry[3] * geometry[4] * geometry[5]
            if chunk % 16 == 0 and geometry[0] * planes * chunk * geometry[6] <= 5 << 29:
                break
        blocks, bs = geometry[6], geometry[2]
        parents = _log_int(rng, 1, max(1, blocks // 16))
        children = _log_int(rng, 1, max(1, blocks // 6))
        hi = max(2, blocks * bs // (2 * (parents + (children if op == "compact" else 0))))
        hi = min(hi, 8192)
        more = dict(grow_hi=rng.choice([1, 1, bs])) if op == "branch" else {}
        return _unnamed(_blocks("", op, geometry, parents, children, (max(1, hi // 8), hi), salt=salt,
                                **more))
    more = dict(block_size=rng.choice([8, 16, 16, 16, 24, 32, 64]), salt=salt)
    if rng.random() < 0.4:
        more.update(e4m3=True, k_scale=rng.uniform(0.02, 0.05), v_scale=rng.uniform(0.01, 0.03))
    heads, group, dim = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16]), rng.choice([64, 128, 128])
    if op == "shared":
        seqs = _log_int(rng, 1, 256)
        cached_hi = _log_int(rng, 1, min(8192, 400000 // seqs))
        blocks = _log_int(rng, 1, 32768 // more["block_size"]) if rng.random() < 0.8 else 0
        return _unnamed(_attend("", op, heads, group, dim, seqs, (1, 1), (0, cached_hi),
                                prefix=blocks * more["block_size"], **more))
    seqs = _log_int(rng, 1, 64)
    if op == "write" and rng.random() < 0.4:
        return _unnamed(_attend("", op, heads, group, dim, seqs, (1, 1), (0, 4000), **more))
    new_hi = _log_int(rng, 2, 16384 // seqs)
    cached_hi = 0 if rng.random() < 0.5 else _log_int(rng, 1, 32768 // seqs)
    if op == "prompt":  # no more scores than the largest listed case has
        while heads * group * seqs * new_hi * (new_hi + 2 * cached_hi) > 6e9:
            new_hi, cached_hi = new_hi * 2 // 3 + 1, cached_hi * 2 // 3
    return _unnamed(_attend("", op, heads, group, dim, seqs, (max(1, new_hi // 8), new_hi),
                            (0, cached_hi), **more))


def _unnamed(c):
    del c["name"]
    return c


def _lengths(c):
    """(rows, tokens cached before them, past the shared prefix) of each sequence."""
    r = random.Random(c["salt"])
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["seqs"])]
    return new, [r.randint(c["cached_lo"], c["cached_hi"]) for _ in range(c["seqs"])]


def _held(c):
    """Tokens of each parent, then of each child (a branch's children take
    their parents')."""
    r = random.Random(c["salt"])
    got = [r.randint(c["tokens_lo"], c["tokens_hi"]) for _ in range(c["parents"])]
    if c["op"] == "branch":
        parent = [r.randrange(c["parents"]) for _ in range(c["children"])]
        return got, parent, [r.randint(c["grow_lo"], c["grow_hi"]) for _ in range(c["children"])]
    got += [r.randint(c["tokens_lo"], c["tokens_hi"]) for _ in range(c["children"])]
    ended = sorted(r.sample(range(len(got)), len(got) // 2))
    return got, ended, None


def _cdiv(a, b):
    return -(-a // b)


# ------------------------------------------------------------------ inputs


def _geometry(c, blocks):
    from paper_2606_01387_amd.synth import Geometry

    return Geometry(c["layers"], c.get("planes", 2), c["block_size"], c["heads"], c["dim"],
                    c.get("elem_bytes", 1 if c.get("e4m3") else 2), blocks)


def _handle(s, c, blocks):
    """What a serving program keeps: the pool's handle and its sequences."""
    from paper_2606_01387_amd import claimkv, sequences

    pool = claimkv.Pool(_geometry(c, blocks), 7, s["kv"].view(torch.uint8), max_claims=256,
                        max_footprint=1 << 14, event_capacity=1 << 10)
    s["pool"] = pool
    s["seqs"] = sequences.Sequences(pool, tables=s["tables"], lengths=s["lengths"], refs=s["refs"])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_blocks if case["op"] in ("branch", "compact") else _prepare_attend)(case, g)


def _prepare_attend(c, g):
    dev = "cuda"
    H, G, D, bs = c["heads"], c["group"], c["dim"], c["block_size"]
    new, cached = _lengths(c)
    shared = c["prefix"] // bs
    total = [n + m for n, m in zip(new, cached)]
    need = [_cdiv(t, bs) for t in total]
    used = shared + sum(need)
    blocks = used + used // 8 + 8
    wide = shared + max(need)
    perm = torch.randperm(blocks, generator=g, device=dev)[:used].to(torch.int32)
    tables = torch.full((c["seqs"], wide), NONE, device=dev, dtype=torch.int32)
    tables[:, :shared] = perm[:shared]
    need_t = torch.tensor(need, device=dev)
    inside = torch.arange(wide - shared, device=dev)[None] < need_t[:, None]
    tables[:, shared:][inside] = perm[shared:]
    lengths = torch.tensor([c["prefix"] + t for t in total], device=dev, dtype=torch.int32)
    refs = torch.zeros(blocks, device=dev, dtype=torch.int32)
    refs[perm.long()] = 1
    if shared:
        refs[perm[:shared].long()] = c["seqs"]
    offsets = torch.zeros(c["seqs"] + 1, device=dev, dtype=torch.int32)
    offsets[1:] = torch.cumsum(torch.tensor(new, device=dev), 0)
    T = sum(new)

    # keys have a few large channels, as rotary keys do; queries point at some
    # of the keys, so that a row's weights are neither flat nor all on one
    chan = 1 + 3 * (torch.rand(D, generator=g, device=dev) < 0.06).float()
    kv = torch.empty(2 * c["layers"], blocks, bs, H, D, device=dev, dtype=torch.bfloat16)
    kv.normal_(generator=g)
    kv[0::2] *= chan.to(torch.bfloat16)
    if c["e4m3"]:
        kv[0::2] *= 0.5 / c["k_scale"] / 16
        kv[1::2] *= 0.5 / c["v_scale"] / 16
        kv = kv.to(torch.float8_e4m3fn)
    s = dict(c, kv=kv, tables=tables, lengths=lengths, refs=refs, offsets=offsets,
             k_scale=c.get("k_scale", 1.0), v_scale=c.get("v_scale", 1.0),
             prefix_blocks=perm[:shared].clone())
    if c["op"] == "write":
        # a slice of one fused projection, as a layer has them
        qkv = torch.empty(T, (G + 2) * H * D, device=dev, dtype=torch.bfloat16).normal_(generator=g)
        s["k"] = qkv[:, G * H * D:(G + 1) * H * D].view(T, H, D)
        s["v"] = qkv[:, (G + 1) * H * D:].view(T, H, D)
    else:
        s["q"] = (1.5 * torch.randn(T, H * G, D, generator=g, device=dev)).to(torch.bfloat16)
    s["rows_at_most"], s["longest"] = max(new), max(total)
    if own:
        _handle(s, c, blocks)
    return s


def _prepare_blocks(c, g):
    dev = "cuda"
    bs, nb = c["block_size"], c["blocks"]
    chunk = bs * c["heads"] * c["dim"] * c["elem_bytes"]
    kv = torch.randint(-2**62, 2**62, (c["layers"] * c["planes"], nb, chunk // 8), generator=g,
                       device=dev)
    held, second, grow = _held(c)
    n = c["parents"] + c["children"]
    wide = max(_cdiv(t, bs) for t in held) + _cdiv(c["grow_hi"], bs) + 1
    tables = torch.full((n, wide), NONE, device=dev, dtype=torch.int32)
    lengths = torch.zeros(n, device=dev, dtype=torch.int32)
    refs = torch.zeros(nb, device=dev, dtype=torch.int32)
    need = torch.tensor([_cdiv(t, bs) for t in held], device=dev)
    used = int(need.sum())
    perm = torch.randperm(nb, generator=g, device=dev)[:used].to(torch.int32)
    inside = torch.arange(wide, device=dev)[None] < need[:, None]
    tables[:len(held)][inside] = perm
    lengths[:len(held)] = torch.tensor(held, device=dev, dtype=torch.int32)
    refs[perm.long()] = 1
    s = dict(c, kv=kv, tables=tables, lengths=lengths, refs=refs)
    if c["op"] == "branch":
        s["parent_ids"] = torch.tensor(second, device=dev, dtype=torch.int32)
        s["child_ids"] = torch.arange(c["parents"], n, device=dev, dtype=torch.int32)
        s["grow_by"] = torch.tensor(grow, device=dev, dtype=torch.int32)
    else:
        s["ended"] = torch.tensor(second, device=dev, dtype=torch.int32)
        s["before"] = (tables.clone(), lengths.clone(), refs.clone())
    if own:
        _handle(s, c, nb)
    return s


# ------------------------------------------------------------------ one pass


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    q, scales = s["seqs"], dict(k_scale=s.get("k_scale", 1.0), v_scale=s.get("v_scale", 1.0))
    if s["op"] == "write":
        q.write(s["layer"], s["k"], s["v"], offsets=s["offsets"], **scales)
        return s["kv"]
    if s["op"] == "prompt":
        return q.attend(s["layer"], s["q"], offsets=s["offsets"], **scales)
    if s["op"] == "shared":
        return q.attend_shared(s["layer"], s["q"], s["prefix_blocks"], **scales)
    if s["op"] == "branch":
        q.free(s["child_ids"])
        forked = q.fork(s["parent_ids"], s["child_ids"])
        grown = q.grow(s["child_ids"], s["grow_by"])
        return s["kv"], s["tables"], s["lengths"], s["refs"], forked, grown
    s["tables"].copy_(s["before"][0])
    s["lengths"].copy_(s["before"][1])
    s["refs"].copy_(s["before"][2])
    q.free(s["ended"])
    moved = q.compact()
    return s["kv"], s["tables"], s["lengths"], s["refs"], moved


def _run_plain(s):
    if s["op"] == "write":
        return _plain_write(s)
    if s["op"] == "prompt":
        return _plain_prompt(s)
    if s["op"] == "shared":
        return _plain_shared(s)
    if s["op"] == "branch":
        _plain_free(s, s["child_ids"].long())
        forked = _plain_fork(s, s["parent_ids"].long(), s["child_ids"].long())
        grown = _plain_grow(s, s["child_ids"].long(), s["grow_by"])
        return s["kv"], s["tables"], s["lengths"], s["refs"], forked, grown
    s["tables"].copy_(s["before"][0])
    s["lengths"].copy_(s["before"][1])
    s["refs"].copy_(s["before"][2])
    _plain_free(s, s["ended"].long())
    moved = _plain_compact(s)
    return s["kv"], s["tables"], s["lengths"], s["refs"], moved


def _row_places(s):
    """Each packed row's sequence, index in it and position."""
    offsets, rows = s["offsets"].long(), s["k" if s["op"] == "write" else "q"].shape[0]
    at = torch.arange(rows, device=offsets.device)
    seq = torch.searchsorted(offsets, at, right=True) - 1
    i = at - offsets[seq]
    return seq, i, s["lengths"].long()[seq] - (offsets[seq + 1] - offsets[seq]) + i


def _plain_write(s):
    seq, _, pos = _row_places(s)
    block = s["tables"].long()[seq, pos // s["block_size"]]
    token = pos % s["block_size"]
    k, v = s["k"].float(), s["v"].float()
    if s["e4m3"]:
        k = (k / s["k_scale"]).clamp(-448, 448)
        v = (v / s["v_scale"]).clamp(-448, 448)
    held = s["kv"].view(torch.uint8) if s["e4m3"] else s["kv"]
    held[2 * s["layer"]][block, token] = k.to(s["kv"].dtype).view(held.dtype)
    held[2 * s["layer"] + 1][block, token] = v.to(s["kv"].dtype).view(held.dtype)
    return s["kv"]


def _gather(s, plane, blocks, scale):
    """[..., blocks] of a plane as [..., head, token, dim], in 32 bits."""
    x = s["kv"][plane].view(torch.uint8 if s["e4m3"] else torch.bfloat16)[blocks.long().clamp(min=0)]
    x = x.view(s["kv"].dtype).float() * scale
    x = x.flatten(-4, -3) if x.dim() == 4 else x.flatten(1, 2)
    return x.transpose(-3, -2).contiguous()


def _weights(scores, visible):
    """exp(scores - row maximum) at the visible places, in place, and the sums."""
    scores.masked_fill_(~visible, float("-inf"))
    scores.sub_(scores.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    return scores, scores.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_prompt(s):
    H, G, D = s["heads"], s["group"], s["dim"]
    seq, i, pos = _row_places(s)
    N, S = s["rows_at_most"], s["seqs"]
    q = torch.zeros(S, N, H, G, D, device=s["kv"].device)
    q[seq, i] = s["q"].float().view(-1, H, G, D)
    last = torch.full((S, N), -1, device=s["kv"].device)
    last[seq, i] = pos
    k = _gather(s, 2 * s["layer"], s["tables"], s["k_scale"])
    v = _gather(s, 2 * s["layer"] + 1, s["tables"], s["v_scale"])
    q = q.permute(0, 2, 3, 1, 4).reshape(S, H, G * N, D)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(D**-0.5).view(S, H, G, N, -1)
    visible = torch.arange(k.shape[2], device=k.device) <= last[:, None, None, :, None]
    p, total = _weights(scores, visible)
    out = torch.matmul(p.view(S, H, G * N, -1), v).view(S, H, G, N, D).div_(total)
    return out.permute(0, 3, 1, 2, 4)[seq, i].reshape(-1, H * G, D).to(torch.bfloat16)


def _plain_shared(s):
    H, G, D, B, P = s["heads"], s["group"], s["dim"], s["seqs"], s["prefix"]
    mine = s["tables"][:, P // s["block_size"]:]
    q = s["q"].float().view(B, H, G, D)
    k = _gather(s, 2 * s["layer"], mine, s["k_scale"])
    v = _gather(s, 2 * s["layer"] + 1, mine, s["v_scale"])
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous())
    visible = torch.arange(k.shape[2], device=k.device) + P < s["lengths"][:, None, None, None]
    if P:
        kp = _gather(s, 2 * s["layer"], s["prefix_blocks"], s["k_scale"])
        vp = _gather(s, 2 * s["layer"] + 1, s["prefix_blocks"], s["v_scale"])
        together = q.transpose(0, 1).reshape(H, B * G, D)
        first = torch.matmul(together, kp.transpose(-1, -2).contiguous()).view(H, B, G, P)
        scores = torch.cat([first.transpose(0, 1), scores], -1)
        seen = torch.arange(P, device=k.device) < s["lengths"][:, None, None, None]
        visible = torch.cat([seen, visible], -1)
    p, total = _weights(scores.mul_(D**-0.5), visible)
    out = torch.matmul(p[..., P:].contiguous(), v)
    if P:
        shared = torch.matmul(p[..., :P].transpose(0, 1).reshape(H, B * G, P), vp)
        out += shared.view(H, B, G, D).transpose(0, 1)
    return out.div_(total).reshape(B, H * G, D).to(torch.bfloat16)


def _plain_free(s, ids):
    rows = s["tables"][ids]
    inside = torch.arange(rows.shape[1], device=rows.device) < _cdiv(s["lengths"][ids], s["block_size"])[:, None]
    s["refs"].scatter_add_(0, rows.long().clamp(min=0).flatten(), -inside.to(torch.int32).flatten())
    s["tables"][ids] = NONE
    s["lengths"][ids] = 0


def _free_blocks(s):
    """Blocks in order, the free ones first, and how many are free."""
    used = s["refs"] > 0
    return torch.sort(used.to(torch.uint8), stable=True)[1].to(torch.int32), (~used).sum()


def _plain_fork(s, parents, children):
    bs, tables = s["block_size"], s["tables"]
    length, rows = s["lengths"][parents], s["tables"][parents]
    part = (length % bs > 0).to(torch.int32)
    order, free = _free_blocks(s)
    at = torch.cumsum(part, 0)
    fine = at <= free
    col = torch.arange(rows.shape[1], device=rows.device)
    shared = (col < (length // bs)[:, None]) & fine[:, None]
    s["refs"].scatter_add_(0, rows.long().clamp(min=0).flatten(), shared.to(torch.int32).flatten())
    copied = fine & (part > 0)
    to = order[(at[copied] - 1).long()]
    where = (length[copied] // bs).long()
    src = rows[copied, where].long()
    s["refs"][to.long()] = 1
    tables[children] = torch.where(shared, rows, NONE)
    tables[children[copied], where] = to
    s["lengths"][children] = torch.where(fine, length, 0)
    s["kv"][:, to.long()] = s["kv"][:, src]
    return (~fine).to(torch.int32)


def _plain_grow(s, ids, by):
    bs, tables = s["block_size"], s["tables"]
    length = s["lengths"][ids]
    held = _cdiv(length, bs)
    need = _cdiv(length + by, bs) - held
    order, free = _free_blocks(s)
    at = torch.cumsum(need, 0)
    fine = at <= free
    col = torch.arange(tables.shape[1], device=tables.device)
    k = col - held[:, None]
    fresh = (k >= 0) & (k < need[:, None]) & fine[:, None]
    to = order[((at - need)[:, None] + k)[fresh].long()]
    s["refs"][to.long()] = 1
    rows = tables[ids]
    rows[fresh] = to
    tables[ids] = rows
    s["lengths"][ids] = torch.where(fine, length + by, length)
    return (~fine).to(torch.int32)


def _plain_compact(s):
    refs = s["refs"]
    live = refs > 0
    at = torch.arange(refs.numel(), device=refs.device)
    low = at < live.sum()
    src, dst = at[live & ~low], at[~live & low]
    s["kv"][:, dst] = s["kv"][:, src]
    refs[dst] = refs[src]
    refs[src] = 0
    to = at.to(torch.int32)
    to[src] = dst.to(torch.int32)
    s["tables"].copy_(torch.where(s["tables"] >= 0, to[s["tables"].long().clamp(min=0)], NONE))
    return (live & ~low).sum().to(torch.int32).view(1)


# ------------------------------------------------------------------ work


def work(case):
    c, bs = case, case["block_size"]
    if c["op"] in ("branch", "compact"):
        block = c["layers"] * c["planes"] * bs * c["heads"] * c["dim"] * c["elem_bytes"]
        held, second, grow = _held(c)
        if c["op"] == "branch":  # partly filled last blocks are read and written, table rows too
            copied = sum(held[p] % bs > 0 for p in second)
            entries = sum(_cdiv(held[p], bs) for p in second) * 4
        else:  # every live block past the live count moves
            live = sum(_cdiv(t, bs) for i, t in enumerate(held) if i not in set(second))
            copied = live * (c["blocks"] - live) / c["blocks"]  # of random places, about this share
            entries = 2 * sum(_cdiv(t, bs) for t in held)
        return {"bytes": 2 * copied * block + 4 * (2 * c["blocks"] + entries), "flops": 0}
    new, cached = _lengths(c)
    H, G, D, e = c["heads"], c["group"], c["dim"], 1 if c["e4m3"] else 2
    T = sum(new)
    if c["op"] == "write":
        return {"bytes": 2 * T * H * D * (2 + e) + 8 * c["seqs"] + 4 * T, "flops": 0}
    own_tokens = sum(new) + sum(cached)
    scores = sum(n * (c["prefix"] + m) + n * (n + 1) // 2 for n, m in zip(new, cached))
    keys = 2 * H * D * e * (c["prefix"] + own_tokens)
    return {"bytes": keys + 4 * T * H * G * D + 4 * _cdiv(c["prefix"] + own_tokens, bs),
            "flops": 4 * D * H * G * scores}


# ------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    if case["op"] in ("branch", "compact"):
        return None  # whole blocks and whole numbers: there is nothing to be off from
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return (_exact_write if case["op"] == "write" else _exact_attend)(case, s)


def _exact_write(case, s):
    new, cached = _lengths(case)
    kv, bs, row = s["kv"].double(), case["block_size"], 0
    for b, (n, m) in enumerate(zip(new, cached)):
        where = torch.arange(m, m + n, device="cuda")
        block, token = s["tables"][b].long()[where // bs], where % bs
        for i, x in enumerate((s["k"], s["v"])):
            scale = s["v_scale" if i else "k_scale"] if case["e4m3"] else 1.0
            kv[2 * case["layer"] + i, block, token] = x[row:row + n].double() / scale
        row += n
    return kv


def _exact_attend(case, s):
    new, cached = _lengths(case)
    G, D, bs, P = case["group"], case["dim"], case["block_size"], case["prefix"]
    out = torch.empty(s["q"].shape, device="cuda", dtype=torch.float64)
    row = 0
    for b, (n, m) in enumerate(zip(new, cached)):
        L = P + m + n
        where = torch.arange(L, device="cuda")
        block, token = s["tables"][b].long()[where // bs], where % bs
        for h in range(case["heads"]):
            view = s["kv"].view(torch.uint8) if case["e4m3"] else s["kv"]
            k, v = (view[2 * case["layer"] + i][:, :, h][block, token].view(s["kv"].dtype).double()
                    for i in (0, 1))
            for r in range(0, n, 2048):  # rows whose scores are in hand at once
                e = min(n, r + 2048)
                seen = L - n + e
                q = s["q"][row + r:row + e, h * G:(h + 1) * G].double().transpose(0, 1).reshape(-1, D)
                a = q @ k[:seen].T * (s["k_scale"] / math.sqrt(D))
                late = where[:seen] > (torch.arange(r, e, device="cuda") + L - n)[:, None]
                a.view(G, e - r, seen)[late.expand(G, -1, -1)] = -math.inf
                o = torch.softmax(a, -1) @ v[:seen] * s["v_scale"]
                out[row + r:row + e, h * G:(h + 1) * G] = o.view(G, e - r, D).transpose(0, 1)
        row += n
    return out
