"""Cutting sequences to the tokens that weighed most, against plain Python on host copies."""

import random

import numpy as np
import pytest

from paper_2606_01387_amd.synth import Geometry
from test_gpu_blocks import Pair

pytestmark = pytest.mark.gpu

NONE = -1


def choose(w, L, tokens, sinks, recent):
    """The positions that are kept, by definition."""
    if L <= tokens:
        return list(range(L))
    def worth(p):
        return -np.inf if np.isnan(w[p]) else float(w[p])
    rest = [p for p in range(sinks, L - recent)]
    # NaN below -infinity; of equal ones the first
    rest.sort(key=lambda p: (0 if np.isnan(w[p]) else 1, worth(p)), reverse=True)
    return sorted(list(range(sinks)) + rest[:tokens - sinks - recent] + list(range(L - recent, L)))


def evict(m, weights, ids, tokens, sinks, recent):
    """On the model of tests/test_gpu_blocks.py; (statuses, kept)."""
    n, bs = len(m.lengths), m.bs
    ids = list(range(n)) if ids is None else ids
    before, refs = m.tables.copy(), m.refs.copy()
    free = [b for b in range(len(refs)) if refs[b] == 0]
    old_kv = m.kv.copy()
    asked, status, kept, seen = 0, [], [], set()
    for r in ids:
        kept.append([NONE] * tokens)
        if not 0 <= r < n or r in seen:
            status.append(2)
            continue
        seen.add(r)
        L = int(m.lengths[r]) % (1 << 32)
        held = -(-L // bs)
        if held > before.shape[1] or any(not 0 <= b < len(refs) for b in before[r, :held]):
            status.append(2)
            continue
        w = weights[r]
        keep = choose(w, L, tokens, sinks, recent)
        if L <= tokens:
            status.append(0)
            kept[-1][:L] = keep
            continue
        changed = [j for j in range(tokens) if keep[j] != j]
        blocks = -(-tokens // bs)
        first = changed[0] // bs if changed else blocks
        if tokens % bs:
            first = min(first, blocks - 1)
        need = [j for j in range(first, blocks) if refs[before[r, j]] > 1]
        asked += len(need)
        if need and asked > len(free):
            status.append(1)
            continue
        status.append(0)
        kept[-1] = keep
        for rank, j in enumerate(need):
            b = free[asked - len(need) + rank]
            m.tables[r, j] = b
            m.refs[b] = 1
            m.refs[before[r, j]] -= 1
        for j in range(blocks, held):
            m.refs[before[r, j]] -= 1
            m.tables[r, j] = NONE
        token = m.kv.shape[2] // bs
        for j in range(first * bs, tokens):
            src, dst = before[r, keep[j] // bs], m.tables[r, j // bs]
            s, d = keep[j] % bs * token, j % bs * token
            m.kv[:, dst, d:d + token] = old_kv[:, src, s:s + token]
        w[:tokens] = w[keep]
        w[tokens:L] = 0
        m.lengths[r] = tokens
    return status, kept


class Evicting(Pair):
    def __init__(self, torch, ck, max_seqs, max_blocks, geometry, stream=None, seed=0):
        super().__init__(torch, ck, max_seqs, max_blocks, geometry, stream)
        rng = np.random.default_rng(seed)
        # ties, zeros of both signs, infinities and NaN among them
        w = np.exp(rng.normal(size=(max_seqs, max_blocks * geometry.block_size))).astype(np.float32)
        kind = rng.integers(0, 12, w.shape)
        w[kind < 4] = np.round(w[kind < 4])
        w[kind == 4], w[kind == 5] = 0.0, -0.0
        w[kind == 6] *= -1
        special = rng.integers(0, 60, w.shape)
        w[special == 0], w[special == 1], w[special == 2] = np.nan, np.inf, -np.inf
        self.w = w
        self.weights = torch.from_numpy(w.copy()).cuda()

    def evict(self, ids, tokens, sinks=0, recent=0):
        want, kept = evict(self.model, self.w, ids, tokens, sinks, recent)
        status, got = self.seqs.evict(None if ids is None else self.ints(ids), self.weights, tokens,
                                      sinks=sinks, recent=recent)
        assert status.tolist() == want
        assert got.tolist() == kept
        self.same()
        assert np.array_equal(self.weights.cpu().numpy(), self.w, equal_nan=True)


def geometry(blocks, bs=16, heads=2, dim=64, elem=2, layers=2, planes=2):
    return Geometry(layers, planes, bs, heads, dim, elem, blocks)


@pytest.mark.parametrize("sinks,recent", [(0, 0), (4, 16), (0, 40), (64, 0), (1, 63), (30, 34)])
@pytest.mark.parametrize("tokens", [64, 70])
def test_cut(torch, ck, tokens, sinks, recent):
    p = Evicting(torch, ck, 5, 20, geometry(80), seed=1)
    with p.pool:
        p.do("grow", [0, 1, 2, 3], [300, 64, 71, 200])
        p.evict(None, tokens, sinks, recent)


@pytest.mark.parametrize("bs,heads,dim,elem,planes", [
    (1, 1, 8, 2, 2), (5, 2, 8, 1, 2), (16, 1, 8, 1, 2), (24, 3, 24, 1, 2), (64, 1, 576, 1, 1), (16, 8, 128, 2, 2),
    (2, 5, 8, 1, 1), (8, 8, 64, 1, 2), (2, 20, 128, 2, 1)])
def test_geometries(torch, ck, bs, heads, dim, elem, planes):
    """Tokens of 8 bytes to several slices, blocks of one token to 64."""
    p = Evicting(torch, ck, 4, 400 // bs + 2, geometry(1600 // bs + 12, bs, heads, dim, elem, 3, planes), seed=2)
    with p.pool:
        p.do("grow", [0, 1, 2], [400, 37, 250])
        p.do("fork", [0], [3])
        p.evict([3, 1, 2], 101, 3, 20)
        p.evict([0, 2, 3], 100, 3, 20)
        p.evict([0, 3], 7, 7, 0)


@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 1000])
def test_few_kept(torch, ck, tokens):
    p = Evicting(torch, ck, 4, 10, geometry(60), seed=3)
    with p.pool:
        p.do("grow", [0, 1, 2], [160, 1, 33])
        p.evict([2, 0, 1, 3], tokens)
        p.evict([0, 2], tokens)


def test_long_sequences(torch, ck):
    p = Evicting(torch, ck, 2, 1100, geometry(2300, 16, 1, 64, 1, 1), seed=4)
    with p.pool:
        p.do("grow", [0, 1], [17500, 12345])
        p.evict(None, 9001, 4, 333)
        p.evict([1], 4000, 0, 0)


def test_equal_weights_keep_the_first(torch, ck):
    p = Evicting(torch, ck, 2, 20, geometry(50), seed=5)
    p.w[:] = 1
    p.weights.fill_(1)
    with p.pool:
        p.do("grow", [0, 1], [300, 299])
        p.evict([0], 48)       # a plain cut: nothing moves
        p.evict([1], 50, 0, 3)  # but for the last ones


def test_shared_blocks_are_left(torch, ck):
    """Forked sequences, held blocks, both of a pair at once, and rows that
    share a last block that is not full."""
    p = Evicting(torch, ck, 8, 20, geometry(120), seed=6)
    with p.pool:
        p.do("grow", [0, 1], [200, 170])
        p.do("fork", [0, 0, 1], [2, 3, 4])
        p.evict([0, 2], 100, 4, 10)
        p.evict([3], 100, 4, 10)
        for b in p.model.tables[1, 2:4]:  # the program holds two blocks
            p.model.refs[b] += 1
            p.seqs.refs[int(b)] += 1
        p.evict([1], 90, 4, 10)
        p.do("fork", [1], [5])
        p.w[4] = p.w[5] = 1
        p.weights[4:6] = 1
        p.evict([4, 5], 40)  # cut within a shared block
        p.do("grow", [4, 5], [3, 5])
        p.do("free", [0, 1, 2, 3, 4, 5])


def test_too_few_blocks(torch, ck):
    """Entries in order: those that need blocks stop where the free ones end,
    those that need none go on; the ones that fail are as before."""
    p = Evicting(torch, ck, 8, 16, geometry(34), seed=7)
    with p.pool:
        p.do("grow", [0, 1], [160, 160])
        p.do("fork", [0, 0, 1], [2, 3, 4])
        p.do("grow", [5], [90])
        p.evict([0, 2, 3, 5, 1, 4], 80, 2, 5)
        p.evict([4, 5], 50)


def test_refused_entries(torch, ck):
    p = Evicting(torch, ck, 8, 12, geometry(80), seed=8)
    with p.pool:
        p.do("grow", [0, 1, 2, 3], [160, 100, 100, 100])
        for row, entry, value in ((1, 3, -1), (2, 6, 80), (2, 8, -1)):
            p.model.tables[row, entry] = value
            p.seqs.tables[row, entry] = value
        p.model.lengths[3] = 12 * 16 + 1
        p.seqs.lengths[3] = 12 * 16 + 1
        p.evict([0, 1, 2, 3, -1, 8, 0, 4], 50, 1, 1)
        p.model.lengths[3] = -5
        p.seqs.lengths[3] = -5
        p.evict([3, 3], 50)


@pytest.mark.parametrize("seed", range(6))
def test_lifecycles(torch, ck, seed):
    """Random growing, forking, freeing, cutting and packing, all state and
    every byte after each step."""
    rng = random.Random(seed)
    bs = rng.choice([1, 4, 16])
    p = Evicting(torch, ck, 7, 200 // bs, geometry(500 // bs, bs, 1, 8 * rng.randint(1, 4), 2), seed=seed)
    with p.pool:
        for _ in range(25):
            step = rng.choice(["grow", "grow", "fork", "free", "evict", "evict", "evict", "compact"])
            ids = [rng.randrange(-1, 8) for _ in range(rng.randint(1, 6))]
            if step == "grow":
                p.do("grow", ids, [rng.choice([0, 1, 7, 60, 150]) for _ in ids])
            elif step == "fork":
                p.do("fork", ids, [rng.randrange(7) for _ in ids])
            elif step == "free":
                p.do("free", ids[:2])
            elif step == "compact":
                p.do("compact")
            else:
                tokens = rng.choice([1, 10, 30, 64, 100])
                sinks = rng.randint(0, tokens)
                p.evict(rng.choice([ids, None]), tokens, sinks, rng.randint(0, tokens - sinks))


def test_many_entries(torch, ck):
    """More than a workgroup's threads."""
    n = 1500
    p = Evicting(torch, ck, n, 3, geometry(2 * n + 900, 4, 1, 8, 2, 1), seed=9)
    with p.pool:
        p.do("grow", list(range(1200)), [9 if i % 3 else 3 for i in range(1200)])
        p.do("fork", list(range(0, 300)), list(range(1200, 1500)))
        p.evict(None, 6, 1, 1)
        p.evict(list(range(1400, 300, -1)), 5)


def test_entries_past_what_a_workgroup_looks_through(torch, ck):
    """Thousands of entries, some rows named again by later ones."""
    n = 6000
    p = Evicting(torch, ck, n, 2, geometry(2 * n + 64, 4, 1, 8, 1, 1, 1), seed=14)
    with p.pool:
        p.do("grow", list(range(5900)), [7 if i % 2 else 3 for i in range(5900)])
        p.do("fork", [1, 3, 5], [5900, 5901, 5902])
        ids = list(range(5999, 0, -1))
        ids[4500], ids[5000], ids[5500] = 5999 - 17, 5901, -1
        p.evict(ids, 5, 1, 1)


def test_identities(torch, ck):
    """A rewritten block gives up the prefix that it held; those before it and
    claims' held blocks keep theirs."""
    from types import SimpleNamespace

    p = Evicting(torch, ck, 2, 10, geometry(30), seed=10)
    text = np.arange(100, 260, dtype=np.uint32)
    with p.pool:
        p.do("grow", [0], [160])
        row = p.seqs.tables[0].cpu().numpy()
        batch = ck.DeviceBatch(SimpleNamespace(claim_ids=[7], block_offsets=[0, 10], block_ids=row,
                                               token_offsets=[0, 160], tokens=text))
        p.pool.offload(batch)
        assert p.pool.lookup(batch)["hit_blocks"][0] == 10
        p.do("fork", [0], [1])
        p.w[1] = np.arange(160)
        p.weights[1] = torch.arange(160.0)
        p.evict([1], 60, 32, 0)  # blocks of its own take the place of the later ones
        assert p.pool.lookup(batch)["hit_blocks"][0] == 10
        p.w[0] = np.arange(160)
        p.weights[0] = torch.arange(160.0)
        p.evict([0], 60, 35, 0)  # the first two blocks stay (shared with the other), the third changes
        assert p.pool.lookup(batch)["hit_blocks"][0] == 2


@pytest.mark.parametrize("other", [False, True])
def test_streams_and_graphs(torch, ck, other):
    p = Evicting(torch, ck, 4, 20, geometry(90), torch.cuda.Stream() if other else None, seed=11)
    with p.pool:
        p.do("grow", [0, 1, 2], [300, 200, 100])
        p.do("fork", [0], [3])
        p.evict(None, 150, 4, 20)
        torch.cuda.synchronize()
        saved = [t.clone() for t in (p.seqs.tables, p.seqs.lengths, p.seqs.refs, p.weights, p.kv)]
        graph = torch.cuda.CUDAGraph()
        stream = p.pool.stream if other else torch.cuda.Stream()
        if not other:
            return  # the pool's stream is the default one, which does not capture
        with torch.cuda.graph(graph, stream=stream):
            status, kept = p.seqs.evict(None, p.weights, 90, sinks=2, recent=9)
        m = p.model
        state = [x.copy() for x in (m.tables, m.lengths, m.refs, m.kv, p.w)]
        want = evict(m, p.w, None, 90, 2, 9)
        for _ in range(3):
            for t, x in zip((p.seqs.tables, p.seqs.lengths, p.seqs.refs, p.weights, p.kv), saved):
                t.copy_(x)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert status.tolist() == want[0] and kept.tolist() == want[1]
            p.same()
            assert np.array_equal(p.weights.cpu().numpy(), p.w, equal_nan=True)
        del state


def test_bytes_past_4_gib(torch, ck):
    """Blocks behind 4 GiB of a plane, moved within and into them."""
    from paper_2606_01387_amd.sequences import Sequences

    g = geometry(80000, 16, 8, 128, 2, 1)  # 2.6 GB a plane
    kv = torch.empty(g.pool_bytes, dtype=torch.uint8, device="cuda")
    with ck.Pool(g, 3, kv, max_claims=16, max_footprint=64, event_capacity=64) as pool:
        row = torch.tensor([79999 - 7 * i for i in range(20)], dtype=torch.int32, device="cuda")
        seqs = Sequences(pool, tables=row.view(1, -1).clone(),
                         lengths=torch.tensor([320], dtype=torch.int32, device="cuda"))
        seqs.refs[row[3:6].long()] += 1
        seqs.refs[:79000] += 1  # the free blocks are late ones too
        view = kv.view(2, 80000, 16, 2048)
        gen = torch.Generator(device="cuda").manual_seed(1)
        view[:, row.long()] = torch.randint(0, 256, (2, 20, 16, 2048), generator=gen, dtype=torch.uint8, device="cuda")
        old = view[:, row.long()].reshape(2, 320, 2048)
        weights = torch.rand(1, 320, generator=gen, device="cuda")
        status, kept = seqs.evict(None, weights, 200, sinks=10, recent=5)
        torch.cuda.synchronize()
        assert status.tolist() == [0] and int(seqs.lengths[0]) == 200
        now = view[:, seqs.tables[0, :13].long()].reshape(2, 208, 2048)[:, :200]
        assert torch.equal(now, old[:, kept[0].long()])
        held = view[:, row[3:6].long()].reshape(2, 48, 2048)
        assert torch.equal(held, old[:, 48:96])


def test_refusals(torch, ck):
    p = Evicting(torch, ck, 3, 20, geometry(60), seed=12)
    with p.pool:
        p.do("grow", [0], [200])
        for bad in (dict(tokens=0), dict(tokens=-1), dict(tokens=10, sinks=8, recent=3), dict(tokens=10, sinks=-1),
                    dict(tokens=2**31)):
            with pytest.raises(ValueError):
                p.seqs.evict(None, p.weights, **bad)
        for bad in (p.weights[:2], p.weights[:, :100], p.weights.double(), p.weights.cpu()):
            with pytest.raises(ValueError):
                p.seqs.evict(None, bad, 50)
        with pytest.raises(ValueError):
            p.seqs.evict(p.ints([0]).long(), p.weights, 50)
        with pytest.raises(ck.ClaimError):
            p.seqs.evict(p.ints([0, 1, 2, 0]), p.weights, 50)  # more entries than rows
        status, kept = p.seqs.evict(p.ints([]), p.weights, 50)
        assert status.numel() == 0 and kept.shape == (0, 50)
        p.same()
    odd = Evicting(torch, ck, 1, 4, geometry(8, 16, 1, 3, 1), seed=13)  # tokens of 3 bytes
    with odd.pool:
        with pytest.raises(ck.ClaimError):
            odd.seqs.evict(None, odd.weights, 5)
