"""Sequences' blocks: growing, forking, freeing, compacting, copying, and
writing keys and values, against plain Python on host copies."""

import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

NONE = -1


class Model:
    """The definitions, one sequence and one block after another."""

    def __init__(self, max_seqs, max_blocks, blocks, bs, kv):
        self.tables = np.full((max_seqs, max_blocks), NONE, np.int32)
        self.lengths = np.zeros(max_seqs, np.int32)
        self.refs = np.zeros(blocks, np.int32)
        self.bs, self.kv = bs, kv

    def _take(self, k, free):
        got, free[:] = free[:k], free[k:]
        return got

    def grow(self, ids, tokens):
        free = [b for b in range(len(self.refs)) if self.refs[b] == 0]
        left, status, seen, asked = len(free), [], set(), 0
        for r, t in zip(ids, tokens):
            t %= 1 << 32  # counts are unsigned
            if not 0 <= r < len(self.lengths) or r in seen:
                status.append(2)
                continue
            seen.add(r)
            L = int(self.lengths[r])
            if L + t > self.tables.shape[1] * self.bs:
                status.append(2)
                continue
            held, need = -(-L // self.bs), -(-(L + t) // self.bs) - -(-L // self.bs)
            asked += need
            if asked > left:
                status.append(1)
                continue
            for k, b in enumerate(self._take(need, free)):
                self.tables[r, held + k] = b
                self.refs[b] = 1
            self.lengths[r] = L + t
            status.append(0)
        return status

    def fork(self, parents, children):
        free = [b for b in range(len(self.refs)) if self.refs[b] == 0]
        before, left, asked, status, seen = self.lengths.copy(), len(free), 0, [], set()
        for p, c in zip(parents, children):
            n = len(before)
            if not 0 <= c < n or c in seen:
                status.append(2)
                continue
            seen.add(c)
            if not 0 <= p < n or p == c or before[c]:
                status.append(2)
                continue
            L = int(before[p])
            full, part = L // self.bs, L % self.bs > 0
            asked += part
            if part and asked > left:
                status.append(1)
                continue
            if not part and asked > left:
                status.append(1)
                continue
            self.tables[c, :full] = self.tables[p, :full]
            for b in self.tables[p, :full]:
                if b >= 0:
                    self.refs[b] += 1
            if part:
                b = self._take(1, free)[0]
                src = self.tables[p, full]
                if src >= 0:
                    self.tables[c, full] = b
                    self.refs[b] = 1
                    self.kv[:, b] = self.kv[:, src]
            self.lengths[c] = L
            status.append(0)
        return status

    def free(self, ids):
        for r in ids:
            if 0 <= r < len(self.lengths) and self.lengths[r]:
                for j in range(-(-int(self.lengths[r]) // self.bs)):
                    b = self.tables[r, j]
                    if b >= 0 and self.refs[b]:
                        self.refs[b] -= 1
                self.tables[r] = NONE
                self.lengths[r] = 0

    def compact(self):
        used = [b for b in range(len(self.refs)) if self.refs[b]]
        U = len(used)
        src = [b for b in used if b >= U]
        dst = [b for b in range(U) if self.refs[b] == 0]
        for a, b in zip(src, dst):
            self.kv[:, b] = self.kv[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.tables[self.tables == a] = b
        return len(src)


class Pair:
    """The library's sequences and the model's."""

    def __init__(self, torch, ck, max_seqs, max_blocks, geometry, stream=None):
        from paper_2606_01387_amd.sequences import Sequences

        self.torch, g = torch, geometry
        gen = torch.Generator().manual_seed(5)
        kv = torch.randint(0, 256, (g.planes, g.num_blocks, g.chunk_bytes), generator=gen, dtype=torch.uint8)
        self.kv = kv.cuda()
        self.pool = ck.Pool(g, 3, self.kv, max_claims=16, max_footprint=64, event_capacity=64, stream=stream)
        self.seqs = Sequences(self.pool, max_seqs, max_blocks)
        self.model = Model(max_seqs, max_blocks, g.num_blocks, g.block_size, kv.numpy())

    def ints(self, x):
        return self.torch.tensor(x, dtype=self.torch.int32, device="cuda")

    def do(self, name, *lists):
        got = getattr(self.seqs, name)(*[self.ints(x) for x in lists])
        want = getattr(self.model, name)(*lists)
        if got is not None:
            assert got.tolist() == (want if isinstance(want, list) else [want]), name
        self.same()

    def same(self):
        m = self.model
        assert np.array_equal(self.seqs.lengths.cpu().numpy(), m.lengths)
        assert np.array_equal(self.seqs.tables.cpu().numpy(), m.tables)
        assert np.array_equal(self.seqs.refs.cpu().numpy(), m.refs)
        assert np.array_equal(self.kv.cpu().numpy(), m.kv)


def geometry(**kw):
    from paper_2606_01387_amd.synth import Geometry

    d = dict(num_layers=2, planes_per_layer=2, block_size=16, num_kv_heads=2, head_dim=64, elem_bytes=2,
             num_blocks=64)
    d.update(kw)
    return Geometry(**d)


GEOMETRIES = {
    "small": dict(),
    "latent": dict(num_layers=3, planes_per_layer=1, block_size=64, num_kv_heads=1, head_dim=576,
                   elem_bytes=1, num_blocks=50),
    "one-word-chunks": dict(num_layers=1, block_size=1, num_kv_heads=1, head_dim=8, num_blocks=7),
    "odd": dict(num_layers=1, block_size=24, num_kv_heads=3, head_dim=80, num_blocks=201),
    "chunk of pieces": dict(num_layers=1, block_size=40, num_kv_heads=7, head_dim=128, num_blocks=23),
    "many": dict(num_layers=1, planes_per_layer=1, block_size=2, num_kv_heads=1, head_dim=8, elem_bytes=1,
                 num_blocks=9001),
}


@pytest.mark.parametrize("name", GEOMETRIES)
@pytest.mark.parametrize("seed", range(3))
def test_lifecycles(torch, ck, name, seed):
    """Random calls one after another; all state after each of them."""
    g = geometry(**GEOMETRIES[name])
    rng = random.Random(seed)
    seqs = rng.choice([3, 9, 40])
    wide = max(2, g.num_blocks // rng.choice([2, 4, 8]))
    p = Pair(torch, ck, seqs, wide, g)
    with p.pool:
        for _ in range(30):
            k = rng.randint(1, seqs)
            ids = [rng.randrange(-1, seqs + 1) for _ in range(k)]
            op = rng.choice(["grow", "grow", "grow", "fork", "fork", "free", "compact"])
            if op == "grow":
                most = rng.choice([1, g.block_size, 2 * g.block_size * wide // seqs + 1])
                p.do("grow", ids, [rng.randint(0, most) for _ in ids])
            elif op == "fork":
                p.do("fork", ids, [rng.randrange(-1, seqs + 1) for _ in ids])
            elif op == "free":
                p.do("free", ids[:max(1, k // 2)])
            else:
                p.do("compact")


def test_many_sequences(torch, ck):
    """More entries than a planning workgroup has threads."""
    g = geometry(num_layers=1, planes_per_layer=1, block_size=4, num_kv_heads=1, head_dim=8, elem_bytes=1,
                 num_blocks=6000)
    p = Pair(torch, ck, 2500, 8, g)
    rng = random.Random(1)
    with p.pool:
        p.do("grow", list(range(1200)), [rng.randint(0, 9) for _ in range(1200)])
        p.do("fork", [rng.randrange(1200) for _ in range(1300)], list(range(1200, 2500)))
        p.do("grow", list(range(2500)), [rng.randint(0, 6) for _ in range(2500)])
        p.do("free", rng.sample(range(2500), 1500))
        p.do("compact")
        p.do("grow", list(range(2500)), [rng.randint(0, 20) for _ in range(2500)])


def test_huge_requests_are_refused(torch, ck):
    p = Pair(torch, ck, 4, 8, geometry())
    with p.pool:
        p.do("grow", [0, 1], [5, 17])
        p.do("grow", [0, 1, 2, 3], [-1, 2**31 - 1, 129, 128])
        p.do("grow", [0, 0, 7, -5], [1, 1, 1, 1])


def test_grow_without_ids_and_nothing(torch, ck):
    p = Pair(torch, ck, 3, 4, geometry())
    with p.pool:
        assert p.seqs.grow(None, p.ints([3, 40, 0])).tolist() == p.model.grow([0, 1, 2], [3, 40, 0])
        p.same()
        p.do("grow", [], [])
        p.do("fork", [], [])
        p.do("free", [])


def test_a_parent_with_a_missing_last_block(torch, ck):
    p = Pair(torch, ck, 3, 4, geometry())
    with p.pool:
        p.do("grow", [0], [20])
        p.seqs.tables[0, 1] = NONE
        p.seqs.refs[1] = 0
        p.model.tables[0, 1], p.model.refs[1] = NONE, 0
        p.do("fork", [0], [1])
        p.do("free", [0, 1])


def test_copy_blocks(torch, ck):
    p = Pair(torch, ck, 1, 1, geometry(num_blocks=200, num_kv_heads=8, head_dim=128))
    rng = np.random.RandomState(0)
    perm = rng.permutation(200)
    src, dst = perm[:60].astype(np.int32), perm[60:120].astype(np.int32)
    p.model.kv[:, dst] = p.model.kv[:, src]
    src, dst = np.append(src, [-1, 3, 200]), np.append(dst, [5, -1, perm[130]])
    with p.pool:
        p.pool.copy_blocks(p.ints(src), p.ints(dst))
        p.same()


def test_blocks_handed_out_hold_no_identity(torch, ck):
    """A lookup does not hit a block that was handed out again, copied over
    or moved into; a freed block hits until then."""
    from types import SimpleNamespace

    g = geometry()
    p = Pair(torch, ck, 4, 8, g)

    def batch(ids, blocks, tokens):
        off = np.cumsum([0] + [len(b) for b in blocks])
        tof = np.cumsum([0] + [len(t) for t in tokens])
        return ck.DeviceBatch(SimpleNamespace(claim_ids=ids, block_offsets=off,
                                              block_ids=np.concatenate(blocks), token_offsets=tof,
                                              tokens=np.concatenate(tokens)))

    tokens = [np.arange(k * 100, k * 100 + 32) for k in range(4)]
    with p.pool:
        p.do("grow", [0, 1, 2, 3], [32] * 4)
        rows = batch(np.arange(1, 5), [p.model.tables[s, :2] for s in range(4)], tokens)
        p.pool.offload(rows)
        hits = lambda: p.pool.lookup(rows)["hit_blocks"].tolist()  # noqa: E731
        assert hits() == [2, 2, 2, 2]
        p.do("free", [0])
        assert hits() == [2, 2, 2, 2]
        p.do("grow", [0], [16])  # takes block 0
        assert hits() == [0, 2, 2, 2]
        p.do("fork", [0], [0])  # refused
        p.do("free", [0])
        p.do("compact")  # blocks 6 and 7 (claim 4's) move over 0 and 1
        assert hits() == [0, 2, 2, 2]
        p.pool.copy_blocks(p.ints([2]), p.ints([5]))
        assert hits() == [0, 2, 1, 2]


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("dim,heads,bs", [(64, 2, 16), (128, 8, 16), (8, 1, 4), (80, 3, 24), (128, 1, 1)])
def test_write(torch, ck, dim, heads, bs, elem):
    """Rows from slices of a wider projection, at every place of a block;
    rows without a block, and everything else, stay as they are."""
    g = geometry(num_kv_heads=heads, head_dim=dim, block_size=bs, elem_bytes=elem, num_blocks=300)
    p = Pair(torch, ck, 5, 60, g)
    gen = torch.Generator().manual_seed(1)
    new = [1, 0, 37, 5, 9]
    with p.pool:
        p.do("grow", [0, 1, 2, 3, 4], [min(n + c, 60 * bs) for n, c in zip(new, [7, 3, 11, 0, 40])])
        p.seqs.tables[2, 0] = NONE
        p.model.tables[2, 0] = NONE
        p.seqs.lengths[3] = p.model.lengths[3] = 2  # three of its rows are before position 0
        T = sum(new)
        wide = (torch.randn(T, 2, heads + 1, dim, generator=gen) * 3).to(torch.bfloat16)
        wide.view(-1)[::7] *= 100  # some past the largest e4m3 value
        k, v = wide[:, 0, 1:].cuda(), wide[:, 1, :heads].cuda()
        k_scale, v_scale = (0.37, 0.21) if elem == 1 else (1.0, 1.0)
        off = np.concatenate([[0], np.cumsum(new)])
        p.seqs.write(1, k, v, offsets=p.ints(off), k_scale=k_scale, v_scale=v_scale)
        kv = torch.from_numpy(p.model.kv).view(g.planes, g.num_blocks, bs, heads * dim * elem)
        for plane, x, scale in ((2, wide[:, 0, 1:], k_scale), (3, wide[:, 1, :heads], v_scale)):
            if elem == 1:
                x = (x.float() / scale).clamp(-448, 448).to(torch.float8_e4m3fn)
            x = x.contiguous().view(torch.uint8).view(T, -1)
            for s in range(5):
                for i in range(new[s]):
                    pos = int(p.model.lengths[s]) - new[s] + i
                    if pos >= 0 and p.model.tables[s, pos // bs] >= 0:
                        kv[plane, p.model.tables[s, pos // bs], pos % bs] = x[off[s] + i]
        p.same()


def test_write_rounds_as_torch_does(torch, ck):
    """Every bf16 value to e4m3, NaN and the infinities too."""
    g = geometry(num_layers=1, num_kv_heads=8, head_dim=128, elem_bytes=1, block_size=16, num_blocks=5)
    p = Pair(torch, ck, 1, 5, g)
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(64, 8, 128)
    with p.pool:
        p.seqs.grow(None, p.ints([64]))
        p.seqs.write(0, every.cuda(), every.cuda(), offsets=p.ints([0, 64]), k_scale=1.0, v_scale=0.3)
        got = p.kv.cpu()[:, :4].reshape(2, 64, 8, 128)
    for plane, scale in ((0, 1.0), (1, 0.3)):
        x = every.float() / scale
        want = torch.where(x.isnan(), x, x.clamp(-448, 448)).to(torch.float8_e4m3fn).float()
        have = got[plane].view(torch.float8_e4m3fn).float()
        assert torch.equal(want.isnan(), have.isnan())
        assert torch.equal(want.nan_to_num(), have.nan_to_num())


def test_another_stream(torch, ck):
    g = geometry(num_blocks=400, num_kv_heads=8, head_dim=128)
    p = Pair(torch, ck, 40, 20, g, stream=torch.cuda.Stream())
    rng = random.Random(3)
    with p.pool:
        p.do("grow", list(range(8)), [rng.randint(1, 200) for _ in range(8)])
        for _ in range(5):
            parents = [rng.randrange(8) for _ in range(16)]
            p.do("fork", parents, list(range(8, 24)))
            p.do("grow", list(range(24)), [rng.randint(0, 20) for _ in range(24)])
            p.do("free", list(range(8, 24)))
            p.do("compact")
