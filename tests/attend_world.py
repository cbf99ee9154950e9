"""A pool with sequences in random blocks, and attention over them in 64 bits.

Everything in the pool that no sequence holds is NaN, so that a value read
from a wrong place shows.  The reference follows the definition, row by row,
from host copies of what the kernels are given."""

import math
from types import SimpleNamespace

import numpy as np

from paper_2606_01387_amd.synth import Geometry

NONE = -1


class World:
    """``seqs``: (rows, tokens cached before them past the prefix) of each."""

    def __init__(self, torch, *, seqs, heads=2, group=2, dim=64, block_size=16, e4m3=False, layers=2,
                 layer=1, prefix_blocks=0, seed=0, k_scale=None, v_scale=None, spread=1.0):
        self.torch, self.seqs, self.heads, self.group, self.dim = torch, seqs, heads, group, dim
        self.bs, self.e4m3, self.layer, self.prefix_blocks = block_size, e4m3, layer, prefix_blocks
        self.k_scale = (k_scale or 0.05) if e4m3 else 1.0
        self.v_scale = (v_scale or 0.02) if e4m3 else 1.0
        g = torch.Generator().manual_seed(seed)
        P = prefix_blocks * block_size
        self.length = [P + n + m for n, m in seqs]
        need = [-(-(n + m) // block_size) for n, m in seqs]
        used = prefix_blocks + sum(need)
        self.blocks = used + 5
        perm = torch.randperm(self.blocks, generator=g)[:used].to(torch.int32)
        self.prefix = perm[:prefix_blocks].clone()
        wide = prefix_blocks + max(need + [1])
        tables = torch.full((len(seqs), wide), NONE, dtype=torch.int32)
        at = prefix_blocks
        for s, k in enumerate(need):
            tables[s, :prefix_blocks] = self.prefix
            tables[s, prefix_blocks:prefix_blocks + k] = perm[at:at + k]
            at += k
        self.tables = tables
        nan = torch.full((2 * layers, self.blocks, block_size, heads, dim), float("nan"))
        for s in range(len(seqs)):
            for p in range(self.length[s]):
                b = int(tables[s, p // block_size])
                nan[2 * layer:2 * layer + 2, b, p % block_size] = torch.randn(2, heads, dim, generator=g) * spread
        self.kv = self.round(nan)
        self.rows = sum(n for n, _ in seqs)
        self.q = (torch.randn(self.rows, heads * group, dim, generator=g) * spread).to(torch.bfloat16)
        off = np.concatenate([[0], np.cumsum([n for n, _ in seqs])])
        self.offsets = torch.tensor(off, dtype=torch.int32)
        self.lengths = torch.tensor(self.length, dtype=torch.int32)
        self.geometry = Geometry(layers, 2, block_size, heads, dim, 1 if e4m3 else 2, self.blocks)

    def round(self, x):
        torch = self.torch
        if not self.e4m3:
            return x.to(torch.bfloat16)
        x = x.clone()
        x[0::2] /= self.k_scale
        x[1::2] /= self.v_scale
        return x.clamp(-448, 448).to(torch.float8_e4m3fn)

    def to_gpu(self, ck, stream=None):
        """(pool, sequences, device tensors)."""
        from paper_2606_01387_amd.sequences import Sequences

        d = SimpleNamespace(kv=self.kv.cuda(), tables=self.tables.cuda(), lengths=self.lengths.cuda(),
                            offsets=self.offsets.cuda(), q=self.q.cuda(), prefix=self.prefix.cuda())
        pool = ck.Pool(self.geometry, 3, d.kv.view(self.torch.uint8), max_claims=16, max_footprint=64,
                       event_capacity=64, stream=stream)
        return pool, Sequences(pool, tables=d.tables, lengths=d.lengths), d

    def scales(self):
        return dict(k_scale=self.k_scale, v_scale=self.v_scale)

    def values(self, s, head):
        """K and V of sequence s in 64 bits, and which positions have a block."""
        torch, L = self.torch, self.length[s]
        pos = torch.arange(L)
        block = torch.full((L,), NONE, dtype=torch.int64)
        held = pos // self.bs < self.tables.shape[1]
        block[held] = self.tables[s].long()[pos[held] // self.bs]
        P = self.prefix_blocks * self.bs
        if P:
            block[:P] = self.prefix.long()[pos[:P] // self.bs]
        fine = (block >= 0) & (block < self.blocks)
        raw = self.kv.view(torch.uint8) if self.e4m3 else self.kv
        got = []
        for i, scale in ((0, self.k_scale), (1, self.v_scale)):
            x = raw[2 * self.layer + i][block.clamp(0, self.blocks - 1), pos % self.bs, head]
            got.append((x.view(self.kv.dtype).double() * scale).numpy())
        return got[0], got[1], fine.numpy()

    def expected(self, scale=None):
        """(outputs, bounds) in 64 bits, [rows, heads, dim].

        The bound: the output is rounded to bf16 (2^-8 of it), each weight is
        rounded to bf16 (2^-8 of the sum of w |v|), and a score in 32 bits is
        off by at most (dim + 8) 2^-24 of scale sum |q| |k|, which moves the
        weights by as much, above and below the line."""
        scale = self.dim**-0.5 if scale is None else scale
        out = np.zeros((self.rows, self.heads * self.group, self.dim))
        bound = np.zeros_like(out)
        row = 0
        q = self.q.double().numpy()
        for s, (n, _) in enumerate(self.seqs):
            L = self.length[s]
            for h in range(self.heads):
                if not n:
                    continue
                k, v, fine = self.values(s, h)
                for i in range(n):
                    P = L - n + i
                    for g in range(self.group):
                        x = h * self.group + g
                        if P < 0:
                            continue
                        if not fine[:P + 1].all():
                            out[row + i, x] = math.nan
                            continue
                        with np.errstate(invalid="ignore", over="ignore"):
                            a = k[:P + 1] @ q[row + i, x] * scale
                            big = np.abs(k[:P + 1]) @ np.abs(q[row + i, x]) * scale
                            w = np.exp(a - a.max())
                            w /= w.sum()
                            out[row + i, x] = w @ v[:P + 1]
                            delta = 2 * (self.dim + 8) * 2.0**-24 * big.max()
                            bound[row + i, x] = (2.0**-8 * np.abs(out[row + i, x])
                                                 + (2.0**-8 + delta + 2.0**-20) * (w @ np.abs(v[:P + 1])))
            row += n
        return out, 1.01 * bound + 1e-30


def check(out, expected, bound):
    got = out.double().cpu().numpy()
    assert got.shape == expected.shape
    nan = np.isnan(expected)
    assert np.array_equal(np.isnan(got), nan), (np.isnan(got).sum(), nan.sum())
    off = np.abs(got - expected)[~nan]
    assert (off <= bound[~nan]).all(), (off / bound[~nan]).max()
