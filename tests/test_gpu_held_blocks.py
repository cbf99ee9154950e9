"""Blocks that a program holds by a count of its own: compaction leaves them
where they are."""

import random
from types import SimpleNamespace

import numpy as np
import pytest

from test_gpu_blocks import Model, Pair, geometry

pytestmark = pytest.mark.gpu


class HoldingModel(Model):
    """Blocks with more counts than table entries stay; the others move as
    ever, the i-th of them from U on into the i-th free block below U."""

    def compact(self):
        used = [b for b in range(len(self.refs)) if self.refs[b]]
        U = len(used)
        named = np.bincount(self.tables[self.tables >= 0], minlength=len(self.refs))
        src = [b for b in used if b >= U and self.refs[b] <= named[b]]
        dst = [b for b in range(U) if self.refs[b] == 0]
        for a, b in zip(src, dst):
            self.kv[:, b] = self.kv[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.tables[self.tables == a] = b
        return len(src)


def holding_pair(torch, ck, max_seqs, max_blocks, g):
    p = Pair(torch, ck, max_seqs, max_blocks, g)
    p.model.__class__ = HoldingModel

    def hold(blocks, by):
        for b in blocks:
            p.model.refs[b] += by
        p.seqs.refs.index_add_(0, p.ints(blocks), p.ints([by] * len(blocks)))

    return p, hold


# tables that are counted by the plan, and ones (or a pool) that are not
@pytest.mark.parametrize("max_seqs, max_blocks, blocks", [(6, 40, 64), (9, 1500, 300), (6, 40, 9001)])
@pytest.mark.parametrize("seed", range(3))
def test_held_blocks_stay(torch, ck, max_seqs, max_blocks, blocks, seed):
    g = geometry(num_layers=1, block_size=2, num_kv_heads=1, head_dim=8, num_blocks=blocks)
    p, hold = holding_pair(torch, ck, max_seqs, max_blocks, g)
    rng = random.Random(seed)
    most = min(2 * max_blocks, 2 * blocks // max_seqs)
    with p.pool:
        for _ in range(6):
            p.do("grow", list(range(max_seqs)), [rng.randint(0, most) for _ in range(max_seqs)])
            p.do("fork", [rng.randrange(max_seqs) for _ in range(3)], rng.sample(range(max_seqs), 3))
            kept = sorted(rng.sample(range(blocks), rng.randint(1, blocks // 4)))  # used ones and free ones
            hold(kept, 1)
            p.do("free", rng.sample(range(max_seqs), max_seqs // 2))
            p.do("compact")
            hold(kept[::2], -1)
            p.do("compact")
            hold(kept[1::2], -1)


def test_a_prefix_list_and_its_count(torch, ck):
    """A list kept for attend_shared names the same keys and values after a
    compaction when its blocks are held."""
    g = geometry(num_layers=1, num_blocks=40)
    p = Pair(torch, ck, 4, 16, g)
    p.kv.copy_(torch.randn(2, 40, g.chunk_bytes // 2, generator=torch.Generator().manual_seed(0))
               .to(torch.bfloat16).view(torch.uint8))
    with p.pool:
        p.seqs.grow(p.ints([0]), p.ints([200]))  # blocks 0 to 12
        p.seqs.grow(p.ints([1]), p.ints([64]))  # 13 to 16
        p.seqs.fork(p.ints([1]), p.ints([2]))
        p.seqs.grow(p.ints([2]), p.ints([5]))
        shared = p.seqs.tables[1, :4].clone()
        p.seqs.refs.index_add_(0, shared, torch.ones_like(shared))
        q = torch.randn(1, 4, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        before = p.seqs.attend_shared(0, q, shared, ids=p.ints([2]))
        p.seqs.free(p.ints([0]))
        assert p.seqs.compact().item() == 1  # the child's own block
        assert p.seqs.tables[2, :5].tolist() == [13, 14, 15, 16, 0]
        assert torch.equal(p.seqs.attend_shared(0, q, shared, ids=p.ints([2])), before)


def test_a_held_claim_comes_back(torch, ck):
    """A claim's blocks, held while it is out, take its bytes again after
    sequences ended, the pool was compacted and others grew."""
    g = geometry(num_layers=1, num_blocks=32)
    p, hold = holding_pair(torch, ck, 4, 8, g)
    with p.pool:
        p.do("grow", [0, 1, 2], [48, 48, 48])
        blocks = p.model.tables[2, :3].copy()
        row = ck.DeviceBatch(SimpleNamespace(claim_ids=[5], block_offsets=[0, 3], block_ids=blocks,
                                             token_offsets=[0, 48], tokens=np.arange(48)))
        hold(blocks, 1)
        staging = torch.empty(3 * g.block_bytes, dtype=torch.uint8, device="cuda")
        p.pool.offload(row, staging)
        p.do("free", [0, 2])
        p.do("compact")
        assert p.model.tables[1, :3].tolist() == [3, 4, 5]
        p.do("grow", [0, 3], [100, 100])
        assert not np.isin(blocks, p.model.tables).any()
        p.kv[:, torch.from_numpy(blocks).long()] = 0  # while it is out, anything may be there
        p.pool.restore(row, staging)
        p.pool.check(row)
        assert p.pool.read()[0][0]["code"] == ck.MATERIALIZED
        p.same()
